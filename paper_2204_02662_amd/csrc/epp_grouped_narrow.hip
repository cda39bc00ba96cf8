// Grouped products of narrow fp32 matrices (widths of up to 128) with many entries: what the layers of a graph network are.
// They are bound by memory: 2 F_in F_out operations on 4 (F_in + F_out) bytes of an entry.
//
// Product and input gradient: a workgroup holds a group's weights in LDS and goes through up to 1,024 of its entries, 32 to a
// wavefront at a time.  Eight lanes load 128 bytes of an entry, the next 32 entries' while the matrix cores work on these; 4 KB of LDS
// for each wavefront bring them into the order of the instruction's operand (32x32x2: lane l supplies entry l % 32, and of every eight
// numbers four, for four instructions) and the results back into whole lines.  (Loaded from memory in the operand's order, 32 bytes of 32
// rows at a time, 1,000,000 entries of 64 x 64 took 180 us, of 128 x 16 278.)  No barriers: LDS serves a wavefront in order.
//
// Weight gradient: both operands stride through memory entry by entry, which is the order that the instruction wants: lane l supplies
// column l % 32 of entry l / 32, so that two entries' numbers go from memory to the instruction in whole lines, without LDS.  A
// workgroup's four wavefronts share a chunk of entries and add up their sums; k_grouped_sum adds the chunks'.

#include "epp_grouped.h"

using namespace epp_grouped;

namespace {

constexpr int kMost = 128;       // width
constexpr int kWaves = 8, kUnit = 32 * kWaves, kEntries = 4 * kUnit;  // product, input gradient: entries of a workgroup, at most
constexpr int kListed = 1024;    // weight gradient: entries whose rows are looked up at a time

__device__ __attribute__((aligned(128))) float g_zeros[kMost] = {};

typedef float any_floatx4 __attribute__((ext_vector_type(4), aligned(4)));

// K <= 32 P, N <= 32 NB.
template <int P, int NB>
__global__ __launch_bounds__(64 * kWaves) void k_narrow_rows(GroupedArgs g, int input, int units) {
    constexpr int kThreads = 64 * kWaves, kLd = 32 * P + 4;  // (16 lanes that read 16 bytes of neighbouring columns use all 64 banks)
    __shared__ __attribute__((aligned(16))) float Wl[32 * NB][kLd];  // [column][k]
    __shared__ __attribute__((aligned(128))) float turn[kWaves][32 * 32];
    __shared__ int32_t in_rows[kEntries], out_rows[kEntries];
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), half = lane >> 5;
    const int K = input ? g.F_out : g.F_in, N = input ? g.F_in : g.F_out, per = kUnit * units;
    int64_t total;
    const Span s = find_group(g.offsets, g.G, g.m, per, blockIdx.x, &total);
    if (s.g < 0) return;
    const int64_t m0 = s.first + (blockIdx.x - s.chunk0) * per;
    const int count = (int)min((int64_t)per, s.last - m0);
    for (int i = t; i < per; i += kThreads) {
        in_rows[i] = (int32_t)row_of(g.a, m0 + i, i < count);
        out_rows[i] = (int32_t)row_of(g.out, m0 + i, i < count);
    }
    const float* __restrict__ W = reinterpret_cast<const float*>(g.W) + (int64_t)s.g * g.F_in * g.F_out;
    constexpr int kFill = 32 * NB * 32 * P / kThreads, kAtOnce = kFill % 8 == 0 ? 8 : kFill % 6 == 0 ? 6 : kFill % 4 == 0 ? 4 : 2;
    static_assert(kFill * kThreads == 32 * NB * 32 * P && kFill % kAtOnce == 0, "the weights, and nothing behind them");
#pragma unroll 1
    for (int i0 = 0; i0 < kFill; i0 += kAtOnce) {
        float x[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int at = (i0 + i) * kThreads + t, n = input ? at / (32 * P) : at % (32 * NB), k = input ? at % (32 * P) : at / (32 * NB);
            x[i] = W[input ? min(n, N - 1) * K + min(k, K - 1) : min(k, K - 1) * N + min(n, N - 1)];
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int at = (i0 + i) * kThreads + t, n = input ? at / (32 * P) : at % (32 * NB), k = input ? at % (32 * P) : at / (32 * NB);
            Wl[n][k] = n < N && k < K ? x[i] : 0.f;
        }
    }
    __syncthreads();
    // A line of 32 numbers in `turn` is eight pieces of 16 bytes, permuted by the line's number (16 lanes that read the same piece of
    // neighbouring lines use all banks).  By lines: lane l holds piece l % 8 of lines l / 8 + 8 i; by columns: pieces 2 q + l / 32 of line l % 32.
    float* const mine = turn[w];
    const int line = lane >> 3, piece = lane & 7, row = lane & 31;
    auto by_lines = [&](int i) { return reinterpret_cast<floatx4*>(mine + (line + 8 * i) * 32 + ((piece ^ (((line + 8 * i) >> 1) & 7)) * 4)); };
    auto by_columns = [&](int q) { return reinterpret_cast<floatx4*>(mine + row * 32 + (((2 * q + half) ^ ((row >> 1) & 7)) * 4)); };
    const int rounds = (count - 32 * w + kUnit - 1) / kUnit;  // of this wavefront
    // Numbers 32 p + 4 piece .. of the entries of unit u; zeros behind the last number, and for an entry without a row.
    auto load = [&](int u, floatx4 (&v)[P][4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t r = u < rounds ? in_rows[32 * w + kUnit * u + line + 8 * i] : -1;
            const float* p = r < 0 ? g_zeros : reinterpret_cast<const float*>(g.a.data + (int64_t)r * g.a.ld);
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const int k = 32 * q + 4 * piece;
                if (32 * q + 32 <= K || K % 4 == 0) {
                    v[q][i] = *reinterpret_cast<const any_floatx4*>(32 * q + 32 <= K || k < K ? p + k : g_zeros);
                } else {  // (behind the row's end its last number, which `multiply` leaves out)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[q][i][e] = p[min(k + e, K - 1)];
                }
            }
        }
    };
    auto multiply = [&](int u, floatx4 (&v)[P][4]) {
        floatx16 acc[NB] = {};
#pragma unroll
        for (int q = 0; q < P; ++q) {
            if (32 * q >= K) continue;
            if (32 * q + 32 > K && K % 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[q][i][e] = 32 * q + 4 * piece + e < K ? v[q][i][e] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) *by_lines(i) = v[q][i];
            in_order();
            floatx4 x[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = *by_columns(c);
            in_order();
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (32 * q + 8 * c >= K) continue;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const floatx4 y = *reinterpret_cast<const floatx4*>(&Wl[32 * b + row][32 * q + 8 * c + 4 * half]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(y[j], x[c][j], acc[b], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int q = 0; q < 4; ++q) *by_columns(q) = floatx4{acc[b][4 * q], acc[b][4 * q + 1], acc[b][4 * q + 2], acc[b][4 * q + 3]};
            in_order();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int32_t r = out_rows[32 * w + kUnit * u + line + 8 * i];
                const floatx4 x = *by_lines(i);
                const int c = 32 * b + 4 * piece;
                if (r < 0 || c >= N) continue;
                const float y[4] = {x[0], x[1], x[2], x[3]};
                store4<float>(const_cast<char*>(g.out.data) + (int64_t)r * g.out.ld, c, y, N - c);
            }
            in_order();
        }
    };
    floatx4 x[2][P][4];
    load(0, x[0]);
    for (int u = 0; u < rounds; u += 2) {
        load(u + 1, x[1]);
        multiply(u, x[0]);
        if (u + 1 >= rounds) break;
        load(u + 2, x[0]);
        multiply(u + 1, x[1]);
    }
}

// Partial sums of one chunk: columns 32 MT bx and 32 NT by of the two operands on.
template <int MT, int NT>
__global__ __launch_bounds__(256) void k_narrow_weight(GroupedArgs g) {
    constexpr int kPairs = 8;  // pairs of entries on their way at a time
    __shared__ float sums[2][MT * NT * 16][64];
    __shared__ int32_t list[2][kListed + 2 * kPairs];
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), half = lane >> 5, col = lane & 31;
    int64_t total;
    const Span s = find_group(g.offsets, g.G, g.m, g.per, blockIdx.x, &total);
    if (s.g < 0) return;
    const int64_t chunk_first = s.first + (blockIdx.x - s.chunk0) * g.per, chunk_last = min(chunk_first + g.per, s.last);
    const int m0 = blockIdx.y * 32 * MT, n0 = blockIdx.z * 32 * NT;
    int xc[MT], yc[NT];  // (a column behind the width: somebody's numbers, for a result that is not written)
#pragma unroll
    for (int i = 0; i < MT; ++i) xc[i] = m0 + 32 * i + col < g.F_in ? m0 + 32 * i + col : 0;
#pragma unroll
    for (int j = 0; j < NT; ++j) yc[j] = n0 + 32 * j + col < g.F_out ? n0 + 32 * j + col : 0;
    floatx16 acc[MT][NT] = {};
    for (int64_t e0 = chunk_first; e0 < chunk_last; e0 += kListed) {
        // rows of up to kListed entries (those behind the last: none, and read as zeros)
        const int count = (int)min((int64_t)kListed, chunk_last - e0), share = ((count + 3) / 4 + 2 * kPairs - 1) / (2 * kPairs) * (2 * kPairs);
        __syncthreads();
        for (int i = t; i < kListed + 2 * kPairs; i += 256) {
            list[0][i] = (int32_t)row_of(g.a, e0 + i, i < count);
            list[1][i] = (int32_t)row_of(g.b, e0 + i, i < count);
        }
        __syncthreads();
        const int first = min(w * share, count), last = min(first + share, count);
        float x[2][kPairs][MT], y[2][kPairs][NT];
        auto load = [&](int i0, int z) {
#pragma unroll
            for (int q = 0; q < kPairs; ++q) {
                const int32_t ra = list[0][i0 + 2 * q + half], rb = list[1][i0 + 2 * q + half];
                const float* p = ra < 0 ? g_zeros : reinterpret_cast<const float*>(g.a.data + (int64_t)ra * g.a.ld);
                const float* d = rb < 0 ? g_zeros : reinterpret_cast<const float*>(g.b.data + (int64_t)rb * g.b.ld);
#pragma unroll
                for (int i = 0; i < MT; ++i) x[z][q][i] = p[xc[i]];
#pragma unroll
                for (int j = 0; j < NT; ++j) y[z][q][j] = d[yc[j]];
            }
        };
        auto work = [&](int z) {
#pragma unroll
            for (int q = 0; q < kPairs; ++q)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(y[z][q][j], x[z][q][i], acc[i][j], 0, 0, 0);
        };
        if (first < last) load(first, 0);
        for (int i0 = first; i0 < last; i0 += 4 * kPairs) {
            if (i0 + 2 * kPairs < last) load(i0 + 2 * kPairs, 1);
            work(0);
            if (i0 + 2 * kPairs >= last) break;
            if (i0 + 4 * kPairs < last) load(i0 + 4 * kPairs, 0);
            work(1);
        }
    }
    __syncthreads();
    // wavefronts 2 and 3 to 0 and 1, then 1 to 0
#pragma unroll
    for (int step = 2; step; step /= 2) {
        if (w >= step && w < 2 * step) {
#pragma unroll
            for (int i = 0; i < MT * NT; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) sums[w - step][i * 16 + e][lane] = acc[i / NT][i % NT][e];
        }
        __syncthreads();
        if (w < step) {
#pragma unroll
            for (int i = 0; i < MT * NT; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i / NT][i % NT][e] += sums[w][i * 16 + e][lane];
        }
        __syncthreads();
    }
    if (w) return;
    float* part = g.part + (int64_t)blockIdx.x * g.F_in * g.F_out;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int r = m0 + 32 * i + col;
        if (r >= g.F_in) continue;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = n0 + 32 * j + 8 * q + 4 * half;
                const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                store4<float>(reinterpret_cast<char*>(part + (int64_t)r * g.F_out), c, v, g.F_out - c);
            }
    }
}

template <int P, int NB>
int launch_rows(bool input, const GroupedArgs& g, hipStream_t s) {
    // as many entries to a workgroup as leave two of them to a compute unit
    int units = kEntries / kUnit;
    while (units > 1 && g.m < (int64_t)units * kUnit * 2 * kUnits) units /= 2;
    const int64_t per = kUnit * units, blocks = (g.m + std::min<int64_t>(g.G, g.m) * (per - 1)) / per;
    hipLaunchKernelGGL((k_narrow_rows<P, NB>), dim3((unsigned)blocks), dim3(64 * kWaves), 0, s, g, input ? 1 : 0, units);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}

template <int P>
int launch_rows_n(int N, bool input, const GroupedArgs& g, hipStream_t s) {
    if (N <= 32) return launch_rows<P, 1>(input, g, s);
    if (N <= 64) return launch_rows<P, 2>(input, g, s);
    if (N <= 96) return launch_rows<P, 3>(input, g, s);
    return launch_rows<P, 4>(input, g, s);
}

template <int MT, int NT>
int launch_weight(const GroupedArgs& g, int64_t chunks, hipStream_t s) {
    const dim3 grid((unsigned)chunks, (unsigned)((g.F_in + 32 * MT - 1) / (32 * MT)), (unsigned)((g.F_out + 32 * NT - 1) / (32 * NT)));
    hipLaunchKernelGGL((k_narrow_weight<MT, NT>), grid, dim3(256), 0, s, g);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}

}  // namespace

// Where these are faster than tiles of 64 x 64.  Four groups, rows named by lists, us, tiles / these: 64,000 entries, 16 x 41 10.6 / 9.1, its
// gradient 12.0 / 8.8, 64 x 64 12.9 / 13.2; 250,000, 128 x 16 51 / 53, its gradient 53 / 37, 64 x 64 38 / 45; 1,000,000, 16 x 41 140 / 99,
// 64 x 64 175 / 146, 128 x 128 419 / 377; 16,000, 16 x 41 6.5 / 6.6.
bool epp_grouped::narrow_rows(int64_t m, int K, int N) {
    return std::max(K, N) <= kMost && m >= (std::min(K, N) <= 32 ? 49152 : 1 << 19);
}

int epp_grouped::launch_narrow_rows(bool input, const GroupedArgs& g, hipStream_t s) {
    const int K = input ? g.F_out : g.F_in, N = input ? g.F_in : g.F_out;
    if (K <= 32) return launch_rows_n<1>(N, input, g, s);
    if (K <= 64) return launch_rows_n<2>(N, input, g, s);
    if (K <= 96) return launch_rows_n<3>(N, input, g, s);
    return launch_rows_n<4>(N, input, g, s);
}

// .. 64,000, 16 x 41 17.9 / 15.6; 1,000,000, 128 x 16 193 / 161; but 1,000,000, 64 x 47 133 / 151.
bool epp_grouped::narrow_weight(int64_t m, int F_in, int F_out) {
    return std::max(F_in, F_out) <= kMost && std::min(F_in, F_out) <= 32 && m >= 49152;
}

int64_t epp_grouped::narrow_weight_chunk(int64_t m) {
    // four workgroups to a compute unit, and no chunk that takes less time than its partial sums
    return std::max<int64_t>((m + 4 * kUnits - 1) / (4 * kUnits), 256);
}

int epp_grouped::launch_narrow_weight(const GroupedArgs& g, int64_t chunks, hipStream_t s) {
    if (g.F_in <= 32) return g.F_out <= 32 ? launch_weight<1, 1>(g, chunks, s) : launch_weight<1, 2>(g, chunks, s);
    return launch_weight<2, 1>(g, chunks, s);
}
