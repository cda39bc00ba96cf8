// Grouped products of few rows to a group, as single tokens are served: the time is that of reading the weights once.
//
// A workgroup forms 16 R rows of TN columns.  Its wavefronts share the contraction, a run of steps of 64 bytes each: every one streams
// its part of the weights (and of the rows) from memory into a ring of its own in LDS, without waiting for the others, and they add up
// their sums at the end.  Narrow tiles (32 or 64 columns) make enough workgroups for the chip even where only one or two groups have rows.
// Loads go to LDS directly, kDepth steps ahead; behind the last step the ring is filled with zeros, so that the number of loads on
// their way, which is what a wavefront waits by, is always the same.  Rows that are no multiples of 16 bytes come through registers.
//
// Matrix instructions of 16 x 16: lane l supplies column (row) l % 16 and the contraction's piece of 16 bytes l / 16 of a step: one
// instruction of 16 bits, four of floats.  As in the larger tiles, a piece's place in its line of LDS is permuted by the line's number, so that
// lanes read together from different banks.

#include "epp_grouped.h"

using namespace epp_grouped;

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kStep = 64;  // bytes of the contraction

__device__ __attribute__((aligned(128))) unsigned int g_zeros[32] = {};

template <class T>
__device__ __forceinline__ floatx4 multiply16(uintx4 a, uintx4 b, floatx4 c) {
    if constexpr (sizeof(T) == 4) {
        const floatx4 x = __builtin_bit_cast(floatx4, a), y = __builtin_bit_cast(floatx4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
        return c;
    } else if constexpr (std::is_same_v<T, __bf16>) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfloatx8, a), __builtin_bit_cast(bfloatx8, b), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
    }
}

__device__ __forceinline__ const char* zeros() { return reinterpret_cast<const char*>(g_zeros); }
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

template <class T, int MODE, int R, int TN, bool DIRECT>
__global__ __launch_bounds__(kThreads) void k_grouped_few(GroupedArgs g) {
    constexpr int size = (int)sizeof(T), E = 16 / size, KS = kStep / size, TM = 16 * R;
    constexpr int kX = TM * kStep, kW = TN * kStep, kStage = kX + kW, kLoads = kStage / 1024;
    constexpr int kDepth = !DIRECT ? 1 : kStage * 4 <= 20480 ? 4 : 3;  // steps in the ring
    constexpr int kAhead = kLoads <= 5 ? 4 : 3;                        // not DIRECT: steps on their way to registers
    constexpr int kBlocks = R * (TN / 16), kSums = kBlocks * 1024;     // bytes of a wavefront's results
    constexpr int kWide = TN * size, kPieces = kWide / 16;             // product: a line of the weights, one step of the contraction
    static_assert(kX % 1024 == 0 && kW % 1024 == 0 && kLoads * (kDepth - 1) < 64, "ring");
    __shared__ __attribute__((aligned(128))) char ring[kWaves][kDepth * kStage > kSums ? kDepth * kStage : kSums];
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), q = lane >> 4, l16 = lane & 15;
    const int N = MODE == kInput ? g.F_in : g.F_out, K = MODE == kInput ? g.F_out : g.F_in, nt = (N + TN - 1) / TN;
    // Workgroups b, b + 8, .. run on one XCD: it gets neighbouring columns, whose lines its L2 holds.
    const int64_t all = gridDim.x / 8, mine = (int64_t)(blockIdx.x & 7) * all + (blockIdx.x >> 3);
    int64_t total;
    const Span s = find_group(g.offsets, g.G, g.m, TM, mine / nt, &total);
    if (s.g < 0) return;
    const int64_t m0 = uniform(s.first + (mine / nt - s.chunk0) * TM), m_end = uniform(s.last);
    const int n0 = __builtin_amdgcn_readfirstlane((int)(mine % nt) * TN);

    const int steps = (K + KS - 1) / KS, share = (steps + kWaves - 1) / kWaves;
    const int first = min(w * share, steps), last = min(first + share, steps);
    const char* W = g.W + s.g * ((int64_t)g.F_in * g.F_out * size);
    const int64_t ldw = (int64_t)g.F_out * size;
    // This lane's pieces of a step: of rows (four lanes to a row, 16 rows to a load) ..
    const char* px[R];
    int kx[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = 16 * i + (lane >> 2);
        const int64_t row = row_of(g.a, m0 + r, m0 + r < m_end);
        kx[i] = ((lane & 3) ^ ((r >> 2) & 3)) * E;
        px[i] = row < 0 ? nullptr : g.a.data + row * g.a.ld;
    }
    // .. and of the weights
    constexpr int kWLoads = kW / 1024;
    auto turn = [](int line) {  // what a line's units of 32 bytes are permuted by
        if constexpr (size == 4) return TN == 64 ? ((line >> 2) & 3) << 1 : ((line >> 2) & 1) << 1;
        else return TN == 64 ? ((line >> 1) & 1) | (((line >> 3) & 1) << 1) : (line >> 3) & 1;
    };
    const char* pw[kWLoads];
    int kw[kWLoads], left[kWLoads];  // (product: columns from a piece's first to the end)
#pragma unroll
    for (int i = 0; i < kWLoads; ++i) {
        if constexpr (MODE == kInput) {
            const int n = 16 * i + (lane >> 2);
            kw[i] = ((lane & 3) ^ ((n >> 2) & 3)) * E;
            pw[i] = W + (int64_t)min(n0 + n, N - 1) * ldw;  // (columns behind the width: somebody's numbers, for a result that is not written)
            left[i] = 0;
        } else {
            const int line = (64 * i + lane) / kPieces, c = n0 + (((64 * i + lane) % kPieces) ^ (turn(line) << 1)) * E;
            kw[i] = line;
            pw[i] = W + (int64_t)(c < N ? c : 0) * size;
            left[i] = c < N ? N - c : N;
        }
    }
    const unsigned base = __builtin_amdgcn_readfirstlane(lds_address(ring[w]));
    auto fetch = [&](int st, int slot) {  // (the ring's place has been read)
        const unsigned to = base + (unsigned)slot * kStage;
        const int k0 = st * KS;
        const bool some = st < last;
#pragma unroll
        for (int i = 0; i < R; ++i) load_to_lds(some && px[i] && k0 + kx[i] < K ? px[i] + (int64_t)(k0 + kx[i]) * size : zeros(), to + (unsigned)i * 1024u);
#pragma unroll
        for (int i = 0; i < kWLoads; ++i) {
            const char* p = MODE == kInput ? pw[i] + (int64_t)(k0 + kw[i]) * size : pw[i] + (int64_t)(k0 + kw[i]) * ldw;
            load_to_lds(some && k0 + kw[i] < K ? p : zeros(), to + (unsigned)(kX + i * 1024));
        }
    };
    floatx4 acc[R][TN / 16] = {};
    auto work = [&](const char* tile) {
        uintx4 x[R], y[TN / 16];
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = *reinterpret_cast<const uintx4*>(tile + (16 * i + l16) * kStep + ((q ^ ((l16 >> 2) & 3)) * 16));
        const char* weights = tile + kX;
#pragma unroll
        for (int j = 0; j < TN / 16; ++j) {
            if constexpr (MODE == kInput) {
                y[j] = *reinterpret_cast<const uintx4*>(weights + (16 * j + l16) * kStep + ((q ^ ((l16 >> 2) & 3)) * 16));
            } else if constexpr (size == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int line = 4 * q + e, c = 16 * j + l16;
                    y[j][e] = *reinterpret_cast<const unsigned int*>(weights + line * kWide + (((c >> 3) ^ turn(line)) * 32) + (c & 7) * 4);
                }
            } else {
                typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
                const int l0 = 8 * q + (l16 >> 2), l1 = l0 + 4;
                const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(weights + l0 * kWide + ((j ^ turn(l0)) * 32) + (l16 & 3) * 8));
                const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(weights + l1 * kWide + ((j ^ turn(l1)) * 32) + (l16 & 3) * 8));
                y[j] = __builtin_bit_cast(uintx4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        }
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < TN / 16; ++j) acc[i][j] = multiply16<T>(y[j], x[i], acc[i][j]);
    };
    if constexpr (DIRECT) {
        for (int i = 0; i < kDepth - 1; ++i) fetch(first + i, i);
        int slot = 0;
        for (int st = first; st < last; ++st) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch(st + kDepth - 1, slot == 0 ? kDepth - 1 : slot - 1);
            wait_loads<kLoads * (kDepth - 1)>();
            work(ring[w] + slot * kStage);
            slot = slot + 1 == kDepth ? 0 : slot + 1;
        }
    } else {
        // Pieces of any alignment: through registers, kAhead steps on their way.
        uintx4 held[kAhead][kLoads];
        auto load = [&](int st, uintx4 (&v)[kLoads]) {
            const int k0 = st < last ? st * KS : K;  // (behind the last step: zeros)
#pragma unroll
            for (int i = 0; i < R; ++i)
                v[i] = load_piece<T>(px[i] + (int64_t)(k0 + kx[i]) * size, px[i] ? K - (k0 + kx[i]) : 0, false, zeros());
#pragma unroll
            for (int i = 0; i < kWLoads; ++i) {
                if constexpr (MODE == kInput) v[R + i] = load_piece<T>(pw[i] + (int64_t)(k0 + kw[i]) * size, K - (k0 + kw[i]), false, zeros());
                else v[R + i] = load_piece<T>(pw[i] + (int64_t)(k0 + kw[i]) * ldw, k0 + kw[i] < K ? left[i] : 0, false, zeros());
            }
        };
        auto put = [&](int st, const uintx4 (&v)[kLoads]) {
            const bool end = (st + 1) * KS > K, edge = n0 + TN > N;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                uintx4 x = v[i];
                if (i < R || MODE == kInput) {
                    if (end) x = shifted(x, shift_of<T>(K - (st * KS + (i < R ? kx[i < R ? i : 0] : kw[i < R ? 0 : i - R])), false));
                } else if (edge) {
                    x = shifted(x, shift_of<T>(left[i < R ? 0 : i - R], false));
                }
                *reinterpret_cast<uintx4*>(ring[w] + i * 1024 + lane * 16) = x;
            }
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(first + i, held[i]);
        for (int st = first; st < last; st += kAhead) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (st + i < last) {
                    in_order();
                    put(st + i, held[i]);
                    in_order();
                    load(st + i + kAhead, held[i]);
                    work(ring[w]);
                }
            }
        }
    }
    // The wavefronts' sums, added in order: lane l of a block has columns 4 (l / 16) .. + 3 of row l % 16.
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    floatx4* sums = reinterpret_cast<floatx4*>(&ring[0][0]);
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < TN / 16; ++j) sums[(w * kBlocks + i * (TN / 16) + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int b = w; b < kBlocks; b += kWaves) {
        floatx4 v = sums[b * 64 + lane];
#pragma unroll
        for (int x = 1; x < kWaves; ++x) v += sums[(x * kBlocks + b) * 64 + lane];
        const int64_t r = m0 + 16 * (b / (TN / 16)) + l16, to = row_of(g.out, r, r < m_end);
        const int c = n0 + 16 * (b % (TN / 16)) + 4 * q;
        if (to < 0 || c >= N) continue;
        const float x[4] = {v[0], v[1], v[2], v[3]};
        store4<T>(const_cast<char*>(g.out.data) + to * g.out.ld, c, x, N - c);
    }
}

template <class T, int MODE, int R, int TN, bool DIRECT>
int launch_of(const GroupedArgs& g, hipStream_t s) {
    constexpr int TM = 16 * R;
    const int N = MODE == kInput ? g.F_in : g.F_out;
    const int64_t blocks = ((g.m + std::min<int64_t>(g.G, g.m) * (TM - 1)) / TM * ((N + TN - 1) / TN) + 7) / 8 * 8;
    hipLaunchKernelGGL((k_grouped_few<T, MODE, R, TN, DIRECT>), dim3((unsigned)blocks), dim3(kThreads), 0, s, g);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}

// Whether these kernels serve few rows however many tiles of 128 columns there are.
constexpr bool always(bool fp32, bool input, bool direct) { return fp32 && (direct || !input); }

template <class T, int MODE, int R, bool DIRECT>
int launch_columns(const GroupedArgs& g, hipStream_t s) {
    // (where few_rows leaves 2 kUnits of the wider tiles to these kernels)
    if constexpr (always(sizeof(T) == 4, MODE == kInput, DIRECT)) {
        const int N = MODE == kInput ? g.F_in : g.F_out;
        const int64_t groups = std::min<int64_t>(g.G, g.m);
        if (groups * ((N + 63) / 64) >= 2 * kUnits) return launch_of<T, MODE, R, 64, DIRECT>(g, s);
    }
    return launch_of<T, MODE, R, 32, DIRECT>(g, s);
}

// Rows of a tile: as many as most groups have.  (Floats: never 64, which would mostly be products of rows that are not there: 128 entries in
// 8 groups, 2,048 x 4,096, 84 us with 32 rows and 140 with 64.)
template <class T, int MODE, bool DIRECT>
int launch_mode(const GroupedArgs& g, hipStream_t s) {
    if (g.m <= 8 * (int64_t)g.G) return launch_columns<T, MODE, 1, DIRECT>(g, s);
    if (sizeof(T) == 4 || g.m <= 24 * (int64_t)g.G) return launch_columns<T, MODE, 2, DIRECT>(g, s);
    if constexpr (sizeof(T) == 2) return launch_columns<T, MODE, 4, DIRECT>(g, s);
    return EPP_ERR_INVALID_ARG;  // (not reached)
}

template <class T>
int launch_type(bool input, bool direct, const GroupedArgs& g, hipStream_t s) {
    if (direct) return input ? launch_mode<T, kInput, true>(g, s) : launch_mode<T, kProduct, true>(g, s);
    return input ? launch_mode<T, kInput, false>(g, s) : launch_mode<T, kProduct, false>(g, s);
}

}  // namespace

// Fewer than 32 rows to a group on average (so that no launch has 2^32 threads), and 16 bits only where the larger tiles are not enough to fill the chip with loads.  Larger tiles
// against these, us: bfloat16, 8 groups, 2 entries, 2,048 x 4,096 (64 tiles of 128 x 128) 22.2 / 9.2; 64, 4,096 x 1,024 (64) 38.5 / 23.0;
// 256 of the same 39.1 / 31.4; but 64, 2,048 x 4,096 (256) 25.5 / 35.2 and 64 groups, 256, 2,048 x 4,096 201 / 198.  Floats: 8 groups, 16
// entries, 4,096 x 1,024 250 / 27; 64 groups, 1,024, 2,048 x 4,096 980 / 604; 2,048 of the same 1,077 / 1,105.  Rows of any alignment the same, but for
// the input gradient of floats: 8 groups, 2 entries, 1,777 x 1,333 60 / 17; 64 groups, 256, 800 x 3,329 164 / 148, its gradient 161 / 207.
bool epp_grouped::few_rows(bool fp32, bool input, bool direct, int64_t m, int G, int K, int N) {
    if (std::min(K, N) < 8) return false;  // (rows shorter than a piece)
    if (m >= (fp32 ? 24 : 32) * (int64_t)G) return false;
    return always(fp32, input, direct) || std::min<int64_t>(G, m) * ((N + 127) / 128) < kUnits;
}

int epp_grouped::launch_few(int type, bool input, bool direct, const GroupedArgs& g, hipStream_t s) {
    if (type == EPP_FLOAT32) return launch_type<float>(input, direct, g, s);
    if (type == EPP_BFLOAT16) return launch_type<__bf16>(input, direct, g, s);
    return launch_type<_Float16>(input, direct, g, s);
}
