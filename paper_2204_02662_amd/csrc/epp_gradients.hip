// The norm of many gradients together, and the gradients scaled so that it does not exceed a bound:
//     norm = sqrt(sum over all tensors and elements of x^2),   y = x min(1, max_norm / norm)
//
// Both passes are bound by memory.  The tensors' addresses and sizes travel in the kernels' arguments (a captured launch keeps
// them), so that nothing is copied to the GPU; more tensors than the arguments hold take several launches.  A tensor is cut into
// pieces of kPiece elements, and the workgroups go through the pieces of all tensors.  Squares are added in 64 bits: no square of a
// finite element overflows or vanishes, and the order of additions is fixed.  Every workgroup of the second pass adds the first
// one's sums itself, so the two passes are two launches and nothing counts or waits in between; the sums of more launches than one are added
// by one in between.

#include <cmath>

#include "epp_internal.h"

namespace {

constexpr int kThreads = 256;
constexpr int kTensors = 96;       // to a launch
constexpr int kFewTensors = 12;    // .. and to one whose arguments are short
// Workgroups, and partial sums, of a launch: eight to a compute unit.  With half as many the norm of 2^28 bf16 took 104 us (92), of 2^24 fp32 in
// four tensors 14.5 (15.6); pieces of 16,384 elements cost the norm of 2^29 fp32 367 us (352).
constexpr int kMostBlocks = 2048;
constexpr int64_t kPiece = 8192;   // elements

// (Tables of one record to an entry: with an array for each field, the compiler found the address of an 8-byte field as an entry's number
// plus seven times it, and scalar loads drop the lowest bits of both.)
struct Tensor {
    const char* in;
    char* out;
    int64_t count;
    int64_t first;  // piece
    int64_t type;
};
template <int N>
struct Tensors {
    Tensor t[N];
    int64_t pieces;
    int64_t n;
};

typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));

template <class T> __device__ __forceinline__ T to(float x) { return (T)x; }

// x times a factor of 64 bits, rounded to fp32: the factor as the sum of two floats, which takes two operations a number (conversions to
// 64 bits and back, four times as long each).  A factor so small that its second part would lose bits: as it is.
struct Factor {
    double whole;
    float high, low;
    bool small;
    __device__ __forceinline__ explicit Factor(double f) : whole(f), high((float)f), low((float)(f - (double)(float)f)), small(!(f > 0x1p-90)) {
        if (!(low == low)) low = 0.f;  // (NaN: `high` is)
    }
    __device__ __forceinline__ float operator()(float x) const {
        if (small) return (float)((double)x * whole);
        if (low == 0.f) return x * high;  // (and infinities stay what they are)
        return __builtin_fmaf(x, high, x * low);
    }
};

// The `E` elements of 16 bytes.
template <class T>
__device__ __forceinline__ void unpack(uintx4 v, T (&x)[16 / sizeof(T)]) { __builtin_memcpy(x, &v, 16); }

template <class T>
__device__ __forceinline__ double squares(const T* __restrict__ p, int count) {
    constexpr int E = 16 / (int)sizeof(T);
    double sum = 0.0;
    int head = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T);
    if (head > count) head = count;
    const int vectors = (count - head) / E, t = threadIdx.x;
    if (t < head) { const double x = (double)(float)p[t]; sum += x * x; }
    const uintx4* v = reinterpret_cast<const uintx4*>(p + head);
#pragma unroll 4
    for (int i = t; i < vectors; i += kThreads) {
        T x[E];
        unpack<T>(v[i], x);
#pragma unroll
        for (int e = 0; e < E; ++e) { const double y = (double)(float)x[e]; sum = __builtin_fma(y, y, sum); }
    }
    for (int i = head + vectors * E + t; i < count; i += kThreads) { const double x = (double)(float)p[i]; sum = __builtin_fma(x, x, sum); }
    return sum;
}

template <class T>
__device__ __forceinline__ void scaled(const T* p, T* q, int count, const Factor& scale) {
    constexpr int E = 16 / (int)sizeof(T);
    const int t = threadIdx.x;
    const bool together = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(q)) & 15) == 0;
    int head = together ? (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T) : count;
    if (head > count) head = count;
    const int vectors = (count - head) / E;
    for (int i = t; i < head; i += kThreads) q[i] = to<T>(scale((float)p[i]));
    const uintx4* v = reinterpret_cast<const uintx4*>(p + head);
    uintx4* u = reinterpret_cast<uintx4*>(q + head);
#pragma unroll 4
    for (int i = t; i < vectors; i += kThreads) {
        T x[E];
        unpack<T>(v[i], x);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = to<T>(scale((float)x[e]));
        uintx4 w;
        __builtin_memcpy(&w, x, 16);
        __builtin_nontemporal_store(w, u + i);
    }
    for (int i = head + vectors * E + t; i < count; i += kThreads) q[i] = to<T>(scale((float)p[i]));
}

// The sum of x over a workgroup, for all its threads.
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double part[kThreads / 64];
#pragma unroll
    for (int d = 32; d; d /= 2) x += __shfl_xor(x, d, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) sum += part[w];
    __syncthreads();
    return sum;
}

// The tensor that holds a piece.
template <int N>
__device__ __forceinline__ int tensor_of(const Tensors<N>& x, int64_t piece) {
    int lo = 0, hi = (int)x.n - 1;  // the last tensor whose first piece is not behind it (empty tensors have none)
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (x.t[mid].first <= piece) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <int N>
__global__ __launch_bounds__(kThreads) void k_squares(Tensors<N> x, double* __restrict__ sums) {
    double sum = 0.0;
    for (int64_t piece = blockIdx.x; piece < x.pieces; piece += gridDim.x) {
        const Tensor t = x.t[tensor_of(x, piece)];
        const int64_t begin = (piece - t.first) * kPiece;
        const int count = (int)min(kPiece, t.count - begin);
        if (t.type == EPP_FLOAT32) sum += squares(reinterpret_cast<const float*>(t.in) + begin, count);
        else if (t.type == EPP_BFLOAT16) sum += squares(reinterpret_cast<const __bf16*>(t.in) + begin, count);
        else sum += squares(reinterpret_cast<const _Float16*>(t.in) + begin, count);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ __forceinline__ double total_of(const double* sums, int n) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += kThreads) sum += sums[i];
    return block_sum(sum);
}

__device__ __forceinline__ double norm_of(const double* __restrict__ sums, int n) { return sqrt(total_of(sums, n)); }

// All sums into the first of them.  (One workgroup: what it adds in which order is what norm_of would.)
__global__ __launch_bounds__(kThreads) void k_total(double* sums, int n) {
    const double x = total_of(sums, n);
    if (threadIdx.x == 0) sums[0] = x;
}

__global__ __launch_bounds__(kThreads) void k_norm(const double* __restrict__ sums, int n, float* __restrict__ norm) {
    const double x = norm_of(sums, n);
    if (threadIdx.x == 0) *norm = (float)x;
}

template <int N>
__global__ __launch_bounds__(kThreads) void k_scale(Tensors<N> x, const double* __restrict__ sums, int n, double max_norm, float* norm) {
    const double total = norm_of(sums, n);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    const Factor scale(total <= max_norm ? 1.0 : max_norm / total);
    // (from the last piece on: what the first pass read last is still in the memory-side cache)
    for (int64_t piece = x.pieces - 1 - blockIdx.x; piece >= 0; piece -= gridDim.x) {
        const Tensor t = x.t[tensor_of(x, piece)];
        if (scale.whole == 1.0 && t.in == t.out) continue;
        const int64_t begin = (piece - t.first) * kPiece;
        const int count = (int)min(kPiece, t.count - begin);
        if (t.type == EPP_FLOAT32) scaled(reinterpret_cast<const float*>(t.in) + begin, reinterpret_cast<float*>(t.out) + begin, count, scale);
        else if (t.type == EPP_BFLOAT16) scaled(reinterpret_cast<const __bf16*>(t.in) + begin, reinterpret_cast<__bf16*>(t.out) + begin, count, scale);
        else scaled(reinterpret_cast<const _Float16*>(t.in) + begin, reinterpret_cast<_Float16*>(t.out) + begin, count, scale);
    }
}

// A few small gradients in one launch of one workgroup, which holds them in registers between the norm and the scaling.  `pieces` of up to
// kFewPiece elements, kFewRounds to a wavefront.
constexpr int kFewWaves = 16, kFewRounds = 2, kFewPiece = 1024, kFewPieces = kFewWaves * kFewRounds;
struct FewPiece {
    const char* in;
    char* out;
    int count, type;
};
struct FewPieces {
    FewPiece p[kFewPieces];
    int64_t n;
};

// Sixteen elements of a piece for each lane, as they are in memory: four loads of four, or sixteen where the piece is not a whole one (those
// behind its end get its last element).  No load under a condition of its own, and none converted here: it would be waited for where it
// stands, and the next piece's be issued behind it.
template <class T>
__device__ __forceinline__ void load_few(const char* p, int count, uintx4 (&raw)[4]) {
    typedef T vec4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    typedef unsigned int uintx2 __attribute__((ext_vector_type(2)));
    const T* q = reinterpret_cast<const T*>(p);
    const int at = (int)(threadIdx.x & 63) * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        vec4 v;
        if (count == kFewPiece) {
            v = *reinterpret_cast<const vec4*>(q + 256 * j + at);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = q[min(256 * j + at + i, count - 1)];
        }
        if constexpr (sizeof(T) == 4) {
            raw[j] = __builtin_bit_cast(uintx4, v);
        } else {
            const uintx2 two = __builtin_bit_cast(uintx2, v);
            raw[j][0] = two[0];
            raw[j][1] = two[1];
        }
    }
}
// Four of them.
template <class T>
__device__ __forceinline__ void numbers_few(const uintx4& raw, float (&x)[4]) {
    typedef T vec4 __attribute__((ext_vector_type(4)));
    typedef unsigned int uintx2 __attribute__((ext_vector_type(2)));
    vec4 v;
    if constexpr (sizeof(T) == 4) v = __builtin_bit_cast(vec4, raw);
    else v = __builtin_bit_cast(vec4, uintx2{raw[0], raw[1]});
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)v[i];
}
template <class T>
__device__ __forceinline__ double squares_few(const uintx4 (&raw)[4], int count) {
    const int at = (int)(threadIdx.x & 63) * 4;
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x[4];
        numbers_few<T>(raw[j], x);
        if (count < kFewPiece) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = 256 * j + at + i < count ? x[i] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) { const double y = (double)x[i]; sum = __builtin_fma(y, y, sum); }
    }
    return sum;
}
template <class T>
__device__ __forceinline__ void store_few(char* p, int count, const uintx4 (&raw)[4], const Factor& scale) {
    typedef T vec4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    T* q = reinterpret_cast<T*>(p);
    const int at = (int)(threadIdx.x & 63) * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x[4];
        numbers_few<T>(raw[j], x);
        vec4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to<T>(scale(x[i]));
        if (256 * j + at + 4 <= count) {
            *reinterpret_cast<vec4*>(q + 256 * j + at) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (256 * j + at + i < count) q[256 * j + at + i] = v[i];
        }
    }
}

template <bool CLIP>
__global__ __launch_bounds__(64 * kFewWaves) void k_few(FewPieces p, double max_norm, float* norm) {
    __shared__ double part[kFewWaves];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    FewPiece one[kFewRounds];
    uintx4 raw[kFewRounds][4];
#pragma unroll
    for (int r = 0; r < kFewRounds; ++r) {
        one[r] = p.p[w + kFewWaves * r];
        if (w + kFewWaves * r >= p.n) one[r].count = 0;
    }
#pragma unroll
    for (int r = 0; r < kFewRounds; ++r) {
        if (one[r].count == 0) continue;
        if (one[r].type == EPP_FLOAT32) load_few<float>(one[r].in, one[r].count, raw[r]);
        else load_few<__bf16>(one[r].in, one[r].count, raw[r]);  // (or _Float16: as they are in memory)
    }
    double sum = 0.0;
#pragma unroll
    for (int r = 0; r < kFewRounds; ++r) {
        if (one[r].count == 0) continue;
        if (one[r].type == EPP_FLOAT32) sum += squares_few<float>(raw[r], one[r].count);
        else if (one[r].type == EPP_BFLOAT16) sum += squares_few<__bf16>(raw[r], one[r].count);
        else sum += squares_few<_Float16>(raw[r], one[r].count);
    }
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) == 0) part[w] = sum;
    __syncthreads();
    double total = 0.0;
#pragma unroll
    for (int i = 0; i < kFewWaves; ++i) total += part[i];
    total = sqrt(total);
    if (threadIdx.x == 0) *norm = (float)total;
    if constexpr (CLIP) {
        const Factor scale(total <= max_norm ? 1.0 : max_norm / total);
#pragma unroll
        for (int r = 0; r < kFewRounds; ++r) {
            if (one[r].count == 0 || (scale.whole == 1.0 && one[r].in == one[r].out)) continue;
            if (one[r].type == EPP_FLOAT32) store_few<float>(one[r].out, one[r].count, raw[r], scale);
            else if (one[r].type == EPP_BFLOAT16) store_few<__bf16>(one[r].out, one[r].count, raw[r], scale);
            else store_few<_Float16>(one[r].out, one[r].count, raw[r], scale);
        }
    }
}

int size_of(int type) { return type == EPP_FLOAT32 ? 4 : 2; }
// The pieces of all gradients, if there are few enough of them.
bool few_pieces(const epp_gradient_t* grads, int n, FewPieces* p) {
    p->n = 0;
    for (int k = 0; k < n; ++k) {
        const epp_gradient_t& g = grads[k];
        if (g.count > (int64_t)kFewPiece * (kFewPieces - p->n)) return false;
        const int size = size_of(g.type);
        for (int64_t at = 0; at < g.count; at += kFewPiece, ++p->n) {
            if (p->n == kFewPieces) return false;
            p->p[p->n] = {static_cast<const char*>(g.data) + at * size, static_cast<char*>(g.out ? g.out : g.data) + at * size,
                          (int)std::min<int64_t>(kFewPiece, g.count - at), g.type};
        }
    }
    return true;
}

int launches(int n) { return std::max(1, (n + kTensors - 1) / kTensors); }

// The table of tensors [first, ..) of a launch.
template <int N>
void fill(Tensors<N>* x, const epp_gradient_t* grads, int n, int first) {
    x->n = std::min(N, n - first);
    x->pieces = 0;
    for (int k = 0; k < x->n; ++k) {
        const epp_gradient_t& g = grads[first + k];
        x->t[k] = {static_cast<const char*>(g.data), static_cast<char*>(g.out ? g.out : g.data), g.count, x->pieces, g.type};
        x->pieces += (g.count + kPiece - 1) / kPiece;
    }
}
template <int N>
unsigned blocks_of(const Tensors<N>& x) { return (unsigned)std::min<int64_t>(std::max<int64_t>(x.pieces, 1), kMostBlocks); }

struct Block { uintptr_t begin, end; int tensor; bool written; };

int check(const epp_gradient_t* grads, int n, const float* norm, void* workspace, int64_t workspace_bytes, bool writes) {
    if (n < 0 || n > (1 << 20)) { epp_set_error("%d gradients (0 to %d)", n, 1 << 20); return n < 0 ? EPP_ERR_INVALID_ARG : EPP_ERR_TOO_LARGE; }
    if ((n > 0 && !grads) || !norm || !workspace) { epp_set_error("NULL argument"); return EPP_ERR_INVALID_ARG; }
    if (reinterpret_cast<uintptr_t>(norm) & 3) { epp_set_error("address not aligned to its elements"); return EPP_ERR_INVALID_ARG; }
    const int64_t need = epp_gradient_norm_workspace(n);
    if (workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15)) {
        epp_set_error("workspace of %lld bytes (need %lld, 16-byte aligned)", (long long)workspace_bytes, (long long)need);
        return EPP_ERR_INVALID_ARG;
    }
    for (int k = 0; k < n; ++k) {
        const epp_gradient_t& g = grads[k];
        if (g.type != EPP_FLOAT32 && g.type != EPP_BFLOAT16 && g.type != EPP_FLOAT16) { epp_set_error("gradient %d: unknown element type %d", k, g.type); return EPP_ERR_INVALID_ARG; }
        if (g.count < 0 || g.count >= (1ll << 40)) { epp_set_error("gradient %d: %lld elements", k, (long long)g.count); return g.count < 0 ? EPP_ERR_INVALID_ARG : EPP_ERR_TOO_LARGE; }
        if (g.count > 0 && !g.data) { epp_set_error("gradient %d: NULL argument", k); return EPP_ERR_INVALID_ARG; }
        if ((reinterpret_cast<uintptr_t>(g.data) | reinterpret_cast<uintptr_t>(g.out)) & (unsigned)(size_of(g.type) - 1)) {
            epp_set_error("gradient %d: address not aligned to its elements", k);
            return EPP_ERR_INVALID_ARG;
        }
    }
    // What is written must be nobody else's: an element scaled twice, or read after it was scaled, has no defined value.
    std::vector<Block> b;
    try {
        b.reserve(2 * (size_t)n + 2);
        const uintptr_t ws = reinterpret_cast<uintptr_t>(workspace), nm = reinterpret_cast<uintptr_t>(norm);
        b.push_back({ws, ws + (uintptr_t)need, -1, true});
        b.push_back({nm, nm + 4, -2, true});
        for (int k = 0; k < n; ++k) {
            const epp_gradient_t& g = grads[k];
            if (g.count == 0) continue;
            const uintptr_t bytes = (uintptr_t)g.count * (uintptr_t)size_of(g.type), x = reinterpret_cast<uintptr_t>(g.data), y = reinterpret_cast<uintptr_t>(g.out ? g.out : g.data);
            b.push_back({x, x + bytes, k, writes && x == y});
            if (writes && x != y) b.push_back({y, y + bytes, k, true});
        }
        std::sort(b.begin(), b.end(), [](const Block& p, const Block& q) { return p.begin < q.begin; });
    } catch (...) {
        epp_set_error("no host memory for %d gradients", n);
        return EPP_ERR_ALLOC;
    }
    uintptr_t end = 0, end_written = 0;  // of all blocks so far, of the written ones
    for (const Block& x : b) {
        if (x.begin < end_written || (x.written && x.begin < end)) { epp_set_error("gradients, outputs, norm and workspace must not alias"); return EPP_ERR_INVALID_ARG; }
        end = std::max(end, x.end);
        if (x.written) end_written = std::max(end_written, x.end);
    }
    return EPP_OK;
}

// Sums of squares of all tensors into the workspace; how many.
template <int N>
int sum_squares(const epp_gradient_t* grads, int n, double* sums, int* count, hipStream_t s) {
    Tensors<N> x;
    *count = 0;
    for (int first = 0; first < n; first += N) {
        fill(&x, grads, n, first);
        if (!x.pieces) continue;
        const unsigned blocks = blocks_of(x);
        hipLaunchKernelGGL((k_squares<N>), dim3(blocks), dim3(kThreads), 0, s, x, sums + *count);
        EPP_HIP_TRY(hipGetLastError());
        *count += (int)blocks;
    }
    return EPP_OK;
}

template <int N>
int clip(const epp_gradient_t* grads, int n, double max_norm, float* norm, double* sums, hipStream_t s) {
    int count;
    EPP_TRY(sum_squares<N>(grads, n, sums, &count, s));
    // One launch's sums every workgroup of the scaling adds itself.  Those of more launches are added once: they, the workgroups and the
    // launches that would add them again all grow with the tensors.  bf16, added by every workgroup / once: 200 tensors of 172,027 86 / 79 us, 1,000
    // of 200,000 0.58 / 0.37 ms, 12,288 of 172,027 36.3 / 4.3 ms.
    if (count > kMostBlocks) {
        hipLaunchKernelGGL(k_total, dim3(1), dim3(kThreads), 0, s, sums, count);
        EPP_HIP_TRY(hipGetLastError());
        count = 1;
    }
    Tensors<N> x;
    bool told = false;
    for (int first = 0; first < n; first += N) {
        fill(&x, grads, n, first);
        if (!x.pieces) continue;
        hipLaunchKernelGGL((k_scale<N>), dim3(blocks_of(x)), dim3(kThreads), 0, s, x, sums, count, max_norm, told ? nullptr : norm);
        EPP_HIP_TRY(hipGetLastError());
        told = true;
    }
    return EPP_OK;
}

}  // namespace

extern "C" int64_t epp_gradient_norm_workspace(int n) {
    if (n < 0 || n > (1 << 20)) { epp_set_error("%d gradients (0 to %d)", n, 1 << 20); return n < 0 ? EPP_ERR_INVALID_ARG : EPP_ERR_TOO_LARGE; }
    return (int64_t)launches(n) * kMostBlocks * (int64_t)sizeof(double);
}

extern "C" int epp_gradient_norm(const epp_gradient_t* grads, int n, float* norm, void* workspace, int64_t workspace_bytes, epp_stream_t stream) {
    EPP_TRY(check(grads, n, norm, workspace, workspace_bytes, false));
    hipStream_t s = (hipStream_t)stream;
    FewPieces few = {};
    if (few_pieces(grads, n, &few)) {
        hipLaunchKernelGGL((k_few<false>), dim3(1), dim3(64 * kFewWaves), 0, s, few, 0.0, norm);
        EPP_HIP_TRY(hipGetLastError());
        return EPP_OK;
    }
    double* sums = static_cast<double*>(workspace);
    int count;
    EPP_TRY(n <= kFewTensors ? sum_squares<kFewTensors>(grads, n, sums, &count, s) : sum_squares<kTensors>(grads, n, sums, &count, s));
    hipLaunchKernelGGL(k_norm, dim3(1), dim3(kThreads), 0, s, sums, count, norm);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}

extern "C" int epp_clip_gradients(const epp_gradient_t* grads, int n, double max_norm, float* norm, void* workspace, int64_t workspace_bytes,
                                  epp_stream_t stream) {
    if (!(max_norm >= 0.0)) { epp_set_error("max_norm must be >= 0 (got %g)", max_norm); return EPP_ERR_INVALID_ARG; }
    EPP_TRY(check(grads, n, norm, workspace, workspace_bytes, true));
    hipStream_t s = (hipStream_t)stream;
    FewPieces few = {};
    if (few_pieces(grads, n, &few)) {
        hipLaunchKernelGGL((k_few<true>), dim3(1), dim3(64 * kFewWaves), 0, s, few, max_norm, norm);
        EPP_HIP_TRY(hipGetLastError());
        return EPP_OK;
    }
    double* sums = static_cast<double*>(workspace);
    return n <= kFewTensors ? clip<kFewTensors>(grads, n, max_norm, norm, sums, s) : clip<kTensors>(grads, n, max_norm, norm, sums, s);
}
