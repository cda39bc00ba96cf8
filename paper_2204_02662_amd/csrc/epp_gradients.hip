// The norm of many gradients together, and the gradients scaled so that it does not exceed a bound:
//     norm = sqrt(sum over all tensors and elements of x^2),   y = x min(1, max_norm / norm)
//
// Both passes are bound by memory.  The tensors' addresses and sizes travel in the kernels' arguments (a captured launch keeps
// them), so that nothing is copied to the GPU; more tensors than the arguments hold take several launches.  A tensor is cut into
// pieces of kPiece elements, and the workgroups go through the pieces of all tensors.  Squares are added in 64 bits: no square of a
// finite element overflows or vanishes, and the order of additions is fixed.  Every workgroup of the second pass adds the first
// one's sums itself, so the two passes are two launches and nothing counts or waits in between.

#include <cmath>

#include "epp_internal.h"

namespace {

constexpr int kThreads = 256;
constexpr int kTensors = 96;       // to a launch
constexpr int kMostBlocks = 1024;  // workgroups, and partial sums, of a launch
constexpr int64_t kPiece = 8192;   // elements

struct Tensors {
    const char* in[kTensors];
    char* out[kTensors];
    int64_t count[kTensors];
    int64_t first[kTensors];   // piece
    unsigned char type[kTensors];
    int n;
    int64_t pieces;
};

typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));

template <class T> __device__ __forceinline__ T to(float x) { return (T)x; }

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
__device__ __forceinline__ void scaled(const T* p, T* q, int count, double scale) {
    constexpr int E = 16 / (int)sizeof(T);
    const int t = threadIdx.x;
    const bool together = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(q)) & 15) == 0;
    int head = together ? (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T) : count;
    if (head > count) head = count;
    const int vectors = (count - head) / E;
    for (int i = t; i < head; i += kThreads) q[i] = to<T>((float)((double)(float)p[i] * scale));
    const uintx4* v = reinterpret_cast<const uintx4*>(p + head);
    uintx4* u = reinterpret_cast<uintx4*>(q + head);
#pragma unroll 4
    for (int i = t; i < vectors; i += kThreads) {
        T x[E];
        unpack<T>(v[i], x);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = to<T>((float)((double)(float)x[e] * scale));
        uintx4 w;
        __builtin_memcpy(&w, x, 16);
        u[i] = w;
    }
    for (int i = head + vectors * E + t; i < count; i += kThreads) q[i] = to<T>((float)((double)(float)p[i] * scale));
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
__device__ __forceinline__ int tensor_of(const Tensors& x, int64_t piece) {
    int lo = 0, hi = x.n - 1;  // the last tensor whose first piece is not behind it (empty tensors have none)
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (x.first[mid] <= piece) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__global__ __launch_bounds__(kThreads) void k_squares(Tensors x, double* __restrict__ sums) {
    double sum = 0.0;
    for (int64_t piece = blockIdx.x; piece < x.pieces; piece += gridDim.x) {
        const int k = tensor_of(x, piece);
        const int64_t begin = (piece - x.first[k]) * kPiece;
        const int count = (int)min(kPiece, x.count[k] - begin);
        if (x.type[k] == EPP_FLOAT32) sum += squares(reinterpret_cast<const float*>(x.in[k]) + begin, count);
        else if (x.type[k] == EPP_BFLOAT16) sum += squares(reinterpret_cast<const __bf16*>(x.in[k]) + begin, count);
        else sum += squares(reinterpret_cast<const _Float16*>(x.in[k]) + begin, count);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ __forceinline__ double norm_of(const double* __restrict__ sums, int n) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += kThreads) sum += sums[i];
    return sqrt(block_sum(sum));
}

__global__ __launch_bounds__(kThreads) void k_norm(const double* __restrict__ sums, int n, float* __restrict__ norm) {
    const double x = norm_of(sums, n);
    if (threadIdx.x == 0) *norm = (float)x;
}

__global__ __launch_bounds__(kThreads) void k_scale(Tensors x, const double* __restrict__ sums, int n, double max_norm, float* norm) {
    const double total = norm_of(sums, n);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    const double scale = total <= max_norm ? 1.0 : max_norm / total;
    for (int64_t piece = blockIdx.x; piece < x.pieces; piece += gridDim.x) {
        const int k = tensor_of(x, piece);
        if (scale == 1.0 && x.in[k] == x.out[k]) continue;
        const int64_t begin = (piece - x.first[k]) * kPiece;
        const int count = (int)min(kPiece, x.count[k] - begin);
        if (x.type[k] == EPP_FLOAT32) scaled(reinterpret_cast<const float*>(x.in[k]) + begin, reinterpret_cast<float*>(x.out[k]) + begin, count, scale);
        else if (x.type[k] == EPP_BFLOAT16) scaled(reinterpret_cast<const __bf16*>(x.in[k]) + begin, reinterpret_cast<__bf16*>(x.out[k]) + begin, count, scale);
        else scaled(reinterpret_cast<const _Float16*>(x.in[k]) + begin, reinterpret_cast<_Float16*>(x.out[k]) + begin, count, scale);
    }
}

int size_of(int type) { return type == EPP_FLOAT32 ? 4 : 2; }
int launches(int n) { return std::max(1, (n + kTensors - 1) / kTensors); }

// The table of tensors [first, ..) of a launch.
void fill(Tensors* x, const epp_gradient_t* grads, int n, int first) {
    x->n = std::min(kTensors, n - first);
    x->pieces = 0;
    for (int k = 0; k < x->n; ++k) {
        const epp_gradient_t& g = grads[first + k];
        x->in[k] = static_cast<const char*>(g.data);
        x->out[k] = static_cast<char*>(g.out ? g.out : g.data);
        x->count[k] = g.count;
        x->first[k] = x->pieces;
        x->type[k] = (unsigned char)g.type;
        x->pieces += (g.count + kPiece - 1) / kPiece;
    }
}
unsigned blocks_of(const Tensors& x) { return (unsigned)std::min<int64_t>(std::max<int64_t>(x.pieces, 1), kMostBlocks); }

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
int sum_squares(const epp_gradient_t* grads, int n, double* sums, int* count, hipStream_t s) {
    Tensors x;
    *count = 0;
    for (int first = 0; first < n; first += kTensors) {
        fill(&x, grads, n, first);
        if (!x.pieces) continue;
        const unsigned blocks = blocks_of(x);
        hipLaunchKernelGGL(k_squares, dim3(blocks), dim3(kThreads), 0, s, x, sums + *count);
        EPP_HIP_TRY(hipGetLastError());
        *count += (int)blocks;
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
    double* sums = static_cast<double*>(workspace);
    int count;
    EPP_TRY(sum_squares(grads, n, sums, &count, s));
    hipLaunchKernelGGL(k_norm, dim3(1), dim3(kThreads), 0, s, sums, count, norm);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}

extern "C" int epp_clip_gradients(const epp_gradient_t* grads, int n, double max_norm, float* norm, void* workspace, int64_t workspace_bytes,
                                  epp_stream_t stream) {
    if (!(max_norm >= 0.0)) { epp_set_error("max_norm must be >= 0 (got %g)", max_norm); return EPP_ERR_INVALID_ARG; }
    EPP_TRY(check(grads, n, norm, workspace, workspace_bytes, true));
    hipStream_t s = (hipStream_t)stream;
    double* sums = static_cast<double*>(workspace);
    int count;
    EPP_TRY(sum_squares(grads, n, sums, &count, s));
    Tensors x;
    bool told = false;
    for (int first = 0; first < n; first += kTensors) {
        fill(&x, grads, n, first);
        if (!x.pieces) continue;
        hipLaunchKernelGGL(k_scale, dim3(blocks_of(x)), dim3(kThreads), 0, s, x, sums, count, max_norm, told ? nullptr : norm);
        EPP_HIP_TRY(hipGetLastError());
        told = true;
    }
    if (!told) {  // (no gradients, or only empty ones)
        hipLaunchKernelGGL(k_norm, dim3(1), dim3(kThreads), 0, s, sums, count, norm);
        EPP_HIP_TRY(hipGetLastError());
    }
    return EPP_OK;
}
