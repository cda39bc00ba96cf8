// Products of rows that belong to groups, each group with a weight matrix of its own (the experts of a mixture, the
// types of a graph's vertices).  With entries i of group g at [offsets[g], offsets[g + 1]):
//     out[o(i), :]    = X[a(i), :] W[g]                 (product)
//     grad_X[o(i), :] = grad_out[a(i), :] W[g]^T        (input gradient)
//     grad_W[g]       = sum over i of X[a(i), :]^T grad_out[b(i), :]
// a, b and o are row lists or the entries themselves.  Sizes of groups are known to the GPU only: a launch has as many
// workgroups as m entries in G groups can need, and every one finds its tile by a scan of the offsets.
//
// A workgroup forms a TM x TN tile of the result from operand tiles of 128 bytes of the contraction (64 elements of 16
// bits, 32 floats) in LDS, two of them: while the matrix cores work on one, the other fills.  An operand comes in one of
// two ways:
//   lines of K      the contraction is contiguous in memory (rows of X; W in the input gradient): a line of the tile is 128
//                   bytes of one row
//   lines of width  the contraction strides (W in the product; both operands of the weight gradient): a line is one step of
//                   the contraction, as wide as the tile
// Both are moved in pieces of 16 bytes, a lane each.  A piece's place in its line is permuted by the line's number, so that
// lanes that read the same piece of neighbouring lines use different banks.  Where widths, strides and addresses are
// multiples of 16 bytes, pieces go from global memory to LDS directly (what lies outside is fetched from a block of zeros);
// elsewhere through registers.
//
// Matrix instructions of 32 x 32: lane l supplies row (column) l % 32 and the contraction's piece 2 s + l / 32 of step s:
// eight elements of 16 bits in one instruction, four floats in four.  Which elements those are does not matter as long as
// both operands agree.  Lines of width are read column by column: 16 bits by the transposing LDS load (16 lanes load four
// lines of 16 elements, and lane i gets the four of column i), floats one by one.  The first operand of the instruction is
// the result's column, so that a lane holds four neighbouring columns of one row.
// Sums are fp32; 16-bit results are rounded once, when they are written.

#include "epp_internal.h"

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned int uintx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfloatx8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));

constexpr int kMaxGroups = 2048;
constexpr int kMaxWidth = 1 << 16;
constexpr int kLine = 128;  // bytes of the contraction in a tile

enum Mode { kProduct, kInput, kWeight };

__device__ __attribute__((aligned(128))) unsigned int g_zeros[32] = {};

struct Side {           // a matrix and the rows of it that entries name
    const char* data;
    int64_t n, ld;      // rows, bytes from row to row
    const int32_t* rows;
};
struct GroupedArgs {
    Side a, b;          // product, input gradient: a, weight gradient: both
    Side out;
    const char* W;
    const int32_t* offsets;
    int64_t m;
    int G, F_in, F_out;
    int vec_out;        // results are written four at a time
    int64_t per;        // weight gradient: entries to a chunk (0: whole groups)
    float* part;        // .. and its partial sums
};

// ---------------------------------------------------------------- numbers
template <class T> struct Num;
template <> struct Num<float> {
    static __device__ __forceinline__ float from(float x) { return x; }
};
template <> struct Num<__bf16> {
    static __device__ __forceinline__ __bf16 from(float x) { return (__bf16)x; }
};
template <> struct Num<_Float16> {
    static __device__ __forceinline__ _Float16 from(float x) { return (_Float16)x; }
};

// One piece (16 bytes) of the contraction of both operands.
template <class T>
__device__ __forceinline__ floatx16 multiply(uintx4 a, uintx4 b, floatx16 c) {
    if constexpr (sizeof(T) == 4) {
        const floatx4 x = __builtin_bit_cast(floatx4, a), y = __builtin_bit_cast(floatx4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], y[j], c, 0, 0, 0);
        return c;
    } else if constexpr (std::is_same_v<T, __bf16>) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bfloatx8, a), __builtin_bit_cast(bfloatx8, b), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
    }
}

// ---------------------------------------------------------------- groups
struct Span { int g; int64_t first, last, chunk0; };  // a group (-1: none), its entries, its first tile

// The group that holds the `tile`-th of the tiles of `per` entries, and how many tiles there are.  Offsets are kept inside
// [0, m]; a group that would end before it begins is empty.
__device__ __forceinline__ Span find_group(const int32_t* __restrict__ offsets, int G, int64_t m, int64_t per, int64_t tile, int64_t* total) {
    const int lane = threadIdx.x & 63;
    Span found = {-1, 0, 0, 0};
    int64_t before = 0;
    for (int g0 = 0; g0 < G; g0 += 64) {
        const int g = g0 + lane;
        int64_t lo = 0, hi = 0;
        if (g < G) {
            lo = min(max((int64_t)offsets[g], (int64_t)0), m);
            hi = min(max((int64_t)offsets[g + 1], (int64_t)0), m);
        }
        const int tiles = hi > lo ? (int)((hi - lo + per - 1) / per) : 0;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(upto, d, 64);
            if (lane >= d) upto += x;
        }
        const unsigned long long past = __ballot(before + upto > tile);
        if (found.g < 0 && past) {
            const int l = __ffsll((long long)past) - 1;
            found = {g0 + l, __shfl(lo, l, 64), __shfl(hi, l, 64), before + __shfl(upto - tiles, l, 64)};
        }
        before += __shfl(upto, 63, 64);
    }
    *total = before;
    found.g = __builtin_amdgcn_readfirstlane(found.g);
    return found;
}

// ---------------------------------------------------------------- operand tiles
__device__ __forceinline__ unsigned lds_address(const void* p) {
    return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
// 16 bytes a lane into LDS, lane after lane from `to` on.  Complete once vmcnt says so (wait_and_meet).  (Not the compiler's builtin: it waits
// for all of these loads before every transposing LDS read, those of the next tile included.  The compiler writes m0 right before its own uses.)
__device__ __forceinline__ void load_to_lds(const char* from, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}
// All loads of this wavefront have arrived and all its LDS reads are done; then the same for the workgroup's.
__device__ __forceinline__ void wait_and_meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ int64_t row_of(const Side& s, int64_t i, bool valid) {  // -1: no such row
    if (!valid) return -1;
    const int64_t r = s.rows ? (int64_t)s.rows[i] : i;
    return r >= 0 && r < s.n ? r : -1;
}

// A piece with `valid` elements (0 .. a piece's), through registers.
template <class T>
__device__ __forceinline__ uintx4 load_piece(const char* p, int64_t valid) {
    constexpr int E = 16 / (int)sizeof(T);
    typedef unsigned int any_uintx4 __attribute__((ext_vector_type(4), aligned(2)));
    uintx4 v = {0, 0, 0, 0};
    if (valid >= E) return *reinterpret_cast<const any_uintx4*>(p);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < valid) v[e] = reinterpret_cast<const unsigned int*>(p)[e];
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < valid) v[e / 2] |= (unsigned int)reinterpret_cast<const unsigned short*>(p)[e] << (16 * (e % 2));
    }
    return v;
}

// Lines of K: TD rows, row r's place set once.
template <class T, int TD, int NT, bool DIRECT>
struct LinesOfK {
    static constexpr int E = 16 / (int)sizeof(T), N = TD * 8 / NT, kBytes = TD * kLine;
    const char* p[N];
    uint64_t bad = 0;  // bit i: piece i has no row
    int k;             // element of the contraction where this thread's pieces begin
    int K;
    uintx4 held[DIRECT ? 1 : N];
    // row(i): place of tile row i, null: none
    template <class F> __device__ __forceinline__ void start(int K_, F row) {
        const int t = threadIdx.x;
        K = K_;
        k = ((t & 7) ^ ((t >> 3) & 7)) * E;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            p[i] = row((i * NT + t) >> 3);
            if (!p[i]) bad |= 1ull << i;
            p[i] += (int64_t)k * (int64_t)sizeof(T);
        }
    }
    __device__ __forceinline__ void fetch(char* to) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool no = (bad >> i) & 1;
            if constexpr (DIRECT) {
                load_to_lds(no || k >= K ? reinterpret_cast<const char*>(g_zeros) : p[i],
                            __builtin_amdgcn_readfirstlane(lds_address(to + (i * NT + (threadIdx.x & ~63)) * 16)));
            } else {
                held[i] = load_piece<T>(p[i], no ? 0 : K - k);
            }
            p[i] += kLine;
        }
        k += kLine / (int)sizeof(T);
    }
    __device__ __forceinline__ void put(char* to) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < N; ++i) *reinterpret_cast<uintx4*>(to + (i * NT + threadIdx.x) * 16) = held[i];
        }
    }
    // Piece 2 s + half of rows c0 + l % 32 (c0 a multiple of 32).
    static __device__ __forceinline__ uintx4 piece(const char* tile, int c0, int s) {
        const int l = threadIdx.x & 63;
        return *reinterpret_cast<const uintx4*>(tile + (c0 + (l & 31)) * kLine + (((2 * s + (l >> 5)) ^ (l & 7)) * 16));
    }
};

// Lines of width: the steps of the contraction are the entries [first, last) of `s`, the columns begin at c0.
template <class T, int TD, int NT, bool DIRECT>
struct LinesOfWidth {
    static constexpr int E = 16 / (int)sizeof(T), N = TD * 8 / NT, kBytes = TD * kLine;
    static constexpr int kWide = TD * (int)sizeof(T), kPieces = kWide / 16, kUnits = kWide / 32, kMask = (kUnits < 8 ? kUnits : 8) - 1;
    static constexpr int kSteps = kLine / (int)sizeof(T);
    static_assert(NT % kPieces == 0 && (kMask & (kMask + 1)) == 0, "tile");
    Side s;
    int64_t at, last;   // entry of this thread's first piece in the next tile
    int32_t row[N];     // rows of the next tile's pieces where there is a list of them
    int col, width;
    uintx4 held[DIRECT ? 1 : N];
    __device__ __forceinline__ int column(int i) const {  // of this thread's piece i, in elements
        const int t = threadIdx.x, line = (i * NT + t) / kPieces;
        return col + (((t % kPieces) ^ ((line & kMask) << 1)) * E);
    }
    __device__ __forceinline__ void start(const Side& side, int64_t first, int64_t end, int c0, int w) {
        s = side;
        at = first + threadIdx.x / kPieces;
        last = end;
        col = c0;
        width = w;
        next_rows();
    }
    __device__ __forceinline__ void next_rows() {
        if (!s.rows) return;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t e = at + i * (NT / kPieces);
            row[i] = e < last ? s.rows[e] : -1;
        }
    }
    __device__ __forceinline__ void fetch(char* to) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t e = at + i * (NT / kPieces);
            const int64_t r = s.rows ? (int64_t)row[i] : e;
            const int c = column(i);
            const bool no = e >= last || r < 0 || r >= s.n || c >= width;
            const char* p = s.data + r * s.ld + (int64_t)c * (int64_t)sizeof(T);
            if constexpr (DIRECT) {
                load_to_lds(no ? reinterpret_cast<const char*>(g_zeros) : p,
                            __builtin_amdgcn_readfirstlane(lds_address(to + (i * NT + (threadIdx.x & ~63)) * 16)));
            } else {
                held[i] = load_piece<T>(p, no ? 0 : width - c);
            }
        }
        at += kSteps;
        next_rows();
    }
    __device__ __forceinline__ void put(char* to) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < N; ++i) *reinterpret_cast<uintx4*>(to + (i * NT + threadIdx.x) * 16) = held[i];
        }
    }
    // Piece 2 s + half of the contraction for columns c + l % 32.
    static __device__ __forceinline__ uintx4 piece(const char* tile, int c, int st) {
        const int l = threadIdx.x & 63, q = 2 * st + (l >> 5);
        if constexpr (sizeof(T) == 4) {
            uintx4 v;
            const int x = c + (l & 31);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int line = 4 * q + j;
                v[j] = *reinterpret_cast<const unsigned int*>(tile + line * kWide + (((x >> 3) ^ (line & kMask)) * 32) + (x & 7) * 4);
            }
            return v;
        } else {
            typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
            const int i = l & 15, unit = (c >> 4) + ((l >> 4) & 1);
            const int l0 = 8 * q + (i >> 2), l1 = l0 + 4;
            const char* p0 = tile + l0 * kWide + ((unit ^ (l0 & kMask)) * 32) + (i & 3) * 8;
            const char* p1 = tile + l1 * kWide + ((unit ^ (l1 & kMask)) * 32) + (i & 3) * 8;
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(p0));
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(p1));
            return __builtin_bit_cast(uintx4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// Four neighbouring results of a row; `valid` of them exist.
template <class T>
__device__ __forceinline__ void store4(char* row, int col, const float (&x)[4], int valid, bool vec) {
    T* p = reinterpret_cast<T*>(row) + col;
    if (vec && valid >= 4) {
        typedef T vec4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<vec4*>(p) = vec4{Num<T>::from(x[0]), Num<T>::from(x[1]), Num<T>::from(x[2]), Num<T>::from(x[3])};
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c < valid) p[c] = Num<T>::from(x[c]);
    }
}

// WM x WN wavefronts, each with BM x BN blocks of 32 x 32 of the result.  TO: type of the results.
template <class T, class TO, int MODE, int WM, int WN, int BM, int BN, bool DIRECT>
__global__ __launch_bounds__(64 * WM * WN) void k_grouped(GroupedArgs g) {
    constexpr int NT = 64 * WM * WN, TM = 32 * WM * BM, TN = 32 * WN * BN;
    using A = std::conditional_t<MODE == kWeight, LinesOfWidth<T, TM, NT, DIRECT>, LinesOfK<T, TM, NT, DIRECT>>;
    using B = std::conditional_t<MODE == kInput, LinesOfK<T, TN, NT, DIRECT>, LinesOfWidth<T, TN, NT, DIRECT>>;
    __shared__ __attribute__((aligned(128))) char tiles[2][A::kBytes + B::kBytes];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w % WM, wn = w / WM;
    A a;
    B b;
    int64_t K;                        // steps of the contraction
    int64_t m0 = 0, m_end = 0;        // rows of the result: entries (product, input gradient) or rows of grad_W
    int n0;
    const int N = MODE == kInput ? g.F_in : g.F_out;
    const int nt = (N + TN - 1) / TN;
    char* out_base = const_cast<char*>(g.out.data);
    if constexpr (MODE != kWeight) {
        // Workgroups b, b + 8, .. run on one XCD: it gets neighbouring tiles, which share rows and weights in its L2.
        int64_t total;
        Span s = find_group(g.offsets, g.G, g.m, TM, -1, &total);
        const int64_t per = (total * nt + 7) / 8, mine = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
        if ((int64_t)(blockIdx.x >> 3) >= per || mine >= total * nt) return;
        s = find_group(g.offsets, g.G, g.m, TM, mine / nt, &total);
        m0 = s.first + (mine / nt - s.chunk0) * TM;
        m_end = s.last;
        n0 = (int)(mine % nt) * TN;
        const int64_t w_bytes = (int64_t)g.F_in * g.F_out * (int64_t)sizeof(T);
        const char* W = g.W + s.g * w_bytes;
        const int64_t ldw = (int64_t)g.F_out * (int64_t)sizeof(T);
        K = MODE == kInput ? g.F_out : g.F_in;
        a.start((int)K, [&](int i) -> const char* {
            const int64_t r = row_of(g.a, m0 + i, m0 + i < m_end);
            return r < 0 ? nullptr : g.a.data + r * g.a.ld;
        });
        if constexpr (MODE == kInput) {
            b.start((int)K, [&](int i) -> const char* { return n0 + i < N ? W + (int64_t)(n0 + i) * ldw : nullptr; });
        } else {
            b.start(Side{W, K, ldw, nullptr}, 0, K, n0, N);
        }
    } else {
        const int mt = (g.F_in + TM - 1) / TM;
        // (the tiles of one group or chunk are dealt to all XCDs: groups differ in size)
        const int per_group = mt * nt, in = (int)(blockIdx.x % per_group), share = (per_group + 7) / 8;
        const int64_t chunk = blockIdx.x / per_group;
        int tile = in;
        if (per_group % 8 == 0) tile = (in & 7) * share + (in >> 3);
        int64_t first, last;
        if (g.per) {
            int64_t total;
            const Span s = find_group(g.offsets, g.G, g.m, g.per, chunk, &total);
            if (s.g < 0) return;
            first = s.first + (chunk - s.chunk0) * g.per;
            last = min(first + g.per, s.last);
            out_base = reinterpret_cast<char*>(g.part + chunk * g.F_in * g.F_out);
        } else {
            first = min(max((int64_t)g.offsets[chunk], (int64_t)0), g.m);
            last = max(first, min((int64_t)g.offsets[chunk + 1], g.m));
            out_base += chunk * g.F_in * g.F_out * (int64_t)sizeof(TO);
        }
        K = last - first;
        m0 = (int64_t)(tile / nt) * TM;
        m_end = g.F_in;
        n0 = (tile % nt) * TN;
        a.start(g.a, first, last, (int)m0, g.F_in);
        b.start(g.b, first, last, n0, g.F_out);
    }

    floatx16 acc[BM][BN] = {};
    constexpr int kSteps = kLine / (int)sizeof(T);
    const int64_t steps = (K + kSteps - 1) / kSteps;
    if (steps > 0) {
        a.fetch(tiles[0]);
        b.fetch(tiles[0] + A::kBytes);
        a.put(tiles[0]);
        b.put(tiles[0] + A::kBytes);
    }
    for (int64_t st = 0; st < steps; ++st) {
        const char* now = tiles[st & 1];
        char* next = tiles[(st & 1) ^ 1];
        wait_and_meet();
        if (st + 1 < steps) {
            a.fetch(next);
            b.fetch(next + A::kBytes);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            uintx4 x[BM], y[BN];
#pragma unroll
            for (int i = 0; i < BM; ++i) x[i] = A::piece(now, 32 * (BM * wm + i), s);
#pragma unroll
            for (int j = 0; j < BN; ++j) y[j] = B::piece(now + A::kBytes, 32 * (BN * wn + j), s);
#pragma unroll
            for (int i = 0; i < BM; ++i)
#pragma unroll
                for (int j = 0; j < BN; ++j) acc[i][j] = multiply<T>(y[j], x[i], acc[i][j]);
        }
        if (st + 1 < steps) {
            a.put(next);
            b.put(next + A::kBytes);
        }
    }

    const bool vec = g.vec_out != 0;
#pragma unroll
    for (int i = 0; i < BM; ++i) {
        const int64_t r = m0 + 32 * (BM * wm + i) + (lane & 31);
        int64_t to;
        if constexpr (MODE == kWeight) to = r < m_end ? r : -1;
        else to = row_of(g.out, r, r < m_end);
        if (to < 0) continue;
        char* row = out_base + to * (MODE == kWeight ? (int64_t)g.F_out * (int64_t)sizeof(TO) : g.out.ld);
#pragma unroll
        for (int j = 0; j < BN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = n0 + 32 * (BN * wn + j) + 8 * q + 4 * (lane >> 5);
                const float x[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                store4<TO>(row, c, x, N - c, vec);
            }
    }
}

// grad_W[g] = the sum of its chunks' partial sums, in order (none: zeros).
template <class TO>
__global__ __launch_bounds__(256) void k_grouped_sum(GroupedArgs g, TO* __restrict__ grad_W) {
    const int64_t size = (int64_t)g.F_in * g.F_out;
    __shared__ int64_t span[2];
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        int64_t before = 0, count = 0;
        for (int h0 = 0; h0 <= (int)blockIdx.y; h0 += 64) {
            const int h = h0 + lane;
            int64_t tiles = 0;
            if (h <= (int)blockIdx.y) {
                const int64_t lo = min(max((int64_t)g.offsets[h], (int64_t)0), g.m), hi = min(max((int64_t)g.offsets[h + 1], (int64_t)0), g.m);
                tiles = hi > lo ? (hi - lo + g.per - 1) / g.per : 0;
            }
            if (h == (int)blockIdx.y) count = tiles;
            else before += tiles;
        }
#pragma unroll
        for (int d = 32; d; d /= 2) {
            before += __shfl_xor(before, d, 64);
            count += __shfl_xor(count, d, 64);
        }
        if (lane == 0) {
            span[0] = before;
            span[1] = count;
        }
    }
    __syncthreads();
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= size) return;
    const float* p = g.part + span[0] * size + e;
    const int64_t count = span[1];
    float sum = 0.f;
    int64_t c = 0;
    for (; c + 8 <= count; c += 8) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = p[(c + i) * size];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i];
    }
    for (; c < count; ++c) sum += p[c * size];
    grad_W[blockIdx.y * size + e] = Num<TO>::from(sum);
}

// ---------------------------------------------------------------- host side
int size_of(int type) { return type == EPP_FLOAT32 ? 4 : 2; }

int check_type(int type) {
    if (type != EPP_FLOAT32 && type != EPP_BFLOAT16 && type != EPP_FLOAT16) { epp_set_error("unknown element type %d", type); return EPP_ERR_INVALID_ARG; }
    return EPP_OK;
}

int check_groups(int64_t m, int G, int F_in, int F_out) {
    if (m < 0 || m >= (1ll << 31)) { epp_set_error("%lld entries (0 to 2^31 - 1)", (long long)m); return m < 0 ? EPP_ERR_INVALID_ARG : EPP_ERR_TOO_LARGE; }
    if (G < 1 || G > kMaxGroups) { epp_set_error("%d groups (1 to %d)", G, kMaxGroups); return G < 1 ? EPP_ERR_INVALID_ARG : EPP_ERR_TOO_LARGE; }
    if (F_in < 1 || F_out < 1) { epp_set_error("F_in=%d, F_out=%d must be >= 1", F_in, F_out); return EPP_ERR_INVALID_ARG; }
    if (F_in > kMaxWidth || F_out > kMaxWidth) { epp_set_error("F_in=%d, F_out=%d (up to %d)", F_in, F_out, kMaxWidth); return EPP_ERR_TOO_LARGE; }
    return EPP_OK;
}

int check_rows(const epp_rows_t* x, int64_t m, int width, int size, const char* what) {
    if (!x || (!x->data && m > 0 && x->n > 0)) { epp_set_error("%s: NULL argument", what); return EPP_ERR_INVALID_ARG; }
    if (x->n < 0 || x->n >= (1ll << 31)) { epp_set_error("%s: %lld rows", what, (long long)x->n); return x->n < 0 ? EPP_ERR_INVALID_ARG : EPP_ERR_TOO_LARGE; }
    if (x->ld < width || x->ld >= (1ll << 31)) { epp_set_error("%s: rows of %d elements, %lld from row to row", what, width, (long long)x->ld); return EPP_ERR_INVALID_ARG; }
    if (!x->rows && x->n < m) { epp_set_error("%s: %lld rows, %lld entries and no list of rows", what, (long long)x->n, (long long)m); return EPP_ERR_INVALID_ARG; }
    if (reinterpret_cast<uintptr_t>(x->data) % (unsigned)size || reinterpret_cast<uintptr_t>(x->rows) % 4) {
        epp_set_error("%s: address not aligned to its elements", what);
        return EPP_ERR_INVALID_ARG;
    }
    return EPP_OK;
}

// Whether rows of two matrices share memory: their spans do, and they are not different columns of one wider matrix.
bool overlap(const epp_rows_t& x, int wx, const epp_rows_t& y, int wy, int size) {
    if (x.n <= 0 || y.n <= 0) return false;
    const uintptr_t bx = reinterpret_cast<uintptr_t>(x.data), by = reinterpret_cast<uintptr_t>(y.data);
    const uintptr_t ex = bx + (uintptr_t)((x.n - 1) * x.ld + wx) * (uintptr_t)size, ey = by + (uintptr_t)((y.n - 1) * y.ld + wy) * (uintptr_t)size;
    if (ex <= by || ey <= bx) return false;
    if (x.ld != y.ld) return true;
    const uintptr_t pitch = (uintptr_t)x.ld * (uintptr_t)size;
    const uintptr_t lx = (uintptr_t)wx * (uintptr_t)size, ly = (uintptr_t)wy * (uintptr_t)size;
    const uintptr_t d = (by >= bx ? by - bx : pitch - (bx - by) % pitch) % pitch;  // y's first column, seen from x's
    return !(d >= lx && d + ly <= pitch);
}
bool overlaps_block(const epp_rows_t& x, int wx, int size, const void* p, int64_t bytes) {
    if (x.n <= 0 || bytes <= 0) return false;
    const uintptr_t bx = reinterpret_cast<uintptr_t>(x.data), ex = bx + (uintptr_t)((x.n - 1) * x.ld + wx) * (uintptr_t)size;
    const uintptr_t bp = reinterpret_cast<uintptr_t>(p);
    return bx < bp + (uintptr_t)bytes && bp < ex;
}
int aliased() { epp_set_error("matrices must not alias"); return EPP_ERR_INVALID_ARG; }

bool aligned(const Side& s, int width_bytes) { return (reinterpret_cast<uintptr_t>(s.data) | (uintptr_t)s.ld | (uintptr_t)width_bytes) % 16 == 0; }
Side side(const epp_rows_t& x, int size) { return {static_cast<const char*>(x.data), x.n, x.ld * size, x.rows}; }

// Tiles of `tile` entries that m entries in G groups can make.
int64_t most_tiles(int64_t m, int64_t G, int64_t tile) { return (m + std::min(G, m) * (tile - 1)) / tile; }

template <class T, class TO, int MODE, int WM, int WN, int BM, int BN>
int launch(const GroupedArgs& g, int64_t blocks, bool direct, hipStream_t s) {
    if (blocks > 0x7FFFFFFF) { epp_set_error("%lld workgroups in one launch", (long long)blocks); return EPP_ERR_TOO_LARGE; }
    if (direct) hipLaunchKernelGGL((k_grouped<T, TO, MODE, WM, WN, BM, BN, true>), dim3((unsigned)blocks), dim3(64 * WM * WN), 0, s, g);
    else hipLaunchKernelGGL((k_grouped<T, TO, MODE, WM, WN, BM, BN, false>), dim3((unsigned)blocks), dim3(64 * WM * WN), 0, s, g);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}

template <class T, int MODE>
int launch_rows(const GroupedArgs& g, bool direct, hipStream_t s) {
    const int N = MODE == kInput ? g.F_in : g.F_out;
    const int64_t blocks = (most_tiles(g.m, g.G, 128) * ((N + 127) / 128) + 7) / 8 * 8;
    return launch<T, T, MODE, 2, 2, 2, 2>(g, blocks, direct, s);
}

// product (X, W -> out) and input gradient (grad_out, W -> grad_X)
int grouped_rows(int mode, int type, const epp_rows_t* in, const void* W, const int32_t* offsets, int G, int64_t m, int F_in, int F_out,
                 const epp_rows_t* out, hipStream_t s) {
    EPP_TRY(check_type(type));
    EPP_TRY(check_groups(m, G, F_in, F_out));
    const int size = size_of(type), w_in = mode == kInput ? F_out : F_in, w_out = mode == kInput ? F_in : F_out;
    EPP_TRY(check_rows(in, m, w_in, size, mode == kInput ? "grad_out" : "X"));
    EPP_TRY(check_rows(out, m, w_out, size, mode == kInput ? "grad_X" : "out"));
    if (!W || !offsets) { epp_set_error("NULL argument"); return EPP_ERR_INVALID_ARG; }
    if (reinterpret_cast<uintptr_t>(W) % (unsigned)size || reinterpret_cast<uintptr_t>(offsets) % 4) { epp_set_error("address not aligned to its elements"); return EPP_ERR_INVALID_ARG; }
    if (overlap(*in, w_in, *out, w_out, size) || overlaps_block(*out, w_out, size, W, (int64_t)G * F_in * F_out * size) ||
        overlaps_block(*out, w_out, size, offsets, 4 * ((int64_t)G + 1)))
        return aliased();
    if (m == 0) return EPP_OK;
    GroupedArgs g = {};
    g.a = side(*in, size);
    g.out = side(*out, size);
    g.W = static_cast<const char*>(W);
    g.offsets = offsets;
    g.m = m;
    g.G = G;
    g.F_in = F_in;
    g.F_out = F_out;
    g.vec_out = (reinterpret_cast<uintptr_t>(out->data) | (uintptr_t)g.out.ld) % (4 * (unsigned)size) == 0;
    const bool direct = aligned(g.a, w_in * size) && reinterpret_cast<uintptr_t>(W) % 16 == 0 && (F_out * size) % 16 == 0;
    if (mode == kInput) {
        if (type == EPP_FLOAT32) return launch_rows<float, kInput>(g, direct, s);
        if (type == EPP_BFLOAT16) return launch_rows<__bf16, kInput>(g, direct, s);
        return launch_rows<_Float16, kInput>(g, direct, s);
    }
    if (type == EPP_FLOAT32) return launch_rows<float, kProduct>(g, direct, s);
    if (type == EPP_BFLOAT16) return launch_rows<__bf16, kProduct>(g, direct, s);
    return launch_rows<_Float16, kProduct>(g, direct, s);
}

// How the weight gradient cuts its entries: chunks of `per` entries of a group, at most `count` of them; per = 0: whole groups.
struct Chunks { int64_t per, count; };
Chunks chunking(int64_t m, int G, int F_in, int F_out) {
    const int64_t tiles = (int64_t)((F_in + 127) / 128) * ((F_out + 127) / 128);
    // (one group may hold nearly all entries: its tiles alone have to fill the chip)
    const int64_t wanted = 512 / tiles;
    if (wanted <= 1 || m < 512) return {0, G};
    const int64_t per = std::max<int64_t>((m + wanted - 1) / wanted, 256);
    return {per, most_tiles(m, G, per)};
}

template <class T, class TO>
int launch_weight(GroupedArgs g, const Chunks& c, bool direct, TO* grad_W, hipStream_t s) {
    const int64_t tiles = (int64_t)((g.F_in + 127) / 128) * ((g.F_out + 127) / 128);
    if (!c.per) {
        g.out.data = reinterpret_cast<const char*>(grad_W);
        g.vec_out = g.F_out % 4 == 0 && reinterpret_cast<uintptr_t>(grad_W) % (4 * sizeof(TO)) == 0;
        return launch<T, TO, kWeight, 2, 2, 2, 2>(g, c.count * tiles, direct, s);
    }
    g.vec_out = g.F_out % 4 == 0;
    EPP_TRY((launch<T, float, kWeight, 2, 2, 2, 2>(g, c.count * tiles, direct, s)));
    const int64_t size = (int64_t)g.F_in * g.F_out;
    hipLaunchKernelGGL((k_grouped_sum<TO>), dim3((unsigned)((size + 255) / 256), (unsigned)g.G), dim3(256), 0, s, g, grad_W);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}

}  // namespace

extern "C" int epp_grouped_product(int type, const epp_rows_t* X, const void* W, const int32_t* offsets, int G, int64_t m, int F_in,
                                   int F_out, const epp_rows_t* out, epp_stream_t stream) {
    return grouped_rows(kProduct, type, X, W, offsets, G, m, F_in, F_out, out, (hipStream_t)stream);
}

extern "C" int epp_grouped_input_gradient(int type, const epp_rows_t* grad_out, const void* W, const int32_t* offsets, int G, int64_t m,
                                          int F_in, int F_out, const epp_rows_t* grad_X, epp_stream_t stream) {
    return grouped_rows(kInput, type, grad_out, W, offsets, G, m, F_in, F_out, grad_X, (hipStream_t)stream);
}

extern "C" int64_t epp_grouped_weight_gradient_workspace(int64_t m, int G, int F_in, int F_out) {
    EPP_TRY(check_groups(m, G, F_in, F_out));
    const Chunks c = chunking(m, G, F_in, F_out);
    return c.per ? c.count * F_in * F_out * (int64_t)sizeof(float) : 16;
}

extern "C" int epp_grouped_weight_gradient(int type, const epp_rows_t* X, const epp_rows_t* grad_out, const int32_t* offsets, int G,
                                           int64_t m, int F_in, int F_out, int grad_W_type, void* grad_W, void* workspace,
                                           int64_t workspace_bytes, epp_stream_t stream) {
    EPP_TRY(check_type(type));
    EPP_TRY(check_type(grad_W_type));
    if (grad_W_type != type && grad_W_type != EPP_FLOAT32) { epp_set_error("grad_W is fp32 or of the operands' type"); return EPP_ERR_INVALID_ARG; }
    EPP_TRY(check_groups(m, G, F_in, F_out));
    const int size = size_of(type), size_w = size_of(grad_W_type);
    EPP_TRY(check_rows(X, m, F_in, size, "X"));
    EPP_TRY(check_rows(grad_out, m, F_out, size, "grad_out"));
    if (!grad_W || !offsets || !workspace) { epp_set_error("NULL argument"); return EPP_ERR_INVALID_ARG; }
    if (reinterpret_cast<uintptr_t>(grad_W) % (unsigned)size_w || reinterpret_cast<uintptr_t>(offsets) % 4) { epp_set_error("address not aligned to its elements"); return EPP_ERR_INVALID_ARG; }
    const int64_t need = epp_grouped_weight_gradient_workspace(m, G, F_in, F_out);
    if (workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15)) {
        epp_set_error("workspace of %lld bytes (need %lld, 16-byte aligned)", (long long)workspace_bytes, (long long)need);
        return EPP_ERR_INVALID_ARG;
    }
    const int64_t w_bytes = (int64_t)G * F_in * F_out * size_w;
    if (overlaps_block(*X, F_in, size, grad_W, w_bytes) || overlaps_block(*grad_out, F_out, size, grad_W, w_bytes) ||
        overlaps_block(*X, F_in, size, workspace, need) || overlaps_block(*grad_out, F_out, size, workspace, need) ||
        (reinterpret_cast<uintptr_t>(workspace) < reinterpret_cast<uintptr_t>(grad_W) + (uintptr_t)w_bytes &&
         reinterpret_cast<uintptr_t>(grad_W) < reinterpret_cast<uintptr_t>(workspace) + (uintptr_t)need))
        return aliased();
    GroupedArgs g = {};
    g.a = side(*X, size);
    g.b = side(*grad_out, size);
    g.offsets = offsets;
    g.m = m;
    g.G = G;
    g.F_in = F_in;
    g.F_out = F_out;
    const Chunks c = chunking(m, G, F_in, F_out);
    g.per = c.per;
    g.part = static_cast<float*>(workspace);
    const bool direct = aligned(g.a, F_in * size) && aligned(g.b, F_out * size);
    hipStream_t s = (hipStream_t)stream;
    if (type == EPP_FLOAT32) return launch_weight<float, float>(g, c, direct, static_cast<float*>(grad_W), s);
    if (type == EPP_BFLOAT16) {
        if (grad_W_type == EPP_FLOAT32) return launch_weight<__bf16, float>(g, c, direct, static_cast<float*>(grad_W), s);
        return launch_weight<__bf16, __bf16>(g, c, direct, static_cast<__bf16*>(grad_W), s);
    }
    if (grad_W_type == EPP_FLOAT32) return launch_weight<_Float16, float>(g, c, direct, static_cast<float*>(grad_W), s);
    return launch_weight<_Float16, _Float16>(g, c, direct, static_cast<_Float16*>(grad_W), s);
}
