// Products of rows that belong to groups, each group with a weight matrix of its own (the experts of a mixture, the
// types of a graph's vertices).  With entries i of group g at [offsets[g], offsets[g + 1]):
//     out[o(i), :]    = X[a(i), :] W[g]                 (product)
//     grad_X[o(i), :] = grad_out[a(i), :] W[g]^T        (input gradient)
//     grad_W[g]       = sum over i of X[a(i), :]^T grad_out[b(i), :]
// a, b and o are row lists or the entries themselves.  Sizes of groups are known to the GPU only: a launch has as many
// workgroups as m entries in G groups can need, and every one finds its tile by a scan of the offsets.
//
// A workgroup forms a TM x TN tile of the result from operand tiles of 128 bytes of the contraction (64 elements of 16
// bits, 32 floats) in LDS, two of each or four: while the matrix cores work on one, the others fill.  An operand comes in one of
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
//
// What bounds them: large tiles of 16 bits the matrix cores together with what feeds them.  8,192 x 2,048 weights, 32 groups of 1,024
// entries in bfloat16 run at 1,160 TFLOP/s (a library product of 8,192 x 4,096 x 2,048 1,300; these kernels without most of their loads of
// operands 1,490); groups of exponentially distributed sizes at 960.  Floats: 122 to 128 TFLOP/s (a library product 153).  The weight gradient
// writes more than the products do: 256 KB a tile of floats, which nothing else in the compute unit overlaps.

#include "epp_grouped.h"

using namespace epp_grouped;

#include <cmath>
#include <numeric>

namespace {

constexpr int kMaxGroups = 2048;
constexpr int kMaxWidth = 1 << 16;
constexpr int kLine = 128;   // bytes of the contraction in a tile

__device__ __attribute__((aligned(128))) unsigned int g_zeros[32] = {};
__device__ int32_t g_none = -1;  // no row

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

// ---------------------------------------------------------------- operand tiles
// All loads of this wavefront have arrived and all its LDS reads are done; then the same for the workgroup's.
// (ALLOWED: but for the last so many loads)
template <int ALLOWED>
__device__ __forceinline__ void wait_and_meet() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(ALLOWED) : "memory"); }

__device__ __forceinline__ const char* zeros() { return reinterpret_cast<const char*>(g_zeros); }

// Lines of K: TD rows, whose places are set once.  DIRECT: what stands in a line without a row is somebody's numbers (the result's row
// is not written, or written as zeros); behind the contraction's end there are zeros.
template <class T, int TD, int NT, bool DIRECT>
struct LinesOfK {
    static constexpr int E = 16 / (int)sizeof(T), kPieces = kLine / 16, N = TD * kPieces / NT, kBytes = TD * kLine, kSteps = kLine / (int)sizeof(T);
    static __device__ __forceinline__ int turn(int row) { return (row >> 1) & 7; }  // what a line's pieces are permuted by
    static_assert((NT / kPieces) % 16 == 0, "all of a thread's pieces are of the same part of their lines");
    const char* base;  // DIRECT: the same for all lanes, moves with the contraction
    unsigned off[DIRECT ? N : 1];
    const char* p[DIRECT ? 1 : N];
    uintx4 held[DIRECT ? 1 : N];
    bool cut;          // .. some of them cut short
    int k, K;          // the contraction's element in this thread's pieces, and its end
    unsigned lds_wave;
    // row_at(i): tile row i, counted from `from`, -1: none
    template <class F> __device__ __forceinline__ void start(const char* from, int64_t pitch, int end, int wave, F row_at) {
        const int t = threadIdx.x;
        K = end;
        k = ((t % kPieces) ^ turn(t / kPieces)) * E;
        base = uniform(from);
        lds_wave = (unsigned)wave * 1024u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t r = row_at((i * NT + t) / kPieces);
            if constexpr (DIRECT) off[i] = (unsigned)(r < 0 ? 0 : r * pitch) + (unsigned)k * (unsigned)sizeof(T);
            else p[i] = r < 0 ? nullptr : from + r * pitch;
        }
    }
    __device__ __forceinline__ void prepare() {}
    // Piece i of the next tile, which the contraction fills (FULL), or as far as it goes.
    template <bool FULL>
    __device__ __forceinline__ void fetch(int i, char* to) {
        if constexpr (DIRECT) {
            const unsigned at = lds_address(to) + lds_wave + (unsigned)(i * NT * 16);
            if (FULL) load_to_lds(base, off[i], at);
            else load_to_lds(k < K ? base + off[i] : zeros(), at);
        } else {
            held[i] = load_piece<T>(p[i] + (int64_t)k * (int64_t)sizeof(T), p[i] ? K - k : 0, K < E, zeros());
            cut = !FULL;
        }
    }
    __device__ __forceinline__ void advance() {  // after all pieces of a tile
        base += kLine;
        k += kSteps;
    }
    __device__ __forceinline__ void put(char* to) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < N; ++i) *reinterpret_cast<uintx4*>(to + (i * NT + threadIdx.x) * 16) = cut ? shifted(held[i], shift_of<T>(K - (k - kSteps), K < E)) : held[i];
        }
    }
    // Piece 2 s + half of rows c0 + l % 32 (c0 a multiple of 32).
    static __device__ __forceinline__ uintx4 piece(const char* tile, int c0, int s) {
        const int l = threadIdx.x & 63;
        return *reinterpret_cast<const uintx4*>(tile + (c0 + (l & 31)) * kLine + (((2 * s + (l >> 5)) ^ turn(l & 31)) * 16));
    }
};

// Lines of width: the steps of the contraction are the entries [first, last) of `s`, the columns begin at c0.  LIST: the entries may name
// rows through a list.
template <class T, int TD, int NT, bool DIRECT, bool LIST>
struct LinesOfWidth {
    static constexpr int E = 16 / (int)sizeof(T), N = TD * kLine / 16 / NT, kBytes = TD * kLine;
    static constexpr int kWide = TD * (int)sizeof(T), kPieces = kWide / 16, kPairs = kWide / 32;
    static constexpr int kSteps = kLine / (int)sizeof(T);
    static_assert(NT % kPieces == 0 && (kPairs == 4 || kPairs % 8 == 0), "tile");
    // What a line's units of 32 bytes are permuted by.
    static __device__ __forceinline__ int turn(int line) {
        if constexpr (sizeof(T) == 4) return ((line >> 2) & 1) << 2;
        else if constexpr (kPairs == 4) return ((line >> 1) & 1) << 1;
        else return (line & 3) << 1;
    }
    static constexpr int kLines = NT / kPieces;  // lines from piece to piece of a thread
    static_assert(kLines % 8 == 0, "all of a thread's pieces are of the same columns");
    Side s;
    uint32_t at, last;  // entry of this thread's first piece in the next tile, and the end
    int c, width;       // column of this thread's pieces; columns
    const char* base;   // DIRECT, no list: place of the next tile's first line, the same for all lanes
    unsigned off;       // .. and of this thread's first piece, seen from there
    const char* col;    // DIRECT, list: place of column c of row 0
    const char* p[DIRECT && LIST ? N : 1];  // .. places of the next tile's pieces
    char* ring;         // .. four tiles' rows in LDS, each 64 of them: arrived two tiles before they are used
    int64_t ask;        // .. entry where the next tile to ask for begins, the same for all lanes
    int slot;           // .. place in the ring of the next tile
    bool asks;          // .. this wavefront loads the list
    int32_t row[!DIRECT && LIST ? N : 1];
    unsigned lds_wave;
    uintx4 held[DIRECT ? 1 : N];
    bool cut;           // .. some of them cut short
    __device__ __forceinline__ void start(const Side& side, int64_t first, int64_t end, int c0, int w, int wave, char* lds_ring = nullptr, bool loads_list = false) {
        const int t = threadIdx.x, line = t / kPieces;
        s = side;
        at = (uint32_t)first + (uint32_t)line;
        last = (uint32_t)end;
        width = w;
        c = c0 + ((t % kPieces) ^ (turn(line) << 1)) * E;
        lds_wave = (unsigned)wave * 1024u;
        if constexpr (DIRECT) {
            if (c >= width) c = 0;  // (somebody's numbers, for a result that is not written)
            base = uniform(s.data + first * s.ld);
            off = (unsigned)line * (unsigned)s.ld + (unsigned)c * (unsigned)sizeof(T);
            col = s.data + (int64_t)c * (int64_t)sizeof(T);
        }
        if constexpr (LIST && DIRECT) {
            ring = lds_ring;
            ask = uniform(first);
            slot = 0;
            asks = loads_list;
            ask_rows(0);
            ask_rows(1);
        }
        if constexpr (!DIRECT) {
            cut = c0 + TD > width;
            if constexpr (LIST) next_rows();
        }
    }
    // The rows of a tile into slot q of the ring.  (Loaded into registers and kept there from tile to tile, they would have to be waited for
    // behind the operands' loads, which the compiler's count of loads does not know: 594 instead of 380 us for 16 groups of 2,048 entries
    // and 2,048 x 2,048 weights.)
    __device__ __forceinline__ void ask_rows(int q) {
        if (asks) {
            const int64_t e = ask + (threadIdx.x & 63);  // (`ask` and `at` pass the last entry, but not 2^32)
            if (s.rows) load4_to_lds(reinterpret_cast<const char*>(e < last ? s.rows + e : &g_none), lds_address(ring) + (unsigned)q * 256u);
            else reinterpret_cast<int32_t*>(ring + q * 256)[threadIdx.x & 63] = e < last ? (int32_t)e : -1;
        }
        ask += kSteps;
    }
    __device__ __forceinline__ void next_rows() {
        if (!s.rows) return;
#pragma unroll
        for (int i = 0; i < N; ++i) row[i] = at + i * kLines < last ? s.rows[at + i * kLines] : -1;
    }
    // The next tile's places.
    __device__ __forceinline__ void prepare() {
        if constexpr (DIRECT && LIST) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t r = *reinterpret_cast<const uint32_t*>(ring + slot * 256 + (i * kLines + threadIdx.x / kPieces) * 4);
                p[i] = r < (uint32_t)s.n ? col + (uint64_t)r * (uint64_t)(uint32_t)s.ld : zeros();
            }
        }
    }
    template <bool FULL>
    __device__ __forceinline__ void fetch(int i, char* to) {
        if constexpr (DIRECT) {
            const unsigned lds = lds_address(to) + lds_wave + (unsigned)(i * NT * 16);
            if constexpr (LIST) load_to_lds(p[i], lds);
            else if (FULL) load_to_lds(base + (int64_t)(i * kLines) * s.ld, off, lds);
            else load_to_lds(at + i * kLines < last ? base + (int64_t)(i * kLines) * s.ld + off : zeros(), lds);
        } else {
            const uint32_t e = at + i * kLines;
            int64_t r = (int64_t)e;
            bool no = e >= last || c >= width;
            if constexpr (LIST) {
                if (s.rows) r = row[i];
                no = no || r < 0 || r >= s.n;
            }
            held[i] = load_piece<T>(s.data + r * s.ld + (int64_t)c * (int64_t)sizeof(T), no ? 0 : width - c, width < E, zeros());
        }
    }
    __device__ __forceinline__ void advance() {
        at += kSteps;
        if constexpr (DIRECT) base += kSteps * s.ld;
        if constexpr (DIRECT && LIST) {
            ask_rows((slot + 2) & 3);
            slot = (slot + 1) & 3;
        }
        if constexpr (!DIRECT && LIST) next_rows();
    }
    __device__ __forceinline__ void put(char* to) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < N; ++i) *reinterpret_cast<uintx4*>(to + (i * NT + threadIdx.x) * 16) = cut ? shifted(held[i], shift_of<T>(width - c, width < E)) : held[i];
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
                v[j] = *reinterpret_cast<const unsigned int*>(tile + line * kWide + (((x >> 3) ^ turn(line)) * 32) + (x & 7) * 4);
            }
            return v;
        } else {
            typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
            const int i = l & 15, unit = (c >> 4) + ((l >> 4) & 1);
            const int l0 = 8 * q + (i >> 2), l1 = l0 + 4;
            const char* p0 = tile + l0 * kWide + ((unit ^ turn(l0)) * 32) + (i & 3) * 8;
            const char* p1 = tile + l1 * kWide + ((unit ^ turn(l1)) * 32) + (i & 3) * 8;
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(p0));
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(p1));
            return __builtin_bit_cast(uintx4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// Where a tile of the result is.
struct Place {
    int g;                  // group (product, input gradient)
    int64_t m0, m_end;      // rows of the result: entries, or rows of grad_W
    int n0;
    int64_t first, last;    // weight gradient: entries
    char* out;              // .. and its matrix
};

// One tile: WM x WN wavefronts, each with BM x BN blocks of 32 x 32 of the result.  TO: type of the results.
template <class T, class TO, int MODE, int WM, int WN, int BM, int BN, bool DIRECT, bool LIST, int STAGES>
__device__ __forceinline__ void form_tile(const GroupedArgs& g, const Place& at, char* lds) {
    constexpr int NT = 64 * WM * WN, TM = 32 * WM * BM, TN = 32 * WN * BN;
    using A = std::conditional_t<MODE == kWeight, LinesOfWidth<T, TM, NT, DIRECT, LIST>, LinesOfK<T, TM, NT, DIRECT>>;
    using B = std::conditional_t<MODE == kInput, LinesOfK<T, TN, NT, DIRECT>, LinesOfWidth<T, TN, NT, DIRECT, LIST>>;
    constexpr int kBytes = A::kBytes + B::kBytes, kSteps = kLine / (int)sizeof(T), kSubs = kLine / 32, kLoads = A::N + B::N;
    static_assert(STAGES == 2 || (DIRECT && !LIST && kLoads * (STAGES - 1) < 64), "stages");
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wn = w % WN, wm = w / WN;
    A a;
    B b;
    int64_t K;  // steps of the contraction
    const int64_t m0 = at.m0, m_end = at.m_end;
    const int n0 = at.n0, N = MODE == kInput ? g.F_in : g.F_out;
    if constexpr (MODE != kWeight) {
        const char* W = g.W + at.g * ((int64_t)g.F_in * g.F_out * (int64_t)sizeof(T));
        const int64_t ldw = (int64_t)g.F_out * (int64_t)sizeof(T);
        K = MODE == kInput ? g.F_out : g.F_in;
        // (with a list a row's place is counted from the first one, else from the tile's)
        a.start(g.a.rows ? g.a.data : g.a.data + m0 * g.a.ld, g.a.ld, (int)K, w, [&](int i) -> int64_t {
            const int64_t r = row_of(g.a, m0 + i, m0 + i < m_end);
            return r < 0 ? -1 : g.a.rows ? r : (int64_t)i;
        });
        if constexpr (MODE == kInput) b.start(W + n0 * ldw, ldw, (int)K, w, [&](int i) -> int64_t { return n0 + i < N ? i : -1; });
        else b.start(Side{W, K, ldw, nullptr}, 0, K, n0, N, w);
    } else {
        K = at.last - at.first;
        char* ring = lds + STAGES * kBytes;
        a.start(g.a, at.first, at.last, (int)m0, g.F_in, w, ring, w == 0);
        b.start(g.b, at.first, at.last, n0, g.F_out, w, ring + 1024, w == 1);
        if (DIRECT && LIST) wait_and_meet<0>();
    }

    // Two sets of operand pieces in registers: while the matrix cores work on one, the other is read.  The wavefronts meet when all have
    // read the last pieces of a tile, before they work on them: the tile's place is then free for another, whose loads are issued at once
    // (in between the last products instead, and thus later, they took 656 instead of 593 us for 32,768 entries, 32 groups, 4,096 x 2,048), and
    // the first pieces of the next arrive behind the last products.
    // kAcross: 32 lanes hold neighbouring columns, and write 128 bytes of a row; else a lane holds four neighbouring columns.  (Where writing
    // floats is most of the work: 256 entries of 16 bits, 64 groups, 1,777 x 2,048, 201 / 171 us; floats from floats, whose tiles are small, 266 / 282.)
    constexpr bool kAcross = MODE == kWeight && sizeof(T) == 2 && sizeof(TO) == 4;
    floatx16 acc[BM][BN] = {};
    uintx4 x[2][BM], y[2][BN];
    auto read = [&](const char* tile, int s, int set) {
#pragma unroll
        for (int j = 0; j < BN; ++j) y[set][j] = B::piece(tile + A::kBytes, 32 * (BN * wn + j), s);
#pragma unroll
        for (int i = 0; i < BM; ++i) x[set][i] = A::piece(tile, 32 * (BM * wm + i), s);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto work = [&](int set) {
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j) acc[i][j] = kAcross ? multiply<T>(x[set][i], y[set][j], acc[i][j]) : multiply<T>(y[set][j], x[set][i], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto put = [&](char* tile) {
        a.put(tile);
        b.put(tile + A::kBytes);
    };
    auto fetch_all = [&](auto full, char* tile) {  // all loads of a tile, whose places are prepared
#pragma unroll
        for (int f = 0; f < A::N; ++f) a.template fetch<full>(f, tile);
#pragma unroll
        for (int f = 0; f < B::N; ++f) b.template fetch<full>(f, tile + A::kBytes);
        a.advance();
        b.advance();
    };
    auto prepare = [&]() {
        a.prepare();
        b.prepare();
    };
    const int64_t full = K / kSteps, steps = (K + kSteps - 1) / kSteps;  // tiles that the contraction fills, and all
    using Yes = std::true_type;
    using No = std::false_type;
    if (steps > 0) {
        prepare();
        fetch_all(No{}, lds);
        put(lds);
        if constexpr (STAGES > 2) {
#pragma unroll
            for (int i = 1; i < STAGES - 1; ++i)
                if (i < steps) fetch_all(No{}, lds + i * kBytes);
        }
        if (STAGES > 2 && steps >= STAGES - 1) wait_and_meet<kLoads * (STAGES - 2)>();
        else wait_and_meet<0>();
        if (STAGES - 1 < steps) {
            prepare();
            fetch_all(No{}, lds + (STAGES - 1) * kBytes);
        }
    }
    auto contract = [&](auto live) {
        int64_t st = 0;
        int stage = 0;
        if (live && steps > 0) read(lds, 0, 0);
        auto step = [&](auto middle) {  // middle: the tile to be loaded into this one's place is a full one
            char* now = lds + stage * kBytes;
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            char* next = lds + stage * kBytes;
            if constexpr (live) read(now, 1, 1);
            if (middle || st + STAGES < steps) prepare();
            if constexpr (live) {
#pragma unroll
                for (int s = 1; s < kSubs; ++s) {
                    work((s - 1) & 1);
                    if (s + 1 < kSubs) read(now, s + 1, (s + 1) & 1);
                }
            }
            if (!DIRECT && (middle || st + 1 < steps)) put(next);
            // (of the loads that are on their way, the next tile's have to have arrived)
            if constexpr (middle) wait_and_meet<kLoads * (STAGES - 2)>();
            else wait_and_meet<0>();
            if constexpr (middle) fetch_all(Yes{}, now);
            else if (st + STAGES < steps) fetch_all(No{}, now);
            if constexpr (live) {
                if (middle || st + 1 < steps) read(next, 0, 0);
                work(1);
            }
        };
        for (; st + STAGES < full; ++st) step(Yes{});
        for (; st < steps; ++st) step(No{});
    };
    // (a wavefront whose rows lie behind the group's last has nothing to do but its share of the loads)
    if (m0 + 32 * BM * wm < m_end) contract(Yes{});
    else contract(No{});

    if constexpr (kAcross) {
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int64_t r = m0 + 32 * (BM * wm + i) + 8 * (e / 4) + 4 * (lane >> 5) + e % 4;
                float* row = reinterpret_cast<float*>(at.out) + r * g.F_out;
#pragma unroll
                for (int j = 0; j < BN; ++j) {
                    const int c = n0 + 32 * (BN * wn + j) + (lane & 31);
                    if (r < m_end && c < N) row[c] = acc[i][j][e];
                }
            }
        return;
    }
#pragma unroll
    for (int i = 0; i < BM; ++i) {
        const int64_t r = m0 + 32 * (BM * wm + i) + (lane & 31);
        int64_t to;
        bool none = false;  // a row of X that does not exist
        if constexpr (MODE == kWeight) to = r < m_end ? r : -1;
        else {
            to = row_of(g.out, r, r < m_end);
            if (DIRECT && g.a.rows) none = row_of(g.a, r, r < m_end) < 0;
        }
        if (to < 0) continue;
        char* row = at.out + to * (MODE == kWeight ? (int64_t)g.F_out * (int64_t)sizeof(TO) : g.out.ld);
#pragma unroll
        for (int j = 0; j < BN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = n0 + 32 * (BN * wn + j) + 8 * q + 4 * (lane >> 5);
                float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if (none) v[0] = v[1] = v[2] = v[3] = 0.f;
                store4<TO>(row, c, v, N - c);
            }
    }
}

// Product and input gradient.  QUARTERS: where the tiles fill the chip's kUnits compute units some times over and then up to half of them
// once more, those last tiles are dealt out in quarters.
template <class T, int MODE, int WM, int WN, int BM, int BN, bool DIRECT, bool QUARTERS, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void k_grouped_rows(GroupedArgs g) {
    constexpr int TM = 32 * WM * BM, TN = 32 * WN * BN;
    __shared__ __attribute__((aligned(128))) char lds[STAGES * (TM + TN) * kLine];
    const int N = MODE == kInput ? g.F_in : g.F_out;
    const int nt = (N + TN - 1) / TN;
    int64_t tiles;
    find_group(g.offsets, g.G, g.m, TM, -1, &tiles);
    tiles *= nt;
    // Workgroups b, b + 8, .. run on one XCD: it gets neighbouring tiles, which share rows and weights in its L2.
    int64_t whole = tiles, b = blockIdx.x;
    if (QUARTERS && tiles % kUnits <= kUnits / 2) whole = tiles / kUnits * kUnits;
    int quarter = -1;
    const bool last = b >= (whole + 7) / 8 * 8;
    if (last) b -= (whole + 7) / 8 * 8;
    const int64_t count = last ? 4 * (tiles - whole) : whole, per = (count + 7) / 8;
    int64_t mine = (b & 7) * per + (b >> 3);
    if ((b >> 3) >= per || mine >= count) return;
    if (last) {
        quarter = (int)(mine & 3);
        mine = whole + (mine >> 2);
    }
    int64_t unused;
    const Span s = find_group(g.offsets, g.G, g.m, TM, mine / nt, &unused);
    Place at = {s.g, uniform(s.first + (mine / nt - s.chunk0) * TM), uniform(s.last), __builtin_amdgcn_readfirstlane((int)(mine % nt) * TN), 0, 0, const_cast<char*>(g.out.data)};
    if (!QUARTERS || quarter < 0) {
        form_tile<T, T, MODE, WM, WN, BM, BN, DIRECT, false, STAGES>(g, at, lds);
    } else if constexpr (QUARTERS) {
        at.m0 += (quarter & 1) * (TM / 2);
        at.n0 += (quarter >> 1) * (TN / 2);
        if (at.m0 < at.m_end && at.n0 < N) form_tile<T, T, MODE, WM, WN, BM / 2, BN / 2, DIRECT, false, STAGES>(g, at, lds);
    }
}

// The group (of up to 64) that `rank` others precede in the order of their sizes, largest first.
__device__ __forceinline__ int group_of_rank(const int32_t* __restrict__ offsets, int G, int64_t m, int rank) {
    const int lane = threadIdx.x & 63;
    const int g = min(lane, G - 1);
    const int lo = (int)min(max((int64_t)offsets[g], (int64_t)0), m), hi = (int)min(max((int64_t)offsets[g + 1], (int64_t)0), m);
    // (one number to compare: the size, to 2^-25 of all entries, and before others of the same size the lower group)
    const int shift = max(0, 39 - __builtin_clzll((unsigned long long)m | 1));
    const unsigned key = lane < G ? ((unsigned)max(hi - lo, 0) >> shift) * 64u + (63u - (unsigned)lane) : 0u;
    int before = 0;
    for (int j = 0; j < G; ++j) before += (unsigned)__builtin_amdgcn_readlane((int)key, j) > key;
    return __ffsll((long long)__ballot(lane < G && before == rank)) - 1;
}

template <class T, class TO, int WM, int WN, int BM, int BN, bool DIRECT, bool LIST, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void k_grouped_weight(GroupedArgs g) {
    constexpr int TM = 32 * WM * BM, TN = 32 * WN * BN;
    __shared__ __attribute__((aligned(128))) char lds[STAGES * (TM + TN) * kLine + (DIRECT && LIST ? 2048 : 0)];
    const int mt = (g.F_in + TM - 1) / TM, nt = (g.F_out + TN - 1) / TN;
    // (the tiles of one group or chunk are dealt to all XCDs: groups differ in size)
    const int per_group = mt * nt, in = (int)(blockIdx.x % per_group), share = per_group / 8;
    int64_t chunk = blockIdx.x / per_group;
    if constexpr (BM * BN >= 8) {
        // (large tiles, a few to a compute unit: the longest groups first, or the last ones to begin end long after the others)
        if (!g.per && g.G <= 64) chunk = group_of_rank(g.offsets, g.G, g.m, (int)chunk);
    }
    const int tile = per_group % 8 == 0 ? (in & 7) * share + (in >> 3) : in;
    Place at = {0, (int64_t)(tile / nt) * TM, g.F_in, (tile % nt) * TN, 0, 0, const_cast<char*>(g.out.data)};
    if (g.per) {
        int64_t total;
        const Span s = find_group(g.offsets, g.G, g.m, g.per, chunk, &total);
        if (s.g < 0) return;
        at.first = uniform(s.first + (chunk - s.chunk0) * g.per);
        at.last = uniform(min(at.first + g.per, s.last));
        at.out = reinterpret_cast<char*>(g.part + chunk * g.F_in * g.F_out);
    } else {
        at.first = min(max((int64_t)g.offsets[chunk], (int64_t)0), g.m);
        at.last = max(at.first, min((int64_t)g.offsets[chunk + 1], g.m));
        at.out += chunk * g.F_in * g.F_out * (int64_t)sizeof(TO);
    }
    form_tile<T, TO, kWeight, WM, WN, BM, BN, DIRECT, LIST, STAGES>(g, at, lds);
}

// grad_W[g] = the sum of its chunks' partial sums, in order (none: zeros).  Four elements to a thread; SLICES threads share the chunks of
// them, every one a run of consecutive chunks.
template <class TO, int SLICES>
__global__ __launch_bounds__(256) void k_grouped_sum(GroupedArgs g, TO* __restrict__ grad_W) {
    constexpr int kThreads = 256 / SLICES;  // that share no element
    const int64_t size = (int64_t)g.F_in * g.F_out;
    __shared__ int64_t span[2];
    __shared__ float part[SLICES > 1 ? SLICES : 1][kThreads][4];
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        int64_t before = 0, count = 0;
        for (int h0 = 0; h0 <= (int)blockIdx.y; h0 += 64) {
            const int h = h0 + lane;
            int64_t tiles = 0;
            if (h <= (int)blockIdx.y) {
                const int64_t lo = min(max((int64_t)g.offsets[h], (int64_t)0), g.m), hi = min(max((int64_t)g.offsets[h + 1], (int64_t)0), g.m);
                tiles = hi > lo ? (uint32_t)(hi - lo + g.per - 1) / (uint32_t)g.per : 0;
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
            span[0] = min(before, g.chunks);
            span[1] = min(count, g.chunks - span[0]);
        }
    }
    __syncthreads();
    const int slice = threadIdx.x / kThreads, lane = threadIdx.x % kThreads;
    const int64_t e = ((int64_t)blockIdx.x * kThreads + lane) * 4;
    const int64_t share = (span[1] + SLICES - 1) / SLICES, first = min(slice * share, span[1]), last = min(first + share, span[1]);
    typedef float any_floatx4 __attribute__((ext_vector_type(4), aligned(4)));
    const float* p = g.part + span[0] * size + e;
    const int valid = (int)max(min(size - e, (int64_t)4), (int64_t)0);
    float sum[4] = {};
    if (valid == 4) {
        int64_t c = first;
        for (; c + 4 <= last; c += 4) {
            floatx4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const any_floatx4*>(p + (c + i) * size);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) sum[q] += x[i][q];
        }
        for (; c < last; ++c) {
            const floatx4 x = *reinterpret_cast<const any_floatx4*>(p + c * size);
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[q] += x[q];
        }
    } else {
        for (int64_t c = first; c < last; ++c)
#pragma unroll
            for (int q = 0; q < 3; ++q)
                if (q < valid) sum[q] += p[c * size + q];
    }
    if constexpr (SLICES > 1) {
#pragma unroll
        for (int q = 0; q < 4; ++q) part[slice][lane][q] = sum[q];
        __syncthreads();
        if (slice) return;
#pragma unroll
        for (int x = 1; x < SLICES; ++x)
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[q] += part[x][lane][q];
    }
    if (valid) store4<TO>(reinterpret_cast<char*>(grad_W + blockIdx.y * size + e), 0, sum, valid);
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
    // (every row of either begins a multiple of `pitch` behind its first: the common divisor of their distances, of which a single row has none)
    const uintptr_t pitch = std::gcd(x.n > 1 ? (uintptr_t)x.ld : 0, y.n > 1 ? (uintptr_t)y.ld : 0) * (uintptr_t)size;
    if (!pitch) return true;
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
// A list of `count` rows or offsets (NULL: none).
bool overlaps_list(const int32_t* list, int64_t count, const void* p, int64_t bytes) {
    if (!list || count <= 0 || bytes <= 0) return false;
    const uintptr_t o = reinterpret_cast<uintptr_t>(list), b = reinterpret_cast<uintptr_t>(p);
    return o < b + (uintptr_t)bytes && b < o + 4 * (uintptr_t)count;
}
int aliased() { epp_set_error("outputs and the workspace must not alias anything else"); return EPP_ERR_INVALID_ARG; }

bool aligned(const Side& s, int width_bytes) { return (reinterpret_cast<uintptr_t>(s.data) | (uintptr_t)s.ld | (uintptr_t)width_bytes) % 16 == 0; }
Side side(const epp_rows_t& x, int size) { return {static_cast<const char*>(x.data), x.n, x.ld * size, x.rows}; }

// Tiles of `tile` entries that m entries in G groups can make.
int64_t most_tiles(int64_t m, int64_t G, int64_t tile) { return (m + std::min(G, m) * (tile - 1)) / tile; }

// (a launch has fewer than 2^32 threads)
int check_blocks(int64_t blocks, int threads) {
    if (blocks * threads <= 0xFFFFFFFFll) return EPP_OK;
    epp_set_error("%lld tiles of the result in one launch", (long long)blocks);
    return EPP_ERR_TOO_LARGE;
}

template <class T, int MODE, int WM, int WN, int BM, int BN, bool DIRECT, bool QUARTERS, int STAGES = 2>
int launch_rows_of(const GroupedArgs& g, hipStream_t s) {
    constexpr int TM = 32 * WM * BM, TN = 32 * WN * BN;
    const int N = MODE == kInput ? g.F_in : g.F_out;
    int64_t blocks = most_tiles(g.m, g.G, TM) * ((N + TN - 1) / TN) + 16;
    if (QUARTERS) blocks += 3 * (kUnits / 2);
    EPP_TRY(check_blocks(blocks, 64 * WM * WN));
    hipLaunchKernelGGL((k_grouped_rows<T, MODE, WM, WN, BM, BN, DIRECT, QUARTERS, STAGES>), dim3((unsigned)blocks), dim3(64 * WM * WN), 0, s, g);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}

// Tiles of 64 x 64 where those of 128 x 128 would not be enough for the chip, and for floats always: their products take 16 times as long, so
// that tiles which are not full, or not there, cost more than fetching.  128 / 64, us: bfloat16, 4 groups, 300 entries, 1,024 x 1,024 (34 tiles)
// 14.1 / 8.2, 2,000 (141) 15.5 / 13.4, 8,000 (516) 25.3 / 35.4; floats, 300 of 4,096 x 1,024 255 / 77, 16 groups, 8,000 733 / 577,
// 4 groups, 30,000 1,934 / 1,898.  With less than one of them to a compute unit, four of their tiles of operands in LDS (16 bits: floats work
// longer on a tile than it takes to load): 4 groups, 300 of 4,096 x 1,024 31.4 / 18.7.
bool small_tiles(int64_t tiles) { return tiles < kUnits; }

// 16 bits: tiles of 256 x 256, which fetch half as much a product as tiles of 128 x 128 but come one to a compute unit, where there are enough
// of them and the width does not waste a part of each.  bfloat16, groups of exponentially distributed sizes, 128 / 256 wide, us: 2,048 entries,
// 16 groups, 4,096 x 4,096 (about 256 tiles of 256) 173 / 154; 32,768, 32, 4,096 x 2,048 663 / 593; 32,768, 64, 2,048 x 512 (320) 112 / 101;
// 60,000, 8, 1,000 x 1,000 178 / 152; but 8,192, 64, 2,048 x 512 (128) 34 / 55, 512, 4, 4,096 x 4,096 (64) 49 / 85, and 32,768, 4, 256 x 384 (a
// quarter wasted) 24 / 29.  Through registers the product would need more of them than there are; with tiles of 128 x 256 it took longer (532
// / 549 for 32,768, 16, 2,047 x 2,047; its gradients 536 / 428 and, of the weights, 579 / 421).
bool fills(int width) { return (width + 255) / 256 * 2048 <= 9 * width || width >= 1024; }
bool large_tiles(int64_t rows, int width) { return fills(width) && rows * ((width + 255) / 256) >= 192; }
// Weight gradients, whose tiles each go through all entries of a group: enough that the longest group's take at most twice as long as the
// average compute unit's share (the longest of G exponentially distributed sizes is 1 + 1/2 + .. + 1/G, about ln G + 0.58, times their
// average).  128 / 256 wide, us: 2 groups, 8,000 entries, 4,096 x 4,096 (512 tiles of 256) 325 / 254, 3,001 x 3,999 of 4,000 (384) 203 / 175; 4,
// 16,000, 1,500 x 3,000 (288) 355 / 267; but 8, 16,000, 2,048 x 1,024 (256) 88 / 122; 64, 32,768, 512 x 512 (256) 56 / 90.  Below the rule's
// bound groups of one size would gain what others lose more of, and the host knows no sizes.  Even / exponentially distributed sizes, 128 wide
// and 256: 8, 16,000, 2,048 x 1,024 77 / 81 and 69 / 147; 64, 32,768, 512 x 512 40 / 48 and 34 / 55; 16, 16,384, 1,024 x 1,024 (256) 54 / 68 and
// 42 / 89; above it 16, 32,768, 2,048 x 2,048 (1,024) 333 / 359 and 275 / 278; 8, 16,384, 2,048 x 2,048 (512) 143 / 151 and 132 / 166.
bool large_weight_tiles(int G, int F_in, int F_out) {
    const int64_t tiles = (int64_t)G * ((F_in + 255) / 256) * ((F_out + 255) / 256);
    return F_in >= 256 && fills(F_out) && (double)tiles >= kUnits / 2 * (std::log((double)G) + 0.58);
}

template <class T, int MODE>
int launch_rows(const GroupedArgs& g, bool direct, hipStream_t s) {
    const int N = MODE == kInput ? g.F_in : g.F_out, K = MODE == kInput ? g.F_out : g.F_in;
    if constexpr (sizeof(T) == 4)
        if (narrow_rows(g.m, K, N)) return launch_narrow_rows(MODE == kInput, g, s);
    if (few_rows(sizeof(T) == 4, MODE == kInput, direct, g.m, g.G, K, N))
        return launch_few(sizeof(T) == 4 ? EPP_FLOAT32 : std::is_same_v<T, __bf16> ? EPP_BFLOAT16 : EPP_FLOAT16, MODE == kInput, direct, g, s);
    if constexpr (sizeof(T) == 2) {
        const bool large = large_tiles(g.m / 256 + g.G / 2, N);
        if (direct && large) return launch_rows_of<T, MODE, 2, 4, 4, 2, true, true>(g, s);
        if constexpr (MODE == kInput)
            if (large) return launch_rows_of<T, MODE, 2, 4, 4, 2, false, true>(g, s);
    }
    if (sizeof(T) == 4 || small_tiles((g.m / 128 + g.G / 2) * ((N + 127) / 128))) {
        if constexpr (sizeof(T) == 2)
            if (direct && (g.m / 64 + g.G / 2) * ((N + 63) / 64) <= kUnits) return launch_rows_of<T, MODE, 2, 2, 1, 1, true, false, 4>(g, s);
        if (direct) return launch_rows_of<T, MODE, 2, 2, 1, 1, true, false>(g, s);
        return launch_rows_of<T, MODE, 2, 2, 1, 1, false, false>(g, s);
    }
    if constexpr (sizeof(T) == 2) {
        if (direct) return launch_rows_of<T, MODE, 2, 2, 2, 2, true, false>(g, s);
        return launch_rows_of<T, MODE, 2, 2, 2, 2, false, false>(g, s);
    }
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
        overlaps_block(*out, w_out, size, offsets, 4 * ((int64_t)G + 1)) ||
        (in->rows && overlaps_block(*out, w_out, size, in->rows, 4 * m)) || (out->rows && overlaps_block(*out, w_out, size, out->rows, 4 * m)))
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
    // (with a list of rows, direct loads find them by 32 bits; and there has to be one)
    const bool direct = aligned(g.a, w_in * size) && reinterpret_cast<uintptr_t>(W) % 16 == 0 && (F_out * size) % 16 == 0 && in->n > 0 && g.a.ld < (1 << 24) &&
                        (!in->rows || g.a.n * g.a.ld < (1ll << 32));
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
Chunks chunking(bool fp32, int64_t m, int G, int F_in, int F_out) {
    if (fp32 && narrow_weight(m, F_in, F_out)) {
        const int64_t per = narrow_weight_chunk(m);
        return {per, std::max<int64_t>(most_tiles(m, G, per), 1)};
    }
    // A group's entries are one workgroup's, about 0.7 us a tile of them; groups differ in size, so the longest is taken to have twice the
    // average.  Cut into n chunks, that takes an n-th, and the partial sums of all chunks are written and read (8 bytes an element at
    // about 2.7 TB/s) and added by a launch of 5 us.  4 groups, bfloat16, whole / cut, us: 30,000 entries, 1,024 x 1,024 162 / 100;
    // 2,000 of the same 17 / 32; 2,000, 160 x 100 17.6 / 10.8.
    const double longest = std::min<double>((double)m, 2.0 * (double)m / G), whole = 0.7 * longest / (fp32 ? 32 : 64);
    const double each = 0.5 * G * F_in * F_out * 3e-6;
    const int64_t tiles = (int64_t)((F_in + 63) / 64) * ((F_out + 63) / 64), at_once = tiles * ((G + 1) / 2);
    const double most = (double)((8 * kUnits + at_once - 1) / at_once);  // (more than eight workgroups to a compute unit gain nothing)
    const double n = std::min(std::sqrt(whole / each), most);
    if (n < 2.0 || whole / n + n * each + 5.0 >= whole) return {0, G};
    const int64_t per = ((int64_t)(longest / n) / 64 + 1) * 64;
    return {per, most_tiles(m, G, per)};
}

template <class T, class TO, int WM, int WN, int BM, int BN, bool DIRECT, bool LIST, int STAGES = 2>
int launch_weight_of(const GroupedArgs& g, int64_t chunks, hipStream_t s) {
    constexpr int TM = 32 * WM * BM, TN = 32 * WN * BN;
    const int64_t blocks = chunks * ((g.F_in + TM - 1) / TM) * ((g.F_out + TN - 1) / TN);
    EPP_TRY(check_blocks(blocks, 64 * WM * WN));
    hipLaunchKernelGGL((k_grouped_weight<T, TO, WM, WN, BM, BN, DIRECT, LIST, STAGES>), dim3((unsigned)blocks), dim3(64 * WM * WN), 0, s, g);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}

template <class T, class TO>
int launch_weight_tiles(const GroupedArgs& g, int64_t chunks, bool direct, hipStream_t s) {
    if constexpr (sizeof(T) == 2)
        if (!g.per && large_weight_tiles(g.G, g.F_in, g.F_out)) {
            if (!direct) return launch_weight_of<T, TO, 2, 4, 4, 2, false, true>(g, chunks, s);
            if (g.a.rows || g.b.rows) return launch_weight_of<T, TO, 2, 4, 4, 2, true, true>(g, chunks, s);
            return launch_weight_of<T, TO, 2, 4, 4, 2, true, false>(g, chunks, s);
        }
    const bool list = g.a.rows || g.b.rows;
    if (sizeof(T) == 4 || small_tiles(chunks * ((g.F_in + 127) / 128) * ((g.F_out + 127) / 128))) {
        if (direct && list) return launch_weight_of<T, TO, 2, 2, 1, 1, true, true>(g, chunks, s);
        if (direct) return launch_weight_of<T, TO, 2, 2, 1, 1, true, false>(g, chunks, s);
        return launch_weight_of<T, TO, 2, 2, 1, 1, false, true>(g, chunks, s);
    }
    if constexpr (sizeof(T) == 2) {
        if (direct && list) return launch_weight_of<T, TO, 2, 2, 2, 2, true, true>(g, chunks, s);
        if (direct) return launch_weight_of<T, TO, 2, 2, 2, 2, true, false>(g, chunks, s);
        return launch_weight_of<T, TO, 2, 2, 2, 2, false, true>(g, chunks, s);
    }
}

template <class TO>
int launch_sum(const GroupedArgs& g, int64_t chunks, TO* grad_W, hipStream_t s) {
    // (many chunks of small matrices: 16 threads to an element)
    const int64_t quads = ((int64_t)g.F_in * g.F_out + 3) / 4;
    if (chunks >= 16 * (int64_t)g.G) hipLaunchKernelGGL((k_grouped_sum<TO, 16>), dim3((unsigned)((quads + 15) / 16), (unsigned)g.G), dim3(256), 0, s, g, grad_W);
    else hipLaunchKernelGGL((k_grouped_sum<TO, 1>), dim3((unsigned)((quads + 255) / 256), (unsigned)g.G), dim3(256), 0, s, g, grad_W);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}

template <class T, class TO>
int launch_weight(GroupedArgs g, const Chunks& c, bool direct, TO* grad_W, hipStream_t s) {
    if constexpr (sizeof(T) == 4)
        if (narrow_weight(g.m, g.F_in, g.F_out)) {
            EPP_TRY(launch_narrow_weight(g, c.count, s));
            return launch_sum<TO>(g, c.count, grad_W, s);
        }
    if (!c.per) {
        g.out.data = reinterpret_cast<const char*>(grad_W);
        return launch_weight_tiles<T, TO>(g, c.count, direct, s);
    }
    EPP_TRY((launch_weight_tiles<T, float>(g, c.count, direct, s)));
    return launch_sum<TO>(g, c.count, grad_W, s);
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
    int64_t bytes = 16;  // (for operands of any type)
    for (const bool fp32 : {false, true}) {
        const Chunks c = chunking(fp32, m, G, F_in, F_out);
        if (c.per) bytes = std::max<int64_t>(bytes, c.count * F_in * F_out * (int64_t)sizeof(float));
    }
    return bytes;
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
         reinterpret_cast<uintptr_t>(grad_W) < reinterpret_cast<uintptr_t>(workspace) + (uintptr_t)need) ||
        overlaps_list(offsets, (int64_t)G + 1, grad_W, w_bytes) || overlaps_list(offsets, (int64_t)G + 1, workspace, need) ||
        overlaps_list(X->rows, m, grad_W, w_bytes) || overlaps_list(X->rows, m, workspace, need) ||
        overlaps_list(grad_out->rows, m, grad_W, w_bytes) || overlaps_list(grad_out->rows, m, workspace, need))
        return aliased();
    GroupedArgs g = {};
    g.a = side(*X, size);
    g.b = side(*grad_out, size);
    g.offsets = offsets;
    g.m = m;
    g.G = G;
    g.F_in = F_in;
    g.F_out = F_out;
    const Chunks c = chunking(type == EPP_FLOAT32, m, G, F_in, F_out);
    g.per = c.per;
    g.chunks = c.count;
    g.part = static_cast<float*>(workspace);
    const bool direct = aligned(g.a, F_in * size) && aligned(g.b, F_out * size) && std::max(g.a.ld, g.b.ld) < (1 << 26);
    hipStream_t s = (hipStream_t)stream;
    if (type == EPP_FLOAT32) return launch_weight<float, float>(g, c, direct, static_cast<float*>(grad_W), s);
    if (type == EPP_BFLOAT16) {
        if (grad_W_type == EPP_FLOAT32) return launch_weight<__bf16, float>(g, c, direct, static_cast<float*>(grad_W), s);
        return launch_weight<__bf16, __bf16>(g, c, direct, static_cast<__bf16*>(grad_W), s);
    }
    if (grad_W_type == EPP_FLOAT32) return launch_weight<_Float16, float>(g, c, direct, static_cast<float*>(grad_W), s);
    return launch_weight<_Float16, _Float16>(g, c, direct, static_cast<_Float16*>(grad_W), s);
}
