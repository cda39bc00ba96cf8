// What the grouped products' kernels share (csrc/epp_grouped.hip, csrc/epp_grouped_narrow.hip, csrc/epp_grouped_few.hip).
#pragma once

#include "epp_internal.h"

namespace epp_grouped {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned int uintx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfloatx8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));

constexpr int kUnits = 256;  // compute units

enum Mode { kProduct, kInput, kWeight };

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
    int64_t per;        // weight gradient: entries to a chunk (0: whole groups)
    int64_t chunks;     // .. how many chunks there can be (offsets that descend name more of them)
    float* part;        // .. and their partial sums
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

// The same value in all lanes, and the compiler told so.
__device__ __forceinline__ int64_t uniform(int64_t x) {
    return (int64_t)((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)x) | (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32);
}
__device__ __forceinline__ const char* uniform(const char* p) { return reinterpret_cast<const char*>(uniform(reinterpret_cast<int64_t>(p))); }

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
        const int tiles = hi > lo ? (int)((uint32_t)(hi - lo + per - 1) / (uint32_t)per) : 0;
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
    *total = uniform(before);
    found.g = __builtin_amdgcn_readfirstlane(found.g);
    return found;
}

__device__ __forceinline__ int64_t row_of(const Side& s, int64_t i, bool valid) {  // -1: no such row
    if (!valid) return -1;
    const int64_t r = s.rows ? (int64_t)s.rows[i] : i;
    return r >= 0 && r < s.n ? r : -1;
}
__device__ __forceinline__ unsigned lds_address(const void* p) {
    return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
// 16 bytes a lane into LDS, lane after lane from `to` on.  Complete once vmcnt says so (wait_and_meet).  (Not the compiler's builtin: it waits
// for all of these loads before every transposing LDS read, those of the next tile included.  m0 is named as
// changed, of which the compiler warns that it is a register that it reserves: it keeps values there from one of its own uses to the next.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(const char* from, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void load_to_lds(const char* base, unsigned off, unsigned to) {  // (base the same in all lanes)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load4_to_lds(const char* from, unsigned to) {  // (4 bytes a lane)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "memory", "m0");
}
#pragma clang diagnostic pop

// Between a wavefront's own writes to LDS and reads by other lanes of it, both ways: LDS serves them in order, and the compiler keeps it.
__device__ __forceinline__ void in_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Pieces through registers.  One that the line's end cuts short is loaded so that it ends there, and shifted into place when it is put into
// LDS: a load under a condition would be waited for where it stands.  Lines shorter than a piece are loaded element by element.
typedef unsigned int any_uintx4 __attribute__((ext_vector_type(4), aligned(2)));

template <class T>
__device__ __forceinline__ uintx4 load_short(const char* p, int valid) {
    constexpr int E = 16 / (int)sizeof(T);
    uintx4 v = {0, 0, 0, 0};
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
// The piece at p, of which `valid` elements are inside its line; zeros for none of them.
template <class T>
__device__ __forceinline__ uintx4 load_piece(const char* p, int valid, bool short_line, const char* zeros) {
    constexpr int E = 16 / (int)sizeof(T);
    if (short_line) return load_short<T>(p, valid);
    return *reinterpret_cast<const any_uintx4*>(valid <= 0 ? zeros : valid >= E ? p : p - (E - valid) * (int)sizeof(T));
}
__device__ __forceinline__ uintx4 shifted(uintx4 v, int bits) {  // to lower addresses, zeros behind
    unsigned long long lo = (unsigned long long)v[1] << 32 | v[0], hi = (unsigned long long)v[3] << 32 | v[2];
    if (bits >= 64) {
        lo = hi;
        hi = 0;
    }
    const int s = bits & 63;
    lo = s ? lo >> s | hi << (64 - s) : lo;
    hi >>= s;
    return uintx4{(unsigned int)lo, (unsigned int)(lo >> 32), (unsigned int)hi, (unsigned int)(hi >> 32)};
}
// What a piece of `valid` elements is to be shifted by.
template <class T>
__device__ __forceinline__ int shift_of(int valid, bool short_line) {
    constexpr int E = 16 / (int)sizeof(T);
    return valid > 0 && valid < E && !short_line ? (E - valid) * 8 * (int)sizeof(T) : 0;
}

// Four neighbouring results of a row; `valid` of them exist.  (A store needs no alignment beyond the element's.)
template <class T>
__device__ __forceinline__ void store4(char* row, int col, const float (&x)[4], int valid) {
    T* p = reinterpret_cast<T*>(row) + col;
    if (valid >= 4) {
        typedef T vec4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
        *reinterpret_cast<vec4*>(p) = vec4{Num<T>::from(x[0]), Num<T>::from(x[1]), Num<T>::from(x[2]), Num<T>::from(x[3])};
    } else {
#pragma unroll
        for (int c = 0; c < 3; ++c)
            if (c < valid) p[c] = Num<T>::from(x[c]);
    }
}

// Kernels for few rows to a group (csrc/epp_grouped_few.hip).
bool few_rows(bool fp32, bool input, bool direct, int64_t m, int G, int K, int N);
int launch_few(int type, bool input, bool direct, const GroupedArgs& g, hipStream_t s);

// Kernels of their own for narrow fp32 matrices (csrc/epp_grouped_narrow.hip).
bool narrow_rows(int64_t m, int K, int N);  // of contraction K onto N columns
int launch_narrow_rows(bool input, const GroupedArgs& g, hipStream_t s);
bool narrow_weight(int64_t m, int F_in, int F_out);
int64_t narrow_weight_chunk(int64_t m);  // entries to a chunk of partial sums
int launch_narrow_weight(const GroupedArgs& g, int64_t chunks, hipStream_t s);

}  // namespace epp_grouped
