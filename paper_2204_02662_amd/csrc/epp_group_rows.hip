// Entries brought into the order of their groups (a counting sort that keeps the order of a group's entries): what the grouped
// products need of a router's choices, or of the types of a graph's active vertices.
//
// Few entries: one workgroup counts, sums and places them.  Many: blocks of consecutive entries are counted, and then place their
// entries; the counts of the blocks before are added up by every block itself where they are few, else by a wavefront per group in a
// launch between.  A wavefront finds an entry's rank among its 64 by ballots over the bits of the group's number; nothing depends on the
// order in which blocks or wavefronts run.  Few bytes, and bound by the steps that wait for each other: 1,000,000 entries of 8 groups, 8 MB,
// take 13.7 us where a copy takes 1.6.
// Group G stands for "no group": its entries come last.

#include "epp_internal.h"

namespace {

constexpr int kMaxGroups = 2048;
constexpr int kFew = 8192, kFewWaves = 16;
constexpr int kWaves = 4, kBlockEntries = 2048, kMostBlocks = 1024;
// Groups whose counts every block adds up itself, one after the other, instead of a launch of its own: 100,000 entries, 8 groups, 9.9 us with two
// launches; 20,000, 256 groups, 45 us with two, 14 with three.
constexpr int kFewSums = 32;

struct GroupRowsArgs {
    const int32_t* group_of;
    const int32_t* rows;  // NULL: entry i is row i
    int64_t n, m, per;    // per: entries to a block
    int G, bits, blocks;
    int32_t *offsets, *order;
    int32_t *counts, *totals;  // counts[group][block], totals[group] (NULL: counts are few, and not yet summed over the blocks)
};

// Rows and groups of up to kAhead times 64 entries [first, last) (at least one), a lane's share: entry first + 64 j + lane.  All of their rows are on
// their way together, and then all of their groups.
constexpr int kAhead = kBlockEntries / kWaves / 64;
struct Entries {
    int32_t row[kAhead], group[kAhead];
    __device__ __forceinline__ void load(const GroupRowsArgs& a, int64_t first, int64_t last) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int64_t i = min(first + 64 * j + lane, last - 1);
            row[j] = a.rows ? a.rows[i] : (int32_t)i;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) group[j] = row[j] >= 0 && row[j] < a.n ? a.group_of[row[j]] : -1;
    }
    // Adds the entries' groups to count[].
    __device__ __forceinline__ void count(const GroupRowsArgs& a, int64_t first, int64_t last, int32_t* count) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (first + 64 * j + lane < last) atomicAdd(&count[group[j] >= 0 && group[j] < a.G ? group[j] : a.G], 1);
    }
    // Places the entries from next[] on, which is the calling wavefront's own.
    __device__ __forceinline__ void place(const GroupRowsArgs& a, int64_t first, int64_t last, volatile int32_t* next) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (first + 64 * j >= last) break;
            const bool have = first + 64 * j + lane < last;
            const int g = group[j] >= 0 && group[j] < a.G ? group[j] : a.G;
            unsigned long long same = __ballot(have);
            for (int b = 0; b < a.bits; ++b) {
                const unsigned long long set = __ballot((g >> b) & 1);
                same &= (g >> b) & 1 ? set : ~set;
            }
            const int rank = __popcll(same & ((1ull << lane) - 1));
            if (have) {
                const int32_t at = next[g];
                __builtin_amdgcn_wave_barrier();
                if (rank == 0) next[g] = at + __popcll(same);
                __builtin_amdgcn_wave_barrier();
                a.order[at + rank] = row[j];
            }
        }
    }
};

// The same for any number of entries of the calling wavefront.
__device__ __forceinline__ void count_entries(const GroupRowsArgs& a, int64_t first, int64_t last, int32_t* count) {
    for (int64_t i = first; i < last; i += 64 * kAhead) {
        Entries e;
        e.load(a, i, last);
        e.count(a, i, last, count);
    }
}
__device__ __forceinline__ void place_entries(const GroupRowsArgs& a, int64_t first, int64_t last, volatile int32_t* next) {
    for (int64_t i = first; i < last; i += 64 * kAhead) {
        Entries e;
        e.load(a, i, last);
        e.place(a, i, last, next);
    }
}

// Exclusive sums over `n` values, 64 at a time, by one wavefront.  Returns the sum of all.
__device__ __forceinline__ int32_t exclusive_sums(int32_t* v, int n) {
    const int lane = threadIdx.x & 63;
    int32_t before = 0;
    for (int i0 = 0; i0 < n; i0 += 64) {
        const int i = i0 + lane;
        const int32_t mine = i < n ? v[i] : 0;
        int32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int32_t x = __shfl_up(upto, d, 64);
            if (lane >= d) upto += x;
        }
        if (i < n) v[i] = before + upto - mine;
        before += __shfl(upto, 63, 64);
    }
    return before;
}

template <int MOST>  // groups
__global__ __launch_bounds__(64 * kFewWaves) void k_group_few(GroupRowsArgs a) {
    __shared__ int32_t next[kFewWaves][MOST + 1];
    __shared__ int32_t begin[MOST + 1];
    const int t = threadIdx.x, w = t >> 6, groups = a.G + 1;
    for (int i = t; i < kFewWaves * groups; i += 64 * kFewWaves) next[i / groups][i % groups] = 0;
    __syncthreads();
    const int64_t per = ((a.m + kFewWaves - 1) / kFewWaves + 63) / 64 * 64;
    const int64_t first = min(w * per, a.m), last = min(first + per, a.m);
    count_entries(a, first, last, next[w]);
    __syncthreads();
    for (int g = t; g < groups; g += 64 * kFewWaves) {
        int32_t sum = 0;
#pragma unroll
        for (int x = 0; x < kFewWaves; ++x) sum += next[x][g];
        begin[g] = sum;
    }
    __syncthreads();
    if (w == 0) exclusive_sums(begin, groups);
    __syncthreads();
    for (int g = t; g < groups; g += 64 * kFewWaves) {
        int32_t sum = begin[g];
        a.offsets[g] = sum;  // (groups = G + 1: the last one is where the rest begins)
#pragma unroll
        for (int x = 0; x < kFewWaves; ++x) {
            const int32_t c = next[x][g];
            next[x][g] = sum;
            sum += c;
        }
    }
    __syncthreads();
    place_entries(a, first, last, next[w]);
}

__global__ __launch_bounds__(64 * kWaves) void k_group_count(GroupRowsArgs a) {
    extern __shared__ int32_t count[];
    const int t = threadIdx.x, groups = a.G + 1;
    for (int g = t; g < groups; g += 64 * kWaves) count[g] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * a.per, share = a.per / kWaves;
    const int64_t mine = min(first + (t >> 6) * share, a.m);
    count_entries(a, mine, min(mine + share, a.m), count);
    __syncthreads();
    for (int g = t; g < groups; g += 64 * kWaves) a.counts[(int64_t)g * a.blocks + blockIdx.x] = count[g];
}

// A wavefront per group: the sums of its counts up to every block, and of all.
__global__ __launch_bounds__(64) void k_group_sums(GroupRowsArgs a) {
    const int32_t total = exclusive_sums(a.counts + (int64_t)blockIdx.x * a.blocks, a.blocks);
    if (threadIdx.x == 0) a.totals[blockIdx.x] = total;
}

__global__ __launch_bounds__(64 * kWaves) void k_group_place(GroupRowsArgs a) {
    extern __shared__ int32_t next[];  // [wavefront][group], and before that the groups' beginnings in the first row
    __shared__ int32_t before_here[kFewSums + 1];
    const int t = threadIdx.x, w = t >> 6, groups = a.G + 1;
    const int64_t first = (int64_t)blockIdx.x * a.per, share = a.per / kWaves;
    const int64_t mine = min(first + w * share, a.m), last = min(mine + share, a.m);
    const bool once = a.per == kBlockEntries && mine < last;  // few enough entries to hold: they are looked up once, and while the counts are added up
    Entries held;
    if (once) held.load(a, mine, last);
    for (int i = groups + t; i < kWaves * groups; i += 64 * kWaves) next[i] = 0;
    if (a.totals) {
        for (int i = t; i < groups; i += 64 * kWaves) next[i] = a.totals[i];
    } else {  // few counts: every block adds them up itself (the second row of next[]: those of the blocks before)
        const int lane = t & 63;
        for (int g = w; g < groups; g += kWaves) {
            int32_t before = 0, all = 0;
#pragma unroll 8
            for (int i = lane; i < a.blocks; i += 64) {
                const int32_t c = a.counts[g * a.blocks + i];
                all += c;
                if (i < (int)blockIdx.x) before += c;
            }
#pragma unroll
            for (int d = 32; d; d /= 2) {
                before += __shfl_xor(before, d, 64);
                all += __shfl_xor(all, d, 64);
            }
            if (lane == 0) {
                next[g] = all;
                before_here[g] = before;
            }
        }
    }
    __syncthreads();
    if (w == 0) exclusive_sums(next, groups);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int g = t; g < groups; g += 64 * kWaves) a.offsets[g] = next[g];
    // next[x][g], x >= 1: what wavefronts before x have of group g, after the sums below
    if (w + 1 < kWaves) {
        if (once) held.count(a, mine, last, next + (w + 1) * groups);
        else count_entries(a, mine, last, next + (w + 1) * groups);
    }
    __syncthreads();
    for (int g = t; g < groups; g += 64 * kWaves) {
        int32_t sum = next[g] + (a.totals ? a.counts[(int64_t)g * a.blocks + blockIdx.x] : before_here[g]);
        next[g] = sum;
#pragma unroll
        for (int x = 1; x < kWaves; ++x) {
            sum += next[x * groups + g];
            next[x * groups + g] = sum;
        }
    }
    __syncthreads();
    if (once) held.place(a, mine, last, next + w * groups);
    else place_entries(a, mine, last, next + w * groups);
}

int check(int64_t m, int G) {
    if (m < 0) { epp_set_error("%lld entries", (long long)m); return EPP_ERR_INVALID_ARG; }
    if (m >= (1ll << 31)) { epp_set_error("%lld entries (up to 2^31 - 1)", (long long)m); return EPP_ERR_TOO_LARGE; }
    if (G < 1) { epp_set_error("%d groups", G); return EPP_ERR_INVALID_ARG; }
    if (G > kMaxGroups) { epp_set_error("%d groups (up to %d)", G, kMaxGroups); return EPP_ERR_TOO_LARGE; }
    return EPP_OK;
}
bool few(int64_t m) { return m <= kFew; }
// Entries to a block: enough blocks to fill the chip, and not so many that their counts would be what takes time.
int64_t block_entries(int64_t m) {
    const int64_t least = (m + kMostBlocks - 1) / kMostBlocks;
    return std::max<int64_t>((least + kBlockEntries - 1) / kBlockEntries, 1) * kBlockEntries;
}

}  // namespace

extern "C" int64_t epp_group_rows_workspace(int64_t m, int G) {
    EPP_TRY(check(m, G));
    if (few(m)) return 16;
    const int64_t per = block_entries(m), blocks = (m + per - 1) / per;
    return (std::max<int64_t>(blocks, 1) + 1) * ((int64_t)G + 1) * 4;
}

extern "C" int epp_group_rows(const int32_t* group_of, int64_t n, const int32_t* rows, int64_t m, int G, int32_t* offsets, int32_t* order,
                              void* workspace, int64_t workspace_bytes, epp_stream_t stream) {
    EPP_TRY(check(m, G));
    if (n < 0 || n >= (1ll << 31)) { epp_set_error("%lld rows", (long long)n); return n < 0 ? EPP_ERR_INVALID_ARG : EPP_ERR_TOO_LARGE; }
    if (!offsets || !workspace || (m > 0 && !order) || (m > 0 && n > 0 && !group_of)) { epp_set_error("NULL argument"); return EPP_ERR_INVALID_ARG; }
    if (!rows && n != m) { epp_set_error("%lld entries, %lld rows and no list of rows", (long long)m, (long long)n); return EPP_ERR_INVALID_ARG; }
    if ((reinterpret_cast<uintptr_t>(group_of) | reinterpret_cast<uintptr_t>(rows) | reinterpret_cast<uintptr_t>(offsets) | reinterpret_cast<uintptr_t>(order)) & 3) {
        epp_set_error("address not aligned to its elements");
        return EPP_ERR_INVALID_ARG;
    }
    const int64_t need = epp_group_rows_workspace(m, G);
    if (workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15)) {
        epp_set_error("workspace of %lld bytes (need %lld, 16-byte aligned)", (long long)workspace_bytes, (long long)need);
        return EPP_ERR_INVALID_ARG;
    }
    const struct { const void* p; int64_t bytes; } blocks[] = {{order, 4 * m}, {offsets, 4 * ((int64_t)G + 1)}, {workspace, need}, {group_of, 4 * n}, {rows, rows ? 4 * m : 0}};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 5; ++j) {
            const uintptr_t x = reinterpret_cast<uintptr_t>(blocks[i].p), y = reinterpret_cast<uintptr_t>(blocks[j].p);
            if (blocks[i].bytes > 0 && blocks[j].bytes > 0 && x < y + (uintptr_t)blocks[j].bytes && y < x + (uintptr_t)blocks[i].bytes) {
                epp_set_error("arrays must not alias");
                return EPP_ERR_INVALID_ARG;
            }
        }
    GroupRowsArgs a = {};
    a.group_of = group_of;
    a.rows = rows;
    a.n = n;
    a.m = m;
    a.G = G;
    while ((1 << a.bits) <= G) ++a.bits;
    a.offsets = offsets;
    a.order = order;
    hipStream_t s = (hipStream_t)stream;
    if (few(m)) {
        if (G <= 256) hipLaunchKernelGGL((k_group_few<256>), dim3(1), dim3(64 * kFewWaves), 0, s, a);
        else hipLaunchKernelGGL((k_group_few<kMaxGroups>), dim3(1), dim3(64 * kFewWaves), 0, s, a);
        EPP_HIP_TRY(hipGetLastError());
        return EPP_OK;
    }
    a.per = block_entries(m);
    a.blocks = (int)std::max<int64_t>((m + a.per - 1) / a.per, 1);
    a.counts = static_cast<int32_t*>(workspace);
    const bool sums = G > kFewSums;
    if (sums) a.totals = a.counts + (int64_t)a.blocks * (G + 1);
    hipLaunchKernelGGL(k_group_count, dim3((unsigned)a.blocks), dim3(64 * kWaves), (size_t)(G + 1) * 4, s, a);
    EPP_HIP_TRY(hipGetLastError());
    if (sums) {
        hipLaunchKernelGGL(k_group_sums, dim3((unsigned)(G + 1)), dim3(64), 0, s, a);
        EPP_HIP_TRY(hipGetLastError());
    }
    hipLaunchKernelGGL(k_group_place, dim3((unsigned)a.blocks), dim3(64 * kWaves), (size_t)kWaves * (size_t)(G + 1) * 4, s, a);
    EPP_HIP_TRY(hipGetLastError());
    return EPP_OK;
}
