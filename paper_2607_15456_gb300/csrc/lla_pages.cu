// lla_pages.cu -- sequences that share pages of the paged caches: fork, growth, freeing and compaction
// (lla_pages_*).  The ledger is ref_count alone: block b is free where ref_count[b] is 0, and a new page is
// always the free block of the lowest number.  So every result is a function of the inputs, whatever order
// threads run in: counts are integer sums, block ids are ranks from prefix sums.
//
// What bounds them: latency until pages are copied (a table row of the headline batch is 200 bytes, the ledger of a
// 280 GB pool of 24 layers 90 KB), HBM where they are.  Fork 3.7 us a launch for 64 sequences of 4 k tokens, 8 us for
// 1024 of 32 k; copied last pages of 64 beams in 24 layers (128 MB, 18.9 us at the copy rate) 20 us, with 4-byte granules (136 MB,
// runs of 4 to 252 bytes) 30 us; compaction at the copy rate (1.31 GB in 196 us).  A growth by one token without copies, both
// launches, takes 5 us with 4 k blocks, 6 with 64 k, 11 with a million and 99 with 2^24; a compaction without pools, 60 % of the blocks in use,
// 8, 13, 97 and 1512 us: the ledger is gone through twice by at most eight SMs (280 GB hold 2e4 to 1e5 blocks of the models here).
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "lla_device.cuh"
#include "lla_internal.h"
#include "lla_units.cuh"

namespace lla {
namespace {

namespace cg = cooperative_groups;

// Pages that hold `len` tokens (0 <= len <= 64 * LLA_MAX_BLOCKS).
__device__ __forceinline__ int pages_of(int len) {
    return static_cast<int>((static_cast<unsigned>(len) + kBlockTokens - 1) / kBlockTokens);
}

// A sequence's length if its table row can hold it, else -1.
__device__ __forceinline__ int checked_len(int len, int max_blocks) {
    return len >= 0 && len <= static_cast<int64_t>(max_blocks) * kBlockTokens ? len : -1;
}

// ------------------------------------------------------------------------------------------------ fork

constexpr int kForkThreads = 128;
constexpr int kForkSpan = 1024;  // table entries of a CTA

struct ForkArgs {
    int32_t *ref;
    int nb;
    const int32_t *from_table, *from_lens;
    int from_max, from_S;
    int32_t *to_table, *to_lens;
    int to_max, to_S;
    const int32_t *parents;
    int keep;  // parent -1 stands for the sequence itself (from_S == to_S)
    unsigned *err;
};
__device__ __forceinline__ int parent_of(const ForkArgs &a, int s) {
    const int p = a.parents[s];
    return p == -1 && a.keep ? s : p;
}

// Rows 0 .. to_S-1 of the grid copy a child's table (a CTA per kForkSpan entries, so that one long parent of many
// children spreads over the SMs); rows to_S .. to_S+from_S-1 change the counts of a parent's
// pages by its children - 1, once for all of its children, and not at all for the usual parent of one child.
__global__ void __launch_bounds__(kForkThreads) fork_kernel(const ForkArgs a) {
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x;
    unsigned bad = 0;
    if (static_cast<int>(blockIdx.x) < a.to_S) {
        const int s = blockIdx.x;
        const int p = parent_of(a, s);
        int len = 0;
        if (p < -1 || p >= a.from_S) {
            bad = LLA_DEVERR_SEQUENCE;
        } else if (p >= 0) {
            len = checked_len(a.from_lens[p], a.from_max);
            if (len < 0 || pages_of(len) > a.to_max) {
                bad = LLA_DEVERR_CONTEXT;
                len = 0;
            }
        }
        const int n = pages_of(len);
        const int32_t *src = a.from_table + static_cast<int64_t>(p < 0 ? 0 : p) * a.from_max;
        int32_t *dst = a.to_table + static_cast<int64_t>(s) * a.to_max;
        for (int lo = blockIdx.y * kForkSpan; lo < n; lo += gridDim.y * kForkSpan) {
            const int hi = min(n, lo + kForkSpan);
            int v[kForkSpan / kForkThreads];
#pragma unroll
            for (int j = 0; j < kForkSpan / kForkThreads; ++j)
                if (lo + tid + j * kForkThreads < hi) v[j] = src[lo + tid + j * kForkThreads];
#pragma unroll
            for (int j = 0; j < kForkSpan / kForkThreads; ++j)
                if (lo + tid + j * kForkThreads < hi) dst[lo + tid + j * kForkThreads] = v[j];
        }
        if (blockIdx.y == 0 && tid == 0) {
            a.to_lens[s] = len;
            if (bad) atomicOr(a.err, bad);
        }
        return;
    }
    const int p = blockIdx.x - a.to_S;
    const int len = checked_len(a.from_lens[p], a.from_max), n = pages_of(max(0, len));
    const int lo0 = blockIdx.y * kForkSpan;
    if (len < 0 && blockIdx.y == 0 && tid == 0) atomicOr(a.err, LLA_DEVERR_CONTEXT);  // its pages stay counted
    if (lo0 >= n) return;
    const int32_t *row = a.from_table + static_cast<int64_t>(p) * a.from_max;
    constexpr int kEach = kForkSpan / kForkThreads;
    int v[kEach];  // the first span's blocks, read while the children are counted
#pragma unroll
    for (int j = 0; j < kEach; ++j) v[j] = lo0 + tid + j * kForkThreads < n ? row[lo0 + tid + j * kForkThreads] : 0;
    int mine = 0;
    if (n <= a.to_max) {
#pragma unroll
        for (int j = 0; j < LLA_MAX_BATCH / kForkThreads; ++j) {
            const int i = tid + j * kForkThreads;
            if (i < a.to_S) mine += parent_of(a, i) == p;
        }
    }
    __shared__ int children[kForkThreads / 32];
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (tid % 32 == 0) children[tid / 32] = mine;
    __syncthreads();
    int change = -1;
#pragma unroll
    for (int w = 0; w < kForkThreads / 32; ++w) change += children[w];
    for (int lo = lo0; lo < n; lo += gridDim.y * kForkSpan) {
        const int hi = min(n, lo + kForkSpan);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int i = lo + tid + j * kForkThreads;
            if (i >= hi) break;
            const int b = lo == lo0 ? v[j] : row[i];
            if (b < 0 || b >= a.nb)
                bad = LLA_DEVERR_BLOCK_ID;
            else if (change)
                atomicAdd(a.ref + b, change);
        }
    }
    if (bad) atomicOr(a.err, bad);
}

// ------------------------------------------------------------------------------------------------ free

constexpr int kFreeThreads = 256;

// One CTA per listed sequence.  The exchange of the length makes a second mention of a sequence find it empty.
__global__ void __launch_bounds__(kFreeThreads)
free_kernel(int32_t *ref, int nb, const int32_t *table, int max_blocks, int32_t *lens, int S, const int32_t *seqs,
            unsigned *err) {
    __shared__ int held;
    pdl_wait();
    pdl_trigger();
    const int s = seqs[blockIdx.x];
    if (s < 0) return;
    if (s >= S) {
        if (threadIdx.x == 0) atomicOr(err, LLA_DEVERR_SEQUENCE);
        return;
    }
    if (threadIdx.x == 0) {
        const int len = checked_len(atomicExch(lens + s, 0), max_blocks);
        if (len < 0) atomicOr(err, LLA_DEVERR_CONTEXT);
        held = pages_of(max(0, len));
    }
    __syncthreads();
    const int n = held;
    const int32_t *row = table + static_cast<int64_t>(s) * max_blocks;
    bool bad = false;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kFreeThreads) {
        const int b = row[i];
        if (b < 0 || b >= nb)
            bad = true;
        else
            atomicSub(ref + b, 1);
    }
    if (bad) atomicOr(err, LLA_DEVERR_BLOCK_ID);
}

// ------------------------------------------------------------------------------- prefix sums of a cluster

constexpr int kPlanThreads = 1024;  // a sequence each, too
static_assert(kPlanThreads == LLA_MAX_BATCH, "thread s plans sequence s");

// Exclusive prefix sums of two values over a CTA's threads, and the CTA's totals.  `part` has 33 entries.  Three barriers.
struct Two {
    unsigned long long a;
    int b;
};
__device__ __forceinline__ Two block_scan(Two v, Two *part, Two &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto scan = [&](Two x) {  // inclusive, of a warp
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long ua = __shfl_up_sync(0xffffffffu, x.a, o);
            const int ub = __shfl_up_sync(0xffffffffu, x.b, o);
            if (lane >= o) {
                x.a += ua;
                x.b += ub;
            }
        }
        return x;
    };
    const Two inc = scan(v);
    __syncthreads();  // part is free
    if (lane == 31) part[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        const Two w = part[lane], all = scan(w);
        part[lane] = Two{all.a - w.a, all.b - w.b};
        if (lane == 31) part[32] = all;
    }
    __syncthreads();
    total = part[32];
    return Two{part[warp].a + inc.a - v.a, part[warp].b + inc.b - v.b};
}

// The ledger entries [begin, end) of a warp of the cluster, 128 at a time: lane l has entries 4 l to 4 l + 3 of them.
struct Segment {
    int begin, end;
};
__device__ __forceinline__ Segment my_segment(int nb, int rank, int ctas) {
    const int warps = ctas * (kPlanThreads / 32);
    const int64_t per = (static_cast<int64_t>(nb) + warps * 128 - 1) / (warps * 128) * 128;
    const int64_t b = (rank * (kPlanThreads / 32) + (threadIdx.x >> 5)) * per;
    Segment s;
    s.begin = static_cast<int>(b < nb ? b : nb);
    s.end = static_cast<int>(b + per < nb ? b + per : nb);
    return s;
}
// The lane's four entries of those from i on; what lies behind the ledger is `none`.
__device__ __forceinline__ int4 ledger_four(const int32_t *ref, int nb, int i, int none) {
    i += (threadIdx.x & 31) * 4;
    if (i + 4 <= nb) return *reinterpret_cast<const int4 *>(ref + i);
    return make_int4(i < nb ? ref[i] : none, i + 1 < nb ? ref[i + 1] : none, i + 2 < nb ? ref[i + 2] : none, none);
}
// Bit k: the k-th of four entries is free, or (FREE false) in use.
template <bool FREE>
__device__ __forceinline__ unsigned four_flags(int4 v) {
    return static_cast<unsigned>((v.x == 0) == FREE) | static_cast<unsigned>((v.y == 0) == FREE) << 1 |
           static_cast<unsigned>((v.z == 0) == FREE) << 2 | static_cast<unsigned>((v.w == 0) == FREE) << 3;
}
// How many of the segment's entries (below `limit`) are free, or in use: a lane's part of it.
template <bool FREE>
__device__ __forceinline__ int count_ledger(const int32_t *ref, int nb, Segment s, int limit) {
    int n = 0;
#pragma unroll 4
    for (int i = s.begin; i < s.end; i += 128) {
        unsigned m = four_flags<FREE>(ledger_four(ref, nb, i, FREE ? 1 : 0));
        const int left = limit - (i + static_cast<int>(threadIdx.x & 31) * 4);
        if (left < 4) m &= left > 0 ? (1u << left) - 1 : 0u;
        n += __popc(m);
    }
    return n;
}
// f(id, counted, rank) for every entry of the segment, rank being the number of counted entries before it; `rank` is that
// of the segment's first entry.  Ends early where no rank below `enough` is left.
template <bool FREE, typename F>
__device__ __forceinline__ void rank_ledger(const int32_t *ref, int nb, Segment s, int rank, int64_t enough, F f) {
    const unsigned lane = threadIdx.x & 31, below = (1u << lane) - 1;
    for (int i = s.begin; i < s.end && rank < enough; i += 128) {
        const unsigned m = four_flags<FREE>(ledger_four(ref, nb, i, FREE ? 1 : 0));
        int r = rank;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned b = __ballot_sync(0xffffffffu, m >> k & 1);
            r += __popc(b & below);
            rank += __popc(b);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int id = i + static_cast<int>(lane) * 4 + k;
            if (id < nb) f(id, (m >> k & 1) != 0, r);
            r += m >> k & 1;
        }
    }
}

// Sums `mine` over the CTAs of the cluster: what the CTAs before this one have, and all.  A cluster barrier lies in
// it: what any CTA did before the call is done after it.  Every CTA must have started (a barrier of the cluster
// before), since its shared memory is written.
struct ClusterSums {
    int before, all;
};
__device__ __forceinline__ ClusterSums cluster_sums(int mine, int *totals /* shared, 16 */) {
    cg::cluster_group cl = cg::this_cluster();
    const int rank = static_cast<int>(cl.block_rank()), n = static_cast<int>(cl.num_blocks());
    if (n == 1) {
        __syncthreads();
        return ClusterSums{0, mine};
    }
    if (threadIdx.x < static_cast<unsigned>(n)) cl.map_shared_rank(totals, threadIdx.x)[rank] = mine;
    cl.sync();
    ClusterSums s = {0, 0};
    for (int r = 0; r < n; ++r) {
        if (r < rank) s.before += totals[r];
        s.all += totals[r];
    }
    return s;
}

// ---------------------------------------------------------------------------------------------- extend

struct ExtendCopy {  // one page to copy: `rows` rows of block src to block dst
    int src, dst, rows, unused;
};
// The workspace: what the plan tells the kernel behind it.
struct ExtendPlan {
    int copies, unused[3];
    ExtendCopy copy[LLA_MAX_BATCH];
    int grow[LLA_MAX_BATCH];    // tokens that sequence s gets
    int before[LLA_MAX_BATCH];  // its length before the call
};

struct ExtendArgs {
    int32_t *ref;
    int nb;
    int32_t *table;
    int max_blocks;
    int32_t *lens;
    int S;
    const int32_t *cu_new;
    int N, per;
    const uint8_t *skip;
    int32_t *lens_before, *free_blocks;
    ExtendPlan *plan;
    unsigned *err;
};

// The plan of a growth, by one cluster.  Thread s of every CTA works out sequence s (the CTAs do the same sums: it
// is less than passing them on), all threads count the free blocks of their part of the ledger, and after the
// cluster's exchange of counts each free block whose rank is below the need knows its sequence by a binary search.
// Everything that is read and later changed (lengths, counts, last pages) is read before that exchange.  The chain is
// length, last page, its count, the meeting in shared memory, the sums: about 5 us, whatever the sizes.
__global__ void __launch_bounds__(kPlanThreads, 1) extend_plan_kernel(const ExtendArgs a) {
    constexpr int kSlots = 2 * LLA_MAX_BATCH;
    __shared__ int key[kSlots], growers[kSlots], lowest[kSlots];
    __shared__ int first[LLA_MAX_BATCH];  // blocks that sequences before s take
    __shared__ int old_pages[LLA_MAX_BATCH], copy_of[LLA_MAX_BATCH];
    __shared__ Two part[33];
    __shared__ int totals[16];
    cg::cluster_group cl = cg::this_cluster();
    const int tid = threadIdx.x, rank = static_cast<int>(cl.block_rank()), ctas = static_cast<int>(cl.num_blocks());
    for (int i = tid; i < kSlots; i += kPlanThreads) {
        key[i] = -1;
        growers[i] = 0;
        lowest[i] = kSlots;
    }
    if (ctas > 1) cl.sync();  // every CTA has started
    pdl_wait();
    pdl_trigger();
    // free blocks of my part of the ledger: its loads are under way beside those of the sequences
    const Segment seg = my_segment(a.nb, rank, ctas);
    const int mine = count_ledger<true>(a.ref, a.nb, seg, a.nb);
    // sequence tid: its growth, and whether others hold its last page
    int len = 0, n = 0, tail = -1, holders = 0;
    unsigned bad = 0;
    if (tid < a.S) {
        len = a.lens[tid];
        int64_t asked = a.per;
        bool in_range = true;
        if (a.cu_new) {
            const int64_t c0 = a.cu_new[tid], c1 = a.cu_new[tid + 1];
            asked = c1 - c0;
            in_range = c0 >= 0 && asked >= 0 && c1 <= a.N;
        }
        if (a.skip && a.skip[tid]) asked = 0;
        if (!in_range || checked_len(len, a.max_blocks) < 0 ||
            len + asked > static_cast<int64_t>(a.max_blocks) * kBlockTokens) {
            bad = LLA_DEVERR_CONTEXT;
            asked = 0;
        }
        n = static_cast<int>(asked);
        if (n > 0 && len % kBlockTokens) {
            tail = a.table[static_cast<int64_t>(tid) * a.max_blocks + len / kBlockTokens];
            if (tail < 0 || tail >= a.nb) {
                bad = LLA_DEVERR_BLOCK_ID;
                n = 0;
            } else {
                holders = a.ref[tail];
            }
        }
    }
    if (bad && rank == 0) atomicOr(a.err, bad);
    int slot = 0;
    const bool shared_tail = n > 0 && holders > 1;
    const bool some_shared = __syncthreads_or(shared_tail);  // (and the table is clear)
    if (shared_tail) {  // the growing holders of a page meet in a hash table: their number and the lowest of them
        slot = (static_cast<unsigned>(tail) * 2654435769u) >> 21;  // golden-ratio hashing to 2048 slots
        for (;;) {
            const int was = atomicCAS(&key[slot], -1, tail);
            if (was == -1 || was == tail) break;
            slot = (slot + 1) % kSlots;
        }
        atomicAdd(&growers[slot], 1);
        atomicMin(&lowest[slot], tid);
    }
    if (some_shared) __syncthreads();
    const int copy = shared_tail && !(growers[slot] >= holders && lowest[slot] == tid);
    const int rows = len % kBlockTokens;
    unsigned long long need = 0;
    if (n > 0) need = static_cast<unsigned long long>(pages_of(len + n) - pages_of(len) + copy);
    // copies in the high bits: at most 2^10, and at most 2^10 * 2^24 blocks in the low ones
    Two total;
    const Two at = block_scan(Two{need | static_cast<unsigned long long>(copy) << 40, mine}, part, total);
    const unsigned long long low40 = (1ull << 40) - 1;
    const int64_t wanted = static_cast<int64_t>(total.a & low40);
    // a need beyond the ledger is not granted, so that what is used of `first` is below 2^24
    const int copy_index = static_cast<int>(at.a >> 40);
    first[tid] = static_cast<int>(min(static_cast<unsigned long long>(LLA_MAX_BLOCKS) * 2, at.a & low40));
    old_pages[tid] = n > 0 ? pages_of(len) : 0;
    copy_of[tid] = copy ? copy_index : -1;
    const ClusterSums free = cluster_sums(total.b, totals);
    const bool granted = wanted <= free.all;
    if (rank == 0) {
        if (tid < a.S) {
            if (a.lens_before) a.lens_before[tid] = len;
            a.plan->grow[tid] = granted ? n : 0;
            a.plan->before[tid] = len;
            if (granted && n > 0) a.lens[tid] = len + n;
            if (granted && copy) {
                ExtendCopy *c = &a.plan->copy[copy_index];
                c->src = tail;
                c->rows = rows;
                atomicSub(a.ref + tail, 1);
            }
        }
        if (tid == 0) {
            a.plan->copies = granted ? static_cast<int>(total.a >> 40) : 0;
            if (a.free_blocks) *a.free_blocks = free.all - (granted ? static_cast<int>(wanted) : 0);
            if (!granted) atomicOr(a.err, LLA_DEVERR_PAGES);
        }
    }
    if (!granted || wanted == 0) return;
    // the k-th free block: to sequence s = the last with first[s] <= k
    const int warp_first = free.before + __shfl_sync(0xffffffffu, at.b, 0);
    rank_ledger<true>(a.ref, a.nb, seg, warp_first, wanted, [&](int id, bool is_free, int k) {
        if (!is_free || k >= wanted) return;
        int lo = 0, hi = a.S - 1;  // first[lo] <= k
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (first[mid] <= k) lo = mid;
            else hi = mid - 1;
        }
        const int i = k - first[lo], c = copy_of[lo];
        // the copied last page comes first, then the fresh ones
        a.table[static_cast<int64_t>(lo) * a.max_blocks + old_pages[lo] + i - (c >= 0)] = id;
        if (c >= 0 && i == 0) a.plan->copy[c].dst = id;
        a.ref[id] = 1;
    });
}

constexpr int kCopyThreads = 256, kCopyWarps = kCopyThreads / 32;
constexpr int kCopyCtas = 4;        // of an SM
constexpr int kSliceBytes = 4096;   // of a full page's plane, moved by a warp at once

// Up to LLA_MAX_POOLS pools.  A page of pool l has slices[l] slices (of its K-plane, then of its V-plane); a CTA takes
// kCopyWarps of them at once, of one page or of several: first[l] is the number of such units that a block has in the
// pools before l.
struct PoolSet {
    lla_pool p[LLA_MAX_POOLS];
    int first[LLA_MAX_POOLS + 1];
    uint16_t slices[LLA_MAX_POOLS];
    int L, alike;     // alike: every pool has first[1] units
    FastDiv by_pool;  // a division by first[1]
};
__host__ __device__ __forceinline__ int k_slices(const lla_pool &p) { return (kBlockTokens * p.k_row_bytes + kSliceBytes - 1) / kSliceBytes; }
__host__ __device__ __forceinline__ int v_slices(const lla_pool &p) { return (kBlockTokens * p.v_row_bytes + kSliceBytes - 1) / kSliceBytes; }

__device__ __forceinline__ int pool_of(const int *first, int L, int unit) {
    int lo = 0, hi = L - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= unit) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

constexpr int kSliceWords = kSliceBytes / 512;  // of 16 bytes, a lane's

// One load or store where `on`.
__device__ __forceinline__ uint4 load_if(const char *p, bool on) {
    uint4 v;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t@p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p), "r"(static_cast<uint32_t>(on)));
    return v;
}
__device__ __forceinline__ void store_if(char *p, const uint4 &v, bool on) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t@p st.global.v4.u32 [%4], {%0, %1, %2, %3};\n\t}" ::"r"(v.x),
                 "r"(v.y), "r"(v.z), "r"(v.w), "l"(p), "r"(static_cast<uint32_t>(on))
                 : "memory");
}

// Behind the plan: the rows of copied pages in every pool, and the slots of the new tokens.  Of a page only the rows
// that hold tokens are read and written: the first `rows` of each K granule, and a prefix of the V-plane.  A warp moves
// a slice, eight words of 16 bytes in flight a lane, and each CTA takes every stride-th unit, so that long and short copies
// mix on every SM.  Slices of 4 KB with four CTAs an SM measured 20.4 us (16-byte granules) and 30 us (4-byte ones); 4 KB and
// five CTAs 23 and 34, 2 KB and six 27 and 45, two slices a warp in flight 3 us more than one.
__global__ void __launch_bounds__(kCopyThreads, kCopyCtas)
extend_finish_kernel(const ExtendArgs a, const __grid_constant__ PoolSet ps, int64_t *slots) {
    pdl_wait();
    pdl_trigger();
    const ExtendPlan *plan = a.plan;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int copies = plan->copies, per_copy = max(1, ps.first[ps.L]), stride = gridDim.x;
    // units in the order of copies, then pools and pages; a CTA takes every stride-th
    const int step_c = stride / per_copy, step_in = stride - step_c * per_copy;
    int c = blockIdx.x / per_copy, in_copy = blockIdx.x - c * per_copy;
    for (; ps.L > 0 && c < copies; c += step_c, in_copy += step_in) {
        if (in_copy >= per_copy) {
            in_copy -= per_copy;
            if (++c >= copies) break;
        }
        const int l = ps.alike ? div_by(in_copy, ps.by_pool) : pool_of(ps.first, ps.L, in_copy);
        const lla_pool pool = ps.p[l];
        const int slices = ps.slices[l], units = (slices + kCopyWarps - 1) / kCopyWarps, in_pool = in_copy - ps.first[l];
        int page, slice;
        if (slices < kCopyWarps) {  // several pages
            const int at_once = kCopyWarps / slices, p = warp / slices;
            page = in_pool * at_once + p;
            slice = warp - p * slices;
            if (p >= at_once) continue;
        } else {
            page = in_pool / units;
            slice = (in_pool - page * units) * kCopyWarps + warp;
        }
        if (page >= pool.pages || slice >= slices) continue;
        const ExtendCopy job = plan->copy[c];
        const int kb = pool.k_row_bytes, vb = pool.v_row_bytes, rows = job.rows;
        const int64_t page_bytes = static_cast<int64_t>(kBlockTokens) * (kb + vb), block = page_bytes * pool.pages;
        const char *src = static_cast<const char *>(pool.base) + page * page_bytes + job.src * block;
        char *dst = static_cast<char *>(pool.base) + page * page_bytes + job.dst * block;
        // The lane's words j * 32 + lane of 16 bytes, where bit j of `mask` is set, and words of 4 bytes at off_a and off_b.
        const int ks = k_slices(pool);
        unsigned mask;
        int off_a = -1, off_b = -1;
        if (slice < ks) {
            // The plane as words of 16 bytes in a row: with granules of 16 bytes word w is row w % 64, with granules of 4
            // it is rows 4 (w % 16) to 4 (w % 16) + 3, of which the last rows % 4 go as words of 4 bytes.
            src += slice * kSliceBytes;
            dst += slice * kSliceBytes;
            const int bytes = min(kSliceBytes, kBlockTokens * kb - slice * kSliceBytes);  // a multiple of 256
            const unsigned all = (1u << (bytes - lane * 16 + 511) / 512) - 1;  // bytes > lane * 16 - 512
            if (kb % 16 == 0) {
                mask = all & ((lane < rows ? 0x5555u : 0u) | (lane + 32 < rows ? 0xaaaau : 0u));
            } else {
                mask = lane % 16 < rows / 4 ? all : 0u;
                const int r = lane % 4, at = lane / 4 * 256 + rows / 4 * 16 + r * 4;
                if (r < rows % 4 && at < bytes) off_a = at;
                if (r < rows % 4 && at + 2048 < bytes) off_b = at + 2048;
            }
        } else {
            const int words = vb * rows / 16, rest = vb * rows % 16 / 4;  // of 16 bytes, and of 4 behind them
            const int share = (words + (slices - ks) - 1) / (slices - ks);
            const int w0 = (slice - ks) * share, n = min(words - w0, share) - lane;
            src += kBlockTokens * kb + w0 * 16;
            dst += kBlockTokens * kb + w0 * 16;
            mask = (1u << (max(0, n) + 31) / 32) - 1;
            if (slice == slices - 1 && lane < rest) off_a = (words - w0) * 16 + lane * 4;
        }
        uint32_t rest_a = 0, rest_b = 0;
        if (off_a >= 0) rest_a = *reinterpret_cast<const uint32_t *>(src + off_a);
        if (off_b >= 0) rest_b = *reinterpret_cast<const uint32_t *>(src + off_b);
        uint4 v[kSliceWords];
#pragma unroll
        for (int j = 0; j < kSliceWords; ++j) v[j] = load_if(src + lane * 16 + j * 512, mask >> j & 1);
#pragma unroll
        for (int j = 0; j < kSliceWords; ++j) store_if(dst + lane * 16 + j * 512, v[j], mask >> j & 1);
        if (off_a >= 0) *reinterpret_cast<uint32_t *>(dst + off_a) = rest_a;
        if (off_b >= 0) *reinterpret_cast<uint32_t *>(dst + off_b) = rest_b;
    }
    // (64 bits: the last step over N near 2^31 passes it by a grid of threads)
    for (int64_t at = static_cast<int64_t>(blockIdx.x) * kCopyThreads + threadIdx.x; at < a.N; at += static_cast<int64_t>(stride) * kCopyThreads) {
        const int i = static_cast<int>(at);
        int s, j;
        if (a.cu_new) {
            int lo = 0, hi = a.S - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (a.cu_new[mid] <= i) lo = mid;
                else hi = mid - 1;
            }
            s = lo;
            j = a.cu_new[s] <= i && i < a.cu_new[s + 1] ? i - a.cu_new[s] : INT32_MAX;
        } else {
            s = i / a.per;
            j = i - s * a.per;
        }
        int64_t slot = -1;
        if (j < plan->grow[s]) {
            const int pos = plan->before[s] + j;
            const int b = a.table[static_cast<int64_t>(s) * a.max_blocks + pos / kBlockTokens];
            slot = static_cast<int64_t>(b) * kBlockTokens + pos % kBlockTokens;
        }
        slots[i] = slot;
    }
}

// --------------------------------------------------------------------------------------------- compact

// The workspace: counts, then holes [nb / 2] (free blocks below R in order) and movers [nb / 2] (blocks in use
// from R on in order): as many of the one as of the other.
struct CompactPlan {
    int moves, live_below, unused[2];
};
struct CompactArgs {
    int32_t *ref;
    int nb;
    int32_t *table;
    int max_blocks;
    const int32_t *lens;
    int S;
    int32_t *remap, *live;
    CompactPlan *plan;
    int32_t *holes, *movers;
    unsigned *err;
};

__global__ void __launch_bounds__(kPlanThreads, 1) compact_plan_kernel(const CompactArgs a) {
    __shared__ Two part[33];
    __shared__ int totals[16];
    cg::cluster_group cl = cg::this_cluster();
    const int tid = threadIdx.x, rank = static_cast<int>(cl.block_rank()), ctas = static_cast<int>(cl.num_blocks());
    auto sync_all = [&]() {
        if (ctas > 1) cl.sync();
        else __syncthreads();
    };
    if (ctas > 1) cl.sync();  // every CTA has started
    pdl_wait();
    pdl_trigger();
    const Segment seg = my_segment(a.nb, rank, ctas);
    const int mine = count_ledger<false>(a.ref, a.nb, seg, a.nb);
    Two total;
    const Two before_me = block_scan(Two{0, mine}, part, total);
    const ClusterSums live = cluster_sums(total.b, totals);
    const int R = live.all, my_rank = live.before + __shfl_sync(0xffffffffu, before_me.b, 0);
    // blocks in use below R, known to the one warp whose entries hold R (nobody where all are in use)
    if (R == a.nb) {
        if (rank == 0 && tid == 0) a.plan->live_below = R;
    } else if (seg.begin <= R && R < seg.end) {
        const int below_r = __reduce_add_sync(0xffffffffu, count_ledger<false>(a.ref, a.nb, seg, R));
        if (tid % 32 == 0) a.plan->live_below = my_rank + below_r;
    }
    sync_all();
    const int below = *static_cast<volatile int *>(&a.plan->live_below);
    rank_ledger<false>(a.ref, a.nb, seg, my_rank, INT64_MAX, [&](int id, bool in_use, int r) {
        if (in_use) {
            if (id < R) a.remap[id] = id;
            else a.movers[r - below] = id;
        } else {
            a.remap[id] = -1;
            if (id < R) a.holes[id - r] = id;
        }
    });
    sync_all();
    const int moves = R - below;
    for (int k = rank * kPlanThreads + tid; k < moves; k += ctas * kPlanThreads) {
        const int from = a.movers[k], to = a.holes[k];
        a.remap[from] = to;
        a.ref[to] = a.ref[from];
        a.ref[from] = 0;
    }
    if (rank == 0 && tid == 0) {
        a.plan->moves = moves;
        *a.live = R;
    }
}

constexpr int kMoveBytes = kCopyThreads * 16 * 4;  // of a block, moved at once by a CTA

// Up to LLA_MAX_POOLS pools; first[l] is the number of kMoveBytes chunks that a block has in the pools before l.
struct BlockSet {
    char *base[LLA_MAX_POOLS];
    int64_t bytes[LLA_MAX_POOLS];
    int first[LLA_MAX_POOLS + 1];
    int L;
};

// Behind the plan: whole blocks from movers to holes (no hole is a mover, so the order does not matter), and the tables.
// At the copy rate with two to eight words a thread and four to eight CTAs an SM alike.
__global__ void __launch_bounds__(kCopyThreads) compact_move_kernel(const CompactArgs a, const __grid_constant__ BlockSet bs) {
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x;
    bool bad_len = false, bad_id = false;
    for (int s = blockIdx.x; s < a.S; s += gridDim.x) {
        const int len = checked_len(a.lens[s], a.max_blocks);
        bad_len |= len < 0;
        const int n = pages_of(max(0, len));
        int32_t *row = a.table + static_cast<int64_t>(s) * a.max_blocks;
        for (int i = tid; i < n; i += kCopyThreads) {
            const int b = row[i];
            const int to = b >= 0 && b < a.nb ? a.remap[b] : -1;
            if (to < 0) bad_id = true;  // no block, or a free one: left as it is
            else if (to != b) row[i] = to;
        }
    }
    if (bad_len) atomicOr(a.err, LLA_DEVERR_CONTEXT);
    if (bad_id) atomicOr(a.err, LLA_DEVERR_BLOCK_ID);
    const int per_block = bs.first[bs.L];
    const int64_t units = static_cast<int64_t>(a.plan->moves) * per_block;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int k = static_cast<int>(u / per_block), in_block = static_cast<int>(u - static_cast<int64_t>(k) * per_block);
        const int lo = pool_of(bs.first, bs.L, in_block);
        const int64_t bytes = bs.bytes[lo], off = static_cast<int64_t>(in_block - bs.first[lo]) * kMoveBytes;
        const char *src = bs.base[lo] + a.movers[k] * bytes + off;
        char *dst = bs.base[lo] + a.holes[k] * bytes + off;
        const int n = static_cast<int>(bytes - off < kMoveBytes ? bytes - off : kMoveBytes);
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if ((tid + j * kCopyThreads) * 16 < n) v[j] = __ldcs(reinterpret_cast<const uint4 *>(src) + tid + j * kCopyThreads);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if ((tid + j * kCopyThreads) * 16 < n) __stcs(reinterpret_cast<uint4 *>(dst) + tid + j * kCopyThreads, v[j]);
    }
}

// ------------------------------------------------------------------------------------------- launches

// CTAs of a plan's cluster.  One takes 4.1 us (growth) and 6 us (compaction) with 4096 blocks and 4.6 and 10.6 with 16384,
// eight take 5.0 and 8.4, and 5.2 and 8.4.
int plan_ctas(int64_t num_blocks) { return num_blocks > 8192 ? 8 : 1; }

template <typename A>
lla_status launch_plan(void (*kern)(A), int ctas, const A &a, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kPlanThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, a) == cudaSuccess ? LLA_OK : LLA_ERR_CUDA;
}

}  // namespace

lla_status launch_pages_fork(const lla_pages &from, const lla_pages &to, const int32_t *parents, bool keep, cudaStream_t stream) {
    lla_status st;
    ForkArgs a = {};
    a.ref = from.ref_count; a.nb = static_cast<int>(from.num_blocks);
    a.from_table = from.block_table; a.from_lens = from.context_lens;
    a.from_max = from.max_blocks_per_seq; a.from_S = from.S;
    a.to_table = to.block_table; a.to_lens = to.context_lens;
    a.to_max = to.max_blocks_per_seq; a.to_S = to.S;
    a.parents = parents;
    a.keep = keep;
    a.err = device_error_word(&st);
    if (!a.err) return st;
    const int most = from.max_blocks_per_seq;
    const int spans = (most + kForkSpan - 1) / kForkSpan;
    return launch_ex(fork_kernel, dim3(to.S + from.S, spans < 32 ? spans : 32), kForkThreads, 0, stream, a);
}

lla_status launch_pages_free(const lla_pages &p, const int32_t *seqs, int n, cudaStream_t stream) {
    lla_status st;
    unsigned *err = device_error_word(&st);
    if (!err) return st;
    return launch_ex(free_kernel, dim3(n), kFreeThreads, 0, stream, p.ref_count, static_cast<int>(p.num_blocks),
                     static_cast<const int32_t *>(p.block_table), p.max_blocks_per_seq, p.context_lens, p.S, seqs, err);
}

size_t pages_extend_workspace_bytes() { return sizeof(ExtendPlan); }

lla_status launch_pages_extend(const lla_pages &p, const lla_pool *pools, int L, int64_t *slots, int N, const int32_t *cu_new,
                               const uint8_t *skip, int32_t *lens_before, int32_t *free_blocks, void *workspace,
                               cudaStream_t stream) {
    lla_status st;
    ExtendArgs a = {};
    a.ref = p.ref_count; a.nb = static_cast<int>(p.num_blocks);
    a.table = p.block_table; a.max_blocks = p.max_blocks_per_seq; a.lens = p.context_lens; a.S = p.S;
    a.cu_new = cu_new; a.N = N; a.per = cu_new || p.S == 0 ? 0 : N / p.S;
    a.skip = skip; a.lens_before = lens_before; a.free_blocks = free_blocks;
    a.plan = static_cast<ExtendPlan *>(workspace);
    a.err = device_error_word(&st);
    if (!a.err) return st;
    PoolSet ps = {};
    ps.L = L;
    for (int l = 0; l < L; ++l) {
        const int slices = k_slices(pools[l]) + v_slices(pools[l]);
        ps.p[l] = pools[l];
        ps.slices[l] = static_cast<uint16_t>(slices);
        const int at_once = slices < kCopyWarps ? kCopyWarps / slices : 1;
        const int units = slices < kCopyWarps ? (pools[l].pages + at_once - 1) / at_once
                                              : pools[l].pages * ((slices + kCopyWarps - 1) / kCopyWarps);
        ps.first[l + 1] = ps.first[l] + units;
    }
    ps.alike = 1;
    for (int l = 1; l < L; ++l) ps.alike &= ps.first[l + 1] - ps.first[l] == ps.first[1];
    ps.by_pool = fast_div(static_cast<uint32_t>(L > 0 ? ps.first[1] : 1));
    if ((st = launch_plan(extend_plan_kernel, plan_ctas(p.num_blocks), a, stream)) != LLA_OK) return st;
    const int sms = num_sms();
    if (sms <= 0) return LLA_ERR_CUDA;
    // every CTA resident at once; no more than there can be work for
    const int64_t work = static_cast<int64_t>(p.S) * ps.first[L] + (static_cast<int64_t>(N) + kCopyThreads - 1) / kCopyThreads;
    return launch_ex(extend_finish_kernel, dim3(static_cast<unsigned>(work < sms * kCopyCtas ? (work > 0 ? work : 1) : sms * kCopyCtas)),
                     kCopyThreads, 0, stream, a, ps, slots);
}

size_t pages_compact_workspace_bytes(int64_t num_blocks) {
    return sizeof(CompactPlan) + 2 * static_cast<size_t>(num_blocks / 2 + 1) * sizeof(int32_t);
}

lla_status launch_pages_compact(const lla_pages &p, const lla_pool *pools, int L, int32_t *remap, int32_t *live, void *workspace,
                                cudaStream_t stream) {
    lla_status st;
    CompactArgs a = {};
    a.ref = p.ref_count; a.nb = static_cast<int>(p.num_blocks);
    a.table = p.block_table; a.max_blocks = p.max_blocks_per_seq; a.lens = p.context_lens; a.S = p.S;
    a.remap = remap; a.live = live;
    a.plan = static_cast<CompactPlan *>(workspace);
    a.holes = reinterpret_cast<int32_t *>(a.plan + 1);
    a.movers = a.holes + a.nb / 2 + 1;
    a.err = device_error_word(&st);
    if (!a.err) return st;
    BlockSet bs = {};
    bs.L = L;
    for (int l = 0; l < L; ++l) {
        bs.base[l] = static_cast<char *>(pools[l].base);
        bs.bytes[l] = static_cast<int64_t>(kBlockTokens) * (pools[l].k_row_bytes + pools[l].v_row_bytes) * pools[l].pages;
        const int64_t chunks = (bs.bytes[l] + kMoveBytes - 1) / kMoveBytes;
        bs.first[l + 1] = bs.first[l] + static_cast<int>(chunks);  // at most 128 pools of 2^18 chunks
    }
    if ((st = launch_plan(compact_plan_kernel, plan_ctas(p.num_blocks), a, stream)) != LLA_OK) return st;
    const int sms = num_sms();
    if (sms <= 0) return LLA_ERR_CUDA;
    return launch_ex(compact_move_kernel, dim3(sms * 8), kCopyThreads, 0, stream, a, bs);
}

}  // namespace lla
