// lla_prefix_plan.cu -- which sequences of a batch share which pages (lla_prefix_plan): from the block table and the
// lengths the groups whose shared pages lla_decode_attn_prefix reads once.
//
// A level refines the sets of the level before it (at first the whole batch): sequences of a set with the same block in
// the set's next full page form a set of their own.  Its pages go on from there to
//   end = min over its members s of min(full_s, full_leader, first page where the rows of s and of the leader differ or hold no block),
// and with two members and min_pages pages it becomes ceil(n / 64) groups, member of rank r in part ((r + 1) k - 1) / n.
//
// Bound by latency: three levels one after the other, each a hash table in shared memory (of a size for the largest batch), a comparison
// of rows, prefix sums, and the barriers of a CTA's 32 warps, or for many long rows a cluster's.  12.6 us for 64 sequences, by one CTA; 26 for 1024 with up to 512 pages (39 with eight CTAs, atomics of every thread on its
// set's words, and rows compared one load at a time), of which reading 1.6 MB of table rows takes 0.3.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "lla_device.cuh"
#include "lla_internal.h"
#include "lla_plan.cuh"

namespace lla {
namespace {

namespace cg = cooperative_groups;

constexpr int kLevels = LLA_PREFIX_LEVELS;
constexpr int kMembers = LLA_PREFIX_MEMBERS;
constexpr int kSlots = 2 * LLA_MAX_BATCH;
constexpr unsigned long long kNoKey = ~0ull;

struct PrefixArgs {
    const int32_t *table;
    int nb, max_blocks;
    const int32_t *lens;
    int B, max_ctx, min_pages;
    lla_prefix plan;
    unsigned *err;
};

struct PrefixShared {
    unsigned long long key[kSlots];  // set and block of a slot of the hash table
    int lowest[kSlots], count[kSlots];
    int end[kLevels][LLA_MAX_BATCH];  // (the first CTA's) end of each leader's set
    int full[LLA_MAX_BATCH];          // full pages of each sequence
    int lead[LLA_MAX_BATCH];          // leader of each sequence's set, -1 where it is in none
    int page[LLA_MAX_BATCH], last[LLA_MAX_BATCH], size[LLA_MAX_BATCH], group[LLA_MAX_BATCH], member[LLA_MAX_BATCH];  // by leader
    Two part[33];
};

// The first page of [from, limit) where two rows differ or hold no block (one of `nb`), or limit: by a warp, with kLoads loads of either
// row in flight in a lane.  (Four int4 where both rows start on 16 bytes took as long; twelve entries 4 us more for 1024 long rows, and a
// flag set in here for entries that are no blocks 6 us.)
constexpr int kLoads = 8;
__device__ __forceinline__ int first_difference(const int32_t *a, const int32_t *b, int from, int limit, int nb) {
    const int lane = threadIdx.x & 31;
    for (int p = from; p < limit; p += 32 * kLoads) {
        int va[kLoads], vb[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int i = p + 32 * j + lane;
            va[j] = i < limit ? a[i] : 0;
            vb[j] = i < limit ? b[i] : 0;
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const unsigned m = __ballot_sync(0xffffffffu, va[j] != vb[j] || static_cast<unsigned>(va[j]) >= static_cast<unsigned>(nb));
            if (m) return p + 32 * j + __ffs(m) - 1;
        }
    }
    return limit;
}

// One cluster.  Thread s of every CTA works out sequence s (the CTAs do the same sums), the sequences' rows are compared by
// all warps of the cluster, and each CTA ranks and writes its part of the sequences.
__global__ void __launch_bounds__(kPlanThreads, 1) prefix_plan_kernel(const PrefixArgs a) {
    extern __shared__ __align__(16) char smem[];
    PrefixShared &sh = *reinterpret_cast<PrefixShared *>(smem);
    cg::cluster_group cl = cg::this_cluster();
    const int tid = threadIdx.x, warp = tid >> 5, rank = static_cast<int>(cl.block_rank()), ctas = static_cast<int>(cl.num_blocks());
    auto sync_all = [&]() {
        if (ctas > 1) cl.sync();
        else __syncthreads();
    };
    pdl_wait();
    pdl_trigger();
    const int cap = min(a.max_ctx, static_cast<int>(min(static_cast<int64_t>(a.max_blocks) * kBlockTokens, static_cast<int64_t>(INT32_MAX))));
    int full = 0;
    if (tid < a.B) {
        const int len = a.lens[tid];
        if (len < 0 || len > cap) {
            if (rank == 0) atomicOr(a.err, LLA_DEVERR_CONTEXT);
        } else {
            full = len / kBlockTokens;
        }
    }
    // the rows on their way to L2 while the first blocks are sorted (each CTA fetches its part of them)
    if (full > 1) {
        const char *row = reinterpret_cast<const char *>(a.table + static_cast<int64_t>(tid) * a.max_blocks);
        for (int i = rank * 128; i < full * 4; i += ctas * 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + i));
    }
    sh.full[tid] = full;
#pragma unroll
    for (int l = 0; l < kLevels; ++l) sh.end[l][tid] = full;
    sync_all();  // every CTA has started, and the first one's `end` is set
    int *ends = ctas > 1 ? cl.map_shared_rank(&sh.end[0][0], 0) : &sh.end[0][0];

    // the part of the sequences that this CTA ranks: P threads each
    const int per = (a.B + ctas - 1) / ctas, mine0 = rank * per, mine = max(0, min(a.B - mine0, per));
    int P = 32;
    while (P > 1 && P * per > kPlanThreads) P >>= 1;
    const int my_seq = mine0 + tid / P, my_part = tid % P;
    const bool ranks = tid / P < mine;

    bool alive = full > 0;
    int lead = 0, page = 0, groups = 0, members = 0, level = 0;
    for (; level < kLevels; ++level) {
        for (int i = tid; i < kSlots; i += kPlanThreads) {
            sh.key[i] = kNoKey;
            sh.lowest[i] = kSlots;
            sh.count[i] = 0;
        }
        alive = alive && full > page;
        int block = 0;
        if (alive) {
            block = a.table[static_cast<int64_t>(tid) * a.max_blocks + page];
            if (block < 0 || block >= a.nb) {
                if (rank == 0) atomicOr(a.err, LLA_DEVERR_BLOCK_ID);
                alive = false;
            }
        }
        __syncthreads();
        // The sequences of a warp with one key send their lowest, for all of them: a thousand atomics on one word took longer than
        // the rest of a level.
        int slot = 0;
        const unsigned long long key = alive ? static_cast<unsigned long long>(lead) << 32 | static_cast<unsigned>(block) : kNoKey;
        const unsigned same = __match_any_sync(0xffffffffu, key);
        const int sender = __ffs(same) - 1;
        if (alive && tid % 32 == sender) {
            slot = (static_cast<unsigned>(block) * 2654435769u + static_cast<unsigned>(lead) * 40503u) >> 21;  // golden-ratio hashing
            for (;;) {
                const unsigned long long was = atomicCAS(&sh.key[slot], kNoKey, key);
                if (was == kNoKey || was == key) break;
                slot = (slot + 1) % kSlots;
            }
            atomicMin(&sh.lowest[slot], tid);
            atomicAdd(&sh.count[slot], __popc(same));
        }
        slot = __shfl_sync(0xffffffffu, slot, sender);
        __syncthreads();
        const int n = alive ? sh.count[slot] : 0;
        const int lead_new = alive ? sh.lowest[slot] : tid;
        alive = n >= 2;
        sh.lead[tid] = alive ? lead_new : -1;
        sh.page[tid] = page;
        if (!__syncthreads_or(alive)) break;  // nobody shares further (in every CTA alike)
        for (int i = rank * (kPlanThreads / 32) + warp; i < a.B; i += ctas * (kPlanThreads / 32)) {
            const int j = sh.lead[i];
            if (j < 0 || j == i) continue;
            const int limit = min(sh.full[i], sh.full[j]);
            const int e = first_difference(a.table + static_cast<int64_t>(i) * a.max_blocks, a.table + static_cast<int64_t>(j) * a.max_blocks,
                                           sh.page[i] + 1, limit, a.nb);
            if (tid % 32 == 0) atomicMin(ends + level * LLA_MAX_BATCH + j, e);
        }
        sync_all();
        const int end = alive ? *static_cast<volatile int *>(ends + level * LLA_MAX_BATCH + lead_new) : 0;
        alive = alive && end - page >= a.min_pages;
        sh.lead[tid] = alive ? lead_new : -1;
        const bool first = alive && lead_new == tid;
        const int k = (n + kMembers - 1) / kMembers;
        Two total;
        const Two at = block_scan(Two{first ? static_cast<unsigned long long>(k) << 32 | static_cast<unsigned>(n) : 0ull, 0}, sh.part, total);
        if (first) {
            sh.last[tid] = end;
            sh.size[tid] = n;
            sh.group[tid] = groups + static_cast<int>(at.a >> 32);
            sh.member[tid] = members + static_cast<int>(at.a & 0xffffffffu);
        }
        __syncthreads();
        // rank: the members of the set before this one, counted by P threads
        int r = 0;
        const int j = ranks ? sh.lead[my_seq] : -1;
        if (j >= 0) {
            for (int i = 4 * my_part; i < my_seq; i += 4 * P) {
                const int4 v = *reinterpret_cast<const int4 *>(&sh.lead[i]);
                r += (v.x == j) + (v.y == j && i + 1 < my_seq) + (v.z == j && i + 2 < my_seq) + (v.w == j && i + 3 < my_seq);
            }
        }
        for (int o = 1; o < P; o <<= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
        if (ranks && my_part == 0) {
            int column = -1;
            if (j >= 0) {
                const int size = sh.size[j], parts = (size + kMembers - 1) / kMembers;
                const int part = ((r + 1) * parts - 1) / size, begin = part * size / parts;
                const int group = sh.group[j] + part, member = sh.member[j];
                column = group * kMembers + r - begin;
                a.plan.members[member + r] = my_seq;
                if (r == begin)
                    reinterpret_cast<int4 *>(a.plan.groups)[group] =
                        make_int4(sh.page[j], sh.last[j], member + begin, (part + 1) * size / parts - begin);
            }
            a.plan.column[static_cast<int64_t>(level) * a.B + my_seq] = column;
        }
        groups += static_cast<int>(total.a >> 32);
        members += static_cast<int>(total.a & 0xffffffffu);
        if (alive) {
            page = end;
            lead = lead_new;
        }
        __syncthreads();
    }
    // the page behind the last level's pages (a level looks at those behind the ones of the level before it)
    if (alive && full > page && rank == 0) {
        const int block = a.table[static_cast<int64_t>(tid) * a.max_blocks + page];
        if (block < 0 || block >= a.nb) atomicOr(a.err, LLA_DEVERR_BLOCK_ID);
    }
    // what no group holds
    const int at = rank * kPlanThreads + tid, step = ctas * kPlanThreads;
    for (int i = level * a.B + at; i < kLevels * a.B; i += step) a.plan.column[i] = -1;
    for (int i = members + at; i < kLevels * a.B; i += step) a.plan.members[i] = -1;
    for (int i = groups + at; i < kLevels * max(1, a.B / 2); i += step)
        reinterpret_cast<int4 *>(a.plan.groups)[i] = make_int4(0, 0, 0, 0);
    if (rank == 0) {
        if (tid < a.B) a.plan.own_page[tid] = page;
        if (tid == 0) *a.plan.num_groups = groups;
    }
    if (ctas > 1) cl.sync();  // the first CTA's shared memory is read until here
}

}  // namespace

lla_status launch_prefix_plan(const int32_t *block_table, int64_t num_blocks, int max_blocks, const int32_t *context_lens, int B,
                              int max_ctx, int min_pages, const lla_prefix &plan, cudaStream_t stream) {
    lla_status st;
    PrefixArgs a = {};
    a.table = block_table; a.nb = static_cast<int>(num_blocks); a.max_blocks = max_blocks;
    a.lens = context_lens; a.B = B; a.max_ctx = max_ctx; a.min_pages = min_pages;
    a.plan = plan;
    a.err = device_error_word(&st);
    if (!a.err) return st;
    static DeviceOnce configured, configured_cluster;
    constexpr int smem = static_cast<int>(sizeof(PrefixShared));
    if ((st = raise_smem_limit(prefix_plan_kernel, smem, configured)) != LLA_OK) return st;
    if ((st = allow_clusters_of_16(prefix_plan_kernel, configured_cluster)) != LLA_OK) return st;
    const int64_t entries = static_cast<int64_t>(B) * (max_ctx / kBlockTokens);
    return launch_plan(prefix_plan_kernel, entries > 32768 ? 16 : entries > 8192 ? 8 : 1, a, stream, smem);
}

}  // namespace lla
