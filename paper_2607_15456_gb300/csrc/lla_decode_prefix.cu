// lla_decode_prefix.cu -- decode of a batch whose sequences share pages of the paged latent cache (lla_decode_attn_prefix):
// the absorbed decode (App. J "Absorbed attention") with every page of a group of up to 64 sequences read once for all of
// them, with or without the decoupled rotary branch.
//
// A node of the batch is a run of pages with the sequences that read them: a group of the plan, or a sequence with the
// pages that it reads alone; a unit is a node and a head.  For query n of a unit and token i of its pages
//   q~_n = W_up,t^K^T q_n [; rot(q^R_n, P_n)],  beta_n = q_n . mu^K_t
//   s_n,i = scale (q~_n . [c_k,i; k^R_i] + beta_n),  m_n = max_i s_n,i,  l_n = sum_i e^(s_n,i - m_n),
//   o~_n = sum_i e^(s_n,i - m_n) c_v,i
// and a sequence's output joins the states of its nodes j (at most three groups and its own pages) and, in pass 1, the
// current token:
//   o = (W_up,t^V sum_j w_j o~_j + (sum_j w_j l_j) mu^V_t + w_cur v_cur) / (sum_j w_j l_j + w_cur),  w_j = e^(m_j - M).
//
// Four launches on the caller's stream, chained by programmatic dependent launch (three for few sequences, see leaf_alone):
//   absorb_kernel  q~ (scaled into the exp2 domain) and beta of every (sequence, head); the prefix sums of the nodes' pages and
//                  the checks of lengths and plan
//   trunk_kernel   nodes of more than kLeaf queries, one CTA per SM.  Their pages, unit by unit in the order of the nodes, are
//                  split evenly over the CTAs; a CTA takes its pages as runs (parts of one unit).  A page is two products on
//                  the tensor cores, with 128 rows for the up to 64 queries of a run, each of them 2, 4 or 8 times:
//                    S [128 x 64 tokens] = sum_i Q~_i [C_k | K^R]^T      i = 2, 1, 0: q~ as three bf16 parts, in TMEM
//                    O [128 x r_v]      += P C_v                         P in TMEM
//                  All rows of a query have its scores; each thread works out the weights p of some of its tokens and gives them
//                  as bf16(p) or as bf16(p - bf16(p)), so that the query's rows of O add up to a sum with p in two parts, for
//                  the tensor cores' price of one.
//                    warp 0        producer of K-planes (and rotary planes): bulk copies
//                    warp 2        producer of V-planes: TMA boxes of 64 columns with 128-byte swizzle
//                    warp 1        issuer of S, and owner of TMEM
//                    warp 3        issuer of O
//                    warps 4-11    softmax: two groups that take the pages in turn (as in the prefill, a page's step from scores
//                                  to weights takes longer than its products); the running maximum goes from page to page
//                                  through shared memory and a named barrier per pair of warps; lazy rescale of O
//                    warps 12-15   q~ of the next unit into TMEM as soon as the last S of the one before is done; a run's O through
//                                  shared memory, its maxima and its sums to the workspace, joined with what the unit's
//                                  runs before it have left there
//                  Bound by HBM and, at run ends, by latency: 393 MB of pages that 4 sequences each share take 74 us (5.3 TB/s),
//                  287 MB that 64 share 70 us, with the tensor pipe busy for 58 % and the step from S to P for the rest
//   leaf_kernel    nodes of up to kLeaf queries (a sequence's own pages; all nodes where there is no trunk kernel): one page at a time in
//                  each of as many warps as pages fit in an SM's shared memory beside a CTA of the join, on the CUDA cores.  It starts on
//                  each SM as the trunk kernel leaves it.  Bound by HBM while all warps run (6 TB/s)
//   join_kernel    per head and up to 16 sequences: joins the runs of each sequence's nodes and the current token, and applies
//                  W_up,t^V once for all of them.  One CTA per SM, beside the leaf kernel's, so that the weights and the
//                  instructions are there when the records are: 13 us behind the leaves of 128 sequences in 16 heads (22 us where
//                  it started when they had left, with the projection on the CUDA cores).  Bound by latency
// 64 sequences over 16 prompts of 2048 to 4096 tokens, 16 heads, r 96 + 160: 108 us, of 83 us that HBM takes for the bytes.
//
// Storage bf16, d = 128; accumulators fp32 in TMEM, for at most kRunPages pages.  Three parts of q~, and of p, hold the 24 bits of fp32.
// For bf16 outputs p has two, for the price of one (see replica_rows): they are off by at most 2^-18 of p, half a step of the second
// part and to both sides, where an output is rounded by up to 2^-8.  (With two for fp32 outputs, too, a few tokens' outputs were
// off by 2e-6.)  The sums l take p itself.
#include <cuda_runtime.h>

#include <algorithm>

#include "lla_device.cuh"
#include "lla_internal.h"
#include "lla_tcgen05.cuh"
#include "lla_tmap.h"
#include "lla_units.cuh"

namespace lla {
namespace {

constexpr int kPT = 64;          // tokens per page
constexpr int kD = 128;          // head width
constexpr int kRows = 128;       // rows of the products: every query 2, 4 or 8 times
constexpr int kLevels = LLA_PREFIX_LEVELS;
constexpr int kMembers = LLA_PREFIX_MEMBERS;
constexpr int kMaxNodes = kLevels * (LLA_MAX_BATCH / 2) + LLA_MAX_BATCH;
constexpr int kTrunkThreads = 512;
constexpr int kSoftmaxWarp = 4, kAuxWarp = 12;
constexpr int kLeaf = 2;         // most queries of a node that the leaf kernel takes beside a trunk kernel
constexpr int kLeafAlone = 4;    // and without one: most sequences of a call that has none (see leaf_alone)
constexpr int kMaxGrid = 256;
constexpr int kJoinSeqs = 16;    // most sequences of a head that the join works on together
constexpr int kSmemCap = 227 * 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleLog2 = 8.f;  // rescale O^T only when a query's maximum grows by more

struct PlanView {
    const int32_t *num_groups, *groups, *members, *column, *own_page;
};

struct TrunkParams {
    int H, B, max_ctx, max_blocks, pass1;
    int leaf_max;  // queries of a node that the leaf kernel takes, at most
    int trunk_max; // queries of a node that the trunk kernel takes, at most; 0 without one
    const char *pool;
    int64_t num_blocks, page_bytes;
    const char *rope_pool;
    const int32_t *block_table, *context_lens;
    PlanView plan;
    uint16_t *qt;  // [B][H][3][RKT]: q~ * scale * log2 e as three bf16 parts, zero past r_k, then the rotary part
    float *qf;     // [B][H][RKT]: the same in fp32, for the leaves
    float *beta;   // [B][H]: q . mu^K * scale * log2 e
    float *part;   // run records, see record_of
    int *pstart;   // [2][kMaxNodes + 1]: pages of the trunk's nodes, and of the leaves, before each node; then all of them
    int *next;     // share of the leaves that is taken next
    int64_t leaf;  // first record of the leaf kernel
    unsigned *err;
};

struct AbsorbParams {
    TrunkParams t;
    int T, loop, io_bf16;
    float scale_log2;
    const void *w_up_k;  // [H][T][d][r_k]
    const float *mu_k;   // [H][T*d] or NULL
    const void *q, *q_rope;
    const int32_t *positions;  // [3][B] or NULL
    int pairing;
    uint8_t axis[kMaxRopePairs];
    unsigned long long phi[kMaxRopePairs];
};

struct JoinParams {
    TrunkParams t;
    int T, loop, io_bf16, grid, workers, spb, d_rope;
    float scale_log2;
    const void *w_up_v;  // [H][T][d][r_v]
    const float *mu_v;
    const void *q, *q_rope, *cur_k, *cur_v, *cur_k_rope;
    void *out;
};

// ------------------------------------------------------------------------------------------------ nodes

struct Node {
    int pages, first;  // pages of the node, and the first in its table row
    int n, member;     // queries, and the index of the first among all nodes' queries
    int row, len;      // table row, and tokens of it that may be read
};

__device__ __forceinline__ int count_groups(const TrunkParams &p) {
    return max(0, min(*p.plan.num_groups, kLevels * max(1, p.B / 2)));
}

// Node i of the groups and, behind them, the sequences.  One that the plan or the lengths get wrong has no pages.
__device__ __forceinline__ Node node_at(const TrunkParams &p, int groups, int i) {
    const int cap = static_cast<int>(min(static_cast<int64_t>(p.max_ctx), static_cast<int64_t>(p.max_blocks) * kPT));
    Node d = {0, 0, 0, 0, 0, INT32_MAX};
    if (i < groups) {
        const int4 g = reinterpret_cast<const int4 *>(p.plan.groups)[i];
        if (g.x < 0 || g.y <= g.x || g.y > cap / kPT || g.w < 1 || g.w > min(kMembers, p.B) || g.z < 0 || g.z > kLevels * p.B - g.w) return d;
        d.row = p.plan.members[g.z];
        if (d.row < 0 || d.row >= p.B) return d;
        d.pages = g.y - g.x;
        d.first = g.x;
        d.n = g.w;
        d.member = g.z;
        return d;
    }
    d.row = i - groups;
    d.n = 1;
    d.member = kLevels * p.B + d.row;
    d.len = p.context_lens[d.row];
    d.first = p.plan.own_page[d.row];
    if (d.len < 0 || d.len > cap || d.first < 0 || d.first > d.len / kPT) return d;
    d.pages = (d.len + kPT - 1) / kPT - d.first;
    return d;
}

__device__ __forceinline__ bool is_leaf(const TrunkParams &p, const Node &d) { return d.n <= p.leaf_max; }

// Record of the first query of node d at head h, from CTA (or leaf warp) c: r_v latent values, the maximum, the sum.  The
// records of a unit's runs lie as far apart as a node of its kind can have queries, so that no two of them meet: units and
// CTAs grow together.
__device__ __forceinline__ int64_t record_of(const TrunkParams &p, const Node &d, int h, int c) {
    const int64_t at = static_cast<int64_t>(p.H) * d.member + static_cast<int64_t>(h) * d.n;
    return is_leaf(p, d) ? p.leaf + at + static_cast<int64_t>(p.leaf_max) * c : at + static_cast<int64_t>(p.trunk_max) * c;
}
__host__ __device__ constexpr int record_floats(int rv) { return rv + 4; }

// np pages over w workers (0 < w <= np): the first np % w of them take a page more than the others.  32-bit arithmetic: a
// 64-bit division is a called subroutine.
struct Split {
    int each, more;  // pages of a worker, and workers that take one more
    __device__ __forceinline__ Split(int np, int w) : each(np / max(w, 1)), more(np - each * w) {}
    __device__ __forceinline__ int begin(int c) const { return c * each + min(c, more); }
    __device__ __forceinline__ int worker(int page) const {
        const int wide = more * (each + 1);
        return page < wide ? page / (each + 1) : more + (page - wide) / each;
    }
};

// Most pages of a run: a CTA's pages are cut into even pieces of at most as many, a run is a piece's part of a unit, and the epilogue
// joins the runs of a unit in fp32, in the CTA's record of it.  The tensor cores cut off what an addition leaves behind the last bits of
// O, all to one side, so that a sum loses the more the larger it gets.  Measured on sums of one sign, mean over the outputs of 64
// queries: 1.6e-6 of themselves with 24 pages, 9.9e-6 with 64, 2.9e-5 with 128 (of 20 queries, whose rows hold fewer tokens, 0.5, 2.9 and
// 9.5e-6).  fp32 outputs: 24; 64 samples of two videos, d_rope 64, take 174 us so, 178 with 16, 169 with 40.  bf16 outputs: 128, where
// the loss is 1/130 of their half steps of up to 2^-8; 64 samples of 65536 tokens take 116 us so, and 125 with 64.  (A run that
// ends a CTA's share waits for the record that it is joined with, 7 us for 64 queries.)
template <bool FP32>
constexpr int kRunPages = FP32 ? 24 : 128;

// The shares that the pages of the leaves are split into, for `workers` warps: one each of kLeafFirst / 8 of the pages, and the
// rest in up to kLeafRest as many small ones, which the warps take as they get there.  A share's record does not depend on the
// warp that took it, and so neither do the results.  (With one share of each warp the leaf kernel ended when the SM that the trunk
// kernel left last had done its part: 102 us after the start for 128 sequences over 8 documents, 91 so.  Between 3/8 and 6/8, and
// with 2 or 4, it is the same to 2 %; more shares are more records to join.)
constexpr int kLeafFirst = 5, kLeafRest = 2;
struct LeafShares {
    int np, n1, w1, w2;  // pages; pages of the first shares, their number, the number of the small ones
    Split first, rest;
    __device__ __forceinline__ LeafShares(int pages, int workers)
        : np(pages), n1(min(pages, max(workers, pages / 8 * kLeafFirst))), w1(min(workers, pages)), w2(min(kLeafRest * workers, pages - n1)),
          first(n1, w1), rest(pages - n1, w2) {}
    __device__ __forceinline__ int count() const { return w1 + w2; }
    __device__ __forceinline__ int begin(int c) const { return c < w1 ? first.begin(c) : n1 + rest.begin(c - w1); }
    __device__ __forceinline__ int share(int page) const { return page < n1 ? first.worker(page) : w1 + rest.worker(page - n1); }
};

// ----------------------------------------------------------------------------------------- absorb kernel

// One CTA: the prefix sums of the nodes' pages, and the flags of what node_at leaves out.
__device__ void node_prefix(const TrunkParams &p) {
    __shared__ int pages[kMaxNodes];  // a leaf's as -1 - pages
    __shared__ int wsum[2][8];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int groups = count_groups(p), nodes = groups + p.B;
    const int cap = static_cast<int>(min(static_cast<int64_t>(p.max_ctx), static_cast<int64_t>(p.max_blocks) * kPT));
    unsigned bad = 0;
    if (*p.plan.num_groups != groups) bad |= LLA_DEVERR_SEQUENCE;
    for (int i = tid; i < nodes; i += 256) {
        const Node d = node_at(p, groups, i);
        pages[i] = is_leaf(p, d) ? -1 - d.pages : d.pages;
        if (i < groups && d.pages == 0) bad |= LLA_DEVERR_SEQUENCE;
        if (i >= groups) {
            if (d.len < 0 || d.len > cap || d.first < 0 || d.first > d.len / kPT) bad |= LLA_DEVERR_CONTEXT;
            if (d.len == 0 && !p.pass1) bad |= LLA_DEVERR_EMPTY_PASS2;
        }
    }
    for (int b = tid; b < p.B; b += 256) {
        const int len = p.context_lens[b];
#pragma unroll
        for (int l = 0; l < kLevels; ++l) {
            const int col = p.plan.column[static_cast<int64_t>(l) * p.B + b];
            if (col < 0) continue;
            const Node d = col / kMembers < groups ? node_at(p, groups, col / kMembers) : Node{};
            if (d.pages == 0 || col % kMembers >= d.n || p.plan.members[d.member + col % kMembers] != b) bad |= LLA_DEVERR_SEQUENCE;
            else if (d.first + d.pages > len / kPT) bad |= LLA_DEVERR_CONTEXT;
        }
    }
    if (bad) atomicOr(p.err, bad);
    __syncthreads();
    const int per = (nodes + 255) / 256;
    int tot[2] = {0, 0};  // pages of the trunk's nodes, of the leaves
    for (int i = tid * per; i < min(nodes, (tid + 1) * per); ++i) {
        tot[0] += max(0, pages[i]);
        tot[1] += max(0, -1 - pages[i]);
    }
    int x[2] = {tot[0], tot[1]};  // inclusive scans over the warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y0 = __shfl_up_sync(0xffffffffu, x[0], o), y1 = __shfl_up_sync(0xffffffffu, x[1], o);
        if (lane >= o) {
            x[0] += y0;
            x[1] += y1;
        }
    }
    if (lane == 31) {
        wsum[0][warp] = x[0];
        wsum[1][warp] = x[1];
    }
    __syncthreads();
    int ex[2] = {x[0] - tot[0], x[1] - tot[1]};
    for (int w = 0; w < warp; ++w) {
        ex[0] += wsum[0][w];
        ex[1] += wsum[1][w];
    }
    for (int i = tid * per; i < min(nodes, (tid + 1) * per); ++i) {
        const int v = pages[i];
        p.pstart[i] = ex[0];
        p.pstart[kMaxNodes + 1 + i] = ex[1];
        if (v < 0) ex[1] += -1 - v;
        else ex[0] += v;
    }
    if (tid == 255) {
        p.pstart[nodes] = ex[0];
        p.pstart[kMaxNodes + 1 + nodes] = ex[1];
        *p.next = 0;
    }
}

// v as three bf16 parts, `stride` apart.
__device__ __forceinline__ void store_parts(uint16_t *dst, int stride, float v) {
    float part[3];
    bf16_parts(v, part);
#pragma unroll
    for (int k = 0; k < 3; ++k) dst[k * stride] = __bfloat16_as_ushort(__float2bfloat16_rn(part[k]));
}

// Grid (H, RKX / 32 [+ 1 with a rotary branch] + 1, ceil(B / 16)), 256 threads = 32 columns x 8 slices of 16 rows: q~ of 32
// columns of one head for 16 sequences, every weight load of a thread in flight at once; beta by the CTAs of the first
// column chunk; the rotary queries, turned at the current tokens' positions, by those behind the columns; the nodes' prefix
// sums by one CTA of the last row.
template <int RK, int DR>
__global__ void __launch_bounds__(256) absorb_kernel(const __grid_constant__ AbsorbParams a) {
    constexpr int RKX = (RK + 15) / 16 * 16, RKT = RKX + DR, CHUNKS = (RKX + 31) / 32;
    __shared__ float qs[16][kD];
    __shared__ float red[8][16][33];
    const TrunkParams &p = a.t;
    const int h = blockIdx.x, j0 = blockIdx.y * 32, b0 = blockIdx.z * 16, tid = threadIdx.x;
    const int warp = tid >> 5, lane = tid & 31;
    const int nb = min(16, p.B - b0);
    const int64_t th = static_cast<int64_t>(h) * a.T + a.loop;
    pdl_wait();  // the inputs may come from the previous kernel; the workspace is free after it
    // The trunk kernel may start: once every CTA is here the caller's previous kernel is complete, so its producers may read
    // any input of the call, and q~, beta and the workspace only after their own wait.
    pdl_trigger();
    if (blockIdx.y == gridDim.y - 1) {
        if (blockIdx.x == 0 && blockIdx.z == 0) node_prefix(p);
        return;
    }
    if constexpr (DR > 0) {
        if (blockIdx.y == CHUNKS) {
            for (int i = tid; i < nb * (DR / 2); i += 256) {
                const int bi = i / (DR / 2), j = i - bi * (DR / 2), b = b0 + bi;
                int at = a.positions ? a.positions[static_cast<int64_t>(a.axis[j]) * p.B + b] : p.context_lens[b] - (p.pass1 ? 0 : 1);
                if (at < 0) {
                    if (a.positions) atomicOr(p.err, LLA_DEVERR_CONTEXT);
                    at = 0;
                }
                float sn, cs;
                turn_sincos(at, a.phi[j], &sn, &cs);
                const int ia = a.pairing ? 2 * j : j, ic = a.pairing ? 2 * j + 1 : j + DR / 2;
                const int64_t src = (static_cast<int64_t>(b) * p.H + h) * DR;
                const float x = load_elem(a.q_rope, src + ia, a.io_bf16), y = load_elem(a.q_rope, src + ic, a.io_bf16);
                uint16_t *dst = p.qt + (static_cast<int64_t>(b) * p.H + h) * 3 * RKT + RKX;
                const float u = (x * cs - y * sn) * a.scale_log2, v = (x * sn + y * cs) * a.scale_log2;
                store_parts(dst + ia, RKT, u);
                store_parts(dst + ic, RKT, v);
                float *qf = p.qf + (static_cast<int64_t>(b) * p.H + h) * RKT + RKX;
                qf[ia] = u;
                qf[ic] = v;
            }
            return;
        }
    }
    const int col = j0 + lane;
    // this thread's 16 weights: column j0 + lane, rows 16 warp .. 16 warp + 15
    const uint16_t *W = static_cast<const uint16_t *>(a.w_up_k) + th * kD * RK + col;
    float wv[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) wv[u] = col < RK ? bf_to_f(W[(warp * 16 + u) * RK]) : 0.f;
    for (int i = tid; i < 16 * kD; i += 256) {
        const int bi = i >> 7, e = i & (kD - 1);
        qs[bi][e] = bi < nb ? load_elem(a.q, (static_cast<int64_t>(b0 + bi) * p.H + h) * kD + e, a.io_bf16) : 0.f;
    }
    __syncthreads();
#pragma unroll 4
    for (int bi = 0; bi < 16; ++bi) {
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < 16; ++u) s = fmaf(wv[u], qs[bi][warp * 16 + u], s);
        red[warp][bi][lane] = s;
    }
    __syncthreads();
    for (int o = tid; o < 16 * 32; o += 256) {
        const int bi = o >> 5, c = o & 31;
        float s = 0.f;
#pragma unroll
        for (int sl = 0; sl < 8; ++sl) s += red[sl][bi][c];
        if (bi < nb && j0 + c < RKX) {
            const int64_t row = static_cast<int64_t>(b0 + bi) * p.H + h;
            s = j0 + c < RK ? s * a.scale_log2 : 0.f;
            store_parts(p.qt + row * 3 * RKT + j0 + c, RKT, s);
            p.qf[row * RKT + j0 + c] = s;
        }
    }
    if (blockIdx.y == 0) {
        for (int bi = warp; bi < nb; bi += 8) {
            float s = 0.f;
            if (a.mu_k)
                for (int e = lane; e < kD; e += 32) s = fmaf(qs[bi][e], a.mu_k[th * kD + e], s);
            s = warp_sum(s);
            if (lane == 0) p.beta[static_cast<int64_t>(b0 + bi) * p.H + h] = s * a.scale_log2;
        }
    }
}

// ------------------------------------------------------------------------------------------ trunk kernel

// Shared memory and TMEM of the trunk kernel.  Offsets from a 1024-byte aligned base (128-byte swizzle atoms of the V stages).
// THIRD: p in three parts (24 bits, for fp32 outputs); the third in rows of an operand of its own.
template <int RK, int RV, int DR, bool THIRD>
struct Z {
    static constexpr int RKX = (RK + 15) / 16 * 16;   // content contraction, zero-padded
    static constexpr int RKT = RKX + DR;              // with the rotary one
    static constexpr int RVX = (RV + 15) / 16 * 16;   // columns of O (a box reads zeros past r_v)
    static constexpr int NBOX = (RV + 63) / 64;       // TMA boxes of a V-plane
    static constexpr int BOX = kPT * 128;             // one: 64 rows x 128 bytes
    static constexpr int KPLANE = kPT * RK * 2, KPAD = kPT * RKX * 2, RPLANE = kPT * DR * 2;
    static constexpr int KPAGE = KPAD + RPLANE;
    static constexpr int VPAGE = NBOX * BOX;
    // TMEM columns: the parts of q~ (the third in shared memory where it does not fit), O, S of either group, P of either
    // group (in the columns of its S where it does not fit: then S of its next page waits for O of this one)
    static constexpr int PART = RKT / 2, PW = THIRD ? kPT : kPT / 2;  // columns of a part of q~, of a group's P
    static constexpr int QT = 3 * PART + RVX + 2 * kPT + 2 * PW <= 512 ? 3 : 2;
    static constexpr bool ALIAS = QT * PART + RVX + 2 * kPT + 2 * PW > 512;
    static constexpr uint32_t TM_Q = 0, TM_O = QT * PART, TM_S = TM_O + RVX, TM_P = ALIAS ? TM_S : TM_S + 2 * kPT;
    static constexpr uint32_t P_STEP = ALIAS ? kPT : PW;  // from one group's P to the other's
    static constexpr bool P3 = THIRD;
    static constexpr uint32_t TM_COLS = 512;
    static constexpr int QB = QT < 3 ? kRows * RKT * 2 : 0;  // the third part as an operand in shared memory
    static constexpr int QROW = 3 * RKT * 2;                // bytes of a query's parts
    // O on its way to the records: all of its columns at once, or half of them where the rotary plane needs the room
    static constexpr int XCOLS = DR > 0 ? RVX / 2 : RVX, XROW = XCOLS + 4;  // columns, floats of a row
    static constexpr int NBAR = 40;
    static constexpr int EXCH = kRows * XROW * 4;
    // running maxima; maxima and sums of three runs and two groups; a page's maxima of either group
    static constexpr int RED = (kRows + 3 * 2 * 64 * 2 + 2 * 64) * 4;
    static constexpr int FIXED = QB + EXCH + RED + NBAR * 8 + kMaxNodes * 2;
    static constexpr int ST0 = (kSmemCap - 2048 - FIXED) / (KPAGE + VPAGE);
    static constexpr int ST = ST0 > 5 ? 5 : ST0;
    static constexpr int oV = 0;
    static constexpr int oK = oV + ST * VPAGE;
    static constexpr int oQ = oK + ST * KPAGE;
    static constexpr int oExch = oQ + QB;
    static constexpr int oRed = oExch + EXCH;
    static constexpr int oBar = oRed + RED;
    static constexpr int oList = oBar + NBAR * 8;
    // (at least half of an SM's: one CTA per SM, which holds all of TMEM)
    static constexpr int SMEM0 = 1024 + oList + kMaxNodes * 2, SMEM = SMEM0 > 116 * 1024 ? SMEM0 : 116 * 1024;
    static constexpr uint32_t IDESC_S = umma_idesc_bf16(kRows, kPT, 0, 0);
    static constexpr uint32_t IDESC_O = umma_idesc_bf16(kRows, RVX, 0, 1);
    static_assert(RKT % 16 == 0 && RV % 8 == 0 && RVX % 32 == 0, "ranks");
    static_assert(TM_P + P_STEP + PW <= TM_COLS && TM_S + 2 * kPT <= TM_COLS, "TMEM columns");
    static_assert(ST >= 2 && SMEM + 1024 <= kSmemCap, "shared memory");
};

// barrier indices
enum {
    bKfull = 0 /* [5] */, bKempty = 5, bVfull = 10, bVempty = 15, bSfull = 20 /* [2] */, bSfree = 22, bPfull = 24, bPfree = 26,
    bQfull = 28, bQfree = 29, bOdone = 30, bOfree = 31 /* [2] */, bMfull = 33 /* [2] */, bAbort = 35, bTslot = 36
};

// Pages of a unit that go through O together.
struct TrunkRun {
    Node d;
    int h, page, pages;  // page: the first in the table row
    bool first, last;    // of the CTA's runs of the unit
};

struct Share {
    int g0, g1;    // pages of this CTA, among all of the kind
    int nodes, s;  // nodes in `list`, first page of the first
};

// This CTA's share of the pages of the nodes with more queries than a leaf, and the nodes that it lies in: worked out from the
// inputs of the call by all threads, so that copies can start while the absorb kernel still runs.
template <int THREADS>
__device__ Share find_share(const TrunkParams &p, int groups, uint16_t *list) {
    __shared__ int wsum[THREADS / 32], wcnt[THREADS / 32], first;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int nodes = groups + p.B, per = (nodes + THREADS - 1) / THREADS;
    auto scan = [&](int v) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += y;
        }
        return v;
    };
    auto pages = [&](int i) {
        const Node d = node_at(p, groups, i);
        return is_leaf(p, d) ? 0 : d.pages * p.H;
    };
    int tot = 0;
    for (int i = tid * per; i < min(nodes, (tid + 1) * per); ++i) tot += pages(i);
    const int x = scan(tot);
    if (lane == 31) wsum[warp] = x;
    __syncthreads();
    int ex0 = x - tot, np = 0;
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) ex0 += wsum[w];
        np += wsum[w];
    }
    // with fewer pages than CTAs the first np take one each
    const int c = blockIdx.x, we = min(static_cast<int>(gridDim.x), np);
    const Split split(np, we);
    Share r;
    r.g0 = c < we ? split.begin(c) : 0;
    r.g1 = c < we ? split.begin(c + 1) : 0;
    int mine = 0, ex = ex0;
    for (int i = tid * per; i < min(nodes, (tid + 1) * per); ++i) {
        const int n = pages(i);
        mine += n > 0 && ex < r.g1 && ex + n > r.g0;
        ex += n;
    }
    const int y = scan(mine);
    if (lane == 31) wcnt[warp] = y;
    __syncthreads();
    int at = y - mine;
    r.nodes = 0;
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) at += wcnt[w];
        r.nodes += wcnt[w];
    }
    ex = ex0;
    for (int i = tid * per; mine > 0 && i < min(nodes, (tid + 1) * per); ++i) {
        const int n = pages(i);
        if (n > 0 && ex < r.g1 && ex + n > r.g0) {
            if (at == 0) first = ex;
            list[at++] = static_cast<uint16_t>(i);
        }
        ex += n;
    }
    __syncthreads();
    r.s = r.nodes > 0 ? first : 0;
    return r;
}

// The runs of a share, in order, of at most MOST pages.
template <int MOST>
struct RunWalk {
    const TrunkParams &p;
    const uint16_t *list;
    int groups, g0, g1, nodes, i, s, u, stop, in;  // node i of the list starts at page s; u: page of the node, head by head
    Split split;
    int piece, cut;  // the run's piece of the share, and its end
    TrunkRun r;
    __device__ __forceinline__ RunWalk(const TrunkParams &pp, int gr, const Share &sh, const uint16_t *l)
        : p(pp), list(l), groups(gr), g0(sh.g0), g1(sh.g1), nodes(sh.nodes), i(-1), s(sh.s), u(0), stop(0), in(0),
          split(sh.g1 - sh.g0, (sh.g1 - sh.g0 + MOST - 1) / MOST), piece(0), cut(sh.g0 + split.begin(1)) {
        r.pages = 0;
        r.d.pages = 0;
        r.last = true;
    }
    // The next run, or false behind the last.
    __device__ __forceinline__ bool next() {
        u += r.pages;
        r.first = r.last;
        if (u < stop) {
            in += r.pages;
            if (in == r.d.pages) {
                ++r.h;
                in = 0;
            }
        } else {
            if (i >= 0) s += r.d.pages * p.H;
            if (++i >= nodes) {
                r.pages = 0;
                r.d.pages = 0;
                i = nodes;
                u = stop = 0;
                return false;
            }
            r.d = node_at(p, groups, list[i]);
            u = max(g0, s) - s;
            stop = min(g1, s + r.d.pages * p.H) - s;
            r.h = u / r.d.pages;
            in = u - r.h * r.d.pages;
        }
        if (s + u >= cut) cut = g0 + split.begin(++piece + 1);
        const int left = min(stop - u, r.d.pages - in);
        r.pages = min(left, cut - s - u);
        r.last = r.pages == left;
        r.page = r.d.first + in;
        return true;
    }
};

// Sequence * H + head of query i of a run, or -1 where it has none.
__device__ __forceinline__ int64_t query_row(const TrunkParams &p, const TrunkRun &r, int i) {
    if (i >= r.d.n) return -1;
    int b = r.d.row;
    if (r.d.member < kLevels * p.B) b = p.plan.members[r.d.member + i];
    if (b < 0 || b >= p.B) return -1;
    return static_cast<int64_t>(b) * p.H + r.h;
}

// A value that every lane has, for a warp that issues products (their descriptors are in uniform registers then).
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

// The 128 rows hold R queries 128 / R times: replica i = row / R has part i % 2 of their weights p (in the operand behind it the
// third part, where i is odd: those rows' sums are small, and what is added to them is not rounded to the size of the whole) for the tokens
// R (i / 2) to R (i / 2) + R - 1 of each page, and zeros for the others, so that a thread works on R tokens and the sum of a
// query's rows of O is the sum over all tokens of both parts.  (With R = 64 for all, two of the four schedulers did the
// work of up to 32 queries.)
__device__ __forceinline__ int replica_rows(int n) { return n > 32 ? 64 : n > 16 ? 32 : 16; }
struct SoftmaxCtx {
    uint64_t *bar;
    volatile int *abort_flag;
    unsigned *err;
    float *running, *page_max;
    float2 *states;
    int total, g;  // pages of the CTA, this group
};

template <int N>
__device__ __forceinline__ void tmem_ld_n(uint32_t taddr, float (&v)[N]) {
    static_assert(N == 16 || N == 32 || N == 64, "columns");
    if constexpr (N == 16) {
        tmem_ld16(taddr, v);
    } else {
        uint32_t a[32], b[32];
        tmem_ld32_nowait(taddr, a);
        if constexpr (N == 64) tmem_ld32_nowait(taddr + 32, b);
        tmem_wait_ld(a);
        if constexpr (N == 64) tmem_wait_ld(b);
#pragma unroll
        for (int c = 0; c < 32; ++c) {
            v[c] = __uint_as_float(a[c]);
            if constexpr (N == 64) v[32 + c] = __uint_as_float(b[c]);
        }
    }
}

template <typename ZZ, int R>
__device__ __forceinline__ void softmax_run(const SoftmaxCtx &x, int run, int it, int pages) {
    const int g = x.g, quarter = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, row = 32 * quarter + lane;
    const int replica = row / R, slice = replica >> 1, q = row % R;
    const bool second = replica & 1;
    const uint32_t tl = static_cast<uint32_t>(32 * quarter) << 16;
    const int col0 = R == 64 ? 0 : R == 32 ? 32 * (quarter >> 1) : 16 * quarter;  // the slice's tokens (of a whole warp)
    const uint32_t ts = tl + ZZ::TM_S + g * kPT + col0, tp = tl + ZZ::TM_P + g * ZZ::P_STEP;
    float m = -INFINITY, l = 0.f;
    const int first = it + ((it ^ g) & 1), end = it + pages;
    for (int j = first; j < end; j += 2) {
        const int jj = j >> 1, k = j - it;
        mbar_wait(&x.bar[bSfull + g], jj & 1, x.abort_flag, x.err);
        tc_fence_after();
        float s[R];
        tmem_ld_n<R>(ts, s);
        tc_fence_before();
        mbar_arrive(&x.bar[bSfree + g]);
        float t[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) t[c] = s[c];
#pragma unroll
        for (int c = 4; c < R; c += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = c + 4 + e < R ? fmaxf(fmaxf(t[e], s[c + e]), s[c + 4 + e]) : fmaxf(t[e], s[c + e]);
        float mx = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
        // The running maximum after the page before, from the other group's thread of this row; each page's weights are
        // relative to the running maximum that its own step leaves.  Also between runs, where nothing is handed over:
        // what the other group reads here is not written again before it has.
        if (j > 0) {
            named_bar_sync(1 + quarter * 2 + ((j - 1) & 1), 64);
            const float mp = k > 0 ? x.running[row] : m;
            if (mp != m) {
                l *= ex2_approx(m - mp);  // (m = -inf: no page yet, l = 0)
                m = mp;
            }
        }
        // the page's maximum over the slices, where one of them raises it
        if (R < 64 && named_bar_or(10 + g, 128, mx > m + kRescaleLog2)) {
            if (!second) x.page_max[g * 64 + slice * R + q] = mx;
            named_bar_sync(10 + g, 128);
#pragma unroll
            for (int i = 0; i < 64 / R; ++i) mx = fmaxf(mx, x.page_max[g * 64 + i * R + q]);
        }
        const float m_new = fmaxf(m, mx);
        const bool need = m_new > m + kRescaleLog2;  // also the first page
        const float factor = need ? ex2_approx(m - m_new) : 1.f;
        if (need) {
            l *= factor;
            m = m_new;
        }
        if (j + 1 < x.total) {
            x.running[row] = m;
            named_bar_arrive(1 + quarter * 2 + (j & 1), 64);
        }
        const bool any = __any_sync(0xffffffffu, need && k > 0);
        // this group's page before has been read by its product (and O holds it)
        if (jj > 0) mbar_wait(&x.bar[bPfree + g], (jj - 1) & 1, x.abort_flag, x.err);
        if (any) {
            // O holds the run's pages before this one: wait for the last of them, which is the other group's (products
            // complete in order, so that its barrier is at most one phase behind), and rescale
            mbar_wait(&x.bar[bPfree + (g ^ 1)], ((j - 1) >> 1) & 1, x.abort_flag, x.err);
            tc_fence_after();
#pragma unroll 1
            for (int c0 = 0; c0 < ZZ::RVX; c0 += 16) {
                float v[16];
                tmem_ld16(tl + ZZ::TM_O + c0, v);
#pragma unroll
                for (int c = 0; c < 16; ++c) v[c] *= factor;
                tmem_st16(tl + ZZ::TM_O + c0, v);
            }
        }
        tc_fence_after();
        if (R < 64 && (ZZ::ALIAS || j == first)) {  // the other slices' tokens
            uint32_t zero[16];
#pragma unroll
            for (int c = 0; c < 16; ++c) zero[c] = 0;
            tmem_st16u(tp, zero);
            tmem_st16u(tp + 16, zero);
            if constexpr (ZZ::P3) {
                tmem_st16u(tp + kPT / 2, zero);
                tmem_st16u(tp + kPT / 2 + 16, zero);
            }
            tmem_wait_st();
        }
        const float2 mm = make_float2(-m, -m);
        uint32_t pw[R / 2];
        float2 s4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) s4[e] = make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < R; c += 2) {
            float2 y = __fadd2_rn(make_float2(s[c], s[c + 1]), mm);
            y.x = ex2_approx(y.x);
            y.y = ex2_approx(y.y);
            s4[(c >> 1) & 3] = __fadd2_rn(s4[(c >> 1) & 3], y);
            pw[c / 2] = pack_bf16x2(y.x, y.y);
            const float2 f = bf2_to_f2(pw[c / 2]);
            const uint32_t rest = pack_bf16x2(y.x - f.x, y.y - f.y);
            if constexpr (ZZ::P3) {  // (s is free behind its weight: the third part in its place)
                const float2 r = bf2_to_f2(rest);
                s[c] = second ? (y.x - f.x) - r.x : 0.f;
                s[c + 1] = second ? (y.y - f.y) - r.y : 0.f;
            }
            if (second) pw[c / 2] = rest;
        }
        const float2 sa = __fadd2_rn(s4[0], s4[1]), sb = __fadd2_rn(s4[2], s4[3]);
        l += (sa.x + sa.y) + (sb.x + sb.y);
        auto store = [&](uint32_t at) {
            if constexpr (R == 64) tmem_st32u_nowait(at, pw);
            else if constexpr (R == 32) tmem_st16u(at + col0 / 2, pw);
            else tmem_st8u(at + col0 / 2, pw);
        };
        store(tp);
        if constexpr (ZZ::P3) {
#pragma unroll
            for (int c = 0; c < R; c += 2) pw[c / 2] = pack_bf16x2(s[c], s[c + 1]);
            store(tp + kPT / 2);
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&x.bar[bPfull + g]);
    }
    // this group's maxima and sums of the run.  Three slots: when O of run - 2 is free the states of run - 3 have been read.
    if (run >= 2) mbar_wait(&x.bar[bOfree + (run & 1)], ((run - 2) >> 1) & 1, x.abort_flag, x.err);
    if (!second) x.states[((run % 3) * 2 + g) * 64 + slice * R + q] = make_float2(m, l);
    mbar_arrive(&x.bar[bMfull + (run & 1)]);
}

template <int RK, int RV, int DR, bool THIRD>
__global__ void __launch_bounds__(kTrunkThreads, 1)
    trunk_kernel(const __grid_constant__ CUtensorMap tv, const __grid_constant__ TrunkParams p) {
    using ZZ = Z<RK, RV, DR, THIRD>;
    extern __shared__ __align__(1024) char sm_raw[];
    char *sm = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(sm_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint64_t *bar = reinterpret_cast<uint64_t *>(sm + ZZ::oBar);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(bar + bAbort);
    uint32_t *tslot = reinterpret_cast<uint32_t *>(bar + bTslot);
    float *running = reinterpret_cast<float *>(sm + ZZ::oRed);          // [128] maxima
    float2 *states = reinterpret_cast<float2 *>(running + kRows);       // [3 runs][2 groups][64] maxima and sums
    float *page_max = reinterpret_cast<float *>(states + 3 * 2 * 64);    // [2 groups][64]
    uint16_t *list = reinterpret_cast<uint16_t *>(sm + ZZ::oList);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

    const int groups = count_groups(p);
    if (groups == 0) {  // nothing is shared
        pdl_wait();
        return;
    }
    if (tid == 0) {
        for (int s = 0; s < ZZ::ST; ++s) {
            mbar_init(&bar[bKfull + s], 1);
            mbar_init(&bar[bKempty + s], 1);
            mbar_init(&bar[bVfull + s], 1);
            mbar_init(&bar[bVempty + s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bar[bSfull + s], 1);
            mbar_init(&bar[bSfree + s], 128);
            mbar_init(&bar[bPfull + s], 128);
            mbar_init(&bar[bPfree + s], 1);
            mbar_init(&bar[bOfree + s], 128);
            mbar_init(&bar[bMfull + s], 256);
        }
        mbar_init(&bar[bQfull], 128);
        mbar_init(&bar[bQfree], 1);
        mbar_init(&bar[bOdone], 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) tmem_alloc(tslot, ZZ::TM_COLS);
    if constexpr (ZZ::KPAD > ZZ::KPLANE) {  // the K granules past r_k stay zero (against zero q~ columns)
        for (int s = 0; s < ZZ::ST; ++s)
            for (int i = tid; i < (ZZ::KPAD - ZZ::KPLANE) / 16; i += kTrunkThreads)
                reinterpret_cast<uint4 *>(sm + ZZ::oK + s * ZZ::KPAGE + ZZ::KPLANE)[i] = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    constexpr uint32_t tmem = 0;  // the whole of TMEM is allocated (one CTA per SM)
    const Share sh = find_share<kTrunkThreads>(p, groups, list);
    // q~ and beta come from the absorb kernel, and the workspace is free once it has waited for the kernel before it; the
    // producers read only inputs of the call, which that kernel's wait ordered before this launch, and wait at their end
    if (warp != 0 && warp != 2) {
        pdl_wait();
        pdl_trigger();  // the leaf kernel may take this SM as soon as this CTA has left it
    }
    RunWalk<kRunPages<THIRD>> w(p, groups, sh, list);

    if (warp == 0 || warp == 2) {
        // ------------------------------------------------------------------------------ producers
        if (lane == 0) {
            // after a failed wait (or once the abort flag is up) no further copy is issued, so no full barrier receives a
            // second arrival in one phase; the last ST rounds issued are awaited below
            const int full = warp == 0 ? bKfull : bVfull, empty = warp == 0 ? bKempty : bVempty;
            const uint64_t pol = policy_evict_first();
            int it = 0;
            bool stop = false;
            while (!stop && w.next()) {
                const int32_t *bt = p.block_table + static_cast<int64_t>(w.r.d.row) * p.max_blocks + w.r.page;
                for (int k = 0; k < w.r.pages; ++k, ++it) {
                    const int st = it % ZZ::ST;
                    int32_t blk = bt[k];
                    if (blk < 0 || blk >= p.num_blocks) {
                        atomicOr(p.err, LLA_DEVERR_BLOCK_ID);
                        blk = 0;
                    }
                    const int64_t page = static_cast<int64_t>(blk) * p.H + w.r.h;
                    if (!mbar_wait(&bar[empty + st], ((it / ZZ::ST) & 1) ^ 1u, abort_flag, p.err) || *abort_flag) {
                        stop = true;
                        break;
                    }
                    if (warp == 0) {
                        mbar_arrive_expect_tx(&bar[bKfull + st], ZZ::KPLANE + ZZ::RPLANE);
                        char *ks = sm + ZZ::oK + st * ZZ::KPAGE;
                        bulk_g2s(ks, p.pool + page * p.page_bytes, ZZ::KPLANE, &bar[bKfull + st], pol);
                        if constexpr (DR > 0)
                            bulk_g2s(ks + ZZ::KPAD, p.rope_pool + static_cast<int64_t>(blk) * ZZ::RPLANE, ZZ::RPLANE, &bar[bKfull + st], pol);
                    } else {
                        mbar_arrive_expect_tx(&bar[bVfull + st], ZZ::VPAGE);
                        char *vs = sm + ZZ::oV + st * ZZ::VPAGE;
#pragma unroll
                        for (int a = 0; a < ZZ::NBOX; ++a)
                            tma_load_3d(vs + a * ZZ::BOX, &tv, a * 64, 0, static_cast<int>(page), &bar[bVfull + st]);
                    }
                }
            }
            // every copy has landed before the CTA can exit, even after an abort
            volatile int never = 0;
            for (int j = max(0, it - ZZ::ST); j < it; ++j) mbar_wait(&bar[full + j % ZZ::ST], (j / ZZ::ST) & 1, &never, p.err);
        }
        __syncwarp();
        pdl_wait();
    } else if (warp == 1) {
        // ------------------------------------------------------------------------------- S issuer
        const uint32_t base = smem_addr(sm);
        const uint64_t dk0 = umma_desc(base + ZZ::oK, kPT * 16, 128);
        [[maybe_unused]] const uint64_t dq = umma_desc(base + ZZ::oQ, kRows * 16, 128);
        int it = 0, parts = 0;
        while (uniform(w.next())) {
            const int pages = uniform(w.r.pages), last = uniform(w.r.last);
            if (uniform(w.r.first)) mbar_wait_warp(&bar[bQfull], parts++ & 1, abort_flag, p.err);
            for (int k = 0; k < pages; ++k, ++it) {
                const int g = it & 1, st = it % ZZ::ST;
                mbar_wait_warp(&bar[bKfull + st], (it / ZZ::ST) & 1, abort_flag, p.err);
                if (it >= 2) mbar_wait_warp(&bar[(ZZ::ALIAS ? bPfree : bSfree) + g], ((it >> 1) - 1) & 1, abort_flag, p.err);
                tc_fence_after();
                const uint64_t dk = dk0 + static_cast<uint64_t>((st * ZZ::KPAGE) >> 4);
                const uint32_t ts = tmem + ZZ::TM_S + g * kPT;
                // the small parts first: what they add is not rounded to the size of the whole
#pragma unroll
                for (int part = 2; part >= 0; --part)
#pragma unroll
                    for (int ks = 0; ks < ZZ::RKT / 16; ++ks) {
                        const bool more = part < 2 || ks > 0;
                        if (part < ZZ::QT)
                            umma_bf16_ts_warp(ts, tmem + ZZ::TM_Q + part * ZZ::PART + ks * 8, dk + ks * ((2 * kPT * 16) >> 4), ZZ::IDESC_S, more);
                        else
                            umma_bf16_warp(ts, dq + ks * ((2 * kRows * 16) >> 4), dk + ks * ((2 * kPT * 16) >> 4), ZZ::IDESC_S, more);
                    }
                if (last && k == pages - 1) umma_commit_warp(&bar[bQfree]);
                umma_commit_warp(&bar[bKempty + st]);
                umma_commit_warp(&bar[bSfull + g]);
            }
        }
        // every product has completed before TMEM is released, even after an abort: the last commit on each buffer
        volatile int never = 0;
        for (int j = max(0, it - 2); j < it; ++j) mbar_wait_warp(&bar[bSfull + (j & 1)], (j >> 1) & 1, &never, p.err);
        __syncwarp();
    } else if (warp == 3) {
        // ------------------------------------------------------------------------------- O issuer
        const uint32_t base = smem_addr(sm);
        const uint64_t dv0 = umma_desc_sw128_mn(base + ZZ::oV, ZZ::BOX);
        int it = 0;
        for (int run = 0; uniform(w.next()); ++run) {
            const int pages = uniform(w.r.pages);
            for (int k = 0; k < pages; ++k, ++it) {
                const int g = it & 1, st = it % ZZ::ST;
                mbar_wait_warp(&bar[bVfull + st], (it / ZZ::ST) & 1, abort_flag, p.err);
                mbar_wait_warp(&bar[bPfull + g], (it >> 1) & 1, abort_flag, p.err);
                // the first page of a run starts O anew, once the run before has been read
                if (k == 0 && run > 0) mbar_wait_warp(&bar[bOfree + ((run - 1) & 1)], ((run - 1) >> 1) & 1, abort_flag, p.err);
                tc_fence_after();
                const uint64_t dv = dv0 + static_cast<uint64_t>((st * ZZ::VPAGE) >> 4);
#pragma unroll
                for (int ks = 0; ks < kPT / 16; ++ks)
                    umma_bf16_ts_warp(tmem + ZZ::TM_O, tmem + ZZ::TM_P + g * ZZ::P_STEP + ks * 8, dv + ks * (2048 >> 4), ZZ::IDESC_O, k > 0 || ks > 0);
                if constexpr (THIRD) {
#pragma unroll
                    for (int ks = 0; ks < kPT / 16; ++ks)
                        umma_bf16_ts_warp(tmem + ZZ::TM_O, tmem + ZZ::TM_P + g * ZZ::P_STEP + kPT / 2 + ks * 8, dv + ks * (2048 >> 4), ZZ::IDESC_O, true);
                }
                umma_commit_warp(&bar[bVempty + st]);
                if (k == pages - 1) umma_commit_warp(&bar[bOdone]);
                umma_commit_warp(&bar[bPfree + g]);  // also: O holds pages up to it
            }
        }
        // every product has completed before TMEM is released, even after an abort
        volatile int never = 0;
        for (int j = max(0, it - 2); j < it; ++j) mbar_wait_warp(&bar[bPfree + (j & 1)], (j >> 1) & 1, &never, p.err);
        __syncwarp();
    } else if (warp < kAuxWarp) {
        // ------------------------------------------------------------------- softmax, warps 4-7 and 8-11
        SoftmaxCtx x = {bar, abort_flag, p.err, running, page_max, states, sh.g1 - sh.g0, (warp - kSoftmaxWarp) >> 2};
        int it = 0;
        for (int run = 0; w.next(); ++run) {
            if (w.r.d.n > 32) softmax_run<ZZ, 64>(x, run, it, w.r.pages);
            else if (w.r.d.n > 16) softmax_run<ZZ, 32>(x, run, it, w.r.pages);
            else softmax_run<ZZ, 16>(x, run, it, w.r.pages);
            it += w.r.pages;
        }
    } else {
        // --------------------------------------------------------- q~ and epilogue, warps 12-15
        constexpr int RS = record_floats(RV);
        const int quarter = warp & 3, row = 32 * quarter + lane;
        const uint32_t tl = tmem + (static_cast<uint32_t>(32 * quarter) << 16);
        // the parts of a run's queries into TMEM, row by row, a fetch ahead of what is stored
        constexpr int WORDS = ZZ::RKT / 8, AT_ONCE = WORDS <= 12 ? WORDS : WORDS / 2, CHUNKS = 3 * WORDS / AT_ONCE;  // of 16 bytes
        static_assert(AT_ONCE % 2 == 0 && AT_ONCE <= 12, "words of two");
        uint4 v[2][AT_ONCE];
        const char *src = nullptr;
        auto fetch = [&](int c) {
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
                v[c & 1][i] = src ? *reinterpret_cast<const uint4 *>(src + (c * AT_ONCE + i) * 16) : make_uint4(0, 0, 0, 0);
        };
        // the first words of a run's queries, before their place is free
        auto fetch_queries = [&](const TrunkRun &r) {
            const int64_t q = query_row(p, r, row & (replica_rows(r.d.n) - 1));
            src = q < 0 ? nullptr : reinterpret_cast<const char *>(p.qt) + q * ZZ::QROW;
            fetch(0);
        };
        auto store_queries = [&] {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                if (c + 1 < CHUNKS) fetch(c + 1);
                const int part = c * AT_ONCE / WORDS, w0 = c * AT_ONCE - part * WORDS;
                if (part < ZZ::QT) {
#pragma unroll
                    for (int i = 0; i < AT_ONCE; i += 2) {
                        const uint4 a = v[c & 1][i], b = v[c & 1][i + 1];
                        const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                        tmem_st8u(tl + ZZ::TM_Q + part * ZZ::PART + (w0 + i) * 4, u);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i) *reinterpret_cast<uint4 *>(sm + ZZ::oQ + (w0 + i) * (kRows * 16) + row * 16) = v[c & 1][i];
                }
            }
            if (ZZ::QT < 3) fence_proxy_async_smem();
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&bar[bQfull]);
        };
        RunWalk<kRunPages<THIRD>> ahead(p, groups, sh, list);
        if (ahead.next()) {
            fetch_queries(ahead.r);
            store_queries();
        }
        for (int run = 0, parts = 0; w.next(); ++run) {
            if (ahead.next() && ahead.r.first) {  // the next unit's q~, as soon as S of this one's pages is done
                fetch_queries(ahead.r);
                mbar_wait(&bar[bQfree], parts++ & 1, abort_flag, p.err);
                tc_fence_after();
                store_queries();
            }
            const int n = w.r.d.n, R = replica_rows(n);
            const bool joins = !w.r.first;  // the record holds the part's runs before this one
            float *rec = p.part + record_of(p, w.r.d, w.r.h, blockIdx.x) * RS;
            float *exch = reinterpret_cast<float *>(sm + ZZ::oExch);
            float2 *state = reinterpret_cast<float2 *>(rec + row * RS + RV);  // of query `row`: maximum and sum
            const float2 was_state = joins && row < n ? *state : make_float2(0.f, 0.f);
            mbar_wait(&bar[bOdone], run & 1, abort_flag, p.err);
            mbar_wait(&bar[bMfull + (run & 1)], (run >> 1) & 1, abort_flag, p.err);
            tc_fence_after();
            auto run_state = [&] {  // of query `row`: maximum and sum of both groups (whose slices have one maximum)
                const float2 *st = states + (run % 3) * 2 * 64;
                const float m0 = st[row].x, m1 = st[64 + row].x, m = fmaxf(m0, m1);
                float l0 = 0.f, l1 = 0.f;
                for (int i = row; i < 64; i += R) {
                    l0 += st[i].y;
                    l1 += st[64 + i].y;
                }
                return make_float2(m, (m0 == m ? l0 : l0 * ex2_approx(m0 - m)) + (m1 == m ? l1 : l1 * ex2_approx(m1 - m)));
            };
            // every row of O into shared memory, which frees it, and from there the sums of the queries' rows
#pragma unroll 1
            for (int c0 = 0; c0 < ZZ::RVX; c0 += ZZ::XCOLS) {
                if (c0 > 0) named_bar_sync(9, 128);
#pragma unroll 1
                for (int c = 0; c < ZZ::XCOLS; c += 16) {
                    float o[16];
                    tmem_ld16(tl + ZZ::TM_O + c0 + c, o);
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        *reinterpret_cast<float4 *>(exch + row * ZZ::XROW + c + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                }
                if (c0 + ZZ::XCOLS >= ZZ::RVX) {
                    tc_fence_before();
                    mbar_arrive(&bar[bOfree + (run & 1)]);
                }
                if (joins && c0 == 0 && row < n) {
                    const float2 now = run_state(), was = was_state;
                    const float m = fmaxf(was.x, now.x);
                    const float2 f = make_float2(ex2_approx(was.x - m), ex2_approx(now.x - m));
                    *reinterpret_cast<float2 *>(exch + row * ZZ::XROW + ZZ::XCOLS) = f;  // (behind the columns of a row)
                    *state = make_float2(m, fmaf(was.y, f.x, now.y * f.y));
                }
                named_bar_sync(9, 128);
                const int words = min(ZZ::XCOLS, RV - c0) / 4;
                auto sum = [&](int q, int c) {
                    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int k = q; k < kRows; k += R) {
                        const float4 b = *reinterpret_cast<const float4 *>(exch + k * ZZ::XROW + c);
                        a = make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
                    }
                    return a;
                };
                auto at = [&](int q, int c) { return reinterpret_cast<float4 *>(rec + static_cast<int64_t>(q) * RS + c0 + c); };
                if (joins) {  // (a thread has the same words of every run of a part)
#pragma unroll 2
                    for (int i = row; i < n * words; i += 128) {
                        const int q = i / words, c = 4 * (i - q * words);
                        const float4 was = *at(q, c), a = sum(q, c);
                        const float2 f = *reinterpret_cast<const float2 *>(exch + q * ZZ::XROW + ZZ::XCOLS);
                        *at(q, c) = make_float4(fmaf(was.x, f.x, a.x * f.y), fmaf(was.y, f.x, a.y * f.y), fmaf(was.z, f.x, a.z * f.y), fmaf(was.w, f.x, a.w * f.y));
                    }
                } else {
#pragma unroll 2
                    for (int i = row; i < n * words; i += 128) {
                        const int q = i / words, c = 4 * (i - q * words);
                        *at(q, c) = sum(q, c);
                    }
                }
            }
            if (!joins && row < n) *state = run_state();
            named_bar_sync(9, 128);  // the shared memory is free
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, ZZ::TM_COLS);
    }
}

// -------------------------------------------------------------------------------------------- leaf kernel

// Shared memory of the join kernel.
constexpr int kJoinThreads = 512, kJoinWarps = kJoinThreads / 32;
template <int RV>
struct J {
    static constexpr int RVX = (RV + 15) / 16 * 16;     // columns of the projection, zeros past r_v
    static constexpr int WROW = (RVX / 8 | 1) * 16;     // bytes of a row of W_up^V: an odd number of 16-byte words
    static constexpr int OROW = RVX + 8;                // floats of a row of o~
    static constexpr int oO = kD * WROW, oCoef = oO + kJoinWarps * OROW * 4;
    static constexpr int SMEM = oCoef + kJoinSeqs * 16;  // weights, a row of o~ of each warp, coefficients
    static_assert(OROW % 32 == 8, "rows of o~ in other banks");
};

// Shared memory of the leaf kernel: a slot for one page, the queries and the weights of each warp.
constexpr int kMaxWarps = 9;
template <int RK, int RV, int DR, bool ALONE>
struct L {
    static constexpr int NQ = ALONE ? kLeafAlone : kLeaf;  // queries of a node
    static constexpr int RKX = (RK + 15) / 16 * 16, RKT = RKX + DR;
    static constexpr int KPLANE = kPT * RK * 2, RPLANE = kPT * DR * 2, VPLANE = kPT * RV * 2;
    static constexpr int SLOT = KPLANE + RPLANE + VPLANE;
    static constexpr int SCRATCH = NQ * (2 * RKT + kPT) * 4 + 16;  // q~ of two runs, p, two barriers
    // a CTA of the join kernel has room beside this one (1 KB of each is the system's)
    static constexpr int W0 = (kSmemCap + 1024 - 2 * 1024 - 256 - J<RV>::SMEM) / (SLOT + SCRATCH);
    static constexpr int WARPS = W0 > kMaxWarps ? kMaxWarps : W0;
    static constexpr int oScratch = WARPS * SLOT;
    static constexpr int oAbort = oScratch + WARPS * SCRATCH, SMEM = 128 + oAbort + 16;
    static constexpr bool TAIL = RV > 128;  // 4 columns in each lane, and one more behind the 128th
    static_assert(RV <= 160 && (RV <= 128 || RV == 160) && SCRATCH % 16 == 0, "columns of a warp");
};

// A warp's pages in order: of its first share, and of those that it takes then.
struct LeafWalk {
    const TrunkParams &p;
    const LeafShares &sh;
    const int *before;  // pages of the leaves before each node
    int groups, nodes, share, u, end;  // pages u to end of the share are left
    int i, s;                          // the node, and the page that it starts at
    TrunkRun r;                        // the run
    int k;                             // page of the run
    bool ok;
    __device__ __forceinline__ LeafWalk(const TrunkParams &pp, const LeafShares &ss, int gr, int first)
        : p(pp), sh(ss), before(pp.pstart + kMaxNodes + 1), groups(gr), nodes(gr + pp.B), share(first), u(0), end(0), i(-1), s(0), k(0) {
        r.d.pages = 0;
        ok = share < sh.w1;
        if (ok) {
            u = sh.begin(share);
            end = sh.begin(share + 1);
            next_run();
        }
    }
    // The last node with at most u pages of leaves before it: the one that page u lies in.  32 nodes behind node i are looked at
    // first, then 32 parts of what is left.
    __device__ __forceinline__ void find_node() {
        const int page = u / p.H, lane = threadIdx.x & 31;
        int lo = max(i, 0), n = nodes - lo;
        for (int step = 1;; step = (n + 31) / 32) {
            const int at = lo + lane * step;
            const int c = __popc(__ballot_sync(0xffffffffu, lane * step < n && __ldcg(before + at) <= page));  // (at least one)
            lo += (c - 1) * step;
            n -= (c - 1) * step;
            if (c < 32) n = min(n, step);
            if (n == 1 || (step == 1 && c < 32)) break;
        }
        i = lo;
        s = __ldcg(before + i) * p.H;
        r.d = node_at(p, groups, i);
    }
    __device__ __forceinline__ void next_run() {
        if (u >= s + r.d.pages * p.H) find_node();
        r.h = (u - s) / r.d.pages;
        const int in = u - s - r.h * r.d.pages;
        r.page = r.d.first + in;
        r.pages = min(end - u, r.d.pages - in);
        u += r.pages;
        k = 0;
    }
    __device__ __forceinline__ void step() {
        if (++k < r.pages || !ok) return;
        if (u >= end) {
            if ((threadIdx.x & 31) == 0) share = sh.w1 + atomicAdd(p.next, 1);
            share = __shfl_sync(0xffffffffu, share, 0);
            ok = share < sh.count();
            if (!ok) return;
            u = sh.begin(share);
            end = sh.begin(share + 1);
        }
        next_run();
    }
    __device__ __forceinline__ int block() const {
        return ok ? p.block_table[static_cast<int64_t>(r.d.row) * p.max_blocks + r.page + k] : 0;
    }
};

// One page of NQ queries, by a warp: scores of tokens lane and lane + 32 from the K-plane (and the rotary plane), the online
// softmax of each query, and 4 or 5 columns of its value sum in each lane.  `k_read` is called when the K-plane has been read.
template <typename LL, int NQ, typename F>
__device__ __forceinline__ void leaf_page(const char *slot, const float *qs, float *ps, int left, float (&m)[LL::NQ], float (&l)[LL::NQ],
                                          float (&acc)[LL::NQ][5], F k_read) {
    constexpr int RV = LL::VPLANE / (kPT * 2);
    const int lane = threadIdx.x & 31;
    float s[NQ][2][2];  // of two tokens, in two sums each: shorter chains, and less to round
#pragma unroll
    for (int q = 0; q < NQ; ++q) s[q][0][0] = s[q][0][1] = s[q][1][0] = s[q][1][1] = 0.f;
    auto dot = [&](const char *plane, const float *qq, int granules) {
#pragma unroll 2
        for (int g = 0; g < granules; ++g) {
            const uint4 a = *reinterpret_cast<const uint4 *>(plane + g * (kPT * 16) + lane * 16);
            const uint4 b = *reinterpret_cast<const uint4 *>(plane + g * (kPT * 16) + (lane + 32) * 16);
            const float2 a0 = bf2_to_f2(a.x), a1 = bf2_to_f2(a.y), a2 = bf2_to_f2(a.z), a3 = bf2_to_f2(a.w);
            const float2 b0 = bf2_to_f2(b.x), b1 = bf2_to_f2(b.y), b2 = bf2_to_f2(b.z), b3 = bf2_to_f2(b.w);
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const float4 u = *reinterpret_cast<const float4 *>(qq + q * LL::RKT + g * 8), v = *reinterpret_cast<const float4 *>(qq + q * LL::RKT + g * 8 + 4);
                s[q][0][0] = fmaf(a1.y, u.w, fmaf(a1.x, u.z, fmaf(a0.y, u.y, fmaf(a0.x, u.x, s[q][0][0]))));
                s[q][0][1] = fmaf(a3.y, v.w, fmaf(a3.x, v.z, fmaf(a2.y, v.y, fmaf(a2.x, v.x, s[q][0][1]))));
                s[q][1][0] = fmaf(b1.y, u.w, fmaf(b1.x, u.z, fmaf(b0.y, u.y, fmaf(b0.x, u.x, s[q][1][0]))));
                s[q][1][1] = fmaf(b3.y, v.w, fmaf(b3.x, v.z, fmaf(b2.y, v.y, fmaf(b2.x, v.x, s[q][1][1]))));
            }
        }
    };
    dot(slot, qs, LL::KPLANE / (kPT * 16));
    if constexpr (LL::RPLANE > 0) dot(slot + LL::KPLANE, qs + LL::RKX, LL::RPLANE / (kPT * 16));
    k_read();
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const float x0 = lane < left ? s[q][0][0] + s[q][0][1] : -INFINITY, x1 = lane + 32 < left ? s[q][1][0] + s[q][1][1] : -INFINITY;
        const float mn = fmaxf(m[q], warp_max(fmaxf(x0, x1)));
        const float f = m[q] == -INFINITY ? 0.f : ex2_approx(m[q] - mn);
        const float p0 = ex2_approx(x0 - mn), p1 = ex2_approx(x1 - mn);
        m[q] = mn;
        l[q] = fmaf(l[q], f, p0 + p1);
        ps[q * kPT + lane] = p0;
        ps[q * kPT + 32 + lane] = p1;
#pragma unroll
        for (int e = 0; e < 5; ++e) acc[q][e] *= f;
    }
    __syncwarp();
    const char *vp = slot + LL::KPLANE + LL::RPLANE;
    const int c4 = lane * 4 < RV ? lane * 8 : 0;
    auto token = [&](int t, const float (&pv)[NQ]) {
        const uint2 a = *reinterpret_cast<const uint2 *>(vp + t * (RV * 2) + c4);
        const float2 a0 = bf2_to_f2(a.x), a1 = bf2_to_f2(a.y);
        float a4 = 0.f;
        if constexpr (LL::TAIL) a4 = bf_to_f(*reinterpret_cast<const uint16_t *>(vp + t * (RV * 2) + 256 + lane * 2));
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            acc[q][0] = fmaf(pv[q], a0.x, acc[q][0]);
            acc[q][1] = fmaf(pv[q], a0.y, acc[q][1]);
            acc[q][2] = fmaf(pv[q], a1.x, acc[q][2]);
            acc[q][3] = fmaf(pv[q], a1.y, acc[q][3]);
            if constexpr (LL::TAIL) acc[q][4] = fmaf(pv[q], a4, acc[q][4]);
        }
    };
    const int nt = min(left, kPT);  // rows behind the sequence hold no latents
#pragma unroll 2
    for (int t = 0; t + 4 <= nt; t += 4) {
        float4 p4[NQ];
#pragma unroll
        for (int q = 0; q < NQ; ++q) p4[q] = *reinterpret_cast<const float4 *>(ps + q * kPT + t);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float pv[NQ];
#pragma unroll
            for (int q = 0; q < NQ; ++q) pv[q] = i == 0 ? p4[q].x : i == 1 ? p4[q].y : i == 2 ? p4[q].z : p4[q].w;
            token(t + i, pv);
        }
    }
    for (int t = nt & ~3; t < nt; ++t) {
        float pv[NQ];
#pragma unroll
        for (int q = 0; q < NQ; ++q) pv[q] = ps[q * kPT + t];
        token(t, pv);
    }
}

// Every warp streams its own pages through a slot of its own: while it works on the values of a page the K-plane of the next
// one lands, and while it works on that one's scores its V-plane does.  The other warps' copies fill the rest of HBM's time, so
// that a warp's run boundaries (the queries of the next run, the record of this one) cost nothing until the warps of an SM
// together cannot keep up.
template <int RK, int RV, int DR, bool ALONE>
__global__ void __maxnreg__(ALONE ? 160 : 120) leaf_kernel(const __grid_constant__ TrunkParams p) {
    using LL = L<RK, RV, DR, ALONE>;
    constexpr int NQ = LL::NQ;
    constexpr int RS = record_floats(RV);
    extern __shared__ __align__(128) char sm[];
    volatile int *abort_flag = reinterpret_cast<int *>(sm + LL::oAbort);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    char *slot = sm + warp * LL::SLOT;
    uint64_t *bar = reinterpret_cast<uint64_t *>(sm + LL::oScratch + warp * LL::SCRATCH);  // K, V
    float *qbuf = reinterpret_cast<float *>(bar + 2), *ps = qbuf + 2 * NQ * LL::RKT;
    if (lane == 0) {
        mbar_init(&bar[0], 1);
        mbar_init(&bar[1], 1);
        fence_mbar_init();
    }
    if (tid == 0) *abort_flag = 0;
    __syncthreads();
    // The trunk kernel lets this one start when all of its CTAs have waited for the absorb kernel, so that q~ and beta are
    // there and the workspace is free.  Its own records are not read here; the wait for it is at the end.
    if (ALONE) pdl_wait();  // there is no trunk kernel between the absorb kernel and this one
    pdl_trigger();          // the join may take this SM as soon as this CTA has left it
    const int groups = count_groups(p);
    const LeafShares shares(__ldcg(p.pstart + kMaxNodes + 1 + groups + p.B) * p.H, gridDim.x * LL::WARPS);
    LeafWalk ahead(p, shares, groups, blockIdx.x * LL::WARPS + warp);
    if (ahead.ok) {
        const uint64_t pol = policy_evict_first();
        auto checked = [&](int blk) {
            if (blk >= 0 && blk < p.num_blocks) return blk;
            if (lane == 0) atomicOr(p.err, LLA_DEVERR_BLOCK_ID);
            return 0;
        };
        auto issue_k = [&](int blk, int h) {
            if (lane == 0) {
                mbar_arrive_expect_tx(&bar[0], LL::KPLANE + LL::RPLANE);
                bulk_g2s(slot, p.pool + (static_cast<int64_t>(blk) * p.H + h) * p.page_bytes, LL::KPLANE, &bar[0], pol);
                if constexpr (DR > 0)
                    bulk_g2s(slot + LL::KPLANE, p.rope_pool + static_cast<int64_t>(blk) * LL::RPLANE, LL::RPLANE, &bar[0], pol);
            }
        };
        auto issue_v = [&](int blk, int h) {
            if (lane == 0) {
                mbar_arrive_expect_tx(&bar[1], LL::VPLANE);
                bulk_g2s(slot + LL::KPLANE + LL::RPLANE, p.pool + (static_cast<int64_t>(blk) * p.H + h) * p.page_bytes + LL::KPLANE, LL::VPLANE,
                         &bar[1], pol);
            }
        };
        // the queries of a run, as soon as its first page is asked for (loaded at its start, they took 2.6 us a run)
        auto fetch_queries = [&](const TrunkRun &r, int run) {
            for (int q = 0; q < (r.d.n == 3 ? 4 : r.d.n); ++q) {  // (beside three queries there is a fourth of zeros)
                const int64_t row = query_row(p, r, q);
                float *dst = qbuf + ((run & 1) * NQ + q) * LL::RKT;
                for (int i = lane * 4; i < LL::RKT; i += 128) {
                    if (row >= 0) cp_async16(dst + i, p.qf + row * LL::RKT + i);
                    else *reinterpret_cast<float4 *>(dst + i) = make_float4(0.f, 0.f, 0.f, 0.f);
                }
            }
            cp_async_commit();
        };
        int blk = checked(ahead.block());
        issue_k(blk, ahead.r.h);
        issue_v(blk, ahead.r.h);
        fetch_queries(ahead.r, 0);
        int it = 0, run = 0, issued_k = 1, issued_v = 1;
        bool ok = true;
        for (; ok && ahead.ok; ++run) {
            const TrunkRun r = ahead.r;
            const int n = r.d.n, share = ahead.share;
            const float *qs = qbuf + (run & 1) * NQ * LL::RKT;
            cp_async_wait_all();
            __syncwarp();
            float m[NQ], l[NQ], acc[NQ][5];
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                m[q] = -INFINITY;
                l[q] = 0.f;
#pragma unroll
                for (int e = 0; e < 5; ++e) acc[q][e] = 0.f;
            }
            for (int k = 0; ok && k < r.pages; ++k, ++it) {
                const int left = r.d.len - (r.page + k) * kPT;
                ahead.step();
                const int next = ahead.block();  // (in flight while the scores are worked out)
                if (ahead.ok && ahead.k == 0) fetch_queries(ahead.r, run + 1);
                ok = mbar_wait(&bar[0], it & 1, abort_flag, p.err);
                auto k_read = [&] {
                    __syncwarp();
                    blk = checked(next);
                    if (ok && ahead.ok) {
                        issue_k(blk, ahead.r.h);
                        ++issued_k;
                    }
                    ok = mbar_wait(&bar[1], it & 1, abort_flag, p.err) && ok;
                };
                if (n == 1) leaf_page<LL, 1>(slot, qs, ps, left, m, l, acc, k_read);
                else if (NQ == 2 || n == 2) leaf_page<LL, 2>(slot, qs, ps, left, m, l, acc, k_read);
                else leaf_page<LL, NQ>(slot, qs, ps, left, m, l, acc, k_read);
                __syncwarp();
                if (ok && ahead.ok) {
                    issue_v(blk, ahead.r.h);
                    ++issued_v;
                }
            }
            float *dst = p.part + record_of(p, r.d, r.h, share) * RS;
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const float sum = warp_sum(l[q]);
                if (q >= n) continue;
                if (lane * 4 < RV)
                    *reinterpret_cast<float4 *>(dst + q * RS + lane * 4) = make_float4(acc[q][0], acc[q][1], acc[q][2], acc[q][3]);
                if constexpr (LL::TAIL) dst[q * RS + 128 + lane] = acc[q][4];
                if (lane == 0) {
                    dst[q * RS + RV] = m[q];
                    dst[q * RS + RV + 1] = sum;
                }
            }
        }
        cp_async_wait_all();
        if (!ok) {  // a wait ran out: what is in flight lands before the CTA can exit
            volatile int never = 0;
            mbar_wait(&bar[0], (issued_k - 1) & 1, &never, p.err);
            mbar_wait(&bar[1], (issued_v - 1) & 1, &never, p.err);
        }
    }
    pdl_wait();  // behind this kernel the trunk kernel is complete, too
}

// ------------------------------------------------------------------------------------------- join kernel

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void mma_bf16_16816(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

// An item is a head with up to spb sequences, of which a CTA (one per SM) has an even share; with one item or more each, spb is as
// small as that leaves it.  W_up,t^V of the head waits in shared memory, and what a sequence's nodes are in registers, when the
// records are there.  64 registers: as many as leave room beside the leaf kernel.
template <int RV>
__global__ void __launch_bounds__(kJoinThreads, 2) join_kernel(const __grid_constant__ JoinParams a) {
    using JJ = J<RV>;
    constexpr int RS = record_floats(RV);
    extern __shared__ __align__(16) char jw[];
    float *rows = reinterpret_cast<float *>(jw + JJ::oO), *coef = reinterpret_cast<float *>(jw + JJ::oCoef);
    const TrunkParams &p = a.t;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // the projection: this warp's rows 16 tile .. + 15 of the outputs of sequences 8 half .. + 7; this thread's two of either
    const int tile = warp & 7, half = warp >> 3, e = 16 * tile + (lane >> 2), n = 8 * half + 2 * (lane & 3);
    for (int i = tid; i < kD * (JJ::RVX - RV) / 8; i += kJoinThreads) *reinterpret_cast<uint4 *>(jw + i * JJ::WROW + RV * 2) = make_uint4(0, 0, 0, 0);
    for (int i = lane; i < JJ::OROW; i += 32) rows[warp * JJ::OROW + i] = 0.f;
    const int groups = count_groups(p), nodes = groups + p.B;
    const int per_head = (p.B + a.spb - 1) / a.spb, items = per_head * p.H;
    const Split split_items(items, gridDim.x);
    const int i0 = split_items.begin(blockIdx.x), i1 = split_items.begin(blockIdx.x + 1);
    int head = -1;
#pragma unroll 1
    for (int item = i0; item < i1; ++item) {
        const int h = item / per_head, b0 = (item - h * per_head) * a.spb;
        const int nb = min(a.spb, p.B - b0);
        const int64_t th = static_cast<int64_t>(h) * a.T + a.loop;
        auto iorow = [&](int b) { return static_cast<int64_t>(b) * p.H + h; };
        if (h != head) {
            const char *W = static_cast<const char *>(a.w_up_v) + th * kD * RV * 2;
            for (int i = tid; i < kD * (RV / 8); i += kJoinThreads) {
                const int r = i / (RV / 8), c = i - r * (RV / 8);
                cp_async16(jw + r * JJ::WROW + c * 16, W + i * 16);
            }
            cp_async_commit();
            head = h;
        }
        // (inputs of the call, before the wait:) what goes into this thread's outputs
        float mu[2], cv[2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            mu[x] = a.mu_v ? a.mu_v[th * kD + e + 8 * x] : 0.f;
#pragma unroll
            for (int y = 0; y < 2; ++y) cv[x][y] = a.cur_v && n + y < nb ? load_elem(a.cur_v, iorow(b0 + n + y) * kD + e + 8 * x, a.io_bf16) : 0.f;
        }
        // G warps per sequence: warp `sub` of them takes the runs sub + G k
        int G = 1;
        while (2 * G * nb <= kJoinWarps) G *= 2;
        const int bi = warp / G, sub = warp - bi * G, b = b0 + min(bi, nb - 1);
        // lane l < 3 knows level l's node of the sequence, lane 3 its own pages; then the current token's score
        int node = groups + b, rank = 0;
        bool there = lane == kLevels;
        if (lane < kLevels) {
            const int col = p.plan.column[static_cast<int64_t>(lane) * p.B + b];
            there = col >= 0 && col / kMembers < groups;
            if (there) {
                node = col / kMembers;
                rank = col % kMembers;
            }
        }
        Node d = {0, 0, 0, 0, 0, 0};
        if (there) d = node_at(p, groups, node);
        there = d.pages > 0 && rank < d.n;
        float qk = -INFINITY;
        if (a.cur_k) {
            const int64_t row = iorow(b);
            qk = 0.f;
#pragma unroll
            for (int i = 0; i < kD / 32; ++i)
                qk = fmaf(load_elem(a.q, row * kD + lane + 32 * i, a.io_bf16), load_elem(a.cur_k, row * kD + lane + 32 * i, a.io_bf16), qk);
            for (int i = lane; i < a.d_rope; i += 32)  // both stand at one position: the rotation cancels
                qk = fmaf(load_elem(a.q_rope, row * a.d_rope + i, a.io_bf16), load_elem(a.cur_k_rope, static_cast<int64_t>(b) * a.d_rope + i, a.io_bf16), qk);
            qk = warp_sum(qk) * a.scale_log2;
        }
        // The first item twice: at first with weights in the place of a record, and without an output, while the kernels before still
        // write theirs, so that the instructions are there when the records are (fetched behind the wait they took longer than the join).
#pragma unroll 1
        for (int dry = item == i0; dry >= 0; --dry) {
            if (item == i0 && dry == 0) {
                pdl_wait();
                pdl_trigger();
            }
            // the runs of the nodes: records first + step i of run i
            int runs = 0, first = 0, step = 0;
            if (there) {
                const int *before = p.pstart + (is_leaf(p, d) ? kMaxNodes + 1 : 0);
                const int np = before[nodes] * p.H, s0 = before[node] * p.H + h * d.pages, s1 = s0 + d.pages - 1;
                int c0;
                if (is_leaf(p, d)) {
                    const LeafShares shares(np, a.workers);
                    c0 = shares.share(s0);
                    runs = shares.share(s1) - c0 + 1;
                } else {
                    const Split split(np, min(a.grid, np));  // as find_share
                    c0 = split.worker(s0);
                    runs = split.worker(s1) - c0 + 1;
                }
                first = static_cast<int>(record_of(p, d, h, c0)) + rank;
                step = is_leaf(p, d) ? p.leaf_max : p.trunk_max;
            }
            const float *part = p.part;
            if (dry) {  // (one run; a head's weights are many records long)
                runs = lane == kLevels;
                first = step = 0;
                part = static_cast<const float *>(a.w_up_v);
            }
            int upto[kLevels + 1];  // runs of the nodes up to each
#pragma unroll
            for (int l = 0; l <= kLevels; ++l) upto[l] = (l ? upto[l - 1] : 0) + __shfl_sync(0xffffffffu, runs, l);
            const float beta = dry ? 0.f : p.beta[iorow(b)];
            float M = -INFINITY, l = 0.f, acc[5];  // of columns 4 lane .. + 3, and 128 + lane
#pragma unroll
            for (int c = 0; c < 5; ++c) acc[c] = 0.f;
            if (bi < nb) {
#pragma unroll 1
                for (int r0 = 0; r0 < upto[kLevels]; r0 += 32) {
                    const int nr = min(32, upto[kLevels] - r0), r = r0 + min(lane, nr - 1);
                    int level = 0, in = r;
#pragma unroll
                    for (int k = 0; k < kLevels; ++k)
                        if (r >= upto[k]) {
                            level = k + 1;
                            in = r - upto[k];
                        }
                    const int rec = __shfl_sync(0xffffffffu, first, level) + in * __shfl_sync(0xffffffffu, step, level);
                    const float2 ml = *reinterpret_cast<const float2 *>(part + static_cast<int64_t>(rec) * RS + RV);
                    constexpr int KR = 6;  // runs whose loads are in flight together, the first of them beside their maxima and sums
                    float4 v[KR];
                    float t[KR];
                    auto load = [&](int k0) {
#pragma unroll
                        for (int k = 0; k < KR; ++k) {
                            const float *pr = part + static_cast<int64_t>(__shfl_sync(0xffffffffu, rec, min(k0 + k * G, nr - 1))) * RS;
                            v[k] = lane * 4 < RV ? *reinterpret_cast<const float4 *>(pr + lane * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
                            t[k] = RV > 128 ? pr[128 + lane] : 0.f;
                        }
                    };
                    load(sub);
                    const float mi = lane < nr ? ml.x : -INFINITY;
                    const float Mn = fmaxf(M, warp_max(mi)), f = M == -INFINITY ? 0.f : ex2_approx(M - Mn);
                    const float wi = mi == -INFINITY ? 0.f : ex2_approx(mi - Mn);
                    M = Mn;
                    l = fmaf(l, f, warp_sum(lane < nr ? wi * ml.y : 0.f));
#pragma unroll
                    for (int c = 0; c < 5; ++c) acc[c] *= f;
#pragma unroll 1
                    for (int k0 = sub;;) {
#pragma unroll
                        for (int k = 0; k < KR; ++k) {
                            const float wk = __shfl_sync(0xffffffffu, wi, min(k0 + k * G, 31));
                            if (wk != 0.f && k0 + k * G < nr) {  // warp-uniform (a NaN state stays one)
                                acc[0] = fmaf(wk, v[k].x, acc[0]);
                                acc[1] = fmaf(wk, v[k].y, acc[1]);
                                acc[2] = fmaf(wk, v[k].z, acc[2]);
                                acc[3] = fmaf(wk, v[k].w, acc[3]);
                                if constexpr (RV > 128) acc[4] = fmaf(wk, t[k], acc[4]);
                            }
                        }
                        if ((k0 += KR * G) >= nr) break;
                        load(k0);
                    }
                }
                float *row = rows + warp * JJ::OROW;  // (that of sequence bi and warp `sub` of its)
                if (lane * 4 < RV) *reinterpret_cast<float4 *>(row + lane * 4) = make_float4(acc[0], acc[1], acc[2], acc[3]);
                if constexpr (RV > 128) row[128 + lane] = acc[4];
                if (sub == 0 && lane == 0) {
                    M += beta;  // the same for all of a query's cached tokens
                    const float Mx = fmaxf(M, qk);
                    const float al = M == -INFINITY ? 0.f : ex2_approx(M - Mx);
                    const float pc = a.cur_k ? ex2_approx(qk - Mx) : 0.f;
                    const float den = al * l + pc;
                    const float inv = den == 0.f ? 0.f : 1.f / den;
                    coef[bi * 4] = al * inv;
                    coef[bi * 4 + 1] = al * l * inv;
                    coef[bi * 4 + 2] = pc * inv;
                }
            }
            cp_async_wait_all();
            __syncthreads();
            if (G > 1) {
                for (int i = tid; i < nb * RV; i += kJoinThreads) {
                    const int q = i / RV, c = i - q * RV;
                    float o = rows[q * G * JJ::OROW + c];
                    for (int k = 1; k < G; ++k) o += rows[(q * G + k) * JJ::OROW + c];
                    rows[q * G * JJ::OROW + c] = o;
                }
                __syncthreads();
            }
            // out_b[e] = coef0 (W_up^V o~_b)[e] + coef1 mu^V[e] + coef2 v_cur,b[e]; the product with o~ as three bf16 parts (24 bits), the
            // small ones in sums of their own: 1.7 us with the output for 15 sequences, operands and sums in registers.  (On CUDA cores
            // it was bound by the reads of o~ from shared memory: 6 us for 16 sequences.)
            if (8 * half < nb) {
                float big[4] = {0.f, 0.f, 0.f, 0.f}, small[4] = {0.f, 0.f, 0.f, 0.f};
                const uint32_t wa = smem_addr(jw) + (16 * tile + (lane & 15)) * JJ::WROW + (lane >> 4) * 16;
                const float *o = rows + min(8 * half + (lane >> 2), nb - 1) * G * JJ::OROW + 2 * (lane & 3);
#pragma unroll 2
                for (int ks = 0; ks < JJ::RVX / 16; ++ks) {
                    uint32_t w[4], q[3][2];
                    ldmatrix_x4(w, wa + ks * 32);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float2 u = *reinterpret_cast<const float2 *>(o + ks * 16 + 8 * x);
                        q[0][x] = pack_bf16x2(u.x, u.y);
                        const float2 f = bf2_to_f2(q[0][x]);
                        q[1][x] = pack_bf16x2(u.x - f.x, u.y - f.y);
                        const float2 g = bf2_to_f2(q[1][x]);
                        q[2][x] = pack_bf16x2(u.x - f.x - g.x, u.y - f.y - g.y);
                    }
                    mma_bf16_16816(small, w, q[2]);
                    mma_bf16_16816(small, w, q[1]);
                    mma_bf16_16816(big, w, q[0]);
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        if (dry || n + y >= nb) continue;
                        const float *cf = coef + (n + y) * 4;
                        const float v = fmaf(cf[2], cv[x][y], fmaf(cf[1], mu[x], (big[2 * x + y] + small[2 * x + y]) * cf[0]));
                        store_elem(a.out, iorow(b0 + n + y) * kD + e + 8 * x, v, a.io_bf16);
                    }
            }
            __syncthreads();  // o~, the coefficients and the weights are free
        }
    }
}

// ----------------------------------------------------------------------------------------------- host side

struct PrefixWorkspace {
    size_t part, qt, qf, beta, pstart, total;
    size_t leaf;  // first record of the leaf kernel
};

inline size_t al256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// Whether a call goes without a trunk kernel: no group of up to kLeafAlone sequences has more members than the leaf kernel can take,
// and one of two never more than it takes beside a trunk.  For three and four the leaf kernel alone is faster over short contexts (us, four
// sequences over one prompt of 768 / 4096 / 16384 / 65536 / 262144 tokens, alone and with a trunk kernel):
//   16 heads               16.5  24.9  47.5  102  332     26.2  31.1  45.5  104  328
//   2 heads                14.6  17.6  27.2   61  107     21.4  24.6  27.5   38   67
//   16 heads, d_rope 64    17.4  29.1  59.9  148  512     26.3  34.1  52.7  127  414
constexpr int kAloneTokens = 16384;
bool leaf_alone(int B, int max_ctx) { return B <= kLeaf || (B <= kLeafAlone && max_ctx <= kAloneTokens); }

// Queries of a node of either kind, at most, of B sequences.
int leaf_queries(int B, bool alone) { return alone ? std::max(B, 1) : kLeaf; }
int trunk_queries(int B) { return B <= kLeaf ? 0 : std::min(B, kMembers); }

// For B sequences on either path: `warps` and `warps_alone` are the leaf kernel's on an SM.
PrefixWorkspace prefix_workspace(int rkt, int r_v, int B, int H, int grid, int warps, int warps_alone) {
    PrefixWorkspace w;
    w.leaf = trunk_queries(B) > 0 ? static_cast<size_t>(H) * kLevels * B + static_cast<size_t>(trunk_queries(B)) * grid : 0;
    const int of_shares = std::max(trunk_queries(B) > 0 ? leaf_queries(B, false) * warps : 0, leaf_alone(B, 0) ? leaf_queries(B, true) * warps_alone : 0);
    const size_t records = w.leaf + static_cast<size_t>(H) * (kLevels + 1) * B + static_cast<size_t>(of_shares) * (1 + kLeafRest) * grid;
    w.part = 0;
    w.qt = al256(records * record_floats(r_v) * sizeof(float));
    w.qf = w.qt + al256(static_cast<size_t>(B) * H * 3 * rkt * sizeof(uint16_t));
    w.beta = w.qf + al256(static_cast<size_t>(B) * H * rkt * sizeof(float));
    w.pstart = w.beta + al256(static_cast<size_t>(B) * H * sizeof(float));
    w.total = w.pstart + al256((2 * (kMaxNodes + 1) + 1) * sizeof(int));
    return w;
}

template <int RK, int RV, int DR, bool THIRD>
lla_status launch_prefix(const DecodeArgs &a, const lla_prefix &plan, const void *rope_pool, const RotaryAxes &rope,
                         const int32_t *positions, const void *q_rope, const void *cur_k_rope, cudaStream_t stream) {
    using ZZ = Z<RK, RV, DR, THIRD>;
    lla_status st = LLA_OK;
    unsigned *err = device_error_word(&st);
    if (st != LLA_OK) return st;
    const int grid = num_sms();
    if (grid <= 0) return LLA_ERR_CUDA;
    if (grid > kMaxGrid) return LLA_ERR_UNSUPPORTED;
    if (a.num_blocks * a.H >= (int64_t(1) << 31)) return LLA_ERR_UNSUPPORTED;  // TMA coordinate
    using LL = L<RK, RV, DR, false>;
    using LA = L<RK, RV, DR, true>;
    const PrefixWorkspace w = prefix_workspace(ZZ::RKT, RV, a.B, a.H, grid, LL::WARPS, LA::WARPS);
    if (a.workspace_bytes < w.total) return LLA_ERR_WORKSPACE;
    char *ws = static_cast<char *>(a.workspace);
    static DeviceOnce configured, configured_leaf, configured_alone;
    if (raise_smem_limit(leaf_kernel<RK, RV, DR, false>, LL::SMEM, configured_leaf, true) != LLA_OK) return LLA_ERR_CUDA;
    if (raise_smem_limit(leaf_kernel<RK, RV, DR, true>, LA::SMEM, configured_alone, true) != LLA_OK) return LLA_ERR_CUDA;
    if (raise_smem_limit(trunk_kernel<RK, RV, DR, THIRD>, ZZ::SMEM, configured) != LLA_OK) return LLA_ERR_CUDA;
    const int64_t page_bytes = static_cast<int64_t>(head_page_bytes(RK, RV, 2));
    // the V-planes of every page: [num_blocks * H][64 tokens][r_v] bf16
    CUtensorMap tv;
    const uint64_t dims[3] = {static_cast<uint64_t>(RV), static_cast<uint64_t>(kPT), static_cast<uint64_t>(a.num_blocks) * a.H};
    const uint64_t strides[2] = {static_cast<uint64_t>(RV) * 2, static_cast<uint64_t>(page_bytes)};
    const uint32_t box[3] = {64, kPT, 1};
    if (!encode_tmap_bf16(&tv, static_cast<const char *>(a.pool) + kPT * RK * 2, 3, dims, strides, box, true)) return LLA_ERR_CUDA;

    TrunkParams tp = {};
    tp.H = a.H; tp.B = a.B; tp.max_ctx = a.max_ctx; tp.max_blocks = a.max_blocks; tp.pass1 = a.cur_k != nullptr;
    tp.pool = static_cast<const char *>(a.pool);
    tp.num_blocks = a.num_blocks; tp.page_bytes = page_bytes;
    tp.rope_pool = static_cast<const char *>(rope_pool);
    tp.block_table = a.block_table; tp.context_lens = a.context_lens;
    tp.plan = PlanView{plan.num_groups, plan.groups, plan.members, plan.column, plan.own_page};
    tp.qt = reinterpret_cast<uint16_t *>(ws + w.qt);
    tp.qf = reinterpret_cast<float *>(ws + w.qf);
    tp.beta = reinterpret_cast<float *>(ws + w.beta);
    tp.part = reinterpret_cast<float *>(ws + w.part);
    tp.pstart = reinterpret_cast<int *>(ws + w.pstart);
    tp.next = tp.pstart + 2 * (kMaxNodes + 1);
    tp.leaf = static_cast<int64_t>(w.leaf);
    // Beside a trunk kernel, leaves of up to four queries need registers that the join's CTA holds: 64 sequences over 16 prompts, all of
    // them leaves then, take 107 us instead of 109, but 128 samples of 8 documents 105 instead of 97, and of two videos 149 instead of 140.
    const bool alone = leaf_alone(a.B, a.max_ctx);
    tp.leaf_max = leaf_queries(a.B, alone);
    tp.trunk_max = trunk_queries(a.B);
    tp.err = err;

    AbsorbParams ap = {};
    ap.t = tp;
    ap.T = a.T; ap.loop = a.loop; ap.io_bf16 = a.io_bf16;
    ap.scale_log2 = a.scale * kLog2e;
    ap.w_up_k = a.w_up_k; ap.mu_k = a.mu_k; ap.q = a.q; ap.q_rope = q_rope;
    ap.positions = positions; ap.pairing = rope.pairing;
    if (DR > 0) {
        for (int j = 0; j < DR / 2; ++j) ap.axis[j] = rope.axis[j];
        rotary_phases(DR, rope.base, ap.phi);
    }
    if ((st = launch_ex(absorb_kernel<RK, DR>, dim3(a.H, (ZZ::RKX + 31) / 32 + (DR > 0) + 1, (a.B + 15) / 16), 256, 0, stream, ap)) != LLA_OK)
        return st;
    if (alone) {
        st = launch_ex(leaf_kernel<RK, RV, DR, true>, dim3(grid), LA::WARPS * 32, LA::SMEM, stream, tp);
    } else {
        if ((st = launch_ex(trunk_kernel<RK, RV, DR, THIRD>, dim3(grid), kTrunkThreads, ZZ::SMEM, stream, tv, tp)) != LLA_OK) return st;
        st = launch_ex(leaf_kernel<RK, RV, DR, false>, dim3(grid), LL::WARPS * 32, LL::SMEM, stream, tp);
    }
    if (st != LLA_OK) return st;

    JoinParams jp = {};
    jp.t = tp;
    jp.T = a.T; jp.loop = a.loop; jp.io_bf16 = a.io_bf16; jp.grid = grid; jp.workers = grid * (alone ? LA::WARPS : LL::WARPS); jp.d_rope = DR;
    jp.scale_log2 = ap.scale_log2;
    jp.w_up_v = a.w_up_v; jp.mu_v = a.mu_v;
    jp.q = a.q; jp.q_rope = q_rope; jp.cur_k = a.cur_k; jp.cur_v = a.cur_v; jp.cur_k_rope = cur_k_rope;
    jp.out = a.out;
    // one CTA per SM: as many sequences together as leave no CTA two items, where that can be
    const auto items = [&](int spb) { return static_cast<int64_t>(a.H) * ((a.B + spb - 1) / spb); };
    jp.spb = 1;
    while (jp.spb < kJoinSeqs && items(jp.spb) > grid) ++jp.spb;
    const dim3 jg(static_cast<unsigned>(std::min<int64_t>(grid, items(jp.spb))));
    static DeviceOnce configured_join;
    if (raise_smem_limit(join_kernel<RV>, J<RV>::SMEM, configured_join, true) != LLA_OK) return LLA_ERR_CUDA;
    return launch_ex(join_kernel<RV>, jg, kJoinThreads, J<RV>::SMEM, stream, jp);
}

}  // namespace

bool decode_prefix_supported(int es, int d, int r_k, int r_v, int d_rope) {
    if (es != 2 || d != kD) return false;
    if (d_rope == 0) return (r_k == 96 && r_v == 160) || (r_k == 128 && r_v == 128) || (r_k == 72 && r_v == 120);
    return r_k == 96 && r_v == 160 && (d_rope == 32 || d_rope == 64 || d_rope == 96);
}

#define LLA_PREFIX_SHAPES(X) \
    X(96, 160, 0) X(128, 128, 0) X(72, 120, 0) X(96, 160, 32) X(96, 160, 64) X(96, 160, 96)

size_t decode_prefix_workspace_bytes(int r_k, int r_v, int d_rope, int B, int H) {
    const int grid = num_sms();
    if (grid <= 0) return 0;
#define LLA_PREFIX(K, V, R) \
    if (r_k == K && r_v == V && d_rope == R) \
        return prefix_workspace(Z<K, V, R, false>::RKT, V, B, H, grid, \
                                L<K, V, R, false>::WARPS, L<K, V, R, true>::WARPS).total;
    LLA_PREFIX_SHAPES(LLA_PREFIX)
#undef LLA_PREFIX
    return 0;
}

lla_status launch_decode_prefix(const DecodeArgs &a, const lla_prefix &plan, const void *rope_pool, int d_rope,
                                const RotaryAxes &rope, const int32_t *positions, const void *q_rope,
                                const void *cur_k_rope, cudaStream_t stream) {
#define LLA_PREFIX(K, V, R) \
    if (a.r_k == K && a.r_v == V && d_rope == R) \
        return a.io_bf16 ? launch_prefix<K, V, R, false>(a, plan, rope_pool, rope, positions, q_rope, cur_k_rope, stream) \
                         : launch_prefix<K, V, R, true>(a, plan, rope_pool, rope, positions, q_rope, cur_k_rope, stream);
    LLA_PREFIX_SHAPES(LLA_PREFIX)
#undef LLA_PREFIX
    return LLA_ERR_UNSUPPORTED;
}

}  // namespace lla
