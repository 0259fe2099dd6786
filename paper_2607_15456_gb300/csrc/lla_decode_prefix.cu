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
// Three launches on the caller's stream, chained by programmatic dependent launch:
//   absorb_kernel  q~ (fp32, scaled into the exp2 domain) and beta of every (sequence, head); the prefix sums of the nodes'
//                  pages and the checks of lengths and plan
//   trunk_kernel   one CTA per SM.  The units' pages, in the order of the nodes, are split evenly over the CTAs; a CTA takes
//                  its pages as runs (its part of one unit).  A page is two products on the tensor cores,
//                    S^T [64 tokens x 3 NQ]  = [C_k | K^R] [Q~_0; Q~_1; Q~_2]^T   (q~ as three bf16 parts)
//                    O^T [r_v x 2 NQ]       += C_v^T [P_0; P_1]^T                 (p as two)
//                  for 8 or 32 queries; a group of 33 to 64 members is two halves of 32, which take turns on each page
//                  while it is in shared memory.
//                    warp 0        producer: the K-plane (and rotary plane) by bulk copies, the V-plane by TMA boxes
//                    warp 1        issuer of S^T, and owner of TMEM
//                    warp 2        q~ of the next run as an operand, beta
//                    warp 3        issuer of O^T
//                    warps 4-7     softmax: p as an operand, lazy rescale of O^T
//                    warps 8-11    epilogue: O^T, maxima and sums of a finished run to the workspace
//                  S^T, P, q~ and O^T have two buffers each, so that every role works ahead of the next.
//   join_kernel    per head and up to 8 sequences: joins the runs of each sequence's nodes and the current token, and applies
//                  W_up,t^V once for all of them
//
// Storage bf16, d = 128; accumulators fp32 in TMEM.  Three parts of q~ hold the 24 bits of fp32.  Two parts of p are off by at
// most 2^-18 of p (half a step of the second part), which a sum of many p averages below the rounding of its fp32 sums; the
// sums l take p itself.
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
constexpr int kHalf = 32;        // queries of an operand
constexpr int kFew = 8;          // of the small one
constexpr int kLevels = LLA_PREFIX_LEVELS;
constexpr int kMembers = LLA_PREFIX_MEMBERS;
constexpr int kMaxNodes = kLevels * (LLA_MAX_BATCH / 2) + LLA_MAX_BATCH;
constexpr int kTrunkThreads = 384;
constexpr int kQueryWarp = 2, kValueWarp = 3, kSoftmaxWarp = 4, kEpilogueWarp = 8;
constexpr int kMaxGrid = 256;
constexpr int kJoinSeqs = 8;
constexpr int kSmemCap = 227 * 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleLog2 = 8.f;  // rescale O^T only when a query's maximum grows by more

struct PlanView {
    const int32_t *num_groups, *groups, *members, *column, *own_page;
};

struct TrunkParams {
    int H, B, max_ctx, max_blocks, pass1;
    const char *pool;
    int64_t num_blocks, page_bytes;
    const char *rope_pool;
    const int32_t *block_table, *context_lens;
    PlanView plan;
    float *qt;    // [B][H][RKT]: q~ * scale * log2 e, zero past r_k, then the rotary part
    float *beta;  // [B][H]
    float *part;  // run records, see record_of
    int *pstart;  // [groups + B + 1]: pages of the nodes before each
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
    int T, loop, io_bf16, grid, spb, d_rope;
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
        if (g.x < 0 || g.y <= g.x || g.y > cap / kPT || g.w < 1 || g.w > kMembers || g.z < 0 || g.z > kLevels * p.B - g.w) return d;
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

// Record of query r of node d at head h, from CTA c: r_v latent values, the maximum, the sum.  The runs of a unit lie
// kMembers records apart, and so no two of them meet: units and CTAs grow together.
__device__ __forceinline__ int64_t record_of(const TrunkParams &p, const Node &d, int h, int c) {
    return static_cast<int64_t>(p.H) * d.member + static_cast<int64_t>(h) * d.n + static_cast<int64_t>(kMembers) * c;
}
__host__ __device__ constexpr int record_floats(int rv) { return rv + 4; }

// ----------------------------------------------------------------------------------------- absorb kernel

// One CTA: the prefix sums of the nodes' pages, and the flags of what node_at leaves out.
__device__ void node_prefix(const TrunkParams &p) {
    __shared__ int wsum[8];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int groups = count_groups(p), nodes = groups + p.B;
    const int cap = static_cast<int>(min(static_cast<int64_t>(p.max_ctx), static_cast<int64_t>(p.max_blocks) * kPT));
    unsigned bad = 0;
    if (*p.plan.num_groups != groups) bad |= LLA_DEVERR_SEQUENCE;
    for (int b = tid; b < p.B; b += 256) {
        const int len = p.context_lens[b];
        if (len < 0 || len > cap) bad |= LLA_DEVERR_CONTEXT;
        else if (p.plan.own_page[b] < 0 || p.plan.own_page[b] > len / kPT) bad |= LLA_DEVERR_CONTEXT;
        if (len == 0 && !p.pass1) bad |= LLA_DEVERR_EMPTY_PASS2;
        for (int l = 0; l < kLevels; ++l) {
            const int col = p.plan.column[static_cast<int64_t>(l) * p.B + b];
            if (col < 0) continue;
            const Node d = col / kMembers < groups ? node_at(p, groups, col / kMembers) : Node{};
            if (d.pages == 0 || col % kMembers >= d.n || p.plan.members[d.member + col % kMembers] != b) bad |= LLA_DEVERR_SEQUENCE;
            else if (d.first + d.pages > len / kPT) bad |= LLA_DEVERR_CONTEXT;
        }
    }
    for (int g = tid; g < groups; g += 256)
        if (node_at(p, groups, g).pages == 0) bad |= LLA_DEVERR_SEQUENCE;
    if (bad) atomicOr(p.err, bad);
    const int per = (nodes + 255) / 256;
    int tot = 0;
    for (int i = tid * per; i < min(nodes, (tid + 1) * per); ++i) tot += node_at(p, groups, i).pages;
    int x = tot;  // inclusive scan over the warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) wsum[warp] = x;
    __syncthreads();
    int ex = x - tot;
    for (int w = 0; w < warp; ++w) ex += wsum[w];
    for (int i = tid * per; i < min(nodes, (tid + 1) * per); ++i) {
        p.pstart[i] = ex;
        ex += node_at(p, groups, i).pages;
    }
    if (tid == 255) p.pstart[nodes] = ex;
}

// Grid (H, RKX / 32 [+ 1 with a rotary branch], ceil(B / 16)), 256 threads = 32 columns x 8 slices of 16 rows: q~ of 32
// columns of one head for 16 sequences, every weight load of a thread in flight at once; beta by the CTAs of the first
// column chunk; the rotary queries, turned at the current tokens' positions, by those of the last.
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
                float *dst = p.qt + (static_cast<int64_t>(b) * p.H + h) * RKT + RKX;
                dst[ia] = (x * cs - y * sn) * a.scale_log2;
                dst[ic] = (x * sn + y * cs) * a.scale_log2;
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
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) node_prefix(p);
    for (int i = tid; i < 16 * kD; i += 256) {
        const int bi = i >> 7, e = i & (kD - 1);
        qs[bi][e] = bi < nb ? load_elem(a.q, (static_cast<int64_t>(b0 + bi) * p.H + h) * kD + e, a.io_bf16) : 0.f;
    }
    __syncthreads();
#pragma unroll
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
        if (bi < nb && j0 + c < RKX)
            p.qt[(static_cast<int64_t>(b0 + bi) * p.H + h) * RKT + j0 + c] = j0 + c < RK ? s * a.scale_log2 : 0.f;
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
template <int RK, int RV, int DR>
struct Z {
    static constexpr int RKX = (RK + 15) / 16 * 16;   // content contraction, zero-padded
    static constexpr int RKT = RKX + DR;              // with the rotary one
    static constexpr int NCH = (RV + 127) / 128;      // chunks of O^T rows: 128, the last 64 if that holds it
    static constexpr bool LAST64 = RV % 128 != 0 && RV % 128 <= 64;
    static constexpr int NBOX = (RV + 63) / 64;       // TMA boxes of a V-plane
    static constexpr int BOX = kPT * 128;             // one: 64 rows x 128 bytes
    static constexpr int KPLANE = kPT * RK * 2, KPAD = kPT * RKX * 2, RPLANE = kPT * DR * 2;
    static constexpr int KPAGE = KPAD + RPLANE;
    static constexpr int VPAGE = (LAST64 ? 2 * NCH - 1 : 2 * NCH) * BOX;
    static constexpr int QB = 3 * kHalf * RKT * 2;    // q~ operand (one of two)
    static constexpr int PB = kPT * 2 * kHalf * 2;    // P operand (one of two)
    static constexpr int NBAR = 40;
    // floats: maxima [2][4][32], factors [32], sums [2][4][32], beta [4][32], states [2 slots][2][32]
    static constexpr int RED = (256 + 32 + 256 + 128 + 128) * 4;
    static constexpr int FIXED = 2 * QB + 2 * PB + RED + NBAR * 8 + kMaxNodes * 2 + 1024;
    static constexpr int ST0 = (kSmemCap - 1024 - FIXED) / (KPAGE + VPAGE);
    static constexpr int ST = ST0 > 4 ? 4 : ST0;
    static constexpr int oV = 0;
    static constexpr int oK = oV + ST * VPAGE;
    static constexpr int oQ = oK + ST * KPAGE;
    static constexpr int oP = oQ + 2 * QB;
    static constexpr int oRed = oP + 2 * PB;
    static constexpr int oBar = oRed + RED;
    static constexpr int oList = oBar + NBAR * 8;
    // (at least half of an SM's: one CTA per SM, which holds all of TMEM)
    static constexpr int SMEM0 = 1024 + oList + kMaxNodes * 2, SMEM = SMEM0 > 116 * 1024 ? SMEM0 : 116 * 1024;
    static constexpr uint32_t TM_S = 3 * kHalf;             // columns of one S^T buffer
    static constexpr uint32_t TM_O0 = 2 * TM_S, TM_O = NCH * 2 * kHalf, TM_COLS = 512;
    static_assert(RKT % 16 == 0 && RV % 8 == 0 && NCH <= 2, "ranks");
    static_assert(VPAGE == NBOX * BOX, "every box of a V stage is loaded");
    static_assert(ST >= 2 && SMEM + 1024 <= kSmemCap, "shared memory");
    static_assert(TM_O0 + 2 * TM_O <= TM_COLS, "TMEM columns");
};

// barrier indices
enum {
    bKfull = 0 /* [4] */, bKempty = 4, bVfull = 8, bVempty = 12, bSfull = 16 /* [2] */, bSfree = 18, bPfull = 20, bPfree = 22,
    bQfull = 24, bQfree = 26, bOdone = 28, bOfree = 30, bMfull = 32, bAbort = 34, bTslot = 35, bBfull = 36 /* [4] */
};

// A CTA's part of a unit.  Its queries are `subs` operands of up to 32, which take turns on every page.
struct TrunkRun {
    Node d;
    int h, page, pages, subs;  // page: the first in the table row
};

struct Share {
    int g0, g1;      // global pages of this CTA
    int nodes, s;    // nodes in `list`, first global page of the first
};

// This CTA's share of the units' pages, and the nodes that it lies in: worked out from the inputs of the call by all threads,
// so that the producer can start on the pages while the absorb kernel still runs.
__device__ Share find_share(const TrunkParams &p, int groups, uint16_t *list) {
    __shared__ int wsum[kTrunkThreads / 32], wcnt[kTrunkThreads / 32], first;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int nodes = groups + p.B, per = (nodes + kTrunkThreads - 1) / kTrunkThreads;
    auto scan = [&](int v) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += y;
        }
        return v;
    };
    int tot = 0;
    for (int i = tid * per; i < min(nodes, (tid + 1) * per); ++i) tot += node_at(p, groups, i).pages * p.H;
    const int x = scan(tot);
    if (lane == 31) wsum[warp] = x;
    __syncthreads();
    int ex0 = x - tot, np = 0;
#pragma unroll
    for (int w = 0; w < kTrunkThreads / 32; ++w) {
        if (w < warp) ex0 += wsum[w];
        np += wsum[w];
    }
    // with fewer pages than CTAs the first np CTAs take one each
    const int c = blockIdx.x, Ge = min(static_cast<int>(gridDim.x), np);
    Share r;
    r.g0 = c < Ge ? page_lo(c, np, Ge) : 0;
    r.g1 = c < Ge ? page_lo(c + 1, np, Ge) : 0;
    int mine = 0, ex = ex0;
    for (int i = tid * per; i < min(nodes, (tid + 1) * per); ++i) {
        const int n = node_at(p, groups, i).pages * p.H;
        mine += n > 0 && ex < r.g1 && ex + n > r.g0;
        ex += n;
    }
    const int y = scan(mine);
    if (lane == 31) wcnt[warp] = y;
    __syncthreads();
    int at = y - mine;
    r.nodes = 0;
#pragma unroll
    for (int w = 0; w < kTrunkThreads / 32; ++w) {
        if (w < warp) at += wcnt[w];
        r.nodes += wcnt[w];
    }
    ex = ex0;
    for (int i = tid * per; mine > 0 && i < min(nodes, (tid + 1) * per); ++i) {
        const int n = node_at(p, groups, i).pages * p.H;
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

// f(run) for every run of the share, in order, until it says false.
template <typename F>
__device__ __forceinline__ void for_runs(const TrunkParams &p, int groups, const Share &sh, const uint16_t *list, F f) {
    int s = sh.s;
    for (int i = 0; i < sh.nodes; ++i) {
        TrunkRun r;
        r.d = node_at(p, groups, list[i]);
        r.subs = r.d.n > kHalf ? 2 : 1;
        const int end = s + r.d.pages * p.H;
        int u = max(sh.g0, s) - s;  // page of the node, head by head
        const int stop = min(sh.g1, end) - s;
        r.h = u / r.d.pages;
        int in = u - r.h * r.d.pages;
        for (; u < stop; ++r.h) {
            r.pages = min(stop - u, r.d.pages - in);
            r.page = r.d.first + in;
            if (!f(r)) return;
            u += r.pages;
            in = 0;
        }
        s = end;
    }
}

// A value that every lane has, for a warp that issues products (their descriptors are in uniform registers then).
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

struct TrunkCtx {
    char *sm;
    uint64_t *bar;
    volatile int *abort_flag;
    float *red, *factor, *lsum, *beta, *state;
    unsigned *err;
};

// The softmax warps' part of one run with NQ query slots in each of SUBS operands.  Lane l of warp w holds the scores of
// tokens 16 w + l / 4 (+ 8) for the queries 8 k + 2 (l % 4) (+ 1) of every operand.
template <typename ZZ, int NQ, int SUBS>
__device__ __forceinline__ void softmax_run(const TrunkCtx &x, const TrunkRun &r, int &it, int &pgs, int sr) {
    constexpr int NV = NQ / 4, NP = 2 * NQ;  // values of a token in a thread, rows of P
    const int tid = threadIdx.x - 32 * kSoftmaxWarp, w = tid >> 5, lane = tid & 31, l4 = lane >> 2, c2 = 2 * (lane & 3);
    const uint32_t tl = static_cast<uint32_t>(32 * w) << 16;
    auto query = [&](int v) { return 8 * (v >> 1) + c2 + (v & 1); };
    float beta[SUBS][NV], m[SUBS][NV], acc[SUBS][NV];
#pragma unroll
    for (int j = 0; j < SUBS; ++j) {
        mbar_wait(&x.bar[bBfull + ((sr + j) & 3)], ((sr + j) >> 2) & 1, x.abort_flag, x.err);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            beta[j][v] = x.beta[((sr + j) & 3) * kHalf + query(v)];
            m[j][v] = -INFINITY;
            acc[j][v] = 0.f;
        }
    }
    for (int k = 0; k < r.pages; ++k, ++pgs) {
        const int left = r.d.len - (r.page + k) * kPT;  // tokens of the page that are there (more than a page: all)
#pragma unroll
        for (int j = 0; j < SUBS; ++j, ++it) {
            const int s = it & 1;
            mbar_wait(&x.bar[bSfull + s], (it >> 1) & 1, x.abort_flag, x.err);
            tc_fence_after();
            float raw[3][2 * NV];
            const uint32_t ts = tl + s * ZZ::TM_S;
            tmem_ld16x256_three(ts, ts + NQ, ts + 2 * NQ, raw);
            tc_fence_before();
            mbar_arrive(&x.bar[bSfree + s]);
            float sc[2][NV];
            bool mine = false;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bool valid = 16 * w + l4 + 8 * t < left;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int i = 4 * (v >> 1) + 2 * t + (v & 1);
                    sc[t][v] = valid ? (raw[0][i] + raw[1][i]) + (raw[2][i] + beta[j][v]) : -INFINITY;
                    mine = mine || sc[t][v] > m[j][v] + kRescaleLog2;
                }
            }
            // most pages raise no query's maximum by 2^8: one barrier that also votes tells all four warps so
            if (named_bar_or(1, 128, mine)) {
                float *rp = x.red + s * 128;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float mx = fmaxf(sc[0][v], sc[1][v]);
#pragma unroll
                    for (int o = 4; o <= 16; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                    if (l4 == 0) rp[w * kHalf + query(v)] = mx;
                }
                named_bar_sync(1, 128);
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float mx = m[j][v];
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, rp[i * kHalf + query(v)]);
                    const bool grows = mx > m[j][v] + kRescaleLog2;  // also the first page
                    const float f = grows ? ex2_approx(m[j][v] - mx) : 1.f;
                    if (grows) {
                        acc[j][v] *= f;
                        m[j][v] = mx;
                    }
                    if (w == 0 && l4 == 0) x.factor[query(v)] = f;
                }
                named_bar_sync(1, 128);
                if (k > 0) {
                    // O^T holds pages up to the one before of this run (the last product issued has released its P buffer;
                    // the one before it had released the other before this warp wrote the last P): scale its columns
                    mbar_wait(&x.bar[bPfree + ((it - 1) & 1)], ((it - 1) >> 1) & 1, x.abort_flag, x.err);
                    tc_fence_after();
#pragma unroll
                    for (int i = 0; i < ZZ::NCH * NP / 16; ++i) {
                        const uint32_t col = ZZ::TM_O0 + ((sr + j) & 1) * ZZ::TM_O + (i / (NP / 16)) * (2 * kHalf) + (i % (NP / 16)) * 16;
                        float o[16];
                        tmem_ld16(tl + col, o);
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] *= x.factor[((i % (NP / 16)) * 16 + e) % NQ];
                        tmem_st16(tl + col, o);
                    }
                }
            }
            if (it >= 2) mbar_wait(&x.bar[bPfree + s], ((it - 2) >> 1) & 1, x.abort_flag, x.err);
            // P as a K-major operand: row part NQ + query, tokens 8 g .. 8 g + 7 at g NP 16 + row 16
            char *pp = x.sm + ZZ::oP + s * ZZ::PB + l4 * 2;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const float pv = ex2_approx(sc[t][v] - m[j][v]);
                    acc[j][v] += pv;
                    float part[2];
                    bf16_parts(pv, part);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        *reinterpret_cast<uint16_t *>(pp + (2 * w + t) * (NP * 16) + (i * NQ + query(v)) * 16) =
                            __bfloat16_as_ushort(__float2bfloat16_rn(part[i]));
                }
            if (SUBS == 1 && left < kPT) {
                // V rows past the sequence hold no latents: zero them (0 * NaN would poison O^T)
                const int st = pgs % ZZ::ST;
                mbar_wait(&x.bar[bVfull + st], (pgs / ZZ::ST) & 1, x.abort_flag, x.err);
                char *vs = x.sm + ZZ::oV + st * ZZ::VPAGE;
                for (int i = tid; i < (kPT - left) * ZZ::NBOX * 8; i += 128) {
                    const int chunk = i & 7, box = (i >> 3) % ZZ::NBOX, row = left + (i >> 3) / ZZ::NBOX;
                    *reinterpret_cast<uint4 *>(vs + box * ZZ::BOX + row * 128 + chunk * 16) = make_uint4(0, 0, 0, 0);
                }
            }
            fence_proxy_async_smem();
            tc_fence_before();
            mbar_arrive(&x.bar[bPfull + s]);
        }
    }
    // the run's maxima and sums, for the epilogue
#pragma unroll
    for (int j = 0; j < SUBS; ++j) {
        const int slot = (sr + j) & 1;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float a = acc[j][v];
#pragma unroll
            for (int o = 4; o <= 16; o <<= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
            if (l4 == 0) x.lsum[(j * 4 + w) * kHalf + query(v)] = a;
        }
        if (sr + j >= 2) mbar_wait(&x.bar[bOfree + slot], ((sr + j - 2) >> 1) & 1, x.abort_flag, x.err);
        if (w == 0 && l4 == 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) x.state[slot * 2 * kHalf + query(v)] = m[j][v];
        }
    }
    named_bar_sync(1, 128);
#pragma unroll
    for (int j = 0; j < SUBS; ++j) {
        const int slot = (sr + j) & 1;
        if (tid < NQ) {
            const float *ls = x.lsum + j * 4 * kHalf + tid;
            x.state[slot * 2 * kHalf + kHalf + tid] = (ls[0] + ls[kHalf]) + (ls[2 * kHalf] + ls[3 * kHalf]);
        }
        mbar_arrive(&x.bar[bMfull + slot]);
    }
}

template <int RK, int RV, int DR>
__global__ void __launch_bounds__(kTrunkThreads, 1)
    trunk_kernel(const __grid_constant__ CUtensorMap tv, const __grid_constant__ TrunkParams p) {
    using ZZ = Z<RK, RV, DR>;
    extern __shared__ __align__(1024) char sm_raw[];
    TrunkCtx x;
    x.sm = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(sm_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    x.bar = reinterpret_cast<uint64_t *>(x.sm + ZZ::oBar);
    x.abort_flag = reinterpret_cast<volatile int *>(x.bar + bAbort);
    x.red = reinterpret_cast<float *>(x.sm + ZZ::oRed);
    x.factor = x.red + 256;
    x.lsum = x.factor + 32;
    x.beta = x.lsum + 256;
    x.state = x.beta + 128;
    x.err = p.err;
    uint32_t *tslot = reinterpret_cast<uint32_t *>(x.bar + bTslot);
    uint16_t *list = reinterpret_cast<uint16_t *>(x.sm + ZZ::oList);
    char *sm = x.sm;
    uint64_t *bar = x.bar;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

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
            mbar_init(&bar[bQfull + s], 32);
            mbar_init(&bar[bQfree + s], 1);
            mbar_init(&bar[bOdone + s], 1);
            mbar_init(&bar[bOfree + s], 128);
            mbar_init(&bar[bMfull + s], 128);
        }
        for (int s = 0; s < 4; ++s) mbar_init(&bar[bBfull + s], 32);
        *x.abort_flag = 0;
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
    const int groups = count_groups(p);
    const Share sh = find_share(p, groups, list);
    // q~ and beta come from the absorb kernel, and the workspace is free once it has waited for the kernel before it; the
    // producer reads only inputs of the call, which that kernel's wait ordered before this launch, and waits at its end
    if (warp != 0) pdl_wait();

    if (warp == 0) {
        // ------------------------------------------------------------------------------- producer
        if (lane == 0) {
            // after a failed wait (or once the abort flag is up) no further copy is issued, so no full barrier receives a
            // second arrival in one phase; the last ST rounds issued are awaited below
            const uint64_t pol = policy_evict_first();
            int itk = 0, itv = 0;
            for_runs(p, groups, sh, list, [&](const TrunkRun &r) {
                const int32_t *bt = p.block_table + static_cast<int64_t>(r.d.row) * p.max_blocks + r.page;
                for (int k = 0; k < r.pages; ++k) {
                    const int st = itk % ZZ::ST;
                    const uint32_t ph = (itk / ZZ::ST) & 1;
                    int32_t blk = bt[k];
                    if (blk < 0 || blk >= p.num_blocks) {
                        atomicOr(p.err, LLA_DEVERR_BLOCK_ID);
                        blk = 0;
                    }
                    const int64_t page = static_cast<int64_t>(blk) * p.H + r.h;
                    if (!mbar_wait(&bar[bKempty + st], ph ^ 1u, x.abort_flag, p.err) || *x.abort_flag) return false;
                    mbar_arrive_expect_tx(&bar[bKfull + st], ZZ::KPLANE + ZZ::RPLANE);
                    char *ks = sm + ZZ::oK + st * ZZ::KPAGE;
                    bulk_g2s(ks, p.pool + page * p.page_bytes, ZZ::KPLANE, &bar[bKfull + st], pol);
                    if constexpr (DR > 0)
                        bulk_g2s(ks + ZZ::KPAD, p.rope_pool + static_cast<int64_t>(blk) * ZZ::RPLANE, ZZ::RPLANE, &bar[bKfull + st], pol);
                    ++itk;
                    if (!mbar_wait(&bar[bVempty + st], ph ^ 1u, x.abort_flag, p.err) || *x.abort_flag) return false;
                    mbar_arrive_expect_tx(&bar[bVfull + st], ZZ::VPAGE);
                    char *vs = sm + ZZ::oV + st * ZZ::VPAGE;
#pragma unroll
                    for (int a = 0; a < ZZ::NBOX; ++a)
                        tma_load_3d(vs + a * ZZ::BOX, &tv, a * 64, 0, static_cast<int>(page), &bar[bVfull + st]);
                    ++itv;
                }
                return true;
            });
            // every copy has landed before the CTA can exit, even after an abort
            volatile int never = 0;
            for (int j = max(0, itk - ZZ::ST); j < itk; ++j) mbar_wait(&bar[bKfull + j % ZZ::ST], (j / ZZ::ST) & 1, &never, p.err);
            for (int j = max(0, itv - ZZ::ST); j < itv; ++j) mbar_wait(&bar[bVfull + j % ZZ::ST], (j / ZZ::ST) & 1, &never, p.err);
        }
        __syncwarp();
        pdl_wait();
    } else if (warp == 1) {
        // ----------------------------------------------------------------------------- S^T issuer
        const uint32_t base = smem_addr(sm);
        const uint64_t dk0 = umma_desc(base + ZZ::oK, kPT * 16, 128);
        int it = 0, pgs = 0, sr = 0;
        auto run = [&](int pages, int subs, int nq) {
            const uint32_t idesc = umma_idesc_bf16(64, 3 * nq, 0, 0);
            for (int k = 0; k < pages; ++k, ++pgs) {
                const int st = pgs % ZZ::ST;
                const uint64_t dk = dk0 + static_cast<uint64_t>((st * ZZ::KPAGE) >> 4);
                for (int j = 0; j < subs; ++j, ++it) {
                    const int s = it & 1, slot = (sr + j) & 1;
                    if (k == 0) mbar_wait_warp(&bar[bQfull + slot], ((sr + j) >> 1) & 1, x.abort_flag, p.err);
                    if (j == 0) mbar_wait_warp(&bar[bKfull + st], (pgs / ZZ::ST) & 1, x.abort_flag, p.err);
                    if (it >= 2) mbar_wait_warp(&bar[bSfree + s], ((it - 2) >> 1) & 1, x.abort_flag, p.err);
                    tc_fence_after();
                    const uint64_t dq = umma_desc(base + ZZ::oQ + slot * ZZ::QB, 3 * nq * 16, 128);
#pragma unroll
                    for (int ks = 0; ks < ZZ::RKT / 16; ++ks)
                        umma_bf16_warp(tmem + s * ZZ::TM_S, dk + ks * ((2 * kPT * 16) >> 4), dq + ks * ((2 * 3 * nq * 16) >> 4), idesc, ks > 0);
                    if (k == pages - 1) umma_commit_warp(&bar[bQfree + slot]);
                    if (j == subs - 1) umma_commit_warp(&bar[bKempty + st]);
                    umma_commit_warp(&bar[bSfull + s]);
                }
            }
            sr += subs;
        };
        for_runs(p, groups, sh, list, [&](const TrunkRun &r) {
            run(uniform(r.pages), uniform(r.subs), uniform(r.d.n) <= kFew ? kFew : kHalf);
            return true;
        });
        // every product has completed before TMEM is released, even after an abort: the last commit on each buffer
        volatile int never = 0;
        for (int j = max(0, it - 2); j < it; ++j) mbar_wait_warp(&bar[bSfull + (j & 1)], (j >> 1) & 1, &never, p.err);
        __syncwarp();
    } else if (warp == kValueWarp) {
        // ----------------------------------------------------------------------------- O^T issuer
        const uint32_t base = smem_addr(sm);
        const uint64_t dv0 = umma_desc_sw128_mn(base + ZZ::oV, ZZ::BOX);
        int it = 0, pgs = 0, sr = 0;
        for_runs(p, groups, sh, list, [&](const TrunkRun &r) {
            const int pages = uniform(r.pages), subs = uniform(r.subs), np = 2 * (uniform(r.d.n) <= kFew ? kFew : kHalf);
            const uint32_t idesc = umma_idesc_bf16(128, np, 1, 0), idesc64 = umma_idesc_bf16(64, np, 1, 0);
            for (int k = 0; k < pages; ++k, ++pgs) {
                const int st = pgs % ZZ::ST;
                const uint64_t dv = dv0 + static_cast<uint64_t>((st * ZZ::VPAGE) >> 4);
                for (int j = 0; j < subs; ++j, ++it) {
                    const int s = it & 1, slot = (sr + j) & 1;
                    mbar_wait_warp(&bar[bPfull + s], (it >> 1) & 1, x.abort_flag, p.err);
                    if (j == 0) mbar_wait_warp(&bar[bVfull + st], (pgs / ZZ::ST) & 1, x.abort_flag, p.err);
                    // the first page of a run starts O^T anew, once the epilogue has read the run before the last
                    if (k == 0 && sr + j >= 2) mbar_wait_warp(&bar[bOfree + slot], ((sr + j - 2) >> 1) & 1, x.abort_flag, p.err);
                    tc_fence_after();
                    const uint64_t dp = umma_desc(base + ZZ::oP + s * ZZ::PB, np * 16, 128);
#pragma unroll
                    for (int ch = 0; ch < ZZ::NCH; ++ch)
#pragma unroll
                        for (int ks = 0; ks < kPT / 16; ++ks)
                            umma_bf16_warp(tmem + ZZ::TM_O0 + slot * ZZ::TM_O + ch * (2 * kHalf), dv + ((ch * 2 * ZZ::BOX + ks * 2048) >> 4),
                                           dp + ks * ((2 * np * 16) >> 4), ZZ::LAST64 && ch == ZZ::NCH - 1 ? idesc64 : idesc, k > 0 || ks > 0);
                    if (j == subs - 1) umma_commit_warp(&bar[bVempty + st]);
                    if (k == pages - 1) umma_commit_warp(&bar[bOdone + slot]);
                    umma_commit_warp(&bar[bPfree + s]);  // also: O^T holds pages up to it
                }
            }
            sr += subs;
            return true;
        });
        if (it > 0) {  // every product has completed before TMEM is released, even after an abort
            volatile int never = 0;
            mbar_wait_warp(&bar[bPfree + ((it - 1) & 1)], ((it - 1) >> 1) & 1, &never, p.err);
        }
        __syncwarp();
    } else if (warp == kQueryWarp) {
        // ---------------------------------------------------------------------------- q~ operands
        int sr = 0;
        for_runs(p, groups, sh, list, [&](const TrunkRun &r) {
            const int nq = r.d.n <= kFew ? kFew : kHalf;
            for (int j = 0; j < r.subs; ++j, ++sr) {
                const int slot = sr & 1;
                if (sr >= 2) mbar_wait(&bar[bQfree + slot], ((sr - 2) >> 1) & 1, x.abort_flag, p.err);
                auto seq = [&](int n) {  // the sequence of query n of this operand, or none
                    const int i = j * kHalf + n;
                    if (i >= r.d.n) return -1;
                    if (r.d.member >= kLevels * p.B) return r.d.row;
                    const int b = p.plan.members[r.d.member + i];
                    return b < 0 || b >= p.B ? -1 : b;
                };
                // row part nq + n is bf16 part `part` of q~_n; its granule g lies at g (3 nq 16) + row 16
                for (int i = lane; i < nq * (ZZ::RKT / 8); i += 32) {
                    const int n = i / (ZZ::RKT / 8), g = i - n * (ZZ::RKT / 8), b = seq(n);
                    float part[3][8];
#pragma unroll
                    for (int k = 0; k < 3; ++k)
#pragma unroll
                        for (int e = 0; e < 8; ++e) part[k][e] = 0.f;
                    if (b >= 0) {
                        const float4 *src = reinterpret_cast<const float4 *>(p.qt + (static_cast<int64_t>(b) * p.H + r.h) * ZZ::RKT) + 2 * g;
                        const float4 u0 = src[0], u1 = src[1];
                        const float v[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w};
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            float pe[3];
                            bf16_parts(v[e], pe);
#pragma unroll
                            for (int k = 0; k < 3; ++k) part[k][e] = pe[k];
                        }
                    }
                    char *dq = sm + ZZ::oQ + slot * ZZ::QB + g * (3 * nq * 16);
#pragma unroll
                    for (int k = 0; k < 3; ++k)
                        *reinterpret_cast<uint4 *>(dq + (k * nq + n) * 16) =
                            make_uint4(pack_bf16x2(part[k][0], part[k][1]), pack_bf16x2(part[k][2], part[k][3]),
                                       pack_bf16x2(part[k][4], part[k][5]), pack_bf16x2(part[k][6], part[k][7]));
                }
                // Four slots of beta, each with its barrier: while S^T of a run of one page is issued the softmax warps may still
                // be a run behind.  They have read the slot that is written: S^T of operand sr - 2, which has been waited for,
                // needed the buffer of the page two before it, and so one of operand sr - 4 or behind.
                if (lane < nq) {
                    const int b = seq(lane);
                    x.beta[(sr & 3) * kHalf + lane] = b >= 0 ? p.beta[static_cast<int64_t>(b) * p.H + r.h] : 0.f;
                }
                mbar_arrive(&bar[bBfull + (sr & 3)]);
                fence_proxy_async_smem();
                mbar_arrive(&bar[bQfull + slot]);
            }
            return true;
        });
    } else if (warp < kEpilogueWarp) {
        // ------------------------------------------------------------------------ softmax, warps 4-7
        int it = 0, pgs = 0, sr = 0;
        for_runs(p, groups, sh, list, [&](const TrunkRun &r) {
            if (r.d.n <= kFew) softmax_run<ZZ, kFew, 1>(x, r, it, pgs, sr);
            else if (r.subs == 1) softmax_run<ZZ, kHalf, 1>(x, r, it, pgs, sr);
            else softmax_run<ZZ, kHalf, 2>(x, r, it, pgs, sr);
            sr += r.subs;
            return true;
        });
    } else {
        // ----------------------------------------------------------------------- epilogue, warps 8-11
        constexpr int RS = record_floats(RV);
        const int w = warp & 3, et = tid - 32 * kEpilogueWarp;
        const uint32_t tl = static_cast<uint32_t>(32 * w) << 16;
        int sr = 0;
        for_runs(p, groups, sh, list, [&](const TrunkRun &r) {
            for (int j = 0; j < r.subs; ++j, ++sr) {
                const int slot = sr & 1, n = min(kHalf, r.d.n - j * kHalf);
                mbar_wait(&bar[bOdone + slot], (sr >> 1) & 1, x.abort_flag, p.err);
                mbar_wait(&bar[bMfull + slot], (sr >> 1) & 1, x.abort_flag, p.err);
                tc_fence_after();
                float *dst = p.part + (record_of(p, r.d, r.h, blockIdx.x) + j * kHalf) * RS;
#pragma unroll
                for (int ch = 0; ch < ZZ::NCH; ++ch) {
                    const bool half = ZZ::LAST64 && ch == ZZ::NCH - 1;  // 16 rows in each quarter of the lanes
                    const int row = ch * 128 + (half ? 16 : 32) * w + lane;
                    const bool mine = row < RV && (!half || lane < 16);
                    const uint32_t to = tl + ZZ::TM_O0 + slot * ZZ::TM_O + ch * (2 * kHalf);
                    if (r.d.n <= kFew) {
                        float o[16];
                        tmem_ld16(to, o);
#pragma unroll
                        for (int q = 0; q < kFew; ++q)
                            if (mine && q < n) dst[q * RS + row] = o[q] + o[kFew + q];
                    } else {
                        float o0[32], o1[32];
                        tmem_ld32(to, o0);
                        tmem_ld32(to + kHalf, o1);
#pragma unroll
                        for (int q = 0; q < kHalf; ++q)
                            if (mine && q < n) dst[q * RS + row] = o0[q] + o1[q];
                    }
                }
                if (et < n) {
                    dst[et * RS + RV] = x.state[slot * 2 * kHalf + et];
                    dst[et * RS + RV + 1] = x.state[slot * 2 * kHalf + kHalf + et];
                }
                tc_fence_before();
                mbar_arrive(&bar[bOfree + slot]);
            }
            return true;
        });
    }
    pdl_trigger();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, ZZ::TM_COLS);
    }
}

// ------------------------------------------------------------------------------------------- join kernel

// Grid (H, ceil(B / spb)), 128 threads; SPB: the sequences that the projection is unrolled for.
template <int RV, int SPB>
__global__ void __launch_bounds__(128, 1) join_kernel(const __grid_constant__ JoinParams a) {
    constexpr int RS = record_floats(RV), NW = RV / 8, NJ = (RV + 31) / 32;
    constexpr int kMaxRuns = kMaxGrid + kLevels + 1;  // a CTA holds pages of several of a sequence's nodes at their ends only
    __shared__ __align__(16) float ob[SPB][RV];
    __shared__ float wts[4][kMaxRuns];
    __shared__ int recs[4][kMaxRuns];
    __shared__ float coef[SPB][3], scs[SPB];
    const TrunkParams &p = a.t;
    const int h = blockIdx.x, b0 = blockIdx.y * a.spb, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int nb = min(a.spb, p.B - b0);
    const int64_t th = static_cast<int64_t>(h) * a.T + a.loop;
    auto iorow = [&](int b) { return static_cast<int64_t>(b) * p.H + h; };
    // this thread's row of W_up^V and mu^V, the current tokens' scores and values: inputs of the call, before the wait
    const uint4 *W = reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.w_up_v) + (th * kD + tid) * RV);
    uint4 wr[NW];
#pragma unroll
    for (int j = 0; j < NW; ++j) wr[j] = W[j];
    const float muv = a.mu_v ? a.mu_v[th * kD + tid] : 0.f;
    float cv[SPB];
#pragma unroll
    for (int bi = 0; bi < SPB; ++bi) cv[bi] = a.cur_v && bi < nb ? load_elem(a.cur_v, iorow(b0 + bi) * kD + tid, a.io_bf16) : 0.f;
    if (a.cur_k) {
        for (int bi = warp; bi < nb; bi += 4) {
            const int64_t row = iorow(b0 + bi);
            float qk = 0.f;
#pragma unroll
            for (int i = 0; i < kD / 32; ++i)
                qk = fmaf(load_elem(a.q, row * kD + lane + 32 * i, a.io_bf16), load_elem(a.cur_k, row * kD + lane + 32 * i, a.io_bf16), qk);
            for (int i = lane; i < a.d_rope; i += 32)  // both stand at one position: the rotation cancels
                qk = fmaf(load_elem(a.q_rope, row * a.d_rope + i, a.io_bf16),
                          load_elem(a.cur_k_rope, static_cast<int64_t>(b0 + bi) * a.d_rope + i, a.io_bf16), qk);
            qk = warp_sum(qk);
            if (lane == 0) scs[bi] = qk * a.scale_log2;
        }
    }
    __syncthreads();
    pdl_wait();
    const int groups = count_groups(p), nodes = groups + p.B;
    const int NP = p.pstart[nodes] * p.H, Ge = min(a.grid, NP);  // the split of find_share
    // G warps per sequence: warp `sub` of them takes the columns lane + 32 (sub + G q)
    const int G = nb == 1 ? 4 : nb == 2 ? 2 : 1;
    const int grp = warp / G, sub = warp - grp * G;
    float *wt = wts[warp];
    int *rec = recs[warp];
    for (int bi = grp; bi < SPB; bi += 4 / G) {
        if (bi >= nb) {
            for (int j = lane + 32 * sub; j < RV; j += 32 * G) ob[bi][j] = 0.f;
            continue;
        }
        const int b = b0 + bi;
        // the runs of the sequence's nodes
        int nr = 0;
        for (int l = 0; l <= kLevels; ++l) {
            int i = groups + b, q = 0;
            if (l < kLevels) {
                const int col = p.plan.column[static_cast<int64_t>(l) * p.B + b];
                if (col < 0 || col / kMembers >= groups) continue;
                i = col / kMembers;
                q = col % kMembers;
            }
            const Node d = node_at(p, groups, i);
            if (d.pages == 0 || q >= d.n) continue;
            const int s0 = p.pstart[i] * p.H + h * d.pages, c0 = cta_of(s0, NP, Ge), c1 = cta_of(s0 + d.pages - 1, NP, Ge);
            const int64_t r0 = record_of(p, d, h, c0) + q;
            for (int c = lane; c <= c1 - c0 && nr + c < kMaxRuns; c += 32) rec[nr + c] = static_cast<int>(r0 + static_cast<int64_t>(kMembers) * c);
            nr = min(kMaxRuns, nr + c1 - c0 + 1);
        }
        __syncwarp();
        float M = -INFINITY, ls = 0.f;
        for (int i = lane; i < nr; i += 32) M = fmaxf(M, wt[i] = p.part[static_cast<int64_t>(rec[i]) * RS + RV]);
        M = warp_max(M);
        for (int i = lane; i < nr; i += 32) {
            const float w8 = wt[i] == -INFINITY ? 0.f : ex2_approx(wt[i] - M);
            ls = fmaf(w8, p.part[static_cast<int64_t>(rec[i]) * RS + RV + 1], ls);
            wt[i] = w8;
        }
        const float l = warp_sum(ls);
        __syncwarp();
        float acc[NJ];
#pragma unroll
        for (int q = 0; q < NJ; ++q) acc[q] = 0.f;
        constexpr int KR = 4;  // runs whose loads are in flight together
        for (int i0 = 0; i0 < nr; i0 += KR) {
            float v[KR][NJ];
#pragma unroll
            for (int k = 0; k < KR; ++k) {
                const float *pr = p.part + static_cast<int64_t>(rec[min(i0 + k, nr - 1)]) * RS;
#pragma unroll
                for (int q = 0; q < NJ; ++q) {
                    const int j = lane + 32 * (sub + G * q);
                    v[k][q] = j < RV ? pr[j] : 0.f;
                }
            }
#pragma unroll
            for (int k = 0; k < KR; ++k) {
                const float w8 = i0 + k < nr ? wt[i0 + k] : 0.f;
                if (w8 != 0.f) {  // warp-uniform (a NaN state stays one)
#pragma unroll
                    for (int q = 0; q < NJ; ++q) acc[q] = fmaf(w8, v[k][q], acc[q]);
                }
            }
        }
        __syncwarp();  // wt and rec are free for the warp's next sequence
#pragma unroll
        for (int q = 0; q < NJ; ++q) {
            const int j = lane + 32 * (sub + G * q);
            if (j < RV) ob[bi][j] = acc[q];
        }
        if (sub == 0 && lane == 0) {
            const float sc = a.cur_k ? scs[bi] : -INFINITY;
            const float Mx = fmaxf(M, sc);
            const float al = M == -INFINITY ? 0.f : ex2_approx(M - Mx);
            const float pc = a.cur_k ? ex2_approx(sc - Mx) : 0.f;
            const float den = al * l + pc;
            const float inv = den == 0.f ? 0.f : 1.f / den;
            coef[bi][0] = al * inv;
            coef[bi][1] = al * l * inv;
            coef[bi][2] = pc * inv;
        }
    }
    __syncthreads();
    // out_b[e] = coef0 (W_up^V o~_b)[e] + coef1 mu^V[e] + coef2 v_cur,b[e]
    float acc[SPB];
#pragma unroll
    for (int bi = 0; bi < SPB; ++bi) acc[bi] = 0.f;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
        const float2 w0 = bf2_to_f2(wr[j].x), w1 = bf2_to_f2(wr[j].y), w2 = bf2_to_f2(wr[j].z), w3 = bf2_to_f2(wr[j].w);
#pragma unroll
        for (int bi = 0; bi < SPB; ++bi) {
            const float4 o0 = *reinterpret_cast<const float4 *>(&ob[bi][j * 8]);
            const float4 o1 = *reinterpret_cast<const float4 *>(&ob[bi][j * 8 + 4]);
            float s = acc[bi];
            s = fmaf(w0.x, o0.x, s); s = fmaf(w0.y, o0.y, s); s = fmaf(w1.x, o0.z, s); s = fmaf(w1.y, o0.w, s);
            s = fmaf(w2.x, o1.x, s); s = fmaf(w2.y, o1.y, s); s = fmaf(w3.x, o1.z, s); s = fmaf(w3.y, o1.w, s);
            acc[bi] = s;
        }
    }
#pragma unroll
    for (int bi = 0; bi < SPB; ++bi) {
        if (bi >= nb) break;
        float v = acc[bi] * coef[bi][0] + coef[bi][1] * muv;
        if (a.cur_v) v = fmaf(coef[bi][2], cv[bi], v);
        store_elem(a.out, iorow(b0 + bi) * kD + tid, v, a.io_bf16);
    }
    __syncthreads();
    pdl_trigger();
}

// ----------------------------------------------------------------------------------------------- host side

struct PrefixWorkspace {
    size_t part, qt, beta, pstart, total;
};

inline size_t al256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

PrefixWorkspace prefix_workspace(int rkt, int r_v, int B, int H, int grid) {
    PrefixWorkspace w;
    const size_t records = static_cast<size_t>(H) * (kLevels + 1) * B + static_cast<size_t>(kMembers) * grid;
    w.part = 0;
    w.qt = al256(records * record_floats(r_v) * sizeof(float));
    w.beta = w.qt + al256(static_cast<size_t>(B) * H * rkt * sizeof(float));
    w.pstart = w.beta + al256(static_cast<size_t>(B) * H * sizeof(float));
    w.total = w.pstart + al256((kMaxNodes + 1) * sizeof(int));
    return w;
}

template <int RK, int RV, int DR>
lla_status launch_prefix(const DecodeArgs &a, const lla_prefix &plan, const void *rope_pool, const RotaryAxes &rope,
                         const int32_t *positions, const void *q_rope, const void *cur_k_rope, cudaStream_t stream) {
    using ZZ = Z<RK, RV, DR>;
    lla_status st = LLA_OK;
    unsigned *err = device_error_word(&st);
    if (st != LLA_OK) return st;
    const int grid = num_sms();
    if (grid <= 0) return LLA_ERR_CUDA;
    if (grid > kMaxGrid) return LLA_ERR_UNSUPPORTED;
    if (a.num_blocks * a.H >= (int64_t(1) << 31)) return LLA_ERR_UNSUPPORTED;  // TMA coordinate
    const PrefixWorkspace w = prefix_workspace(ZZ::RKT, RV, a.B, a.H, grid);
    if (a.workspace_bytes < w.total) return LLA_ERR_WORKSPACE;
    char *ws = static_cast<char *>(a.workspace);
    static DeviceOnce configured;
    if (raise_smem_limit(trunk_kernel<RK, RV, DR>, ZZ::SMEM, configured) != LLA_OK) return LLA_ERR_CUDA;
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
    tp.qt = reinterpret_cast<float *>(ws + w.qt);
    tp.beta = reinterpret_cast<float *>(ws + w.beta);
    tp.part = reinterpret_cast<float *>(ws + w.part);
    tp.pstart = reinterpret_cast<int *>(ws + w.pstart);
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
    if ((st = launch_ex(absorb_kernel<RK, DR>, dim3(a.H, (ZZ::RKX + 31) / 32 + (DR > 0), (a.B + 15) / 16), 256, 0, stream, ap)) != LLA_OK)
        return st;
    if ((st = launch_ex(trunk_kernel<RK, RV, DR>, dim3(grid), kTrunkThreads, ZZ::SMEM, stream, tv, tp)) != LLA_OK) return st;

    JoinParams jp = {};
    jp.t = tp;
    jp.T = a.T; jp.loop = a.loop; jp.io_bf16 = a.io_bf16; jp.grid = grid; jp.d_rope = DR;
    jp.scale_log2 = ap.scale_log2;
    jp.w_up_v = a.w_up_v; jp.mu_v = a.mu_v;
    jp.q = a.q; jp.q_rope = q_rope; jp.cur_k = a.cur_k; jp.cur_v = a.cur_v; jp.cur_k_rope = cur_k_rope;
    jp.out = a.out;
    // about two CTAs per SM: fewer sequences per CTA for small batches
    const int64_t units = static_cast<int64_t>(a.B) * a.H;
    jp.spb = static_cast<int>(std::min<int64_t>(kJoinSeqs, std::max<int64_t>(1, (units + 2 * grid - 1) / (2 * grid))));
    const dim3 jg(a.H, (a.B + jp.spb - 1) / jp.spb);
    if (jp.spb <= 2) return launch_ex(join_kernel<RV, 2>, jg, 128, 0, stream, jp);
    if (jp.spb <= 4) return launch_ex(join_kernel<RV, 4>, jg, 128, 0, stream, jp);
    return launch_ex(join_kernel<RV, 8>, jg, 128, 0, stream, jp);
}

}  // namespace

bool decode_prefix_supported(int es, int d, int r_k, int r_v, int d_rope) {
    if (es != 2 || d != kD) return false;
    if (d_rope == 0) return (r_k == 96 && r_v == 160) || (r_k == 128 && r_v == 128) || (r_k == 72 && r_v == 120);
    return r_k == 96 && r_v == 160 && (d_rope == 32 || d_rope == 64 || d_rope == 96);
}

size_t decode_prefix_workspace_bytes(int r_k, int r_v, int d_rope, int B, int H) {
    const int grid = num_sms();
    if (grid <= 0) return 0;
    return prefix_workspace((r_k + 15) / 16 * 16 + d_rope, r_v, B, H, grid).total;
}

lla_status launch_decode_prefix(const DecodeArgs &a, const lla_prefix &plan, const void *rope_pool, int d_rope,
                                const RotaryAxes &rope, const int32_t *positions, const void *q_rope,
                                const void *cur_k_rope, cudaStream_t stream) {
#define LLA_PREFIX(K, V, R) \
    if (a.r_k == K && a.r_v == V && d_rope == R) \
        return launch_prefix<K, V, R>(a, plan, rope_pool, rope, positions, q_rope, cur_k_rope, stream);
    LLA_PREFIX(96, 160, 0)
    LLA_PREFIX(128, 128, 0)
    LLA_PREFIX(72, 120, 0)
    LLA_PREFIX(96, 160, 32)
    LLA_PREFIX(96, 160, 64)
    LLA_PREFIX(96, 160, 96)
#undef LLA_PREFIX
    return LLA_ERR_UNSUPPORTED;
}

}  // namespace lla
