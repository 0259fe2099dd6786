// lla_beam.cu -- lla_beam_select: the best K continuations of the W beams of each sequence over the vocabulary.
//
// With z the finite logits of a beam, m any number near their maximum and
//   S = sum_u exp(z_u - m),   s_v = score + ((z_v - m) - log S),
// a continuation's rank is by s_v n^-alpha, and within a beam by z_v alone.  So one pass over the logits gives all
// that is needed: the sum S and the K largest logits.  Two launches:
//
//   beam_scan_kernel   a CTA per (beam, share of its row): the row is read once, 64 bytes a thread and tile, the
//                      next tile in flight while this one is summed.  A threshold that at least K logits seen so
//                      far exceed (or equal) lets few candidates through: a tile is kept only by threads whose
//                      maximum passes it.  Leaves the share's K best, sorted, and its (m, S).
//   beam_finish_kernel a CTA per sequence: merges the shares of each beam, log S, the keys in 64 bits, and a
//                      merge of the W sorted lists.
//
// Bound by HBM for large batches (2 or 4 bytes per logit, about 6 instructions per logit), by the chain of the two
// launches for small ones.
//
// Precision.  Ranks are compared in 64 bits, so what matters is log S, which the candidates of a beam share: it
// decides between beams.  z - m is rounded once and is exact where it counts, near m (Sterbenz); the sum of a tile's
// 16 or 32 terms is a tree, and sums of tiles, threads and shares carry their rounding errors along (Knuth's two-sum),
// so that log S is off by the 2^-22 of ex2.approx on single terms and not by the length of the row.
#include <cuda_runtime.h>
#include <float.h>
#include <math_constants.h>
#include <stdint.h>

#include "lla_device.cuh"
#include "lla_internal.h"
#include "lla_units.cuh"

namespace lla {
namespace {

constexpr int kScanThreads = 256;
constexpr int kWords = 4;                             // 16-byte words of a thread and tile
constexpr int kTileWords = kScanThreads * kWords;     // 16 KB a tile
constexpr int kFew = 64;                              // threads of a tile that may bring candidates
constexpr int kCap = 4096;                            // candidates that a CTA holds
constexpr int kMaxShares = 32;                        // shares of a row: a warp merges them
constexpr int kListLen = LLA_MAX_BEAMS;               // a list is a warp's lanes
constexpr float kRise = 60.f;                         // a logit this far over m moves m (e^60 2^24 is finite)

typedef unsigned long long u64;

// The sum and its offset of a share: S = (hi + lo), in units of exp(m).
struct Share {
    float m, hi, lo, unused;
};

// Numbers in order as unsigned integers: a < b as floats (no NaN) exactly if key(a) < key(b); -0 is made 0 before.
__device__ __forceinline__ uint32_t float_key(float x) {
    const uint32_t u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_float(uint32_t k) {
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
// A candidate: larger is better, a larger logit, then a lower token.  0 is none (a finite logit's key is not 0).
__device__ __forceinline__ u64 candidate(float x, int token) {
    return static_cast<u64>(float_key(x + 0.f)) << 32 | (0xffffffffu - static_cast<uint32_t>(token));
}
__device__ __forceinline__ int candidate_token(u64 c) { return static_cast<int>(0xffffffffu - static_cast<uint32_t>(c)); }
__device__ __forceinline__ float candidate_logit(u64 c) { return key_float(static_cast<uint32_t>(c >> 32)); }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two fp32 numbers in a register pair.
__device__ __forceinline__ u64 pack2(float a, float b) {
    u64 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 unpack2(u64 v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ u64 add2(u64 a, u64 b) {
    u64 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ u64 mul2(u64 a, u64 b) {
    u64 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// (hi, lo) += b, exactly but for the sum of the errors.
__device__ __forceinline__ void two_sum(float &hi, float &lo, float b) {
    const float s = __fadd_rn(hi, b), v = __fsub_rn(s, hi);
    lo += __fadd_rn(__fsub_rn(hi, __fsub_rn(s, v)), __fsub_rn(b, v));
    hi = s;
}

// ---------------------------------------------------------------------------------- sorted lists of a warp

__device__ __forceinline__ u64 shfl_xor64(u64 v, int o) { return __shfl_xor_sync(0xffffffffu, v, o); }

// The warp's 32 keys in descending order (bitonic).
__device__ __forceinline__ u64 sort_desc(u64 v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) {
            const u64 o = shfl_xor64(v, j);
            const bool keep_max = ((lane & j) == 0) == ((lane & k) == 0);
            v = keep_max ? (v > o ? v : o) : (v < o ? v : o);
        }
    return v;
}
// The 32 best of two descending lists, descending.
__device__ __forceinline__ u64 merge_desc(u64 a, u64 b) {
    const int lane = threadIdx.x & 31;
    const u64 r = __shfl_sync(0xffffffffu, b, 31 - lane);
    u64 v = a > r ? a : r;  // bitonic
#pragma unroll
    for (int j = 16; j > 0; j >>= 1) {
        const u64 o = shfl_xor64(v, j);
        v = (lane & j) == 0 ? (v > o ? v : o) : (v < o ? v : o);
    }
    return v;
}
// The same for (key, tag) pairs: a larger key, then a smaller tag, is better.
struct Ranked {
    u64 key;
    uint32_t tag;
};
__device__ __forceinline__ bool better(const Ranked &a, const Ranked &b) {
    return a.key != b.key ? a.key > b.key : a.tag < b.tag;
}
__device__ __forceinline__ Ranked merge_ranked(Ranked a, Ranked b) {
    const int lane = threadIdx.x & 31;
    Ranked r;
    r.key = __shfl_sync(0xffffffffu, b.key, 31 - lane);
    r.tag = __shfl_sync(0xffffffffu, b.tag, 31 - lane);
    Ranked v = better(a, r) ? a : r;
#pragma unroll
    for (int j = 16; j > 0; j >>= 1) {
        Ranked o;
        o.key = shfl_xor64(v.key, j);
        o.tag = __shfl_xor_sync(0xffffffffu, v.tag, j);
        if (better(o, v) == ((lane & j) == 0)) v = o;
    }
    return v;
}

// ------------------------------------------------------------------------------------------------ scan

struct ScanArgs {
    const void *logits;
    int64_t row_stride;
    const float *scores;
    const uint8_t *finished;
    int V, K, shares;
    u64 *lists;     // [row][share][K]
    Share *sums;    // [row][share]
};

template <bool BF16>
struct Row {
    static constexpr int kPer = BF16 ? 8 : 4;  // logits of a 16-byte word
    static constexpr uint32_t kMasked = BF16 ? 0xff80ff80u : 0xff800000u;  // -inf
    const char *base;  // the 16-byte word that holds the row's first logit
    int skip;          // its logits before that one
    int V;

    __device__ __forceinline__ void init(const ScanArgs &a, int row) {
        const char *p = static_cast<const char *>(a.logits) + row * a.row_stride * (BF16 ? 2 : 4);
        const int mis = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15);
        base = p - mis;
        skip = mis / (BF16 ? 2 : 4);
        V = a.V;
    }
    __device__ __forceinline__ int words() const { return (skip + V + kPer - 1) / kPer; }
    // Word w; what of it is no logit of the row is masked, and not read.
    __device__ __forceinline__ uint4 edge(int w) const {
        uint32_t r[4] = {kMasked, kMasked, kMasked, kMasked};
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int64_t i = static_cast<int64_t>(w) * kPer + e - skip;
            if (i >= 0 && i < V) {
                if (BF16) {
                    const uint32_t h = reinterpret_cast<const uint16_t *>(base)[i + skip];
                    r[e / 2] = e % 2 ? (r[e / 2] & 0xffffu) | h << 16 : (r[e / 2] & 0xffff0000u) | h;
                } else {
                    r[e % 4] = reinterpret_cast<const uint32_t *>(base)[i + skip];
                }
            }
        }
        return make_uint4(r[0], r[1], r[2], r[3]);
    }
    __device__ __forceinline__ uint4 whole(int w) const {
        uint4 v;
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "l"(base + static_cast<int64_t>(w) * 16));
        return v;
    }
    __device__ __forceinline__ void load(uint4 (&v)[kWords], int tile) const {
        const int w0 = tile * kTileWords + threadIdx.x;
        const int64_t lo = static_cast<int64_t>(tile) * kTileWords * kPer, hi = lo + kTileWords * kPer;
        if (lo >= skip && hi <= static_cast<int64_t>(skip) + V) {  // the same for the whole CTA
#pragma unroll
            for (int j = 0; j < kWords; ++j) v[j] = whole(w0 + j * kScanThreads);
        } else {
#pragma unroll
            for (int j = 0; j < kWords; ++j) {
                const int64_t i = static_cast<int64_t>(w0 + j * kScanThreads) * kPer;
                if (i >= skip && i + kPer <= static_cast<int64_t>(skip) + V) v[j] = whole(w0 + j * kScanThreads);
                else v[j] = edge(w0 + j * kScanThreads);
            }
        }
    }
    __device__ __forceinline__ int token(int tile, int j, int e) const {
        return (tile * kTileWords + j * kScanThreads + static_cast<int>(threadIdx.x)) * kPer + e - skip;
    }
};

__device__ __forceinline__ uint32_t word_of(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Logit e of a word.
template <bool BF16>
__device__ __forceinline__ float logit(const uint4 &v, int e) {
    if (!BF16) return __uint_as_float(word_of(v, e));
    const uint32_t u = word_of(v, e / 2);
    return __uint_as_float(e % 2 ? u & 0xffff0000u : u << 16);
}

// The largest of a thread's logits; NaN ones are passed over (all NaN: NaN).
template <bool BF16>
__device__ __forceinline__ float tile_max(const uint4 (&v)[kWords]) {
    if constexpr (BF16) {
        __nv_bfloat162 m[kWords];
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            const __nv_bfloat162 *p = reinterpret_cast<const __nv_bfloat162 *>(&v[j]);
            m[j] = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
        }
        const __nv_bfloat162 t = __hmax2(__hmax2(m[0], m[1]), __hmax2(m[2], m[3]));
        return fmaxf(__low2float(t), __high2float(t));
    } else {
        float m[kWords];
#pragma unroll
        for (int j = 0; j < kWords; ++j)
            m[j] = fmaxf(fmaxf(logit<BF16>(v[j], 0), logit<BF16>(v[j], 1)), fmaxf(logit<BF16>(v[j], 2), logit<BF16>(v[j], 3)));
        return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
    }
}

// Infinite and NaN logits become -inf.
template <bool BF16>
__device__ __forceinline__ void mask_infinite(uint4 (&v)[kWords]) {
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        uint32_t *u = reinterpret_cast<uint32_t *>(&v[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (BF16) {
                if ((u[i] & 0x7f80u) == 0x7f80u) u[i] = (u[i] & 0xffff0000u) | 0xff80u;
                if ((u[i] & 0x7f800000u) == 0x7f800000u) u[i] = (u[i] & 0xffffu) | 0xff800000u;
            } else if ((u[i] & 0x7f800000u) == 0x7f800000u) {
                u[i] = 0xff800000u;
            }
        }
    }
}

// sum 2^((z - m) log2 e) over a thread's logits of a tile: a tree of pairs.
template <bool BF16>
__device__ __forceinline__ float tile_sum(const uint4 (&v)[kWords], float m) {
    const u64 minus = pack2(-m, -m), l2e = pack2(1.44269504f, 1.44269504f);
    u64 s[kWords];
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        u64 t[BF16 ? 4 : 2];
#pragma unroll
        for (int i = 0; i < (BF16 ? 4 : 2); ++i) {
            const u64 x = mul2(add2(pack2(logit<BF16>(v[j], 2 * i), logit<BF16>(v[j], 2 * i + 1)), minus), l2e);
            const float2 f = unpack2(x);
            t[i] = pack2(ex2(f.x), ex2(f.y));
        }
        s[j] = BF16 ? add2(add2(t[0], t[1]), add2(t[BF16 ? 2 : 0], t[BF16 ? 3 : 1])) : add2(t[0], t[1]);
    }
    const float2 f = unpack2(add2(add2(s[0], s[1]), add2(s[2], s[3])));
    return f.x + f.y;
}

// Shared state of a scanning CTA.
struct Scan {
    u64 buf[kCap];
    u64 tops[kScanThreads / 32][kListLen];
    float maxima[kScanThreads / 32], his[kScanThreads / 32], los[kScanThreads / 32];
    int count;  // candidates in buf
};

// The best 32 of the CTA's candidates, sorted, in the lanes of warp 0.  Barriers on entry and inside.
__device__ __forceinline__ u64 best_of(Scan &sh) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kWarps = kScanThreads / 32;
    __syncthreads();
    const int n = sh.count;
    u64 top = 0;
    for (int i = warp * 32; i < n; i += kScanThreads) {
        const u64 v = sort_desc(i + lane < n ? sh.buf[i + lane] : 0);
        top = i == warp * 32 ? v : merge_desc(top, v);
    }
    for (int half = kWarps / 2; half > 0; half >>= 1) {  // warps [half, 2 half) hand over and are done
        if (warp >= half && warp < 2 * half) sh.tops[warp][lane] = top;
        __syncthreads();
        if (warp < half) top = merge_desc(top, sh.tops[warp + half][lane]);
    }
    return top;
}

template <bool BF16>
__global__ void __launch_bounds__(kScanThreads, 4) beam_scan_kernel(const ScanArgs a) {
    __shared__ Scan sh;
    const int row = blockIdx.x / a.shares, share = blockIdx.x - row * a.shares;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kWarps = kScanThreads / 32, kPer = Row<BF16>::kPer;
    if (tid == 0) sh.count = 0;
    pdl_wait();
    pdl_trigger();
    // a beam that is dead or has ended has nothing to read
    if ((a.finished && a.finished[row]) || !(fabsf(a.scores[row]) <= FLT_MAX)) return;
    Row<BF16> r;
    r.init(a, row);
    const int tiles = (r.words() + kTileWords - 1) / kTileWords;
    const int t0 = static_cast<int>(static_cast<int64_t>(share) * tiles / a.shares);
    const int t1 = static_cast<int>(static_cast<int64_t>(share + 1) * tiles / a.shares);
    const int K = a.K;
    float thr = -CUDART_INF_F;  // at least K logits of lower tokens are >= thr (or it is -inf): only larger ones count
    float m = 0.f, limit = -FLT_MAX, hi = 0.f, lo = 0.f;
    bool have_m = false;
    int bound = 0;  // at least as many as sh.count
    uint4 v[kWords], next[kWords];
    if (t0 < t1) r.load(v, t0);
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) r.load(next, t + 1);
        float top = tile_max<BF16>(v);
        if (!(top <= FLT_MAX)) {  // +inf or nothing but NaN
            mask_infinite<BF16>(v);
            top = tile_max<BF16>(v);
        }
        int passing = __syncthreads_count(top > thr);
        if (!have_m && passing) {  // (thr is -inf until then) the first finite logits: m is their maximum in the CTA
            have_m = true;
            const float w = warp_max(top);
            if (lane == 0) sh.maxima[warp] = w;
            __syncthreads();
            m = sh.maxima[0];
#pragma unroll
            for (int i = 1; i < kWarps; ++i) m = fmaxf(m, sh.maxima[i]);
            limit = m + kRise;
        }
        if (have_m) {
            if (top > limit) {  // a thread's own m from here on
                const float f = ex2((m - top) * 1.44269504f);
                m = top;
                limit = m + kRise;
                hi *= f;
                lo *= f;
            }
            float s = tile_sum<BF16>(v, m);
            if (!(s <= FLT_MAX)) {  // a NaN beside finite logits
                mask_infinite<BF16>(v);
                s = tile_sum<BF16>(v, m);
            }
            two_sum(hi, lo, s);
        }
        if (passing) {
            // Few enough threads bring candidates, or the threshold rises: to one that at least K of their maxima exceed
            // and at most kFew, found by bisection over the numbers (each step a count), or, where too many are
            // equal, over the tokens of equal logits.
            float over = thr, tie = CUDART_INF_F;
            int last_tie = -1, brings = passing;
            if (passing > kFew) {
                const uint32_t mine = float_key(top + 0.f);
                uint32_t below = float_key(thr), above = 0xff800000u;  // the keys of thr and of +inf
                int n_above = 0;
                bool found = false;
                while (above - below > 1) {
                    const uint32_t mid = below + (above - below) / 2;
                    const int n = __syncthreads_count(mine > mid);
                    if (n > kFew) {
                        below = mid;
                    } else if (n < K) {
                        above = mid;
                        n_above = n;
                    } else {
                        over = key_float(mid == 0x7fffffffu ? mid - 1 : mid);  // never -0, which no maximum's key is
                        brings = n;
                        found = true;
                        break;
                    }
                }
                if (!found) {  // n_above < K maxima are over the number of key `above`, and more than kFew over the one below
                    over = tie = key_float(above);
                    int first = INT32_MAX;  // my first logit equal to it
#pragma unroll
                    for (int j = kWords - 1; j >= 0; --j)
#pragma unroll
                        for (int e = kPer - 1; e >= 0; --e)
                            if (logit<BF16>(v[j], e) == tie) first = r.token(t, j, e);
                    int from = r.token(t, 0, 0) - tid * kPer - 1, to = from + kTileWords * kPer;  // (from, to]: the tile's tokens
                    for (;;) {  // the number with first <= from is below K, with first <= to at least K
                        last_tie = from + (to - from + 1) / 2;
                        const int n = __syncthreads_count(first <= last_tie);
                        if (n < K) from = last_tie;
                        else if (n > kFew) to = last_tie;
                        else {
                            brings = n_above + n;
                            break;
                        }
                    }
                }
            }
            constexpr int kMine = kWords * kPer;
            if (bound + brings * kMine > kCap) {  // keep the K best; K are then at least as large as the least of them
                const u64 best = best_of(sh);
                __syncthreads();
                if (warp == 0 && lane < K) sh.buf[lane] = best;
                if (tid == 0) sh.count = min(sh.count, K);
                __syncthreads();
                bound = K;
                const u64 least = sh.count == K ? sh.buf[K - 1] : 0;
                if (least) over = fmaxf(over, candidate_logit(least));
                __syncthreads();
            }
            bound += brings * kMine;
            if (top > over || top >= tie) {
#pragma unroll
                for (int j = 0; j < kWords; ++j)
#pragma unroll
                    for (int e = 0; e < kPer; ++e) {
                        const float x = logit<BF16>(v[j], e);
                        const int token = r.token(t, j, e);
                        if (x > over || (x == tie && token <= last_tie)) {
                            const int at = atomicAdd(&sh.count, 1);
                            if (at < kCap) sh.buf[at] = candidate(x, token);
                        }
                    }
            }
            if (over > thr) thr = over;
        }
#pragma unroll
        for (int j = 0; j < kWords; ++j) v[j] = next[j];
    }
    // the share's best, and its sum: threads' sums in units of the largest m
    const u64 best = best_of(sh);
    const int at = row * a.shares + share;
    if (warp == 0 && lane < K) a.lists[static_cast<int64_t>(at) * K + lane] = best;
    float M = warp_max(have_m ? m : -CUDART_INF_F);
    if (lane == 0) sh.maxima[warp] = M;
    __syncthreads();
    M = sh.maxima[0];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) M = fmaxf(M, sh.maxima[i]);
    if (have_m && m != M) {
        const float f = ex2((m - M) * 1.44269504f);
        hi *= f;
        lo *= f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float h = __shfl_xor_sync(0xffffffffu, hi, o), l = __shfl_xor_sync(0xffffffffu, lo, o);
        two_sum(hi, lo, h);
        lo += l;
    }
    if (lane == 0) {
        sh.his[warp] = hi;
        sh.los[warp] = lo;
    }
    __syncthreads();
    if (tid == 0) {
#pragma unroll
        for (int i = 1; i < kWarps; ++i) {
            two_sum(hi, lo, sh.his[i]);
            lo += sh.los[i];
        }
        a.sums[at] = Share{M, hi, lo, 0.f};
    }
}

// ---------------------------------------------------------------------------------------------- finish

constexpr int kFinishThreads = 512;
constexpr int kFinishWarps = kFinishThreads / 32;

struct FinishArgs {
    int W, K, shares;
    const u64 *lists;
    const Share *sums;
    const float *scores;
    const uint8_t *finished;
    const int32_t *lengths;
    int eos;
    double alpha;
    int32_t *parents, *tokens;
    float *out_scores;
    uint8_t *out_finished;
    int32_t *out_lengths;
};

// Doubles in order as unsigned integers (no NaN); 0 is below all of them.
__device__ __forceinline__ u64 double_key(double x) {
    const u64 u = static_cast<u64>(__double_as_longlong(x + 0.0));
    return u ^ ((u >> 63) ? ~0ull : 1ull << 63);
}

__global__ void __launch_bounds__(kFinishThreads) beam_finish_kernel(const FinishArgs a) {
    __shared__ u64 cand[LLA_MAX_BEAMS][kListLen];    // each beam's best, sorted
    __shared__ u64 keys[LLA_MAX_BEAMS][kListLen];
    __shared__ uint32_t tags[LLA_MAX_BEAMS][kListLen];
    __shared__ double total[LLA_MAX_BEAMS][kListLen];
    __shared__ u64 part[kFinishWarps][kListLen];
    __shared__ double mass[LLA_MAX_BEAMS], log_mass[LLA_MAX_BEAMS], scale[LLA_MAX_BEAMS];
    __shared__ float offset[LLA_MAX_BEAMS], score[LLA_MAX_BEAMS];
    __shared__ int state[LLA_MAX_BEAMS], length[LLA_MAX_BEAMS];  // state 0: dead, 1: goes on, 2: ended
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int W = a.W, K = a.K, b = blockIdx.x;
    pdl_wait();
    pdl_trigger();
    if (tid < W) {
        const int row = b * W + tid;
        const float s = a.scores[row];
        score[tid] = s;
        const bool ended = a.finished && a.finished[row];
        state[tid] = !(fabsf(s) <= FLT_MAX) ? 0 : ended ? 2 : 1;
        const int64_t n = a.lengths ? static_cast<int64_t>(a.lengths[row]) + (ended ? 0 : 1) : 1;
        length[tid] = static_cast<int>(n < INT32_MAX ? n : INT32_MAX);
        mass[tid] = 0.0;
    }
    __syncthreads();
    // n^-alpha of every beam by the last warp, while the others merge
    if (warp == kFinishWarps - 1 && lane < W)
        scale[lane] = a.alpha == 0.0 ? 1.0 : pow(static_cast<double>(max(1, length[lane])), -a.alpha);
    // parts warps merge a beam's shares, then one of them the parts
    const int parts = max(1, min(4, min(a.shares, kFinishWarps / W)));
    const int at_once = kFinishWarps / parts;
    for (int w0 = 0; w0 < W; w0 += at_once) {
        const int w = w0 + warp / parts, p = warp % parts;
        const bool mine = warp / parts < at_once && w < W && state[w < W ? w : 0] == 1;
        u64 top = 0;
        if (mine) {
            const u64 *list = a.lists + static_cast<int64_t>(b * W + w) * a.shares * K;
            u64 ahead = p < a.shares && lane < K ? list[static_cast<int64_t>(p) * K + lane] : 0;
            for (int s = p; s < a.shares; s += parts) {
                const u64 v = ahead;
                ahead = s + parts < a.shares && lane < K ? list[static_cast<int64_t>(s + parts) * K + lane] : 0;
                top = s == p ? v : merge_desc(top, v);
            }
            if (p == parts - 1) {  // and the sum over the shares
                const Share sum = lane < a.shares ? a.sums[(b * W + w) * a.shares + lane] : Share{-CUDART_INF_F, 0.f, 0.f, 0.f};
                const float M = warp_max(sum.m);
                double S = 0.0;
                if (sum.m > -CUDART_INF_F) {
                    const float f = sum.m == M ? 1.f : expf(sum.m - M);
                    S = (static_cast<double>(sum.hi) + static_cast<double>(sum.lo)) * static_cast<double>(f);
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
                if (lane == 0) {
                    mass[w] = S;
                    offset[w] = M;
                }
            }
        }
        if (parts > 1) {
            part[warp][lane] = top;
            __syncthreads();
            if (mine && p == 0) {
                for (int i = 1; i < parts; ++i) top = merge_desc(top, part[warp + i][lane]);
                cand[w][lane] = top;
            }
            __syncthreads();
        } else if (mine) {
            cand[w][lane] = top;
        }
    }
    __syncthreads();
    if (warp == 0 && lane < W) log_mass[lane] = mass[lane] > 0.0 ? log(mass[lane]) : 0.0;
    __syncthreads();
    for (int w = warp; w < W; w += kFinishWarps) {
        double s = 0.0;
        bool some = false;
        if (state[w] == 2) {
            s = score[w];
            some = lane == 0;
            if (some) cand[w][0] = candidate(0.f, a.eos);
        } else if (state[w] == 1) {
            const u64 c = lane < K ? cand[w][lane] : 0;
            some = c != 0;
            if (some)
                s = static_cast<double>(score[w]) +
                    ((static_cast<double>(candidate_logit(c)) - static_cast<double>(offset[w])) - log_mass[w]);
        }
        total[w][lane] = s;
        keys[w][lane] = some ? double_key(s * scale[w]) : 0;
        tags[w][lane] = w * kListLen + lane;
    }
    __syncthreads();
    for (int n = W; n > 1; n = (n + 1) / 2) {  // list w takes in list w + ceil(n / 2)
        const int half = (n + 1) / 2;
        for (int w = warp; w + half < n; w += kFinishWarps) {
            const Ranked r = merge_ranked(Ranked{keys[w][lane], tags[w][lane]}, Ranked{keys[w + half][lane], tags[w + half][lane]});
            keys[w][lane] = r.key;
            tags[w][lane] = r.tag;
        }
        __syncthreads();
    }
    if (tid < K) {
        const int at = b * K + tid;
        const bool some = keys[0][tid] != 0;
        const int w = tags[0][tid] / kListLen, i = tags[0][tid] % kListLen;
        const int token = some ? candidate_token(cand[w][i]) : -1;
        a.parents[at] = some ? b * W + w : -1;
        a.tokens[at] = token;
        a.out_scores[at] = some ? static_cast<float>(total[w][i]) : -CUDART_INF_F;
        if (a.out_finished) a.out_finished[at] = !some || state[w] == 2 || token == a.eos;
        if (a.out_lengths) a.out_lengths[at] = some ? length[w] : 0;
    }
}

int tiles_of(int V, bool bf16) {  // at most, whatever the alignment of a row
    const int64_t words = (static_cast<int64_t>(V) + (bf16 ? 8 : 4) - 1) / (bf16 ? 8 : 4) + 1;
    return static_cast<int>((words + kTileWords - 1) / kTileWords);
}

}  // namespace

size_t beam_select_workspace_bytes(int B, int W, int V, int K, bool bf16) {
    const int tiles = tiles_of(V, bf16);
    const size_t n = static_cast<size_t>(B) * W * (tiles < kMaxShares ? tiles : kMaxShares);
    return n * (sizeof(Share) + static_cast<size_t>(K) * sizeof(u64));
}

lla_status launch_beam_select(const BeamSelectArgs &b, cudaStream_t stream) {
    const int rows = b.B * b.W, tiles = tiles_of(b.V, b.bf16), sms = num_sms();
    if (sms <= 0) return LLA_ERR_CUDA;
    // shares of a row: the split with the shortest way of its slowest CTA slot, a share costing its tiles and about
    // four more for its threshold and its sort
    int shares = 1;
    int64_t best = INT64_MAX;
    for (int s = 1; s <= kMaxShares && s <= tiles; ++s) {
        const int64_t turns = (static_cast<int64_t>(rows) * s + sms * 4 - 1) / (sms * 4);
        const int64_t cost = turns * ((tiles + s - 1) / s + 4);
        if (cost < best) {
            best = cost;
            shares = s;
        }
    }
    ScanArgs a = {};
    a.logits = b.logits; a.row_stride = b.row_stride;
    a.scores = b.scores; a.finished = b.finished;
    a.V = b.V; a.K = b.K; a.shares = shares;
    a.sums = static_cast<Share *>(b.workspace);
    a.lists = reinterpret_cast<u64 *>(a.sums + static_cast<size_t>(rows) * shares);
    lla_status st = b.bf16 ? launch_ex(beam_scan_kernel<true>, dim3(rows * shares), kScanThreads, 0, stream, a)
                           : launch_ex(beam_scan_kernel<false>, dim3(rows * shares), kScanThreads, 0, stream, a);
    if (st != LLA_OK) return st;
    FinishArgs f = {};
    f.W = b.W; f.K = b.K; f.shares = shares;
    f.lists = a.lists; f.sums = a.sums;
    f.scores = b.scores; f.finished = b.finished; f.lengths = b.lengths;
    f.eos = b.eos; f.alpha = static_cast<double>(b.length_penalty);
    f.parents = b.parents; f.tokens = b.tokens; f.out_scores = b.out_scores;
    f.out_finished = b.out_finished; f.out_lengths = b.out_lengths;
    return launch_ex(beam_finish_kernel, dim3(b.B), kFinishThreads, 0, stream, f);
}

}  // namespace lla
