// lla_beam.cu -- lla_beam_select: the best K continuations of the W beams of each sequence over the vocabulary.
//
// With z the finite logits of a beam, m any number near their maximum and
//   S = sum_u exp(z_u - m),   s_v = score + ((z_v - m) - log S),
// a continuation's rank is by s_v n^-alpha, and within a beam by z_v alone.  So one pass over the logits gives all
// that is needed: the sum S and the K largest logits.  Two launches, the second behind the first's wait:
//
//   beam_scan_kernel   a CTA per (beam, share of its row): the row is read once, in tiles of 16 KB that are copied into
//                      shared memory a tile ahead.  A threshold that at least K logits seen so far reach lets few
//                      candidates through; what passes is looked at warp by warp, without a barrier, and ranked at the
//                      ends of growing groups of tiles.  Leaves the share's K best, sorted, and its sum.
//   beam_finish_kernel a CTA per sequence: merges the shares of each beam, takes the logarithm, forms the keys in 64
//                      bits, and merges the W sorted lists.
//
// Bound by HBM for large batches: 64 x 16 beams of 131072 bf16 logits (268 MB, 39.6 us at the copy rate) take 56.5 us.
// A second 268 MB on top takes 36.7 us, so tiles go by at the rate of HBM; the rest is the start of the two waves of rows (a
// first tile, its threshold: about 3 us each, 5 % of a wave for each look at the candidates), of which the second fills 416 of
// the 608 CTA slots, and the second kernel (4 us).
// Rows cut evenly over resident CTAs took 77 us against 66 then: every piece of a row pays a start.  Three stages and
// three CTAs an SM, four more registers, or candidates found in registers (spills) lost 2 to 20 %.  Small batches are
// bound by the chain of the two launches: 4 beams of 32000 logits take 8.7 us, of which the host call is 4.
//
// Precision.  Ranks are compared in 64 bits, so what matters is log S, which the candidates of a beam share: it
// decides between beams.  A term 2^(z K - c), K the fp32 number next to log2 e, takes one rounding of its exponent: 2^-24 |z - b|
// in log S, b = c / K.  K is off by less than 2^-26 of itself, and since sums are put together as powers of 2^K, with b formed from
// the same K, that counts with |z - b| as well, not with |z|.  b is a largest logit seen (to within 0.35, as c is whole), and a thread
// moves it once a logit is kRise = 5 above, so |z - b| <= max(5, top - z) + 0.35, of which the mean under the softmax, d, counts.
// ex2.approx adds 2^-22; a tile's 16 or 32 terms are summed as a tree of five roundings of 2^-24 (logit by logit, where some are not
// finite, ten); the sums of tiles, threads and shares carry their rounding errors along (Knuth's two-sum) and go to a common base
// exactly; the logarithm adds 4e-9:
//   |error of log S| <= 2^-22 + (5 or 10) 2^-24 + 1.25 2^-24 d + 4e-9 < (6 or 9)e-7 + 7.5e-8 d,
// whatever the length of the row.  Rows with logits beyond +-65536 (Base::wide) pay 2^-22 + 2^-23 + 2^-23 d more for each move of a sum
// to another base, of which there are three, as a rule, and six that count at most.  (d is 5 to 7 for most rows; below one large logit, flat rows have ln V.)  How a row is cut into
// shares decides which b a term meets, so the same beam's score may differ by as much from batch to batch.  With kRise = 60 single
// logits far above the first tile were off by 1.4e-6 in a test and by up to 3.4e-6 on paper.  A move sends its warp past the usual tiles'
// loop: kRise = 60, 5, 4 and 2 took 55.9, 56.5, 57.0 and 58.0 us on the largest batch.
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <math_constants.h>
#include <stdint.h>

#include "lla_beam_math.cuh"
#include "lla_device.cuh"
#include "lla_internal.h"
#include "lla_units.cuh"

namespace lla {
namespace {

constexpr int kScanThreads = 256;
constexpr int kWords = 4;                             // 16-byte words of a thread and tile
constexpr int kTileWords = kScanThreads * kWords;     // 16 KB a tile
constexpr int kStages = 2;                            // tiles in shared memory
constexpr int kScanCtas = 4;                          // of an SM
constexpr int kFew = 4;                               // threads over K that may bring candidates of a tile
constexpr int kCap = (2 * LLA_MAX_BEAMS - 1 + kFew) * kWords * 8 + LLA_MAX_BEAMS;                            // candidates that a CTA holds
constexpr int kMaxShares = 32;                        // shares of a row: a warp merges them
constexpr int kListLen = LLA_MAX_BEAMS;               // a list is a warp's lanes
constexpr float kRise = 5.f;                          // a logit this far over the base's moves it: exponents of terms stay below 8

typedef unsigned long long u64;

// What a share of a row leaves: the sum of its terms, hi + lo, and the base of its terms (Base; c = -inf: no finite logit).
struct Share {
    float c, hi, lo, wide;
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
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) {
    u64 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
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
            v = (v > o) == keep_max ? v : o;  // one comparison and a select
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
        v = (v > o) == ((lane & j) == 0) ? v : o;
    }
    return v;
}
// The same for (key, tag) pairs: a larger key, then a smaller tag, is better.
struct Ranked {
    u64 key;
    uint32_t tag;
};
__device__ __forceinline__ bool better(const Ranked &a, const Ranked &b) {
    return (a.key > b.key) | ((a.key == b.key) & (a.tag < b.tag));
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
    // The tiles [first_whole, end_whole) consist of whole words.
    __device__ __forceinline__ int first_whole() const { return skip ? 1 : 0; }
    __device__ __forceinline__ int end_whole() const { return (skip + V) / (kPer * kTileWords); }
    // A thread's words of a tile (word j * kScanThreads + thread of it) into its place in shared memory, word by word;
    // no group of copies is committed.
    __device__ __forceinline__ void copy(uint4 (*slot)[kScanThreads], int tile) const {
#pragma unroll 1
        for (int j = 0; j < kWords; ++j) {
            const int w = tile * kTileWords + j * kScanThreads + threadIdx.x;
            const int64_t i = static_cast<int64_t>(w) * kPer;
            if (i >= skip && i + kPer <= static_cast<int64_t>(skip) + V)
                cp_async16(&slot[j][threadIdx.x], base + static_cast<int64_t>(w) * 16);
            else
                slot[j][threadIdx.x] = edge(w);
        }
    }
    // The token of logit e of a thread's word j, and a thread's logit i (word i / kPer) from shared memory.
    __device__ __forceinline__ int token(int tile, int j, int e, int thread) const {
        return (tile * kTileWords + j * kScanThreads + thread) * kPer + e - skip;
    }
    __device__ __forceinline__ float staged(const uint4 (*slot)[kScanThreads], int thread, int i) const {
        const uint4 *w = &slot[i / kPer][thread];
        if (BF16) return bf_to_f(reinterpret_cast<const uint16_t *>(w)[i % kPer]);
        return reinterpret_cast<const float *>(w)[i % kPer];
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
#pragma unroll
        for (int n = kWords / 2; n > 0; n /= 2)
#pragma unroll
            for (int j = 0; j < n; ++j) m[j] = __hmax2(m[j], m[j + n]);
        return fmaxf(__low2float(m[0]), __high2float(m[0]));
    } else {
        float m[kWords];
#pragma unroll
        for (int j = 0; j < kWords; ++j)
            m[j] = fmaxf(fmaxf(logit<BF16>(v[j], 0), logit<BF16>(v[j], 1)), fmaxf(logit<BF16>(v[j], 2), logit<BF16>(v[j], 3)));
        #pragma unroll
        for (int n = kWords / 2; n > 0; n /= 2)
#pragma unroll
            for (int j = 0; j < n; ++j) m[j] = fmaxf(m[j], m[j + n]);
        return m[0];
    }
}

// What a thread's terms are scaled by.  Terms are 2^(z kLog2e - c) with a whole number c, so that a change of c is exact
// and a term takes one multiply-add; where the largest logit is beyond +-65536 (a row masked whole by the lowest
// number, say) they are 2^((z - c) kLog2e) (`wide`).
constexpr float kLog2e = 1.44269504f;
struct Base {
    float c;
    bool wide;
    __device__ __forceinline__ void set(float top) {
        wide = !(fabsf(top) <= 65536.f);
        c = wide ? top : rintf(top * kLog2e);
    }
    __device__ __forceinline__ float at() const { return wide ? c : c * (1.f / kLog2e); }  // as a logit, nearly
};
__device__ __forceinline__ bool same(const Base &a, const Base &b) { return a.c == b.c && a.wide == b.wide; }

// A base as a logit in 64 bits: what its sums are in units of the exponential of.
__device__ __forceinline__ double logit_of(const Base &b) {
    return static_cast<double>(b.c) * (b.wide ? 1.0 : 1.0 / static_cast<double>(kLog2e));
}

// The factor of a sum that goes from one base to another, 2^(from - to) with bases in units of 1 / K: a power of two, and exact, where
// neither is wide (0 below 2^-126).  A wide base's c K is taken as a sum of two: near +-65536 its fp32 number is 2^-8 off (1.1e-4 of
// log S in rows on both sides, when this went through fp32 logits).  Beyond 2^20 a wide and another base are too far apart for any sum.
// (In fp64 the same cost small calls 1.2 us, even where no base is wide.)
__device__ __forceinline__ float rebase(const Base &from, const Base &to) {
    float n = from.c - to.c, rest = 0.f;
    if (from.wide || to.wide) {
        float d = n * kLog2e, low = 0.f;
        if (from.wide != to.wide) {
            const float w = fminf(fmaxf(from.wide ? from.c : to.c, -1048576.f), 1048576.f), wk = w * kLog2e, wl = fmaf(w, kLog2e, -wk);
            d = from.wide ? wk - to.c : from.c - wk;
            low = from.wide ? wl : -wl;
        }
        d = fmaxf(d, -1000.f);
        n = rintf(d);
        rest = (d - n) + low;
    }
    n = fminf(n, 127.f);
    const float f = n < -126.f ? 0.f : __int_as_float((static_cast<int>(n) + 127) << 23);
    return f * ex2(rest);
}

// The sum of a thread's terms of a tile, not wide: a tree of pairs.
template <bool BF16>
__device__ __forceinline__ float tile_sum(const uint4 (&v)[kWords], float c) {
    const u64 minus = pack2(-c, -c), l2e = pack2(kLog2e, kLog2e);
    u64 s[kWords];
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        u64 t[BF16 ? 4 : 2];
#pragma unroll
        for (int i = 0; i < (BF16 ? 4 : 2); ++i) {
            const float2 f = unpack2(fma2(pack2(logit<BF16>(v[j], 2 * i), logit<BF16>(v[j], 2 * i + 1)), l2e, minus));
            t[i] = pack2(ex2(f.x), ex2(f.y));
        }
        s[j] = BF16 ? add2(add2(t[0], t[1]), add2(t[BF16 ? 2 : 0], t[BF16 ? 3 : 1])) : add2(t[0], t[1]);
    }
#pragma unroll
    for (int n = kWords / 2; n > 0; n /= 2)
#pragma unroll
        for (int j = 0; j < n; ++j) s[j] = add2(s[j], s[j + n]);
    const float2 f = unpack2(s[0]);
    return f.x + f.y;
}

// Shared state of a scanning CTA.
struct Scan {
    uint4 ring[kStages][kWords][kScanThreads];  // a thread reads the words that it copied itself
    u64 buf[kCap];
    u64 tops[kScanThreads / 32][kListLen];
    uint32_t most[kScanThreads / 32], least[kScanThreads / 32];
    float maxima[kScanThreads / 32], his[kScanThreads / 32], los[kScanThreads / 32];
    Base base;
    int count;  // candidates in buf (over kCap: some were dropped)
};

template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// One more of *count; its value before.
__device__ __forceinline__ int claim(int *count) {
    int old;
    asm volatile("atom.shared.add.u32 %0, [%1], 1;" : "=r"(old) : "r"(smem_addr(count)) : "memory");
    return old;
}

// The best 32 of the first n candidates, sorted, in the lanes of warp 0.
__device__ __forceinline__ u64 best_of(Scan &sh, int n) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 top = 0;
    for (int i = warp * 32; i < n; i += kScanThreads) {
        const u64 v = sort_desc(i + lane < n ? sh.buf[i + lane] : 0);
        top = i == warp * 32 ? v : merge_desc(top, v);
    }
    for (int half = kScanThreads / 64; half > 0; half >>= 1) {  // warps [half, 2 half) hand over and are done
        if (n <= half * 32) continue;                           // they had none
        if (warp >= half && warp < 2 * half) sh.tops[warp][lane] = top;
        __syncthreads();
        if (warp < half) top = merge_desc(top, sh.tops[warp + half][lane]);
    }
    return top;
}

template <bool BF16>
__global__ void __launch_bounds__(kScanThreads, kScanCtas) beam_scan_kernel(const ScanArgs a) {
    extern __shared__ __align__(16) unsigned char scan_smem[];
    Scan &sh = *reinterpret_cast<Scan *>(scan_smem);
    const int row = blockIdx.x / a.shares, share = blockIdx.x - row * a.shares;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kWarps = kScanThreads / 32, kPer = Row<BF16>::kPer, kMine = kWords * kPer;
    if (tid == 0) sh.count = 0;
    pdl_wait();
    pdl_trigger();
    Row<BF16> r;
    r.init(a, row);
    const int tiles = (r.words() + kTileWords - 1) / kTileWords;
    const int t0 = static_cast<int>(static_cast<int64_t>(share) * tiles / a.shares);
    const int t1 = static_cast<int>(static_cast<int64_t>(share + 1) * tiles / a.shares);
    const int K = a.K, few = K + kFew;
    // The ring: tile t is copied kStages - 1 tiles ahead, a thread's words by itself.
    const int in0 = r.first_whole(), in1 = min(t1, r.end_whole());
    const uint32_t ring = smem_addr(&sh.ring[0][0][tid]);
    const char *ahead = r.base + (static_cast<int64_t>(t0) * kTileWords + tid) * 16;
    auto slot_of = [&](int t) { return sh.ring[(t - t0) % kStages]; };
    auto fetch_whole = [&](int t) {
        const uint32_t to = ring + (t - t0) % kStages * (kTileWords * 16);
#pragma unroll
        for (int j = 0; j < kWords; ++j)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + j * kScanThreads * 16),
                         "l"(ahead + j * kScanThreads * 16)
                         : "memory");
        ahead += kTileWords * 16;
        cp_async_commit();
    };
    auto fetch = [&](int t) {
        if (t >= in0 && t < in1) {
            fetch_whole(t);
        } else {
            if (t < t1) r.copy(slot_of(t), t);
            ahead += kTileWords * 16;
            cp_async_commit();
        }
    };
    for (int t = t0; t < t0 + kStages - 1; ++t) fetch(t);
    // a beam that is dead or has ended has nothing more to read (the first tiles are under way while this is known)
    if ((a.finished && a.finished[row]) || !(fabsf(a.scores[row]) <= FLT_MAX)) {
        cp_async_wait<0>();
        return;
    }

    float thr = -CUDART_INF_F;  // at least K logits of lower tokens are >= thr (or it is -inf): only larger ones count
    Base base = {0.f, false};
    float limit = -FLT_MAX, hi = 0.f, lo = 0.f;  // limit: the largest logit that base is good for
    bool have_base = false;
    int kept = 0;  // candidates in buf that are the best so far, sorted
    bool brought = false;
    // buf's best to its front, sorted; with K of them, only larger logits of later tokens count.  For few candidates
    // its place is the number of better ones (no two are equal); more than half as many as threads are sorted, which
    // takes 2.4 to 3.1 k cycles where counting takes 1.3 to 1.8 k.  Barriers, one behind the last candidate of all before.
    auto compact = [&]() {
        const int n = min(sh.count, kCap);
        u64 mine = 0;
        int place = tid;
        if (n <= kScanThreads / 2) {
            if (warp * 32 < n) {
                mine = tid < n ? sh.buf[tid] : 0;
                place = tid < n ? 0 : kScanThreads;
#pragma unroll 8
                for (int i = 0; i < n; ++i) place += sh.buf[i] > mine;
            }
        } else {
            mine = best_of(sh, n);
        }
        __syncthreads();
        kept = min(n, K);
        if (place < kept) sh.buf[place] = mine;
        if (tid == 0) sh.count = kept;
        __syncthreads();
        if (kept == K) thr = fmaxf(thr, candidate_logit(sh.buf[K - 1]));
    };
    // The candidates of a warp's threads `who`, thread by thread: a lane to each of that thread's logits, where pass(x, token).
    auto bring = [&](unsigned who, const uint4(*slot)[kScanThreads], int t, auto pass) {
        brought = true;
        __syncwarp();  // the words that other lanes copied
        const int token0 = r.token(t, lane / kPer, lane % kPer, warp * 32);
        do {
            const int owner = __ffs(who) - 1;
            who &= who - 1;
            if (lane < kMine) {
                const float x = r.staged(slot, warp * 32 + owner, lane);
                const int token = token0 + owner * kPer;
                if (pass(x, token)) {
                    const int at = claim(&sh.count);
                    if (at < kCap) sh.buf[at] = candidate(x, token);
                }
            }
        } while (who);
        __syncwarp();  // before the words are overwritten
    };

    // Tiles go by in groups of 1, 2, 6, 18 ...; within a group each warp goes by itself and brings what passes the
    // threshold, and at its end the threshold rises to the K-th best.  The first tile, those after it while fewer than
    // K logits were finite, and a group that brought too much (rising logits), once more, go tile by tile,
    // carefully: the threshold rises before candidates are brought.  (Groups growing by 2, 3 and 4: 62.0, 61.3, 62.3 us.)
    int from = t0, end = t0, group = 2, redo = -1;  // redo: where a group is gone through once more, its end
    __syncthreads();  // sh.count
    for (int t = t0; t < t1;) {
        const bool careful = redo >= 0 || !have_base || thr == -CUDART_INF_F;
        if (!careful && t == end) {
            from = t;
            end = min(t1, t + group);
            group *= 3;
            brought = false;
        }
        uint4 v[kWords];
        bool taken = false;  // the tile below has been waited for
        if (!careful) {
            // Usual tiles, of whole words and with an ordinary base: one question a tile about all that is not usual.
            const int stop = __any_sync(0xffffffffu, base.wide) ? t : min(end, in1 - (kStages - 1));
            const float usual = fminf(thr, limit);
            for (; t < stop; ++t) {
                fetch_whole(t + kStages - 1);  // over tile t - 1
                cp_async_wait<kStages - 1>();
                const uint4(*slot)[kScanThreads] = slot_of(t);
#pragma unroll
                for (int j = 0; j < kWords; ++j) v[j] = slot[j][tid];
                const float top = tile_max<BF16>(v), s = tile_sum<BF16>(v, base.c);
                if (__any_sync(0xffffffffu, !(top <= usual) || !(s <= FLT_MAX))) {
                    taken = __any_sync(0xffffffffu, !(top <= limit) || !(s <= FLT_MAX));
                    if (taken) break;
                    bring(__ballot_sync(0xffffffffu, top > thr), slot, t, [&](float x, int) { return x > thr; });
                }
                two_sum(hi, lo, s);
            }
        }
        if (careful || t < end) {  // any tile
            uint4(*slot)[kScanThreads] = slot_of(redo >= 0 ? redo - 1 : t);
            if (redo >= 0) {  // nothing is in flight in that slot
                r.copy(slot, t);
                cp_async_commit();
                cp_async_wait<0>();
            } else if (!taken) {
                fetch(t + kStages - 1);
                cp_async_wait<kStages - 1>();
            }
#pragma unroll
            for (int j = 0; j < kWords; ++j) v[j] = slot[j][tid];
            float top = tile_max<BF16>(v);
            if (!(top <= FLT_MAX)) {  // +inf or nothing but NaN: the largest finite one
                top = -CUDART_INF_F;
                for (int i = 0; i < kMine; ++i) {
                    const float x = r.staged(slot, tid, i);
                    if (x <= FLT_MAX) top = fmaxf(top, x);
                }
            }
            const uint32_t mine = float_key(top + 0.f);
            uint32_t most = 0, least = 0;  // keys of the largest and the least of the CTA's maxima
            int passing = 0;
            if (careful) {
                const uint32_t w_most = __reduce_max_sync(0xffffffffu, mine), w_least = __reduce_min_sync(0xffffffffu, mine);
                if (lane == 0) {
                    sh.most[warp] = w_most;
                    sh.least[warp] = w_least;
                }
                passing = __syncthreads_count(top > thr);
                most = sh.most[0];
                least = sh.least[0];
#pragma unroll
                for (int i = 1; i < kWarps; ++i) {
                    most = max(most, sh.most[i]);
                    least = min(least, sh.least[i]);
                }
                if (!have_base && passing) {  // (thr is -inf until then) the first finite logits
                    have_base = true;
                    base.set(key_float(most));
                    limit = key_float(most) + kRise;
                }
            }
            if (have_base && redo < 0) {
                if (top > limit) {  // a thread's own base from here on
                    const Base old = base;
                    base.set(top);
                    limit = top + kRise;
                    const float f = rebase(old, base);
                    hi *= f;
                    lo *= f;
                }
                float s = tile_sum<BF16>(v, base.c);
                if (!(s <= FLT_MAX) || base.wide) {  // a logit that is not finite, or a wide base: one by one, word by word
                    s = 0.f;
                    for (int j = 0; j < kWords; ++j) {
                        float word = 0.f;
                        for (int i = j * kPer; i < (j + 1) * kPer; ++i) {
                            const float x = r.staged(slot, tid, i);
                            if (fabsf(x) <= FLT_MAX) word += ex2(base.wide ? (x - base.c) * kLog2e : fmaf(x, kLog2e, -base.c));
                        }
                        s += word;
                    }
                }
                two_sum(hi, lo, s);
            }
            float over = thr, tie = CUDART_INF_F;
            int last_tie = -1;
            if (passing > few) {
                // Too many threads would bring candidates.  Find a threshold that at least K of their maxima exceed and at
                // most `few`, by bisection over the numbers (each step a count), or, where too many are equal, over the
                // tokens of equal logits.
                uint32_t below = max(float_key(thr), least - 1), above = most;  // more than `few` are over below, none over above
                bool found = false;
                while (above - below > 1) {
                    const uint32_t mid = below + (above - below) / 2;
                    const int n = __syncthreads_count(mine > mid);
                    if (n > few) {
                        below = mid;
                    } else if (n < K) {
                        above = mid;
                    } else {
                        over = key_float(mid == 0x7fffffffu ? mid - 1 : mid);  // never -0, which no maximum's key is
                        found = true;
                        break;
                    }
                }
                if (!found) {  // fewer than K maxima are over the number of key `above`, more than `few` over the one below
                    over = tie = key_float(above);
                    int mine_at = INT32_MAX;  // my first logit equal to it
                    for (int i = kMine - 1; i >= 0; --i)
                        if (r.staged(slot, tid, i) == tie) mine_at = r.token(t, i / kPer, i % kPer, tid);
                    // Threads over the tie, or with a tie up to a token: fewer than K up to lo_t, more than few up to hi_t (the
                    // whole tile), and one more at most from token to token, so that some token gives K to few of them.
                    // Fewer than 20 halvings lead there.
                    int lo_t = r.token(t, 0, 0, 0) - 1, hi_t = lo_t + kTileWords * kPer;
                    for (int step = 0; step < 32; ++step) {
                        last_tie = lo_t + (hi_t - lo_t + 1) / 2;
                        const int n = __syncthreads_count(mine > above || mine_at <= last_tie);
                        if (n < K) lo_t = last_tie;
                        else if (n > few) hi_t = last_tie;
                        else break;
                    }
                }
            }
            // In a careful tile at most K + few threads bring theirs: these and what compact() leaves have room in buf.
            static_assert((2 * LLA_MAX_BEAMS - 1 + kFew) * kMine + LLA_MAX_BEAMS <= kCap, "candidates of a tile");
            const unsigned who = __ballot_sync(0xffffffffu, top > over || top >= tie);
            if (who)
                bring(who, slot, t, [&](float x, int token) { return x <= FLT_MAX && (x > over || (x == tie && token <= last_tie)); });
            ++t;
            if (careful) {
                if (passing) {
                    thr = fmaxf(thr, over);
                    __syncthreads();
                    compact();
                }
                if (t == redo) redo = -1;
                if (redo < 0) end = t;
                continue;
            }
        }
        if (t < end || !__syncthreads_or(brought)) continue;  // the end of a group
        if (sh.count <= kCap) {
            compact();
        } else {  // some were dropped: the group once more
            __syncthreads();
            if (tid == 0) sh.count = kept;
            redo = end;
            t = from;
            __syncthreads();
        }
    }
    // the share's best, and its sum
    const int at = row * a.shares + share;
    if (tid < K) a.lists[static_cast<int64_t>(at) * K + tid] = tid < kept ? sh.buf[tid] : 0;
    __syncthreads();
    // threads' sums in units of the base of the one whose base is highest
    float M = warp_max(have_base ? base.at() : -CUDART_INF_F);
    if (lane == 0) sh.maxima[warp] = M;
    __syncthreads();
    M = sh.maxima[0];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) M = fmaxf(M, sh.maxima[i]);
    // those of equal at() are the same, but that one may be wide and another not
    const bool wide = __syncthreads_or(have_base && base.at() == M && base.wide);
    if (have_base && base.at() == M && base.wide == wide) sh.base = base;
    __syncthreads();
    const Base common = sh.base;
    if (have_base && !same(base, common)) {
        const float f = rebase(base, common);
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
        a.sums[at] = Share{have_base ? common.c : -CUDART_INF_F, hi, lo, have_base && common.wide ? 1.f : 0.f};
    }
}

// ---------------------------------------------------------------------------------------------- finish

constexpr int kFinishThreads = 512;
constexpr int kFinishWarps = kFinishThreads / 32;

struct FinishArgs {
    LogTable logs;
    int W, K, shares;
    const u64 *lists;
    const Share *sums;
    const float *scores;
    const uint8_t *finished;
    const int32_t *lengths;
    const int64_t *slots;
    int eos;
    double alpha;
    int32_t *parents, *tokens;
    float *out_scores;
    uint8_t *out_finished;
    int32_t *out_lengths;
    int32_t *model_tokens;
};

// Doubles in order as unsigned integers (no NaN); 0 is below all of them.
__device__ __forceinline__ u64 double_key(double x) {
    u64 u = static_cast<u64>(__double_as_longlong(x));
    if (u << 1 == 0) u = 0;  // -0
    return u ^ ((u >> 63) ? ~0ull : 1ull << 63);
}

__global__ void __launch_bounds__(kFinishThreads) beam_finish_kernel(const __grid_constant__ FinishArgs a) {
    __shared__ u64 cand[LLA_MAX_BEAMS][kListLen];    // each beam's best, sorted
    __shared__ u64 keys[LLA_MAX_BEAMS][kListLen];
    __shared__ uint32_t tags[LLA_MAX_BEAMS][kListLen];
    __shared__ double total[LLA_MAX_BEAMS][kListLen];
    __shared__ u64 part[kFinishWarps][kListLen];
    __shared__ double offset[LLA_MAX_BEAMS], rest[LLA_MAX_BEAMS];  // S is in units of exp(offset); score - log S
    __shared__ double scale[LLA_MAX_BEAMS];                        // n^-alpha
    __shared__ float2 mass[LLA_MAX_BEAMS];                         // S as a sum of two
    __shared__ float score_of[LLA_MAX_BEAMS];
    __shared__ int state[LLA_MAX_BEAMS], length[LLA_MAX_BEAMS];    // state 0: dead, 1: goes on, 2: ended
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int W = a.W, K = a.K, row0 = blockIdx.x * W;
    pdl_wait();
    pdl_trigger();
    // the last warp keeps the beams' states, and n^-alpha while the others merge
    float my_score = 0.f;
    if (warp == kFinishWarps - 1 && lane < W) {
        const float s = a.scores[row0 + lane];
        const bool ended = a.finished && a.finished[row0 + lane];
        const int64_t n = a.lengths ? static_cast<int64_t>(a.lengths[row0 + lane]) + (ended ? 0 : 1) : 1;
        const bool hole = a.slots && a.slots[row0 + lane] < 0;  // its last token is not cached
        state[lane] = !(fabsf(s) <= FLT_MAX) ? 0 : ended ? 2 : hole ? 0 : 1;
        length[lane] = static_cast<int>(n < INT32_MAX ? n : INT32_MAX);
        score_of[lane] = my_score = s;
        scale[lane] = a.alpha == 0.0 ? 1.0 : exp_of(-a.alpha * log_of(static_cast<double>(n > 1 ? n : 1)));  // |x| <= 16 log 2^31
    }
    // `parts` warps merge the lists of a beam's shares and one of them sums up its shares (of a beam that does not go on,
    // whatever is there, which nobody looks at); then one of them merges the parts
    const int parts = max(1, min(4, min(a.shares, kFinishWarps / W)));
    const int at_once = kFinishWarps / parts;
    // A warp's fp64 instruction holds the SM's one fp64 unit for about 20 cycles, whatever its lanes do: a few beams'
    // logarithms are taken by their warps beside the merges, those of many by one warp behind them.  One sequence of 32000
    // tokens, K = W, beside and behind: W = 2 7.06 and 7.17 us, 4 8.1 and 8.3, 8 8.9 and 9.1, 10 alike, 12 10.2 and 10.1, 16 11.2 and
    // 11.0, 32 16.4 and 15.3 (eight sequences: the same order, 20.8 and 19.8 with 32).
    const bool logs_here = W < 10;
    for (int w0 = 0; w0 < W; w0 += at_once) {
        const int w = w0 + warp / parts, p = warp % parts;
        const bool mine = warp / parts < at_once && w < W;
        u64 top = 0;
        if (mine) {
            const u64 *list = a.lists + static_cast<int64_t>(row0 + w) * a.shares * K;
            u64 ahead = lane < K ? list[static_cast<int64_t>(p) * K + lane] : 0;
            Share sum = {-CUDART_INF_F, 0.f, 0.f, 0.f};
            float score = 0.f;
            if (p == parts - 1) {
                if (lane < a.shares) sum = a.sums[(row0 + w) * a.shares + lane];
                if (logs_here) score = a.scores[row0 + w];
                const Base base = {sum.c, sum.wide != 0.f};
                const float M = warp_max(base.at());
                const unsigned tops = __ballot_sync(0xffffffffu, base.at() == M), wide_tops = __ballot_sync(0xffffffffu, base.wide) & tops;
                const int top_lane = __ffs(wide_tops ? wide_tops : tops) - 1;
                const Base common = {__shfl_sync(0xffffffffu, base.c, top_lane), __shfl_sync(0xffffffffu, base.wide, top_lane) != 0};
                const float f = sum.c > -CUDART_INF_F ? rebase(base, common) : 0.f;  // 1 where they are the same
                float hi = sum.hi * f, lo = sum.lo * f;
                for (int o = 1; o < a.shares; o <<= 1) {
                    const float h = __shfl_xor_sync(0xffffffffu, hi, o), l = __shfl_xor_sync(0xffffffffu, lo, o);
                    two_sum(hi, lo, h);
                    lo += l;
                }
                if (lane == 0) {
                    mass[w] = make_float2(hi, lo);
                    if (logs_here) rest[w] = static_cast<double>(score) - log_sum(hi, lo, a.logs);
                    offset[w] = logit_of(common);
                }
            }
            for (int s = p; s < a.shares; s += parts) {
                const u64 v = ahead;
                ahead = s + parts < a.shares && lane < K ? list[static_cast<int64_t>(s + parts) * K + lane] : 0;
                top = s == p ? v : merge_desc(top, v);
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
    if (!logs_here) {
        if (warp == kFinishWarps - 1 && lane < W)
            rest[lane] = static_cast<double>(my_score) - log_sum(mass[lane].x, mass[lane].y, a.logs);
        __syncthreads();
    }
    for (int w = warp; w < W; w += kFinishWarps) {
        u64 c = 0, key = 0;
        if (state[w] == 2) {
            c = lane == 0 ? candidate(0.f, a.eos) : 0;
            if (lane == 0) cand[w][0] = c;
        } else if (state[w] == 1 && lane < K) {
            c = cand[w][lane];
        }
        if (c) {
            double s = score_of[w];
            if (state[w] == 1) s = rest[w] + (static_cast<double>(candidate_logit(c)) - offset[w]);  // not lost beside a huge offset
            total[w][lane] = s;
            key = double_key(a.alpha == 0.0 ? s : s * scale[w]);
        }
        keys[w][lane] = key;
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
        const int at = blockIdx.x * K + tid;
        const bool some = keys[0][tid] != 0;
        const int w = tags[0][tid] / kListLen, i = tags[0][tid] % kListLen;
        const int token = some ? candidate_token(cand[w][i]) : -1;
        a.parents[at] = some ? row0 + w : -1;
        a.tokens[at] = token;
        a.out_scores[at] = some ? static_cast<float>(total[w][i]) : -CUDART_INF_F;
        if (a.out_finished) a.out_finished[at] = !some || state[w] == 2 || token == a.eos;
        if (a.out_lengths) a.out_lengths[at] = some ? length[w] : 0;
        if (a.model_tokens) a.model_tokens[at] = max(token, 0);
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
    // four more for its threshold and its looks at candidates (phase times of a row: 12 k cycles beside 2.3 k a tile)
    int shares = 1;
    int64_t best = INT64_MAX;
    for (int s = 1; s <= kMaxShares && s <= tiles; ++s) {
        const int64_t turns = (static_cast<int64_t>(rows) * s + sms * kScanCtas - 1) / (sms * kScanCtas);
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
    static DeviceOnce once[2];
    auto kern = b.bf16 ? beam_scan_kernel<true> : beam_scan_kernel<false>;
    lla_status st = raise_smem_limit(kern, static_cast<int>(sizeof(Scan)), once[b.bf16 ? 1 : 0]);
    if (st != LLA_OK) return st;
    st = launch_ex(kern, dim3(rows * shares), kScanThreads, static_cast<int>(sizeof(Scan)), stream, a);
    if (st != LLA_OK) return st;
    FinishArgs f = {};
    f.logs = log_table();
    f.W = b.W; f.K = b.K; f.shares = shares;
    f.lists = a.lists; f.sums = a.sums;
    f.scores = b.scores; f.finished = b.finished; f.lengths = b.lengths; f.slots = b.slots;
    f.eos = b.eos; f.alpha = static_cast<double>(b.length_penalty);
    f.parents = b.parents; f.tokens = b.tokens; f.out_scores = b.out_scores;
    f.out_finished = b.out_finished; f.out_lengths = b.out_lengths; f.model_tokens = b.model_tokens;
    return launch_ex(beam_finish_kernel, dim3(b.B), kFinishThreads, 0, stream, f);
}

}  // namespace lla
