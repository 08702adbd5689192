// logprobs.cu -- the log probability of given tokens under their logits, the
// entropy of the distribution and its k largest entries, in one pass over the
// logits; and the gradient of log probability and entropy (darb_token_logprobs,
// darb_token_logprobs_grad): what turns a layer's product into the perplexity
// that Sec. 4.1 reports and into the loss of its retraining.
//
// For a token with logits x_v:  M = max x,  s = sum exp(x_v - M),
//   lse = M + log s,   log p_v = x_v - lse,
//   H   = -sum p log p = log s - (sum exp(x_v - M) (x_v - M)) / s.
// The kernels work in base 2: with the reference r = M log2(e), rounded once
// and used by every term, d_v = x_v log2(e) - r is one FMA, e_v = 2^d_v one
// instruction, and lse = (r + log2 s) ln 2.  A partial result is (M, s, t) with
// s = sum e_v and t = sum e_v d_v; two of them join by
//   f = 2^(r1 - r),  s += f s1,  t += f (t1 + s1 (r1 - r)).
//
// Masks.  Logits are clamped from below at -2^15 before use, so that a masked
// entry (-inf, the type's lowest value, -1e9) adds 2^-huge = 0 to s and to t
// instead of 0 * inf, and so that d of the largest logit is never far from 0
// (the rounding of r is at most 2^-24 of 2^15 log2(e)).  A token whose largest
// logit is not within +-2^14 (every entry masked, or enormous logits) is done
// again in plain fp32 differences x - M ("wide"), which hold for any finite
// logits.  NaN survives every maximum (max.NaN), so a NaN logit makes the
// token's results NaN.
#include "launch.cuh"
#include "tma.cuh"
#include "tokens.cuh"
#include "trace.h"

#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace cg = cooperative_groups;

namespace darb {

int sm_count();

namespace {

constexpr float kMasked = -0x1p15f;   // logits are read as at least this (exact in bf16)
constexpr float kWide = 0x1p14f;      // the largest logit of a token that takes the fast path, in magnitude
constexpr int kMaxTop = DARB_MAX_TOP;
constexpr int kCandidates = 256;    // candidates for the k largest that are gathered at once (k = 32: some 130)
constexpr int kMaxSplit = 8;        // CTAs that share a token
static_assert(kCandidates >= kMaxSplit * kMaxTop, "what a cluster hands on");

struct ScoreArgs {
    const void *x;
    int64_t ld;
    int64_t tokens;
    int32_t vocab;
    int32_t k;
    const int64_t *targets;   // or null
    float *logprob, *entropy, *lse, *top_logprob;   // or null
    int32_t *top_index;
};

// A partial result over some of a token's logits: its largest (clamped) logit,
// and the sums relative to r = reference(m).
struct Part {
    float m, s, t;
};
__device__ __forceinline__ Part empty_part() { return {kMasked, 0.0f, 0.0f}; }
__device__ __forceinline__ float reference(float m) { return __fmul_rn(m, kLog2e); }
__device__ __forceinline__ Part rescaled(const Part &p, float m) {
    const float d = __fsub_rn(reference(p.m), reference(m));
    const float f = exp2_fast(d);
    return {m, f * p.s, f * (p.t + p.s * d)};
}
__device__ __forceinline__ Part warp_join(Part p) {
    float m = p.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    p = rescaled(p, m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        p.s += __shfl_xor_sync(0xFFFFFFFFu, p.s, o);
        p.t += __shfl_xor_sync(0xFFFFFFFFu, p.t, o);
    }
    return p;
}

// A thread's running sums, and one block of N of its logits (clamped, the
// largest of them `top`) added to them: the block is summed by itself first, so
// that no addition chain is longer than a block plus the number of blocks.
struct Running {
    float m, r;
    Pair s, t;
};
__device__ __forceinline__ Running no_sums() { return {kMasked, reference(kMasked), both(0.0f), both(0.0f)}; }
__device__ __forceinline__ void rebase(Running &a, float top) {
    a.m = max_nan(a.m, top);
    const float r = reference(a.m), d = __fsub_rn(a.r, r), f = exp2_fast(d);
    a.t = mul2(both(f), fma2(a.s, both(d), a.t));
    a.s = mul2(both(f), a.s);
    a.r = r;
}
__device__ __forceinline__ void add_pair(Pair x, float r, Pair &s, Pair &t) {
    const Pair d = fma2(x, both(kLog2e), both(-r));
    const Pair e = pair(exp2_fast(low(d)), exp2_fast(high(d)));
    s = add2(s, e);
    t = fma2(e, d, t);
}

// Logits in order of value: larger logits have larger keys, NaN the largest,
// +0 and -0 one key.  Below it the index, inverted: ties go to the lowest.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x);
    if (x != x) return 0xFFFFFFFFu;
    if (x == 0.0f) return 0x80000000u;
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    if (o == 0xFFFFFFFFu) return __uint_as_float(0x7FC00000u);
    return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint64_t key_of(float x, int32_t index) {
    return (uint64_t(order_of(x)) << 32) | uint32_t(0xFFFFFFFFu - uint32_t(index));
}
__device__ __forceinline__ int32_t index_of(uint64_t key) { return int32_t(0xFFFFFFFFu - uint32_t(key)); }

// What every output of a token is made from.
struct Token {
    float r;       // log2 units: the reference, (finite) M log2(e)
    float m;       // M itself
    float log2s;   // log2 s
    float t_s;     // t / s
    bool wide, empty;
    // (the roundings of a token with one entry can leave its log probability above and its
    // entropy below 0; NaN stays)
    __device__ float logprob(float x) const {
        if (empty) return -INFINITY;
        const float l = (wide ? (x - m) * kLog2e - log2s : fmaf(x, kLog2e, -r) - log2s) * kLn2;
        return l > 0.0f ? 0.0f : l;
    }
    __device__ float entropy() const {
        const float h = empty ? 0.0f : (log2s - t_s) * kLn2;
        return h < 0.0f ? 0.0f : h;
    }
    // r is m log2(e) but for its rounding, which belongs to log2s: one rounding at the size of m is left
    __device__ float lse() const { return empty ? -INFINITY : fmaf(wide ? log2s : log2s + fmaf(-m, kLog2e, r), kLn2, m); }
};
__device__ __forceinline__ Token token_of(const Part &p) {
    return {reference(p.m), p.m, log2f(p.s), p.t / p.s, false, false};
}
// Whether a token's fast partial result does not stand (a NaN one does).
__device__ __forceinline__ bool is_wide(float m) { return m < -kWide || m > kWide; }

__device__ __forceinline__ float target_logprob(const Token &tok, int64_t target, int32_t vocab, float x) {
    if (target < 0) return 0.0f;
    if (target >= vocab) return __uint_as_float(0x7FC00000u);
    return tok.logprob(x);
}

// ---- a CTA's slow paths over the logits base[i * stride], i in [i0, i1) ----

// Sum, maximum or maximum with NaN over the CTA; every thread gets it.  `buf`:
// 33 floats of shared memory.
template <typename Op>
__device__ float cta_reduce(float v, float *buf, Op op) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    __syncthreads();   // the buffer may still be read by an earlier call
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
        float a = buf[0];
        for (unsigned w = 1; w < blockDim.x / 32; ++w) a = op(a, buf[w]);
        buf[32] = a;
    }
    __syncthreads();
    return buf[32];
}

// A token in plain differences from its maximum, for logits of any size.
template <typename T>
__device__ Token wide_token(const T *base, int64_t stride, int32_t n, float *buf) {
    float m = -INFINITY;
    for (int32_t i = threadIdx.x; i < n; i += blockDim.x) m = max_nan(m, widen(base[int64_t(i) * stride]));
    m = cta_reduce(m, buf, [](float a, float b) { return max_nan(a, b); });
    if (m == -INFINITY) return {0.0f, m, 0.0f, 0.0f, true, true};
    float s = 0.0f, t = 0.0f;
    for (int32_t i = threadIdx.x; i < n; i += blockDim.x) {
        const float d = widen(base[int64_t(i) * stride]) - m;   // NaN for m = inf and for NaN logits
        const float l = max_nan(d * kLog2e, -1e3f);
        const float e = exp2_fast(l);
        s += e;
        t += e * l;
    }
    s = cta_reduce(s, buf, [](float a, float b) { return a + b; });
    t = cta_reduce(t, buf, [](float a, float b) { return a + b; });
    return {0.0f, m, log2f(s), t / s, true, false};
}

// The min(k, i1 - i0) largest keys, in any order, to sel[0 .. kMaxTop) (0 where
// there is none), for any logits: the k-th largest key is found 8 bits at a
// time.  hist: 256 words, ctl: 4 words of shared memory.
template <typename T>
__device__ void select_any(const T *base, int64_t stride, int32_t i0, int32_t i1, int k, uint64_t *sel, uint32_t *hist,
                           uint32_t *ctl) {
    const int want = min(k, max(0, i1 - i0));
    __syncthreads();
    if (threadIdx.x < kMaxTop) sel[threadIdx.x] = 0;
    if (threadIdx.x == 0) ctl[0] = want, ctl[1] = 0, ctl[2] = 0;   // rank that is left, gathered, done
    uint64_t prefix = 0;
    int bits = 0;   // of the prefix
    if (want > 0) {
        while (bits < 64) {
            for (int i = threadIdx.x; i < 256; i += blockDim.x) hist[i] = 0;
            __syncthreads();
            const int shift = 64 - bits - 8;
            // a run of equal digits is added at once: masked entries share theirs
            uint32_t run_digit = 0, run = 0;
            for (int32_t i = i0 + int32_t(threadIdx.x); i < i1; i += blockDim.x) {
                const uint64_t key = key_of(widen(base[int64_t(i) * stride]), i);
                if (bits > 0 && (key >> (shift + 8)) != prefix) continue;
                const uint32_t d = uint32_t(key >> shift) & 255u;
                if (d == run_digit) {
                    ++run;
                } else {
                    if (run) atomicAdd(&hist[run_digit], run);
                    run_digit = d;
                    run = 1;
                }
            }
            if (run) atomicAdd(&hist[run_digit], run);
            __syncthreads();
            if (threadIdx.x == 0) {
                uint32_t left = ctl[0];
                int d = 255;
                while (d > 0 && hist[d] < left) left -= hist[d--];
                ctl[0] = left;
                ctl[3] = uint32_t(d);
                ctl[2] = hist[d] == left;   // the whole digit is taken
            }
            __syncthreads();
            prefix = (prefix << 8) | ctl[3];
            bits += 8;
            if (ctl[2]) break;
            __syncthreads();
        }
        for (int32_t i = i0 + int32_t(threadIdx.x); i < i1; i += blockDim.x) {
            const uint64_t key = key_of(widen(base[int64_t(i) * stride]), i);
            if ((key >> (64 - bits)) >= prefix) {
                const uint32_t p = atomicAdd(&ctl[1], 1u);
                if (p < kMaxTop) sel[p] = key;
            }
        }
    }
    __syncthreads();
}

// The k largest of n keys in order, to sorted[0 .. kMaxTop) (the keys all
// different, but for zeros, which are none; zeros where there are fewer), by one
// warp.  Up to 64 keys: every lane counts the keys above its own.  More: the
// largest of all lanes' largest, k times, by two 32-bit maxima over the warp.
__device__ __forceinline__ void warp_sort(const uint64_t *keys, int n, int k, uint64_t *sorted) {
    const int lane = threadIdx.x & 31;
    if (n <= 64) {
        const uint64_t lo = lane < n ? keys[lane] : 0, hi = lane + 32 < n ? keys[lane + 32] : 0;
        int above_lo = 0, above_hi = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) {
            const uint64_t o = keys[j];
            above_lo += o > lo;
            above_hi += o > hi;
        }
        sorted[lane] = 0;
        __syncwarp();
        if (lo != 0 && above_lo < k) sorted[above_lo] = lo;
        if (hi != 0 && above_hi < k) sorted[above_hi] = hi;
    } else {
        uint64_t best = 0, mine = 0;
        for (int i = lane; i < n; i += 32) best = keys[i] > best ? keys[i] : best;
        for (int j = 0; j < k; ++j) {
            const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, uint32_t(best >> 32));
            const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, uint32_t(best >> 32) == hi ? uint32_t(best) : 0u);
            const uint64_t top = (uint64_t(hi) << 32) | lo;
            if (lane == j) mine = top;
            if (best == top) {
                best = 0;
                for (int i = lane; i < n; i += 32) best = keys[i] < top && keys[i] > best ? keys[i] : best;
            }
        }
        sorted[lane] = mine;
    }
    __syncwarp();
}

// The k-th largest of 32 values, one a lane (equal values rank by lane); NaN if
// one of them is.
__device__ __forceinline__ float kth_of_warp(float v, int k) {
    const int lane = threadIdx.x & 31;
    int above = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const float o = __shfl_sync(0xFFFFFFFFu, v, j);
        above += o > v || (o == v && j < lane);
    }
    const unsigned at = __ballot_sync(0xFFFFFFFFu, above == k - 1);
    const float kth = __shfl_sync(0xFFFFFFFFu, v, at ? __ffs(at) - 1 : 0);
    return __any_sync(0xFFFFFFFFu, v != v) ? __uint_as_float(0x7FC00000u) : kth;
}

// ---- token rows ----

// The logits of a block of granules, clamped, and their maximum.
template <int N>
__device__ __forceinline__ void clamp_block(uint4 (&q)[N], float &m, float) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
        uint32_t *w = reinterpret_cast<uint32_t *>(&q[u]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float c = max_nan(__uint_as_float(w[i]), kMasked);
            m = max_nan(m, c);
            w[i] = __float_as_uint(c);
        }
    }
}
template <int N>
__device__ __forceinline__ void clamp_block(uint4 (&q)[N], float &m, __nv_bfloat16) {
    const __nv_bfloat162 lowest = __float2bfloat162_rn(kMasked);
    __nv_bfloat162 mm = lowest;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        __nv_bfloat162 *w = reinterpret_cast<__nv_bfloat162 *>(&q[u]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = __hmax2_nan(w[i], lowest);
            mm = __hmax2_nan(mm, w[i]);
        }
    }
    m = max_nan(m, max_nan(__low2float(mm), __high2float(mm)));
}

// The blocks that a thread's share of the logits is cut into: `rounds` rounds of
// U granules, `per_slot` of them sharing a slot of the table of maxima.
struct Blocks {
    int32_t slots, per_slot;
};
inline Blocks blocks_of(int64_t rounds, int most) {
    const int64_t per = std::max<int64_t>(1, (rounds + most - 1) / most);
    return {int32_t((rounds + per - 1) / per), int32_t(per)};
}
constexpr int kRowSlots = 32;   // of the table of maxima, at most

// One read of the logits; bound by memory, and with alternatives by the barriers
// of the joins.  A CTA, or a cluster where rows are long and tokens few, takes a
// token.  The main loop keeps one maximum, one reference and two pairs of sums a
// thread: a block of U granules is clamped and its maximum taken (in bf16 two
// logits an instruction), the sums are moved to the new reference once a block,
// then a logit costs half an FMA, an exponential and two halves of an addition
// and an FMA.  The k largest come from a table of the blocks' maxima: the few
// blocks that reach the bar are read again.
//   4096 x 32000 bf16: 41.5 us (6.3 TB/s), k = 5 49, k = 20 53
//   1023 x 128001 fp32: 78 us (6.7 TB/s), k = 20 86-88
//   1 x 32000 bf16: 3.4 us, k = 8 5.6
constexpr int kItems = 256;   // blocks that may hold one of the k largest, at most

template <typename T, int THREADS, int U, bool CLUSTER>
__global__ void __launch_bounds__(THREADS) score_rows_kernel(const ScoreArgs a, const Blocks blocks) {
    constexpr int V = kPerGranule<T>;
    constexpr int W = THREADS / 32;
    extern __shared__ float block_max[];   // [slots][THREADS], for k > 0
    __shared__ Part warp_part[W], cta_part, token_part;
    __shared__ float thread_max[THREADS], s_top[32], s_bar;
    __shared__ uint64_t cand[kCandidates], sel[kMaxTop], sorted[kMaxTop];
    __shared__ uint32_t items[kItems], hist[256], ctl[4], nitems, ncand;
    __shared__ float buf[33];
    pdl_wait_previous();
    pdl_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const int split = CLUSTER ? int(cluster.num_blocks()) : 1, rank = CLUSTER ? int(cluster.block_rank()) : 0;
    const int64_t token = blockIdx.x / split;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const T *row = static_cast<const T *>(a.x) + token * a.ld;
    const int head = row_head<T>(row);
    const int32_t n = a.vocab, granules = int32_t(row_granules<T>(head, n)), k = a.k;
    const int32_t g0 = int32_t(int64_t(granules) * rank / split), g1 = int32_t(int64_t(granules) * (rank + 1) / split);
    // a round's granules: at once where all of them lie in the row and in this CTA's share
    const int32_t whole0 = head > 0 ? 1 : 0, whole1 = (head + n) / V;
    const uint4 *aligned = reinterpret_cast<const uint4 *>(row - head);
    const auto fetch = [&](uint4 (&q)[U], int32_t g) {
        if (g >= whole0 && g + THREADS * U <= min(g1, whole1)) {
#pragma unroll
            for (int u = 0; u < U; ++u) q[u] = aligned[g + u * THREADS + tid];
            return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t gu = g + u * THREADS + tid;
            q[u] = load_granule(row, gu < g1 ? int64_t(gu) * V - head : int64_t(n), n, -INFINITY);
        }
    };
    uint4 next[U];
    fetch(next, g0);
    int64_t target = -1;
    float target_x = 0.0f;
    if (tid == 0) {
        nitems = ncand = 0;
        if (rank == 0 && a.targets != nullptr) {
            target = a.targets[token];
            if (target >= 0 && target < n) target_x = widen(row[target]);
        }
    }

    Running sum = no_sums();
    int slot = 0, in_slot = 0;
    float slot_max = kMasked;
    for (int32_t g = g0; g < g1; g += THREADS * U) {
        uint4 q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) q[u] = next[u];
        if (g + THREADS * U < g1) fetch(next, g + THREADS * U);
        float top = kMasked;
        clamp_block(q, top, T());
        if (k > 0) {
            slot_max = max_nan(slot_max, top);
            if (++in_slot == blocks.per_slot) {
                block_max[slot++ * THREADS + tid] = slot_max;
                slot_max = kMasked;
                in_slot = 0;
            }
        }
        rebase(sum, top);
        Pair s2 = both(0.0f), t2 = both(0.0f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Pair v[V / 2];
            unpack(q[u], v);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) add_pair(v[i], sum.r, s2, t2);
        }
        sum.s = add2(sum.s, s2);
        sum.t = add2(sum.t, t2);
    }
    if (k > 0) {
        if (in_slot > 0) block_max[slot++ * THREADS + tid] = slot_max;
        thread_max[tid] = sum.m;
    }
    const Part mine = warp_join({sum.m, across(sum.s), across(sum.t)});
    if (lane == 0) warp_part[warp] = mine;
    __syncthreads();
    // Warp 0 joins the sums; warp 1 finds the bar: the k-th largest of 32 maxima
    // over disjoint sets of the token's logits is at most the k-th largest logit, so
    // only blocks that reach it can hold one of the k largest.
    Part all = empty_part();
    float g = kMasked;
    if (warp == 0) {
        all = warp_join(lane < W ? warp_part[lane] : empty_part());
        if (lane == 0) (CLUSTER ? cta_part : token_part) = all;
    } else if (warp == 1 && k > 0) {
        g = thread_max[lane];
#pragma unroll
        for (int w = 1; w < W; ++w) g = max_nan(g, thread_max[w * 32 + lane]);
        if (CLUSTER) s_top[lane] = g;
    }
    if (CLUSTER) {
        cluster.sync();
        if (warp == 0 && rank == 0) {
            all = warp_join(lane < split ? *cluster.map_shared_rank(&cta_part, lane) : empty_part());
            if (lane == 0) token_part = all;
        } else if (warp == 1 && k > 0) {
#pragma unroll
            for (int q = 0; q < kMaxSplit; ++q)
                if (q < split) g = max_nan(g, cluster.map_shared_rank(s_top, q)[lane]);
        }
    }
    if (warp == 1 && k > 0) {
        const float bar = kth_of_warp(g, k);
        if (lane == 0) s_bar = bar > kMasked ? bar : __uint_as_float(0x7FC00000u);
    }
    __syncthreads();
    if (k > 0) {
        const float bar = s_bar;   // NaN: the maxima say nothing
        if (sum.m >= bar)
            for (int i = 0; i < slot; ++i)
                if (block_max[i * THREADS + tid] >= bar) {
                    const uint32_t p = atomicAdd(&nitems, 1u);
                    if (p < kItems) items[p] = uint32_t(i * THREADS + tid);
                }
        __syncthreads();
        const int listed = int(nitems);
        if (listed <= kItems) {
            // the granules of the listed blocks, all at once
            const int per = U * blocks.per_slot;
            for (int i = tid; i < listed * per; i += THREADS) {
                const int32_t item = int32_t(items[i / per]), j = i % per;
                const int32_t gi = g0 + ((item / THREADS) * blocks.per_slot + j / U) * (THREADS * U) + (j % U) * THREADS + item % THREADS;
                if (gi >= g1) continue;
                float v[V];
                const int64_t j0 = int64_t(gi) * V - head;
                unpack(load_granule(row, j0, n, -INFINITY), v);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (v[e] >= bar) {
                        const uint32_t p = atomicAdd(&ncand, 1u);
                        if (p < kCandidates) cand[p] = key_of(v[e], int32_t(j0 + e));
                    }
            }
        }
        __syncthreads();
        int found = int(ncand);
        if (!(bar == bar) || listed > kItems || found > kCandidates) {
            const int32_t i0 = max(0, g0 * V - head), i1 = min(n, g1 * V - head);
            select_any(row, 1, i0, i1, k, sel, hist, ctl);
            if (tid < kMaxTop) cand[tid] = sel[tid];
            found = kMaxTop;
            if (tid == 0) ncand = found;
            __syncthreads();
        }
        if (CLUSTER) {
            // a CTA hands on at most kMaxTop candidates
            if (warp == 0 && found > kMaxTop) {
                warp_sort(cand, found, k, sorted);
                cand[lane] = sorted[lane];
                if (lane == 0) ncand = kMaxTop;
            }
            cluster.sync();
            uint64_t keys[kMaxSplit];
            uint32_t from[kMaxSplit], total = 0;
            if (rank == 0 && warp == 0) {
                uint32_t n_q[kMaxSplit];
#pragma unroll
                for (int q = 0; q < kMaxSplit; ++q) {
                    n_q[q] = q < split ? *cluster.map_shared_rank(&ncand, q) : 0;
                    keys[q] = q < split ? cluster.map_shared_rank(cand, q)[lane] : 0;
                }
#pragma unroll
                for (int q = 0; q < kMaxSplit; ++q) {
                    from[q] = uint32_t(lane) < n_q[q] ? total + lane : 0xFFFFFFFFu;
                    total += n_q[q];
                }
            }
            cluster.sync();   // the other CTAs may leave, and the lists be written
            if (rank == 0 && warp == 0) {
#pragma unroll
                for (int q = 0; q < kMaxSplit; ++q)
                    if (from[q] != 0xFFFFFFFFu) cand[from[q]] = keys[q];
                __syncwarp();
                found = int(total);
            }
        }
        if (warp == 0 && rank == 0) warp_sort(cand, found, k, sorted);
    } else if (CLUSTER) {
        cluster.sync();   // the sums have been read
    }
    if (rank != 0) return;
    const Part whole = token_part;
    Token tok;
    if (is_wide(whole.m)) tok = wide_token(row, 1, n, buf);   // the same for the CTA
    else if (warp > 0) return;
    else tok = token_of(whole);
    if (tid == 0) {
        if (a.logprob) a.logprob[token] = target_logprob(tok, target, n, target_x);
        if (a.entropy) a.entropy[token] = tok.entropy();
        if (a.lse) a.lse[token] = tok.lse();
    }
    if (tid < k) {
        const uint64_t key = sorted[tid];
        a.top_logprob[token * k + tid] = tok.logprob(value_of(uint32_t(key >> 32)));
        a.top_index[token * k + tid] = index_of(key);
    }
}

// ---- token columns ----

// A tile of CT columns; thread = (slot, column), the slots of a CTA share the
// rows of its part of the vocabulary, so that a warp reads whole runs of a row.  The
// same sums as above, one logit a load: bound by instructions and by the loads
// that one CTA an SM has in flight, not by memory.  The bar and the lists of
// candidates are the columns' own.
//   1011 x 25568: fp32 25.5 us (4.1 TB/s), bf16 25, k = 20 39 and 38
//   20 x 10000 fp32: 5.0 us, k = 5 8.4
constexpr int kColThreads = 1024;
constexpr int kColCandidates = 256;   // a column (k = 32: some 130)
static_assert(kColCandidates >= kMaxSplit * kMaxTop, "as above");
constexpr int kColUnroll = 8;
constexpr int kColSlots = 16;         // of the table of maxima, at most
static_assert(kColSlots * kColThreads <= 65536, "a block's place fits an item");
constexpr int kColItems = 8192;       // blocks that may hold one of the k largest

template <int CT>
struct ColShared {
    static constexpr int kSlots = kColThreads / CT;
    Part part[kSlots][CT + 1];
    Part col[CT];
    float top[CT][32];          // maxima of 32 disjoint sets of a column's logits
    float bar[CT];
    uint32_t ncand[CT];
    uint64_t cand[CT][kColCandidates];
    uint64_t sorted[CT][kMaxTop];
    uint64_t sel[kMaxTop];
    uint32_t hist[256], ctl[4];
    float buf[33];
    Token tok[CT];
    uint32_t nitems;
    uint16_t items[kColItems];
    __nv_bfloat16 block_max[kColSlots][kColThreads];   // rounded up: a bound of the block
};

template <typename T, int CT>
__global__ void __launch_bounds__(kColThreads) score_columns_kernel(const ScoreArgs a, const Blocks blocks) {
    constexpr int SLOTS = kColThreads / CT, U = kColUnroll;
    extern __shared__ __align__(16) unsigned char smem[];
    ColShared<CT> &sh = *reinterpret_cast<ColShared<CT> *>(smem);
    pdl_wait_previous();
    pdl_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const int split = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const int64_t c0 = int64_t(blockIdx.x / split) * CT;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int col = tid % CT, slot = tid / CT;
    const int64_t token = c0 + col;
    const bool in = token < a.tokens;
    // this thread's column (past the last token: the last one, for nobody)
    const T *base = static_cast<const T *>(a.x) + (in ? token : a.tokens - 1);
    const int32_t n = a.vocab, k = a.k;
    const int32_t v0 = int32_t(int64_t(n) * rank / split), v1 = int32_t(int64_t(n) * (rank + 1) / split);
    const int64_t stride = SLOTS * a.ld;
    const T *at = base + int64_t(v0 + slot) * a.ld;   // of the next round
    const auto fetch = [&](float (&x)[U], int32_t v) {
        const T *p = at;
        if (v + SLOTS * U <= v1) {
#pragma unroll
            for (int u = 0; u < U; ++u, p += stride) x[u] = widen(*p);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u, p += stride) x[u] = v + slot + u * SLOTS < v1 ? widen(*p) : -INFINITY;
        }
        at += U * stride;
    };
    float next[U];
    fetch(next, v0);
    if (tid < CT) sh.ncand[tid] = 0;
    if (tid == 0) sh.nitems = 0;

    Running sum = no_sums();
    int block = 0, in_block = 0;
    float slot_max = kMasked;
    for (int32_t v = v0; v < v1; v += SLOTS * U) {
        float x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = max_nan(next[u], kMasked);
        if (v + SLOTS * U < v1) fetch(next, v + SLOTS * U);
        float top = x[0];
#pragma unroll
        for (int u = 1; u < U; ++u) top = max_nan(top, x[u]);
        if (k > 0) {
            slot_max = max_nan(slot_max, top);
            if (++in_block == blocks.per_slot) {
                sh.block_max[block++][tid] = __float2bfloat16_ru(slot_max);
                slot_max = kMasked;
                in_block = 0;
            }
        }
        rebase(sum, top);
        Pair s2 = both(0.0f), t2 = both(0.0f);
#pragma unroll
        for (int u = 0; u < U; u += 2) add_pair(pair(x[u], x[u + 1]), sum.r, s2, t2);
        sum.s = add2(sum.s, s2);
        sum.t = add2(sum.t, t2);
    }
    if (in_block > 0) sh.block_max[block++][tid] = __float2bfloat16_ru(slot_max);
    sh.part[slot][col] = {sum.m, across(sum.s), across(sum.t)};
    __syncthreads();
    // warp c joins column c (c < CT <= 32 warps)
    if (warp < CT) {
        Part p = empty_part();
        float g = kMasked;
        for (int s = lane; s < SLOTS; s += 32) {
            const Part q = sh.part[s][warp];
            g = max_nan(g, q.m);
            const float mm = max_nan(p.m, q.m);
            const Part x = rescaled(p, mm), y = rescaled(q, mm);
            p = {mm, x.s + y.s, x.t + y.t};
        }
        p = warp_join(p);
        if (lane == 0) sh.col[warp] = p;
        sh.top[warp][lane] = g;
    }
    // The bar of a column is that of all CTAs of the cluster: few logits reach it.
    if (split > 1) cluster.sync();
    else __syncthreads();
    Part whole = empty_part();   // of the column, in rank 0's warp of it
    if (warp < CT) {
        if (rank == 0 && lane < split) whole = cluster.map_shared_rank(&sh, lane)->col[warp];
        if (k > 0) {
            float g = kMasked;
#pragma unroll
            for (int q = 0; q < kMaxSplit; ++q)
                if (q < split) g = max_nan(g, cluster.map_shared_rank(&sh, q)->top[warp][lane]);
            const float bar = kth_of_warp(g, k);
            if (lane == 0) sh.bar[warp] = bar > kMasked ? bar : __uint_as_float(0x7FC00000u);
        }
    }
    if (k > 0) {
        __syncthreads();
        const float bar = sh.bar[col];   // NaN: the maxima say nothing
        if (in && sum.m >= bar)
            for (int i = 0; i < block; ++i)
                if (widen(sh.block_max[i][tid]) >= bar) {
                    const uint32_t p = atomicAdd(&sh.nitems, 1u);
                    if (p < kColItems) sh.items[p] = uint16_t(i * kColThreads + tid);
                }
        __syncthreads();
        const bool listed = sh.nitems <= kColItems;
        if (listed) {
            // (several loads at once: they are scattered, and wait for memory one by one)
            const int per = U * blocks.per_slot, total = int(sh.nitems) * per;
            constexpr int B = 4;
            for (int i0 = tid; i0 < total; i0 += B * kColThreads) {
                float x[B];
                int32_t v[B], c[B];
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    const int i = i0 + b * kColThreads, at = i < total ? i / per : 0, j = i - at * per;
                    const int32_t item = int32_t(sh.items[at]), t = item % kColThreads;
                    c[b] = t % CT;
                    v[b] = v0 + ((item / kColThreads) * blocks.per_slot + j / U) * (SLOTS * U) + (j % U) * SLOTS + t / CT;
                    if (i >= total) v[b] = v1;
                    x[b] = v[b] < v1 ? widen(static_cast<const T *>(a.x)[int64_t(v[b]) * a.ld + c0 + c[b]]) : -INFINITY;
                }
#pragma unroll
                for (int b = 0; b < B; ++b)
                    if (v[b] < v1 && x[b] >= sh.bar[c[b]]) {
                        const uint32_t p = atomicAdd(&sh.ncand[c[b]], 1u);
                        if (p < kColCandidates) sh.cand[c[b]][p] = key_of(x[b], v[b]);
                    }
            }
        }
        __syncthreads();
        const auto short_way = [&](int c) { return listed && sh.bar[c] == sh.bar[c] && sh.ncand[c] <= kColCandidates; };
        if (__syncthreads_or(tid < CT && in && !short_way(tid)))
            for (int c = 0; c < CT && c0 + c < a.tokens; ++c) {
                if (short_way(c)) continue;
                select_any(static_cast<const T *>(a.x) + c0 + c, a.ld, v0, v1, k, sh.sel, sh.hist, sh.ctl);
                if (tid < kMaxTop) sh.cand[c][tid] = sh.sel[tid];
                if (tid == 0) sh.ncand[c] = kMaxTop;   // all have asked: select_any has barriers
            }
        __syncthreads();
        // a CTA of a cluster hands on at most kMaxTop candidates of a column
        if (warp < CT && (split == 1 || sh.ncand[warp] > kMaxTop)) {
            warp_sort(sh.cand[warp], int(sh.ncand[warp]), k, sh.sorted[warp]);
            if (split > 1) {
                sh.cand[warp][lane] = sh.sorted[warp][lane];
                if (lane == 0) sh.ncand[warp] = kMaxTop;
            }
        }
    }
    if (split > 1) {
        cluster.sync();
        uint64_t keys[kMaxSplit];
        uint32_t from[kMaxSplit], total = 0;
        if (rank == 0 && warp < CT && k > 0) {
            uint32_t n_q[kMaxSplit];
#pragma unroll
            for (int q = 0; q < kMaxSplit; ++q) {
                n_q[q] = q < split ? cluster.map_shared_rank(&sh, q)->ncand[warp] : 0;
                keys[q] = q < split ? cluster.map_shared_rank(&sh, q)->cand[warp][lane] : 0;
            }
#pragma unroll
            for (int q = 0; q < kMaxSplit; ++q) {
                from[q] = uint32_t(lane) < n_q[q] ? total + lane : 0xFFFFFFFFu;
                total += n_q[q];
            }
        }
        cluster.sync();   // the other CTAs may leave, and the lists be written
        if (rank != 0) return;
        if (warp < CT) {
            whole = warp_join(whole);
            if (lane == 0) sh.col[warp] = whole;
            if (k > 0) {
#pragma unroll
                for (int q = 0; q < kMaxSplit; ++q)
                    if (from[q] != 0xFFFFFFFFu) sh.cand[warp][from[q]] = keys[q];
                __syncwarp();
                warp_sort(sh.cand[warp], int(total), k, sh.sorted[warp]);
            }
        }
    }
    __syncthreads();
    const bool wide = tid < CT && in && is_wide(sh.col[tid].m);
    if (tid < CT && in && !wide) sh.tok[tid] = token_of(sh.col[tid]);
    if (__syncthreads_or(wide))
        for (int c = 0; c < CT && c0 + c < a.tokens; ++c) {
            if (!is_wide(sh.col[c].m)) continue;
            const Token tok = wide_token(static_cast<const T *>(a.x) + c0 + c, a.ld, n, sh.buf);
            if (tid == c) sh.tok[c] = tok;
        }
    __syncthreads();
    if (tid < CT && in) {   // slot 0: col == tid
        const Token tok = sh.tok[tid];
        if (a.logprob) {
            const int64_t target = a.targets[token];
            const float x = target >= 0 && target < n ? widen(base[target * a.ld]) : 0.0f;
            a.logprob[token] = target_logprob(tok, target, n, x);
        }
        if (a.entropy) a.entropy[token] = tok.entropy();
        if (a.lse) a.lse[token] = tok.lse();
    }
    for (int i = tid; i < CT * k; i += kColThreads) {
        const int c = i / k, j = i % k;
        if (c0 + c >= a.tokens) break;
        const uint64_t key = sh.sorted[c][j];
        a.top_logprob[(c0 + c) * k + j] = sh.tok[c].logprob(value_of(uint32_t(key >> 32)));
        a.top_index[(c0 + c) * k + j] = index_of(key);
    }
}

template <typename T, int THREADS, bool CLUSTER>
cudaError_t launch_score_rows(const ScoreArgs &a, cudaStream_t stream, int split) {
    constexpr int U = 4;
    const auto kernel = score_rows_kernel<T, THREADS, U, CLUSTER>;
    const int64_t granules = row_granules<T>(kPerGranule<T> - 1, a.vocab) / split + 1;   // of a CTA, at most
    const Blocks blocks = blocks_of((granules + THREADS * U - 1) / (THREADS * U), kRowSlots);
    const size_t smem = a.k > 0 ? size_t(blocks.slots) * THREADS * 4 : 0;
    const cudaError_t e = allow_smem(kernel, smem + 8 * 1024);   // (and the kernel's own)
    if (e != cudaSuccess) return e;
    return launch_ex(kernel, dim3(unsigned(a.tokens * split)), dim3(THREADS), smem, stream, unsigned(split), true, a, blocks);
}

template <typename T>
cudaError_t launch_score_rows(const ScoreArgs &a, cudaStream_t stream) {
    const int64_t sms = sm_count(), granules = row_granules<T>(0, a.vocab);
    // A cluster where it saves more reading than its exchanges cost (k = 5: one token of
    // 32000 bf16 alone 5.5 us, in a cluster 6.7; of 128000 10.3 and 7.0), while there are SMs
    // without a CTA, or with one that has much to read (130 x 128000 fp32: 2 a token 19.2 us, 4 16.5).
    int split = 1;
    if (granules > (a.k > 0 ? 14000 : 6000))
        while (split < kMaxSplit && (a.tokens * split < sms || (a.tokens * split < 2 * sms && granules / split > 8192))) split *= 2;
    if (split > 1) return launch_score_rows<T, 256, true>(a, stream, split);
    // Fewer threads a token leave less waiting for the joins of its sums, and more tokens
    // at a time on an SM; too few, and the loads in flight are too few.  Rows of one round
    // of 64 threads (8000 x 1000 bf16: 12.1 us, with 128 threads 21.6), or of some rounds
    // with many tokens (8000 x 5000 bf16 19.7, with 128 28.2; 1000 x 10000 fp32 10.4, with 128 8.9):
    if (granules <= 256 || (granules > 512 && granules <= 2048 && a.tokens >= 8 * sms))
        return launch_score_rows<T, 64, false>(a, stream, 1);
    // of up to 128 KB with 128 (4096 x 32000 bf16: 52 us, with 256 63; 400 x 11201 fp32 4.1 and
    // 4.8; but 600 x 32000 fp32 16.0 and 13.8), longer ones with 256 (1023 x 128001 fp32: 88, with 128 137).
    if (granules <= 512 || (granules <= 2048 && a.tokens >= sms) || (granules <= 4096 && a.tokens >= 2 * sms) ||
        (granules <= 8192 && a.tokens >= 4 * sms))
        return launch_score_rows<T, 128, false>(a, stream, 1);
    return launch_score_rows<T, 256, false>(a, stream, 1);
}

template <typename T, int CT>
cudaError_t launch_score_columns_ct(const ScoreArgs &a, cudaStream_t stream) {
    const int64_t tiles = (a.tokens + CT - 1) / CT;
    const size_t smem = sizeof(ColShared<CT>);
    const cudaError_t e = allow_smem(score_columns_kernel<T, CT>, smem);
    if (e != cudaSuccess) return e;
    // A CTA takes an SM.  The split with the least time: waves of clusters, each with a
    // fixed part (the joins, the candidates, in a cluster its exchanges) and its rows, in
    // units of a row of 32 columns (2.6 ns).  4000 x 3000 fp32, k = 5: 94 CTAs 20 us, in
    // clusters of 8 76; 37462 x 566: clusters of 4 30.5, of 8 (two waves) 35.
    const ClusterRoom room = cluster_room(score_columns_kernel<T, CT>, kColThreads, smem);
    static_assert(kMaxSplit == 8, "the clusters that room is known of");
    const auto cost = [&](int i) {
        const int64_t waves = (tiles + room.of[i] - 1) / room.of[i];
        const double fixed = a.k > 0 ? (i > 0 ? 3800 : 3000) : (i > 0 ? 1700 : 1150);
        return double(waves) * (fixed + double(a.vocab >> i) * CT / 32);
    };
    int best = 0;
    for (int i = 1; i < 4; ++i)
        if (a.vocab >> i >= 4 * kColThreads / CT && cost(i) < cost(best)) best = i;
    const int split = 1 << best;
    const int64_t rows = a.vocab / split + 1;   // of a CTA, at most
    constexpr int per_round = kColThreads / CT * kColUnroll;
    const Blocks blocks = blocks_of((rows + per_round - 1) / per_round, kColSlots);
    return launch_ex(score_columns_kernel<T, CT>, dim3(unsigned(tiles * split)), dim3(kColThreads), smem, stream,
                     unsigned(split), true, a, blocks);
}

template <typename T>
cudaError_t launch_score_columns(const ScoreArgs &a, cudaStream_t stream) {
    const int sms = sm_count();
    int ct = 32;
    // narrower tiles where the wider leave SMs idle, down to the 32 bytes that memory moves at a time
    while (ct > 4 && (a.tokens <= ct / 2 || (ct * int(sizeof(T)) > 32 && (a.tokens + ct / 2 - 1) / (ct / 2) * kMaxSplit <= sms)))
        ct /= 2;
    if (ct == 32) return launch_score_columns_ct<T, 32>(a, stream);
    if (ct == 16) return launch_score_columns_ct<T, 16>(a, stream);
    if (ct == 8) return launch_score_columns_ct<T, 8>(a, stream);
    return launch_score_columns_ct<T, 4>(a, stream);
}

// ---- the gradient ----
//
//   dx_v = a ([v = target] - p_v) - b p_v (log p_v + H),
// a and b the incoming gradients of log probability and entropy, p_v =
// exp(x_v - lse).  One pass: reads a logit, writes its gradient.

struct GradArgs {
    const void *x;
    void *dx;
    int64_t ld, ldd;
    int64_t tokens;
    int32_t vocab;
    const int64_t *targets;   // or null
    const float *lse, *entropy, *d_logprob, *d_entropy;   // or null, but lse
};

// lse is one fp32 number: half a unit in its last place is 2^-16 below 512, and
// p_v as far off (relative to itself; the logits of trained models are within
// +-100, where it is 2^-18).  Past 512 it is more, and from 2^24 on lse says nothing
// of log sum exp(x - M) any more.  The sums of such a token are taken again from its
// logits, as differences from their maximum.  A single CTA (of columns, a warp) does
// that and writes the whole token, as the gradient may take the logits' place: the
// others that share the token leave it alone.  Asking costs ordinary columns some 0.1 to
// 0.3 us, rows less.
constexpr float kWideLse = 512.0f;
__device__ __forceinline__ bool is_wide_lse(float lse) { return __builtin_expect(fabsf(lse) > kWideLse, false); }   // (of a token with an entry)

// What a token's gradient is made from:  dx_v = a [v = target] - p_v (b log p_v + c),
// c = a + b H.
struct GradToken {
    float lse, a, b, c;
    int32_t target;   // -1: none
};
__device__ __forceinline__ GradToken grad_token(const GradArgs &g, int64_t token) {
    GradToken t = {g.lse[token], 0.0f, 0.0f, 0.0f, -1};
    if (g.d_logprob != nullptr) {
        const int64_t target = g.targets[token];
        if (target >= g.vocab) {
            t.a = __uint_as_float(0x7FC00000u);
        } else if (target >= 0) {
            t.a = g.d_logprob[token];
            t.target = int32_t(target);
        }
    }
    t.c = t.a;
    if (g.d_entropy != nullptr) {
        t.b = g.d_entropy[token];
        t.c = fmaf(t.b, g.entropy[token], t.a);
    }
    if (t.lse == -INFINITY) t = {0.0f, 0.0f, 0.0f, t.a == t.a ? 0.0f : t.a, -1};   // no entry: no distribution, no gradient
    return t;
}

// A wide token: its maximum and log2 of its sum.
struct WideToken {
    float m, log2s;
    __device__ float grad(const GradToken &t, float x, int32_t v) const {
        const float d = max_nan((x - m) * kLog2e, kMasked) - log2s;
        const float g = m == -INFINITY ? 0.0f * t.c : exp2_fast(d) * fmaf(d * kLn2, -t.b, -t.c);
        return v == t.target ? g + t.a : g;
    }
};

// The gradient of one wide row by the CTA, a granule a thread.  (Not inlined: the
// kernels' registers are for their own way.)
template <typename T, typename Args>
__device__ __noinline__ void wide_row(Args a, int64_t token, const T *row, T *out) {
    constexpr int V = kPerGranule<T>;
    __shared__ float buf[33];
    const int head = row_head<T>(row);
    const int32_t n = a.vocab, granules = int32_t(row_granules<T>(head, n));
    const bool alike = row_head<T>(out) == head;
    const auto fetch = [&](int32_t g, float (&v)[V]) { unpack(load_granule(row, int64_t(g) * V - head, n, -INFINITY), v); };
    float m = -INFINITY, s = 0.0f;
    for (int32_t g = threadIdx.x; g < granules; g += blockDim.x) {
        float v[V];
        fetch(g, v);
#pragma unroll
        for (int e = 0; e < V; ++e) m = max_nan(m, v[e]);
    }
    m = cta_reduce(m, buf, [](float p, float q) { return max_nan(p, q); });
    for (int32_t g = threadIdx.x; g < granules; g += blockDim.x) {
        float v[V], part = 0.0f;
        fetch(g, v);
#pragma unroll
        for (int e = 0; e < V; ++e) part += exp2_fast(max_nan((v[e] - m) * kLog2e, kMasked));
        s += part;
    }
    s = cta_reduce(s, buf, [](float p, float q) { return p + q; });
    const GradToken t = grad_token(a, token);
    const WideToken k = {m, log2f(s)};
    for (int32_t g = threadIdx.x; g < granules; g += blockDim.x) {
        const int64_t j0 = int64_t(g) * V - head;
        float v[V];
        fetch(g, v);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = k.grad(t, v[e], int32_t(j0 + e));
        if (alike) {
            store_granule(out, j0, n, v);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (j0 + e >= 0 && j0 + e < n) out[j0 + e] = narrow<T>(v[e]);
        }
    }
}

// The wide tokens of a tile of 32 columns (PAIRS: and those that are read with one),
// by a CTA of its own: a warp takes 4 of them and 8 rows at a time.
constexpr int kGradThreads = 256;
template <typename T, bool PAIRS>
__device__ __noinline__ void wide_tile(const GradArgs a, int64_t tile) {
    static_assert(kGradThreads == 256, "8 warps of 4 tokens");
    const int lane = threadIdx.x & 31;
    const int64_t token = tile * 32 + (threadIdx.x >> 5) * 4 + (lane & 3);
    bool wide = token < a.tokens && is_wide_lse(a.lse[token]) && a.lse[token] != -INFINITY;
    if (PAIRS) {
        const int other = __shfl_xor_sync(0xFFFFFFFFu, int(wide), 1);   // (all lanes)
        wide = token < a.tokens && (wide || other != 0);
    }
    if (!__any_sync(0xFFFFFFFFu, wide)) return;
    const T *x = static_cast<const T *>(a.x) + token;
    T *dx = static_cast<T *>(a.dx) + token;
    const int32_t n = wide ? a.vocab : 0;   // (a lane without a wide token goes along)
    float m = -INFINITY, s = 0.0f;
#pragma unroll 8
    for (int32_t v = lane >> 2; v < n; v += 8) m = max_nan(m, widen(x[v * a.ld]));
#pragma unroll
    for (int o = 4; o < 32; o *= 2) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    for (int32_t v0 = lane >> 2; v0 < n; v0 += 8 * 256) {   // (256 terms first)
        float block = 0.0f;
        const int32_t end = min(n, v0 + 8 * 256);
#pragma unroll 8
        for (int32_t v = v0; v < end; v += 8) block += exp2_fast(max_nan((widen(x[v * a.ld]) - m) * kLog2e, kMasked));
        s += block;
    }
#pragma unroll
    for (int o = 4; o < 32; o *= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (!wide) return;
    const GradToken t = grad_token(a, token);
    const WideToken k = {m, log2f(s)};
    constexpr int U = 8;   // (rows in flight: the stores may be where the loads are)
    for (int32_t v0 = lane >> 2; v0 < n; v0 += 8 * U) {
        T q[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v0 + 8 * u < n) q[u] = x[(v0 + 8 * u) * a.ld];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v0 + 8 * u < n) dx[(v0 + 8 * u) * a.ldd] = narrow<T>(k.grad(t, widen(q[u]), v0 + 8 * u));
    }
}

// N logits of one token, from v0 on `step` apart, to their gradients.  A masked
// entry has p = 0; log p is held above -2^15 or so, so that it adds 0 there.
template <int N>
__device__ __forceinline__ void grad_of(const GradToken &t, Pair (&x)[N], int32_t v0, int32_t step) {
    const Pair lse = both(-t.lse), log2e = both(kLog2e), b = both(-t.b), c = both(-t.c);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        Pair l = add2(x[i], lse);
        l = pair(max_nan(low(l), kMasked), max_nan(high(l), kMasked));
        const Pair d = mul2(l, log2e);
        x[i] = mul2(pair(exp2_fast(low(d)), exp2_fast(high(d))), fma2(l, b, c));
    }
    const uint32_t at = uint32_t(t.target - v0);
    if (t.target >= 0 && at < uint32_t(2 * N * step)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = pair(low(x[i]) + (at == uint32_t(2 * i * step) ? t.a : 0.0f), high(x[i]) + (at == uint32_t((2 * i + 1) * step) ? t.a : 0.0f));
    }
}

constexpr int kGradUnroll = 4;

// Rows whose logits and gradients start alike past a 16-byte boundary: four
// granules a thread in flight.  Bound by memory: 4096 x 32000 bf16 with an entropy
// gradient 78 us (6.8 TB/s).
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) grad_rows_kernel(const __grid_constant__ GradArgs a, int32_t parts) {
    constexpr int V = kPerGranule<T>, U = kGradUnroll;
    pdl_wait_previous();
    pdl_launch_dependents();
    const int64_t token = blockIdx.x / parts;
    const int32_t part = int32_t(blockIdx.x % parts);
    const T *row = static_cast<const T *>(a.x) + token * a.ld;
    T *out = static_cast<T *>(a.dx) + token * a.ldd;
    const int head = row_head<T>(row);
    const int32_t n = a.vocab, granules = int32_t(row_granules<T>(head, n));
    const int32_t first = part * (THREADS * U), g0 = first + int32_t(threadIdx.x);
    // (plain loads: the gradient may take the logits' place)
    if (first >= (head > 0 ? 1 : 0) && first + THREADS * U <= (head + n) / V) {   // granules all in the row
        const uint4 *in = reinterpret_cast<const uint4 *>(row - head) + g0;
        uint4 *to = reinterpret_cast<uint4 *>(out - head) + g0;
        uint4 q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) q[u] = in[u * THREADS];
        const GradToken t = grad_token(a, token);
        if (is_wide_lse(t.lse)) {
            if (part == 0) wide_row<T, const GradArgs &>(a, token, row, out);
            return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Pair v[V / 2];
            unpack(q[u], v);
            grad_of(t, v, (g0 + u * THREADS) * V - head, 1);
            to[u * THREADS] = pack(v);
        }
        return;
    }
    // Parts with an end of the row, or past it: four granules in flight as well in
    // bf16; in fp32 one, as that leaves 32 registers a thread and not 48, and more threads
    // (2000 x 5000: 14.0 us, with four 16.1; bf16, 5000 x 5000: 27.6 and 17.6).
    constexpr int B = sizeof(T) == 4 ? 1 : U;
    const GradToken t = B == 1 ? grad_token(a, token) : GradToken{};
#pragma unroll 1
    for (int b = 0; b < U / B; ++b) {
        const int32_t at = g0 + b * B * THREADS;
        uint4 q[B];
#pragma unroll
        for (int u = 0; u < B; ++u) {
            const int32_t g = at + u * THREADS;
            if (g < granules) q[u] = load_granule(row, int64_t(g) * V - head, n, -INFINITY);
        }
        const GradToken own = B == 1 ? t : grad_token(a, token);   // (after the loads)
        if (is_wide_lse(own.lse)) {   // (in the first round, and for all threads)
            if (part == 0) wide_row<T, const GradArgs &>(a, token, row, out);
            return;
        }
#pragma unroll
        for (int u = 0; u < B; ++u) {
            const int32_t g = at + u * THREADS;
            if (g >= granules) return;
            const int64_t j0 = int64_t(g) * V - head;
            Pair v[V / 2];
            unpack(q[u], v);
            grad_of(own, v, int32_t(j0), 1);
            float w[V];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) w[2 * i] = low(v[i]), w[2 * i + 1] = high(v[i]);
            store_granule(out, j0, n, w);
        }
    }
}

// Rows that do not start alike, and columns: consecutive threads take
// consecutive elements of the contiguous axis, U of them each.  32 registers a thread
// in fp32 (5184 x 175 columns 2.8 us, with 34 3.6), 40 in bf16 (52783 x 30 3.8 us, with 32 4.3).
template <typename T, bool COLUMNS>
__global__ void __launch_bounds__(kGradThreads, sizeof(T) == 4 ? 8 : 6) grad_any_kernel(const GradArgs a, int32_t parts) {   // (parts of a row; columns need none)
    constexpr int U = 8;
    pdl_wait_previous();
    pdl_launch_dependents();
    // columns: 32 tokens x 8 rows of threads; rows: one token
    // (columns: consecutive CTAs take neighbouring tokens of the same rows, after a CTA a tile for its wide tokens)
    const int32_t tiles = COLUMNS ? int32_t((a.tokens + 31) / 32) : 1;
    const int32_t cta = COLUMNS ? int32_t(blockIdx.x) - tiles : int32_t(blockIdx.x);
    if (COLUMNS && cta < 0) return wide_tile<T, false>(a, blockIdx.x);
    const int64_t token = COLUMNS ? int64_t(cta % tiles) * 32 + (threadIdx.x & 31) : cta / parts;
    if (token >= a.tokens) return;
    const int32_t part = COLUMNS ? cta / tiles : cta % parts, step = COLUMNS ? kGradThreads / 32 : kGradThreads;
    const int32_t v0 = part * (step * U) + int32_t(COLUMNS ? threadIdx.x >> 5 : threadIdx.x);
    const T *x = static_cast<const T *>(a.x) + (COLUMNS ? v0 * a.ld + token : token * a.ld + v0);
    T *dx = static_cast<T *>(a.dx) + (COLUMNS ? v0 * a.ldd + token : token * a.ldd + v0);
    const int64_t by = COLUMNS ? step * a.ld : step, by_out = COLUMNS ? step * a.ldd : step;
    const bool whole = v0 + (U - 1) * step < a.vocab;
    Pair v[U / 2];
#pragma unroll
    for (int u = 0; u < U; u += 2) {
        const float lo = whole || v0 + u * step < a.vocab ? widen(x[u * by]) : 0.0f;
        v[u / 2] = pair(lo, whole || v0 + (u + 1) * step < a.vocab ? widen(x[(u + 1) * by]) : 0.0f);
    }
    const GradToken t = grad_token(a, token);
    const bool wide = is_wide_lse(t.lse);
    grad_of(t, v, v0, step);
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (!wide && (whole || v0 + u * step < a.vocab)) dx[u * by_out] = narrow<T>(u & 1 ? high(v[u / 2]) : low(v[u / 2]));
    if (!COLUMNS && wide && part == 0)
        wide_row<T, GradArgs>(a, token, static_cast<const T *>(a.x) + token * a.ld, static_cast<T *>(a.dx) + token * a.ldd);
}

// Rows v0, v0 + ROWS, ... of two neighbouring tokens, N of them, or with GUARD those
// below the vocabulary's end.
template <typename T, int N, int ROWS, bool GUARD>
__device__ __forceinline__ void grad_pairs(const GradArgs &a, int64_t token, const T *x, T *dx, int64_t by, int64_t by_out, int32_t v0) {
    using Two = typename std::conditional<sizeof(T) == 4, uint2, uint32_t>::type;
    Two q[N];
#pragma unroll
    for (int u = 0; u < N; ++u, x += by)
        if (!GUARD || v0 + u * ROWS < a.vocab) q[u] = *reinterpret_cast<const Two *>(x);
    const GradToken t0 = grad_token(a, token), t1 = grad_token(a, token + 1);
    const Pair lse = pair(-t0.lse, -t1.lse), log2e = both(kLog2e), b = pair(-t0.b, -t1.b), c = pair(-t0.c, -t1.c);
    const bool wide = is_wide_lse(t0.lse) || is_wide_lse(t1.lse);
#pragma unroll
    for (int u = 0; u < N; ++u, dx += by_out) {
        if (GUARD && v0 + u * ROWS >= a.vocab) return;
        Pair l;
        if constexpr (sizeof(T) == 4) l = pair(__uint_as_float(q[u].x), __uint_as_float(q[u].y));
        else l = pair(widen2(q[u]).x, widen2(q[u]).y);
        l = add2(l, lse);
        l = pair(max_nan(low(l), kMasked), max_nan(high(l), kMasked));
        const Pair d = mul2(l, log2e), g = mul2(pair(exp2_fast(low(d)), exp2_fast(high(d))), fma2(l, b, c));
        const int32_t v = v0 + u * ROWS;
        const float g0 = low(g) + (v == t0.target ? t0.a : 0.0f), g1 = high(g) + (v == t1.target ? t1.a : 0.0f);
        if (wide) continue;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float2 *>(dx) = make_float2(g0, g1);
        else *reinterpret_cast<__nv_bfloat162 *>(dx) = __floats2bfloat162_rn(g0, g1);
    }
}

// Columns whose rows can be read two tokens at a time: 64 tokens x 8 rows of
// threads, U rows each, a pair the same entry of two tokens.  Consecutive CTAs
// take neighbouring tokens, so that whole rows are read at about the same time.
// 700 x 10000 fp32 10.5 us (5.4 TB/s), 300 x 128000 fp32 45 (6.8 TB/s; consecutive
// CTAs down the rows of the same tokens: 65), 860 x 50000 bf16 35 (39).
template <typename T>
__global__ void __launch_bounds__(kGradThreads, 5) grad_columns_kernel(const GradArgs a) {
    constexpr int U = 8, ROWS = kGradThreads / 32;
    pdl_wait_previous();
    pdl_launch_dependents();
    // (consecutive CTAs take neighbouring tokens of the same rows, after one for the wide tokens of every 32)
    const int32_t tiles = int32_t((a.tokens + 63) / 64), cta = int32_t(blockIdx.x) - int32_t((a.tokens + 31) / 32);
    if (cta < 0) return wide_tile<T, true>(a, blockIdx.x);
    const int64_t token = int64_t(cta % tiles) * 64 + 2 * (threadIdx.x & 31);
    if (token >= a.tokens) return;
    const int32_t v0 = cta / tiles * (ROWS * U) + int32_t(threadIdx.x >> 5);
    const T *x = static_cast<const T *>(a.x) + v0 * a.ld + token;
    T *dx = static_cast<T *>(a.dx) + v0 * a.ldd + token;
    const int64_t by = ROWS * a.ld, by_out = ROWS * a.ldd;
    if (token + 1 == a.tokens) {   // the last one, alone
        const GradToken t = grad_token(a, token);
        if (is_wide_lse(t.lse)) return;
        for (int32_t u = 0, v = v0; v < a.vocab && u < U; ++u, v += ROWS) {
            Pair g[1] = {both(widen(x[u * by]))};
            grad_of(t, g, v, a.vocab);   // (the second value is nobody's)
            dx[u * by_out] = narrow<T>(low(g[0]));
        }
        return;
    }
    if (v0 + (U - 1) * ROWS < a.vocab) {
        grad_pairs<T, U, ROWS, false>(a, token, x, dx, by, by_out, v0);
    } else {   // (fewer at a time: the registers are the other way's)
        for (int32_t u = 0; u < U && v0 + u * ROWS < a.vocab; u += U / 4)
            grad_pairs<T, U / 4, ROWS, true>(a, token, x + u * by, dx + u * by_out, by, by_out, v0 + u * ROWS);
    }
}

template <typename T>
cudaError_t launch_grad(const GradArgs &a, darb_layout_t layout, cudaStream_t stream) {
    const auto grid = [](int64_t n) { return dim3(unsigned(n)); };
    if (layout == DARB_TOKEN_COLUMNS) {
        const int32_t parts = int32_t((a.vocab + 63) / 64);
        const bool pairs = a.tokens > 32 && a.ld % 2 == 0 && a.ldd % 2 == 0 && aligned_to(a.x, 2 * sizeof(T)) && aligned_to(a.dx, 2 * sizeof(T));
        const int64_t tiles = (a.tokens + 31) / 32, blocks = (pairs ? (a.tokens + 63) / 64 : tiles) * parts + tiles;
        if (blocks > INT32_MAX) return cudaErrorNotSupported;
        if (pairs) return launch_ex(grad_columns_kernel<T>, grid(blocks), dim3(kGradThreads), 0, stream, 1, true, a);
        return launch_ex(grad_any_kernel<T, true>, grid(blocks), dim3(kGradThreads), 0, stream, 1, true, a, parts);
    }
    // logits and gradients of every row start alike past a 16-byte boundary
    const bool alike = row_head<T>(a.x) == row_head<T>(a.dx) && (a.tokens == 1 || (a.ld - a.ldd) * int64_t(sizeof(T)) % 16 == 0);
    if (alike) {
        const int64_t granules = row_granules<T>(kPerGranule<T> - 1, a.vocab);
        const auto rows = [&](auto threads) {
            const int64_t parts = (granules + threads.value * kGradUnroll - 1) / (threads.value * kGradUnroll);
            if (a.tokens * parts > INT32_MAX) return cudaErrorNotSupported;
            return launch_ex(grad_rows_kernel<T, threads.value>, grid(a.tokens * parts), dim3(threads.value), 0, stream, 1, true, a,
                             int32_t(parts));
        };
        // Small CTAs: the loads of one in the time of another's stores.  bf16: one part a row
        // or 64 threads (1896 x 2783: 4.3 us, with 64 5.3, with 256 5.5; 4096 x 32000 78, with
        // 256 87).  fp32: 64 for many short rows (3230 x 1656: 9.4 us, with 256 11.1; 700 x 10000
        // 11.4 and 10.5; 100 x 1000 2.4 and 1.7).
        if constexpr (sizeof(T) == 2) {
            if (granules > 256 && granules <= 512) return rows(std::integral_constant<int, 128>());
            return rows(std::integral_constant<int, 64>());
        } else {
            if (granules <= 512 && a.tokens >= 4 * sm_count()) return rows(std::integral_constant<int, 64>());
            return rows(std::integral_constant<int, kGradThreads>());
        }
    }
    const int32_t parts = int32_t((a.vocab + kGradThreads * 8 - 1) / (kGradThreads * 8));
    const int64_t blocks = a.tokens * parts;
    if (blocks > INT32_MAX) return cudaErrorNotSupported;
    return launch_ex(grad_any_kernel<T, false>, grid(blocks), dim3(kGradThreads), 0, stream, 1, true, a, parts);
}

}  // namespace
}  // namespace darb

using namespace darb;

extern "C" {

darb_status_t darb_token_logprobs(const void *logits, darb_dtype_t dtype, darb_layout_t layout, int64_t tokens,
                                  int64_t vocab, int64_t ld, const int64_t *targets, int32_t k, float *logprob,
                                  float *entropy, float *lse, float *top_logprob, int32_t *top_index,
                                  cudaStream_t stream) {
    DARB_TRACE("darb_token_logprobs");
    if (!token_dtype(dtype) || !token_layout(layout) || tokens < 0 || vocab <= 0 || k < 0 || k > DARB_MAX_TOP || k > vocab)
        return DARB_ERR_INVALID_ARG;
    if (ld < (layout == DARB_TOKEN_ROWS ? vocab : tokens)) return DARB_ERR_INVALID_ARG;
    if (tokens == 0) return DARB_OK;
    if (logits == nullptr || !aligned_to(logits, dtype_size(dtype)) || (targets == nullptr) != (logprob == nullptr) ||
        !aligned_to(targets, 8) || !aligned_to(logprob, 4) || !aligned_to(entropy, 4) || !aligned_to(lse, 4))
        return DARB_ERR_INVALID_ARG;
    if (k > 0 && (top_logprob == nullptr || top_index == nullptr || !aligned_to(top_logprob, 4) || !aligned_to(top_index, 4)))
        return DARB_ERR_INVALID_ARG;
    if (tokens > kMaxTokens || vocab > kMaxFeatures) return DARB_ERR_UNSUPPORTED;
    if (token_span(layout, 1, tokens, vocab, ld) < 0) return DARB_ERR_UNSUPPORTED;
    const Range outs[] = {{logprob, tokens * 4}, {entropy, tokens * 4}, {lse, tokens * 4}, {k ? top_logprob : nullptr, tokens * k * 4},
                          {k ? top_index : nullptr, tokens * k * 4}};
    const Range ins[] = {token_range(logits, layout, 1, tokens, vocab, ld, dtype_size(dtype)), {targets, tokens * 8}};
    if (!outputs_apart(outs, ins)) return DARB_ERR_INVALID_ARG;
    if (layout == DARB_TOKEN_COLUMNS && tokens == 1 && ld == 1) layout = DARB_TOKEN_ROWS;   // (a single row: ld is not used)
    const ScoreArgs a = {logits, ld, tokens, int32_t(vocab), k, targets, logprob, entropy, lse, top_logprob, top_index};
    if (layout == DARB_TOKEN_ROWS)
        return enqueue([&] { return dtype == DARB_BF16 ? launch_score_rows<__nv_bfloat16>(a, stream) : launch_score_rows<float>(a, stream); });
    return enqueue([&] { return dtype == DARB_BF16 ? launch_score_columns<__nv_bfloat16>(a, stream) : launch_score_columns<float>(a, stream); });
}

darb_status_t darb_token_logprobs_grad(const void *logits, darb_dtype_t dtype, darb_layout_t layout, int64_t tokens,
                                       int64_t vocab, int64_t ld, const int64_t *targets, const float *lse,
                                       const float *entropy, const float *d_logprob, const float *d_entropy,
                                       void *d_logits, int64_t ld_grad, cudaStream_t stream) {
    DARB_TRACE("darb_token_logprobs_grad");
    if (!token_dtype(dtype) || !token_layout(layout) || tokens < 0 || vocab <= 0) return DARB_ERR_INVALID_ARG;
    const int64_t least = layout == DARB_TOKEN_ROWS ? vocab : tokens;
    if (ld < least || ld_grad < least) return DARB_ERR_INVALID_ARG;
    if (tokens == 0) return DARB_OK;
    const size_t es = dtype_size(dtype);
    if (logits == nullptr || d_logits == nullptr || lse == nullptr || !aligned_to(logits, es) || !aligned_to(d_logits, es) ||
        !aligned_to(lse, 4) || !aligned_to(entropy, 4) || !aligned_to(d_logprob, 4) || !aligned_to(d_entropy, 4) ||
        !aligned_to(targets, 8))
        return DARB_ERR_INVALID_ARG;
    if ((d_logprob != nullptr && targets == nullptr) || (d_entropy != nullptr && entropy == nullptr)) return DARB_ERR_INVALID_ARG;
    if (tokens > kMaxTokens || vocab > kMaxFeatures) return DARB_ERR_UNSUPPORTED;
    if (token_span(layout, 1, tokens, vocab, ld) < 0 || token_span(layout, 1, tokens, vocab, ld_grad) < 0) return DARB_ERR_UNSUPPORTED;
    // the gradient may take the logits' place: every element is read before it is written
    const bool in_place = logits == d_logits && ld == ld_grad;
    const Range outs[] = {token_range(d_logits, layout, 1, tokens, vocab, ld_grad, es)};
    const Range ins[] = {token_range(in_place ? nullptr : logits, layout, 1, tokens, vocab, ld, es), {targets, tokens * 8}, {lse, tokens * 4},
                         {entropy, tokens * 4}, {d_logprob, tokens * 4}, {d_entropy, tokens * 4}};
    if (!outputs_apart(outs, ins)) return DARB_ERR_INVALID_ARG;
    if (layout == DARB_TOKEN_COLUMNS && tokens == 1 && ld == 1 && ld_grad == 1) layout = DARB_TOKEN_ROWS;
    const GradArgs a = {logits, d_logits, ld, ld_grad, tokens, int32_t(vocab), targets, lse, entropy, d_logprob, d_entropy};
    return enqueue([&] { return dtype == DARB_BF16 ? launch_grad<__nv_bfloat16>(a, layout, stream) : launch_grad<float>(a, layout, stream); });
}

}  // extern "C"
