// policy.cu -- the clipped policy loss of drawn answers with a KL term and an
// entropy bonus, and its gradients (darb_policy_loss): between darb_token_logprobs,
// whose log probabilities and entropies it takes, and darb_token_logprobs_grad, which
// takes what it leaves.
//
// Per token that counts, with d = logprob - old (or its mean over the token's
// sequence), r = e^d, A the sequence's advantage and w the token's weight:
//   loss = sum w (-min(r A, clip(r, 1 - low, 1 + high) A) + kl_coef k - entropy_coef H),
//   k = e^x - 1 - x with x = ref - logprob,
//   d_logprob = w (-[not clipped] A r - kl_coef (e^x - 1)),  d_entropy = -entropy_coef w.
// A mean over a sequence shares its gradient among n tokens and gets it back from as
// many, so the formula is the same with one ratio a sequence.
//
// w needs how many tokens count in a sequence, and in all: the inputs are read twice
// (the mask, and log probabilities where the ratio is the sequence's; then everything).
// A CTA takes a chunk of consecutive tokens.  It finds the sequences in it by a search
// among the offsets in which all its threads take part; the place where a sequence starts
// in the chunk stands for it from then on, so that scratch goes by tokens and any
// number of empty sequences costs nothing but reading their offsets.  A chunk's sums of
// a sequence go to that place, those of a sequence from an earlier chunk to the chunk,
// and who needs the sum of a sequence that spans chunks adds the chunks up, in their
// order.  Up to 4096 tokens are one chunk: one CTA, one launch, no scratch.
//
// What bounds it is latency.  A token costs 25 bytes and 225 instructions, 57 in the counting
// kernel and 167 in the one with the losses: 64-bit arithmetic would be too slow to spend on a
// token (one operation takes as long as 6 bytes), so that a border is decided in 32 bits, and by
// the exact difference in the rare thread that meets one, and 64 bits hold sums from a warp on.
// But a chunk is a chain of ten loads and barriers that need one another: 1.5 million tokens of
// 1000 sequences take 27 us (37 MB: 5.5 us), of which the first reading is 6.  So all that does
// without the weights -- exponentials, gradients but for a factor -- comes before the wait for
// the first reading, and the chunks' sums are added up by a launch of its own (a ticket, and the
// last CTA: 2 us more).  300 tokens take 5.0 us, 4096 take 7.2.  Where every sequence counts the
// same, the chunks of a long one before the first that counts are looked through one after the
// other: 15 of 100000 tokens, their first nine tenths masked, 70 us against 24.
#include "launch.cuh"
#include "tma.cuh"
#include "tokens.cuh"
#include "trace.h"

#include <algorithm>
#include <cmath>
#include <limits>

namespace darb {

cudaError_t stream_alloc(void **p, size_t bytes, cudaStream_t stream);

namespace {

constexpr int kE = 8;                       // tokens of a thread
// Tokens of a single CTA of 512 or 128 threads (1024 tokens: 4.7 us by 128 threads, 6.8 by 512; 1025 to 4096: 6.7 to 7.2 by
// one CTA of 512, 9.5 by three launches).
constexpr int kFew = 4096, kVeryFew = 1024;
constexpr int kChunkThreads = 256;
constexpr int kChunkTokens = kChunkThreads * kE;
// Chunks that every CTA adds up itself, not a launch of its own.  Us without that launch and with it, every token counting
// the same, and every sequence: 400000 tokens 11.5 and 15.9, 11.7 and 15.3; 1.5 million 24.0 and 25.5, 25.5 and 25.2;
// 1.8 million 27.2 and 27.2, 29.7 and 27.3; 8 million 116 and 92, 148 and 92.
constexpr int kInline = 800;
constexpr int kStats = 5;                   // loss, policy, kl, entropy, clipped
constexpr int kSums = 4;                    // the sums that they come from
constexpr int kOutside = -2, kNone = -1;    // in place of a sequence

constexpr int kWhole = 1 << 30;             // a chunk that is all of one sequence that started before

struct PolicyWork {
    double *slot_sum;     // per token: of the sequence that starts there, what its first chunk has of it
    double *head_sum;     // per chunk: of the sequence that started before it
    double *partial;      // per chunk and sum
    int4 *info;           // per chunk: the tokens that count; sequences that start in it and have one of them; of the
                          // sequence that started before it; of the one that goes on behind it (kWhole: the same one)
    int32_t *slot_count;
    long long *norm;      // the tokens, or sequences, that count
};

struct PolicyArgs {
    const float *logprob, *old, *ref, *entropy, *advantage;
    const uint8_t *mask;
    const int64_t *offsets;
    float *stats, *d_logprob, *d_entropy;
    PolicyWork w;
    int64_t n, sequences, chunks;
    double log_low, log_high;     // log(1 - low), log(1 + high)
    float low[3], high[3];        // the same, as sums of 32-bit numbers
    float used_low, used_high;    // 1 - low, 1 + high
    float kl_coef, entropy_coef;
    int32_t per_sequence;         // the mean: every sequence counts the same
    int32_t counted;              // w.norm has been summed by a launch of its own
    int32_t vector;
};

// How many of the offsets are <= at: offsets[0 .. n] do not fall.
template <int THREADS>
__device__ __forceinline__ int64_t offsets_upto(const int64_t *offsets, int64_t n, int64_t at) {
    int64_t lo = 0, hi = n + 1;   // the answer is in [lo, hi]
    while (hi > lo) {
        const int64_t span = hi - lo, step = (span + THREADS - 1) / THREADS;
        // thread i looks at the last of the i-th run of `step` offsets
        const int64_t i = lo + (int64_t(threadIdx.x) + 1) * step - 1;
        const int below = __syncthreads_count(i < hi && offsets[i] <= at);
        lo = min(lo + below * step, hi);
        hi = min(lo + step - 1, hi);
    }
    return lo;
}

template <int THREADS>
struct ChunkShared {
    static constexpr int T = THREADS * kE;
    alignas(16) int start[T];   // at the first token of a sequence: the sequence; elsewhere kNone
    uint16_t places[T];         // where the sequences start, in any order
    int sequences;              // how many
    int warp_max[THREADS / 32];
    double scan_sum[THREADS / 32];
    int scan_count[THREADS / 32], scan_flag[THREADS / 32];
    int last;            // where the last sequence of the chunk starts
    int64_t before;      // where the sequence of the first token starts
    int64_t after;       // where the last one ends
};

// What a thread's tokens have to do with sequences.
struct Tokens {
    int first;           // where the last sequence before the thread's tokens starts (0 in the first thread)
    uint32_t starts;     // a bit for each token at which one starts
    uint32_t inside;     // a bit for each token that belongs to one
};

// Which sequences start where in the chunk at c0.
template <int THREADS>
__device__ __forceinline__ Tokens find_sequences(const PolicyArgs &a, int64_t c0, ChunkShared<THREADS> &sh) {
    constexpr int T = THREADS * kE;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int4 *const mine = reinterpret_cast<int4 *>(sh.start + tid * kE);
    mine[0] = mine[1] = make_int4(kNone, kNone, kNone, kNone);
    if (tid == 0) sh.sequences = 0;
    const int64_t s0 = offsets_upto<THREADS>(a.offsets, a.sequences, c0) - 1;   // (its barriers order the writes above)
    if (tid == 0) {
        const bool inside = s0 >= 0 && s0 < a.sequences;
        sh.start[0] = inside ? int(s0) : kOutside;
        // (outside of 0 .. c0 only where offsets are wrong: it is a place in the scratch)
        sh.before = inside ? min(max(a.offsets[s0], int64_t(0)), c0) : c0;
        if (inside) sh.places[atomicAdd(&sh.sequences, 1)] = 0;
    }
    for (int64_t base = s0 + 1;; base += THREADS) {
        const int64_t s = base + tid;
        const int64_t at = s <= a.sequences ? a.offsets[s] - c0 : T, next = s < a.sequences ? a.offsets[s + 1] - c0 : 0;
        const bool in = at < T;
        if (in && at > 0 && c0 + at < a.n) {
            if (s == a.sequences) {
                sh.start[at] = kOutside;
            } else if (next > at) {
                sh.start[at] = int(s);
                const int place = atomicAdd(&sh.sequences, 1);
                if (place < T) sh.places[place] = uint16_t(at);
            }
        }
        const int starts = __syncthreads_count(in);
        if (starts < THREADS) {
            if (tid == starts) sh.after = c0 + at;
            break;
        }
    }
    const int4 x = mine[0], y = mine[1];
    const int id[kE] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    Tokens t = {};
#pragma unroll
    for (int e = 0; e < kE; ++e) t.starts |= uint32_t(id[e] != kNone) << e;
    // the last start of a lane before, of a warp before
    const int mine_last = tid * kE + 31 - __clz(t.starts);
    const uint32_t lanes = __ballot_sync(~0u, t.starts != 0), lower = lanes & ((1u << lane) - 1);
    int before = __shfl_sync(~0u, mine_last, 31 - __clz(lower | 1));
    if (lower == 0) before = -1;
    const int warp_last = __shfl_sync(~0u, mine_last, 31 - __clz(lanes | 1));
    if (lane == 0) sh.warp_max[warp] = lanes != 0 ? warp_last : -1;
    __syncthreads();
    if (lower == 0)
        for (int w = 0; w < warp; ++w) before = max(before, sh.warp_max[w]);
    if (tid == THREADS - 1) sh.last = t.starts != 0 ? mine_last : before;
    t.first = tid == 0 ? 0 : before;
    bool in = sh.start[t.first] >= 0;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
        if (id[e] != kNone) in = id[e] >= 0;
        t.inside |= uint32_t(in) << e;
    }
    const int64_t left = a.n - c0 - tid * kE;
    t.inside &= left >= kE ? (1u << kE) - 1 : left > 0 ? (1u << int(left)) - 1 : 0u;
    return t;
}

// kE tokens from i on (`rest` where n ends before them).
__device__ __forceinline__ void load8(const float *p, int64_t i, int64_t n, bool vector, float (&v)[kE]) {
    if (vector && i + kE <= n) {
        const float4 x = reinterpret_cast<const float4 *>(p + i)[0], y = reinterpret_cast<const float4 *>(p + i)[1];
        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
        return;
    }
#pragma unroll
    for (int e = 0; e < kE; ++e) v[e] = i + e < n ? p[i + e] : 0.0f;
}
// The mask of kE tokens, a bit each.
__device__ __forceinline__ uint32_t load_mask(const uint8_t *p, int64_t i, int64_t n, bool vector) {
    uint32_t bits = 0;
    if (p == nullptr) {
        return i >= n ? 0u : n - i >= kE ? (1u << kE) - 1 : (1u << int(n - i)) - 1;
    }
    if (vector && i + kE <= n) {
        const uint2 q = *reinterpret_cast<const uint2 *>(p + i);
        // the top bit of every byte that is not 0, then byte i's to bit i
        const uint32_t x = (((q.x & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | q.x) >> 7 & 0x01010101u, y = (((q.y & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | q.y) >> 7 & 0x01010101u;
        return (x * 0x01020408u) >> 24 & 15u | ((y * 0x01020408u) >> 24 & 15u) << 4;
    }
#pragma unroll
    for (int e = 0; e < kE; ++e)
        if (i + e < n && p[i + e] != 0) bits |= 1u << e;
    return bits;
}

// a - b exactly, as a rounded difference and what that leaves.
__device__ __forceinline__ void difference(float a, float b, float &hi, float &lo) {
    hi = __fsub_rn(a, b);
    const float bb = __fsub_rn(a, hi);
    lo = __fadd_rn(__fsub_rn(a, __fadd_rn(hi, bb)), __fsub_rn(bb, b));
}

// Whether the exact difference a - b is above (UP) or below a border, `d` being the
// rounded one, which tells unless it is the rounded border.
template <bool UP>
__device__ __forceinline__ bool past(float a, float b, float d, const float (&border)[3]) {
    if (d != border[0]) return UP ? d > border[0] : d < border[0];
    float hi, lo;
    difference(a, b, hi, lo);
    if (lo != border[1]) return UP ? lo > border[1] : lo < border[1];
    return UP ? border[2] < 0.0f : border[2] > 0.0f;
}

// Of every sequence in the chunk, how many of its tokens count: added to counts[] by the
// place of the start (whole numbers: in any order).  A warp without a start has one.
template <int THREADS>
__device__ __forceinline__ void sequence_counts(const Tokens &t, uint32_t on, int *counts) {
    const int tid = threadIdx.x, lane = tid & 31;
    if (__all_sync(~0u, t.starts == 0)) {   // (then all have the same one)
        const int n = __reduce_add_sync(~0u, __popc(on));
        if (lane == 0 && n > 0) atomicAdd(counts + t.first, n);
        return;
    }
    int cur = t.first, from = 0;
    for (uint32_t left = tid == 0 ? t.starts & ~1u : t.starts;; left &= left - 1) {
        const int to = left != 0 ? __ffs(left) - 1 : kE;
        const int n = __popc(on >> from & ((1u << (to - from)) - 1));
        if (n > 0) atomicAdd(counts + cur, n);
        if (left == 0) break;
        cur = tid * kE + to, from = to;
    }
}

// Of every sequence in the chunk, how many of its tokens count and the sum of their
// differences: put(start, count, sum) once for each.
template <int THREADS, bool SUMS, typename Put>
__device__ __forceinline__ void sequence_sums(const Tokens &t, uint32_t on, const float (&lp)[kE],
                                              const float (&old)[kE], ChunkShared<THREADS> &sh, Put put) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int cur = t.first, count = 0, head_count = 0;
    float hi = 0.0f, lo = 0.0f;
    double head_sum = 0.0;
    bool flag = false;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
        const int p = tid * kE + e;
        if ((t.starts >> e & 1) && p > 0) {
            if (!flag) head_count = count, head_sum = SUMS ? double(hi) + double(lo) : 0.0;
            else put(cur, count, SUMS ? double(hi) + double(lo) : 0.0);
            flag = true;
            cur = p, count = 0, hi = 0.0f, lo = 0.0f;
        }
        if (on >> e & 1) {
            ++count;
            if (SUMS) {
                // what the difference and the sum round away is summed beside it
                float d, r, err;
                difference(lp[e], old[e], d, r);
                const float sum = __fadd_rn(hi, d), back = __fsub_rn(sum, hi);
                err = __fadd_rn(__fsub_rn(hi, __fsub_rn(sum, back)), __fsub_rn(d, back));
                hi = sum;
                lo = isfinite(sum) ? lo + (err + r) : 0.0f;
            }
        }
    }
    // from the last start of each thread on, over the threads that have none
    const int tail_count = count;
    const double tail_sum = SUMS ? double(hi) + double(lo) : 0.0;
    int c = tail_count;
    double s = tail_sum;
    int f = flag;
    for (int d = 1; d < 32; d <<= 1) {
        const int oc = __shfl_up_sync(~0u, c, d), of = __shfl_up_sync(~0u, f, d);
        const double os = SUMS ? __shfl_up_sync(~0u, s, d) : 0.0;
        if (lane >= d) {
            if (!f) c += oc, s = os + s;
            f |= of;
        }
    }
    if (lane == 31) sh.scan_count[warp] = c, sh.scan_sum[warp] = s, sh.scan_flag[warp] = f;
    int bc = __shfl_up_sync(~0u, c, 1), bf = __shfl_up_sync(~0u, f, 1);
    double bs = SUMS ? __shfl_up_sync(~0u, s, 1) : 0.0;
    if (lane == 0) bc = 0, bf = 0, bs = 0.0;
    __syncthreads();
    int wc = 0;
    double ws = 0.0;   // of the warps before
    for (int w = 0; w < warp; ++w) {
        if (sh.scan_flag[w]) wc = sh.scan_count[w], ws = sh.scan_sum[w];
        else wc += sh.scan_count[w], ws += sh.scan_sum[w];
    }
    if (!bf) bc += wc, bs = ws + bs;
    // the thread's first start ends the sequence before it, the chunk's end the last one
    if (flag) put(t.first, bc + head_count, bs + head_sum);
    if (tid == THREADS - 1) {
        if (flag) put(cur, tail_count, tail_sum);
        else put(cur, bc + tail_count, bs + tail_sum);
    }
}

__device__ __forceinline__ double warp_sum(double v) {
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
    return v;
}
__device__ __forceinline__ long long warp_sum(long long v) {
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
    return v;
}

template <int THREADS>
__device__ __forceinline__ long long block_sum(long long v) {
    __shared__ long long part[THREADS / 32];
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < THREADS / 32; ++w) v += part[w];
    return v;
}

// The part of thread `at` of `threads` of the tokens (or sequences) that count.
__device__ __forceinline__ long long counted(const PolicyArgs &a, int64_t at, int64_t threads) {
    const int4 *const info = a.w.info;
    long long sum = 0;
#pragma unroll 4
    for (int64_t c = at; c < a.chunks; c += threads) {
        const int4 here = __ldcg(info + c);
        const int tail = __ldcg(&info[c > 0 ? c - 1 : 0].w);
        if (!a.per_sequence) {
            sum += here.x;
            continue;
        }
        sum += here.y;
        // a sequence none of whose tokens count before this chunk
        if (here.z > 0) {
            bool first = (tail & ~kWhole) == 0;
            for (int64_t b = c - 1; first && b > 0 && (__ldcg(&info[b].w) & kWhole) != 0; --b) first = (__ldcg(&info[b - 1].w) & ~kWhole) == 0;
            sum += first;
        }
    }
    return sum;
}

// What a token needs to know of its sequence.
struct Piece {
    float weight, advantage;
    float used, slope;   // of one ratio a sequence: what it is clipped to, and -A r where it is not clipped
};

template <bool SUMS>
__device__ __forceinline__ Piece piece_of(const PolicyArgs &a, float advantage, int count, double sum, long long norm) {
    Piece p;
    const long long n = a.per_sequence ? norm * count : norm;
    p.weight = count > 0 ? 1.0f / __ll2float_rn(n) : 0.0f;
    p.advantage = advantage;
    p.used = p.slope = 0.0f;
    if (SUMS && count > 0) {
        const double d = sum / count;
        const bool up = p.advantage >= 0.0f, cut = up ? d > a.log_high : d < a.log_low;
        const float r = expf(float(d));
        p.used = cut ? (up ? a.used_high : a.used_low) : r;
        p.slope = cut ? 0.0f : -p.advantage * r;
        if (cut) p.weight = -p.weight;   // (the sign says so)
    }
    return p;
}

// e^x - 1 and e^x - 1 - x: the second by its series where the terms cancel (|x| < 1; what
// is left out is below 2^-27 of the sum), and the first from it.
__device__ __forceinline__ void divergence(float x, float &em1, float &excess) {
    float s = 1.0f / 39916800.0f;
    s = fmaf(s, x, 1.0f / 3628800.0f);
    s = fmaf(s, x, 1.0f / 362880.0f);
    s = fmaf(s, x, 1.0f / 40320.0f);
    s = fmaf(s, x, 1.0f / 5040.0f);
    s = fmaf(s, x, 1.0f / 720.0f);
    s = fmaf(s, x, 1.0f / 120.0f);
    s = fmaf(s, x, 1.0f / 24.0f);
    s = fmaf(s, x, 1.0f / 6.0f);
    s = fmaf(s, x, 0.5f);
    const float far = expf(x) - 1.0f;
    const bool near = fabsf(x) < 1.0f;
    excess = near ? s * x * x : far - x;
    em1 = near ? x + s * x * x : far;
}

// e^x of two numbers between -80 and 80, to two units: 2^t with t = x log2 e rounded, and
// what that rounding left taken to first order.
__device__ __forceinline__ Pair exp_pair(Pair x) {
    constexpr float kLog2eRest = 1.925963033500e-08f;   // log2 e - kLog2e
    const Pair t = mul2(x, both(kLog2e)), r = fma2(x, both(kLog2eRest), fma2(x, both(kLog2e), mul2(t, both(-1.0f))));
    const Pair e = pair(exp2_fast(low(t)), exp2_fast(high(t)));
    return fma2(e, mul2(r, both(kLn2)), e);
}
// divergence() of two of them.
__device__ __forceinline__ void divergence_pair(Pair x, Pair &em1, Pair &excess) {
    Pair s = both(1.0f / 39916800.0f);
    constexpr float terms[] = {1.0f / 3628800.0f, 1.0f / 362880.0f, 1.0f / 40320.0f, 1.0f / 5040.0f, 1.0f / 720.0f, 1.0f / 120.0f, 1.0f / 24.0f, 1.0f / 6.0f, 0.5f};
#pragma unroll
    for (int i = 0; i < 9; ++i) s = fma2(s, x, both(terms[i]));
    const Pair near = mul2(s, mul2(x, x)), far = add2(exp_pair(x), both(-1.0f)), rest = fma2(x, both(-1.0f), far), em1_near = add2(x, near);
    const bool n0 = fabsf(low(x)) < 1.0f, n1 = fabsf(high(x)) < 1.0f;
    excess = pair(n0 ? low(near) : low(rest), n1 ? high(near) : high(rest));
    em1 = pair(n0 ? low(em1_near) : low(far), n1 ? high(em1_near) : high(far));
}

__device__ __forceinline__ void store8(float *p, int64_t i, uint32_t inside, bool vector, const float (&v)[kE]) {
    if (vector && inside == (1u << kE) - 1) {
        reinterpret_cast<float4 *>(p + i)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p + i)[1] = make_float4(v[4], v[5], v[6], v[7]);
        return;
    }
#pragma unroll
    for (int e = 0; e < kE; ++e)
        if (inside >> e & 1) p[i + e] = v[e];
}

// ---- the first reading of many tokens: the sums of sequences ----

template <bool SUMS>
__global__ void __launch_bounds__(kChunkThreads) policy_count_kernel(const PolicyArgs a) {
    __shared__ ChunkShared<kChunkThreads> sh;
    const int tid = threadIdx.x;
    const int64_t c = blockIdx.x, c0 = c * kChunkTokens, i = c0 + tid * kE;
    pdl_wait_previous();
    // after the wait, so that the next kernel may read the inputs before it waits for this one
    pdl_launch_dependents();
    uint32_t on = load_mask(a.mask, i, a.n, a.vector);
    float lp[kE] = {}, old[kE] = {};
    if (SUMS) {
        load8(a.logprob, i, a.n, a.vector, lp);
        load8(a.old, i, a.n, a.vector, old);
    }
    if (c == 0 && tid == 0) *a.w.norm = 0;
    const Tokens t = find_sequences<kChunkThreads>(a, c0, sh);
    on &= t.inside;
    const int64_t before = sh.before, end = c0 + kChunkTokens;
    __shared__ int s_head, s_tail, s_starts;
    if (tid == 0) s_head = s_tail = s_starts = 0;
    const bool goes_on = sh.after > end;
    __syncthreads();
    auto put = [&](int start, int count, double sum) {
        if (sh.start[start] < 0) return;
        const bool head = start == 0 && before < c0;
        if (head) {
            s_head = count;
            if (SUMS) a.w.head_sum[c] = sum;
        } else {
            if (count > 0) atomicAdd(&s_starts, 1);
            a.w.slot_count[c0 + start] = count;
            if (SUMS) a.w.slot_sum[c0 + start] = sum;
        }
        if (start == sh.last && goes_on) s_tail = count | (head ? kWhole : 0);
    };
    if (SUMS) {
        sequence_sums<kChunkThreads, SUMS>(t, on, lp, old, sh, put);
    } else {
        __shared__ int counts[SUMS ? 1 : kChunkTokens];
        const int sequences = min(sh.sequences, kChunkTokens);
        for (int k = tid; k < sequences; k += kChunkThreads) counts[sh.places[k]] = 0;
        __syncthreads();
        sequence_counts<kChunkThreads>(t, on, counts);
        __syncthreads();
        for (int k = tid; k < sequences; k += kChunkThreads) put(sh.places[k], counts[sh.places[k]], 0.0);
    }
    const long long all = block_sum<kChunkThreads>(__popc(on));
    if (tid == 0) a.w.info[c] = make_int4(int(all), s_starts, s_head, s_tail);
}

__global__ void __launch_bounds__(kChunkThreads) policy_norm_kernel(const PolicyArgs a) {
    pdl_wait_previous();
    pdl_launch_dependents();
    const long long v = block_sum<kChunkThreads>(counted(a, int64_t(blockIdx.x) * kChunkThreads + threadIdx.x, int64_t(gridDim.x) * kChunkThreads));
    if (threadIdx.x == 0 && v != 0) atomicAdd(reinterpret_cast<unsigned long long *>(a.w.norm), static_cast<unsigned long long>(v));
}

// ---- the loss and its gradients ----

// The sum of a sequence over all chunks that it spans, by one warp.
template <bool SUMS>
__device__ __forceinline__ void across_chunks(const PolicyArgs &a, int64_t lo, int64_t hi, int &count, double &sum) {
    const int lane = threadIdx.x & 31;
    int n = 0;
    double v = 0.0;
    const int64_t c0 = lo / kChunkTokens + 1, c1 = min((hi - 1) / kChunkTokens, a.chunks - 1);
    for (int64_t c = c0 + lane; c <= c1; c += 32) {
        n += __ldcg(&a.w.info[c].z);
        if (SUMS) v += a.w.head_sum[c];
    }
    for (int d = 16; d > 0; d >>= 1) n += __shfl_xor_sync(~0u, n, d);
    if (SUMS) v = warp_sum(v);
    count = a.w.slot_count[lo] + n;
    sum = SUMS ? a.w.slot_sum[lo] + v : 0.0;
}

// The sums of a CTA's warps, in the first warp: lane 8 k has the k-th.
template <int THREADS>
__device__ __forceinline__ double warps_sum(const double (&part)[kSums][THREADS / 32], int lane) {
    double v = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; w += 8)
        if (w + (lane & 7) < THREADS / 32) v += part[lane >> 3][w + (lane & 7)];
    for (int d = 4; d > 0; d >>= 1) v += __shfl_down_sync(~0u, v, d, 8);
    return v;
}
// loss, policy, kl, entropy, clipped from their sums (lane 8 k has the k-th)
__device__ __forceinline__ void write_stats(const PolicyArgs &a, double sum, int lane) {
    const double kl = __shfl_sync(~0u, sum, 8), entropy = __shfl_sync(~0u, sum, 16);
    if (lane == 0) {
        double loss = sum;
        if (a.kl_coef != 0.0f) loss += double(a.kl_coef) * kl;
        if (a.entropy_coef != 0.0f) loss -= double(a.entropy_coef) * entropy;
        a.stats[0] = float(loss);
    }
    if ((lane & 7) == 0) a.stats[1 + (lane >> 3)] = float(sum);
}

// The same for one token, whatever it holds.
template <bool SUMS>
__device__ __noinline__ void rarely_one(const PolicyArgs &a, float lp, float old, float ref, float adv, float &d, float &excess, float &loss, bool &cut) {
    d = excess = loss = 0.0f;
    cut = false;
    if (a.ref != nullptr) {
        float em1;
        divergence(ref - lp, em1, excess);
        if (a.kl_coef != 0.0f) d = -a.kl_coef * em1;
    }
    if (!SUMS) {
        const float diff = lp - old;
        const bool up = adv >= 0.0f;
        cut = up ? past<true>(lp, old, diff, a.high) : past<false>(lp, old, diff, a.low);
        const float r = expf(diff);
        loss = -adv * (cut ? (up ? a.used_high : a.used_low) : r);
        if (!cut) d += -adv * r;
    }
}

// SINGLE: all tokens in one CTA, which counts them itself.
template <int THREADS, bool SINGLE, bool SUMS>
__global__ void __launch_bounds__(THREADS, SINGLE ? 1 : 3) policy_kernel(const PolicyArgs a) {
    constexpr int T = THREADS * kE;
    extern __shared__ __align__(16) unsigned char raw[];
    ChunkShared<THREADS> &sh = *reinterpret_cast<ChunkShared<THREADS> *>(raw);
    Piece *const pieces = reinterpret_cast<Piece *>(raw + (sizeof(ChunkShared<THREADS>) + 15) / 16 * 16);   // by the place of the start
    __shared__ double stat_part[kSums][THREADS / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t c = SINGLE ? 0 : blockIdx.x, c0 = c * T, i = c0 + tid * kE;
    if (SINGLE) {
        pdl_launch_dependents();
        pdl_wait_previous();
    }
    // (many: whatever filled the inputs was complete when the kernel before this one let it start)
    uint32_t on = load_mask(a.mask, i, a.n, a.vector);
    float lp[kE], old[kE], ref[kE], ent[kE];
    load8(a.logprob, i, a.n, a.vector, lp);
    load8(a.old, i, a.n, a.vector, old);
    if (a.ref != nullptr) load8(a.ref, i, a.n, a.vector, ref);
    if (a.entropy != nullptr) load8(a.entropy, i, a.n, a.vector, ent);
    const Tokens t = find_sequences<THREADS>(a, c0, sh);
    const int sequences = min(sh.sequences, T);
    for (int k = tid; k < sequences; k += THREADS) {
        const int id = sh.start[sh.places[k]];
        if (id >= 0) pieces[sh.places[k]].advantage = a.advantage[id];   // (below 0 only where offsets fall)
    }
    on &= t.inside;
    __syncthreads();

    // all that does without the weight, of tokens that do not count as of differences of 0
    float d[kE], excess[kE], loss[kE], advantage[kE];   // gradient; e^x - 1 - x; -min(..)
    uint32_t cut = 0;
    if (!SUMS) {
        float adv = pieces[t.first].advantage;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            if (t.starts >> e & 1) adv = pieces[tid * kE + e].advantage;
            advantage[e] = on >> e & 1 ? adv : 0.0f;
        }
    }
    // two tokens at a time; `rare`: a difference on a border, whose exact value decides,
    // or one too large for exp_pair
    bool rare = false;
#pragma unroll
    for (int e = 0; e < kE; e += 2) {
        const bool c0 = on >> e & 1, c1 = on >> (e + 1) & 1;
        Pair grad = both(0.0f), far_off = both(0.0f);
        if (a.ref != nullptr) {
            const Pair x = pair(c0 ? ref[e] - lp[e] : 0.0f, c1 ? ref[e + 1] - lp[e + 1] : 0.0f);
            rare |= !(fmaxf(fabsf(low(x)), fabsf(high(x))) < 80.0f);
            Pair em1;
            divergence_pair(x, em1, far_off);
            if (a.kl_coef != 0.0f) grad = mul2(em1, both(-a.kl_coef));
        }
        excess[e] = low(far_off), excess[e + 1] = high(far_off);
        if (!SUMS) {
            const Pair diff = pair(c0 ? lp[e] - old[e] : 0.0f, c1 ? lp[e + 1] - old[e + 1] : 0.0f);
            rare |= !(fmaxf(fabsf(low(diff)), fabsf(high(diff))) < 80.0f);
            const bool up0 = advantage[e] >= 0.0f, up1 = advantage[e + 1] >= 0.0f;
            const float b0 = up0 ? a.high[0] : a.low[0], b1 = up1 ? a.high[0] : a.low[0];
            const bool k0 = up0 ? low(diff) > b0 : low(diff) < b0, k1 = up1 ? high(diff) > b1 : high(diff) < b1;
            rare |= low(diff) == b0 || high(diff) == b1;
            const Pair gain = mul2(exp_pair(diff), pair(-advantage[e], -advantage[e + 1]));
            loss[e] = k0 ? -advantage[e] * (up0 ? a.used_high : a.used_low) : low(gain);
            loss[e + 1] = k1 ? -advantage[e + 1] * (up1 ? a.used_high : a.used_low) : high(gain);
            grad = add2(grad, pair(k0 ? 0.0f : low(gain), k1 ? 0.0f : high(gain)));
            cut |= uint32_t(k0) << e | uint32_t(k1) << (e + 1);
        }
        d[e] = low(grad), d[e + 1] = high(grad);
        if (!c0) ent[e] = 0.0f;
        if (!c1) ent[e + 1] = 0.0f;
    }
    if (rare) {
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            if (!(on >> e & 1)) continue;
            bool k;
            rarely_one<SUMS>(a, lp[e], old[e], a.ref != nullptr ? ref[e] : 0.0f, SUMS ? 0.0f : advantage[e], d[e], excess[e], loss[e], k);
            cut = (cut & ~(1u << e)) | uint32_t(k) << e;
        }
    }

    // what the tokens of a sequence share
    if (SINGLE) {
        // the sums stand in the pieces until what tokens need takes their place
        sequence_sums<THREADS, SUMS>(t, on, lp, old, sh, [&](int start, int count, double sum) {
            pieces[start].weight = __int_as_float(count);
            if (SUMS) *reinterpret_cast<double *>(&pieces[start].used) = sum;
        });
        __syncthreads();
        long long mine = a.per_sequence ? 0 : __popc(on);
        if (a.per_sequence)
            for (int k = tid; k < sequences; k += THREADS) mine += __float_as_int(pieces[sh.places[k]].weight) > 0;
        const long long norm = block_sum<THREADS>(mine);
        for (int k = tid; k < sequences; k += THREADS) {
            Piece &p = pieces[sh.places[k]];
            const double sum = SUMS ? *reinterpret_cast<const double *>(&p.used) : 0.0;
            p = piece_of<SUMS>(a, p.advantage, __float_as_int(p.weight), sum, norm);
        }
    } else {
        pdl_launch_dependents();
        pdl_wait_previous();
        __syncthreads();   // (the advantages have been read where they are written again)
        const int64_t before = sh.before;
        const int last = sh.last;
        const bool from_before = before < c0, goes_on = sh.after > c0 + T;
        int n_across = 0;
        double sum_across = 0.0;
        // the sequences at the chunk's ends may go on beyond it
        const int p_across = warp == 0 ? 0 : last;
        const bool across = warp < 2 && !(warp == 1 && last == 0) && sh.start[p_across] >= 0 &&
                            ((p_across == 0 && from_before) || (p_across == last && goes_on));
        if (across)
            across_chunks<SUMS>(a, p_across == 0 ? before : c0 + p_across, p_across == last ? min(sh.after, a.n) : c0 + T, n_across, sum_across);
        const int place = tid < sequences ? sh.places[tid] : 0;
        int n_mine = 0;
        double sum_mine = 0.0;
        if (tid < sequences && c0 + place < a.n) {   // (on its way while the chunks are added up)
            n_mine = __ldcg(a.w.slot_count + c0 + place);
            if (SUMS) sum_mine = __ldcg(a.w.slot_sum + c0 + place);
        }
        const long long norm = a.counted ? __ldcg(a.w.norm) : block_sum<THREADS>(counted(a, tid, THREADS));
        for (int k = tid; k < sequences; k += THREADS) {
            const int p = sh.places[k];
            if ((p == 0 && from_before) || (p == last && goes_on)) continue;
            if (k != tid) {
                n_mine = __ldcg(a.w.slot_count + c0 + p);
                if (SUMS) sum_mine = __ldcg(a.w.slot_sum + c0 + p);
            }
            pieces[p] = piece_of<SUMS>(a, pieces[p].advantage, n_mine, sum_mine, norm);
        }
        if (across && lane == 0) pieces[p_across] = piece_of<SUMS>(a, pieces[p_across].advantage, n_across, sum_across, norm);
    }
    __syncthreads();

    float d_ent[kE];
    Pair sum_loss = both(0.0f), sum_excess = both(0.0f), sum_ent = both(0.0f);
    float sum_cut = 0.0f;
    Piece piece = pieces[t.first];
#pragma unroll
    for (int e = 0; e < kE; e += 2) {
        float w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (t.starts >> (e + i) & 1) piece = pieces[tid * kE + e + i];
            const bool counts = on >> (e + i) & 1;
            w[i] = counts ? fabsf(piece.weight) : 0.0f;
            if (SUMS) {
                loss[e + i] = counts ? -piece.advantage * piece.used : 0.0f;
                d[e + i] += counts ? piece.slope : 0.0f;
                cut |= uint32_t(piece.weight < 0.0f) << (e + i);
            }
            sum_cut += cut >> (e + i) & 1 ? w[i] : 0.0f;
        }
        const Pair ww = pair(w[0], w[1]), dd = mul2(ww, pair(d[e], d[e + 1])), ee = mul2(ww, both(-a.entropy_coef));
        sum_loss = fma2(ww, pair(loss[e], loss[e + 1]), sum_loss);
        sum_excess = fma2(ww, pair(excess[e], excess[e + 1]), sum_excess);
        if (a.entropy != nullptr) sum_ent = fma2(ww, pair(ent[e], ent[e + 1]), sum_ent);
        d[e] = low(dd), d[e + 1] = high(dd);
        d_ent[e] = low(ee), d_ent[e + 1] = high(ee);
    }
    // policy, kl, entropy, clipped: lanes 16 apart share two of the sums, 8 apart one, and lane 8 k ends with the k-th
    const float stat[kSums] = {across(sum_loss), across(sum_excess), across(sum_ent), sum_cut};
    const bool up = lane & 16, odd = lane & 8;
    const float s0 = (up ? stat[2] : stat[0]) + __shfl_xor_sync(~0u, up ? stat[0] : stat[2], 16);
    const float s1 = (up ? stat[3] : stat[1]) + __shfl_xor_sync(~0u, up ? stat[1] : stat[3], 16);
    float sum = (odd ? s1 : s0) + __shfl_xor_sync(~0u, odd ? s0 : s1, 8);
    for (int d = 4; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
    if ((lane & 7) == 0) stat_part[lane >> 3][warp] = double(sum);
    __syncthreads();
    if (warp == 0) {
        const double v = warps_sum<THREADS>(stat_part, lane);
        if (SINGLE) write_stats(a, v, lane);
        else if ((lane & 7) == 0) a.w.partial[c * kSums + (lane >> 3)] = v;
    }
    store8(a.d_logprob, i, t.inside, a.vector, d);
    if (a.d_entropy != nullptr) store8(a.d_entropy, i, t.inside, a.vector, d_ent);
}

// The chunks' sums, in their order.
__global__ void __launch_bounds__(kChunkThreads) policy_stats_kernel(const PolicyArgs a) {
    __shared__ double stat_part[kSums][kChunkThreads / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_launch_dependents();
    pdl_wait_previous();
    double v[kSums] = {};
#pragma unroll 4
    for (int64_t j = tid; j < a.chunks; j += kChunkThreads)
#pragma unroll
        for (int k = 0; k < kSums; ++k) v[k] += __ldcg(a.w.partial + j * kSums + k);
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        v[k] = warp_sum(v[k]);
        if (lane == 0) stat_part[k][warp] = v[k];
    }
    __syncthreads();
    if (warp == 0) write_stats(a, warps_sum<kChunkThreads>(stat_part, lane), lane);
}

// ---- host ----

int64_t chunks_of(int64_t n) { return (n + kChunkTokens - 1) / kChunkTokens; }

// The parts of the scratch one after the other; its size.
int64_t lay_work(char *base, int64_t n, PolicyWork &w) {
    const int64_t c = chunks_of(n);
    int64_t at = 0;
    const auto take = [&](auto *&p, int64_t count) {
        p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at);
        at += (count * int64_t(sizeof(*p)) + 15) / 16 * 16;
    };
    take(w.slot_sum, n);
    take(w.head_sum, c);
    take(w.partial, kSums * c);
    take(w.info, c);
    take(w.slot_count, n);
    take(w.norm, 1);
    return at;
}
int64_t policy_work(int64_t n) {
    PolicyWork w;
    return n <= kFew ? 0 : lay_work(nullptr, n, w);
}

void split_border(double v, float (&b)[3]) {
    b[0] = float(v);
    if (!std::isfinite(v)) {
        b[1] = b[2] = 0.0f;
        return;
    }
    b[1] = float(v - double(b[0]));
    b[2] = float(v - double(b[0]) - double(b[1]));
}

template <int THREADS, bool SINGLE, bool SUMS>
cudaError_t launch_policy_kernel(const PolicyArgs &a, cudaStream_t stream) {
    const auto kernel = policy_kernel<THREADS, SINGLE, SUMS>;
    const size_t smem = (sizeof(ChunkShared<THREADS>) + 15) / 16 * 16 + THREADS * kE * sizeof(Piece);
    const cudaError_t e = allow_smem(kernel, smem + 4096);
    if (e != cudaSuccess) return e;
    return launch_ex(kernel, dim3(unsigned(SINGLE ? 1 : a.chunks)), dim3(THREADS), smem, stream, 1, true, a);
}

template <bool SUMS>
cudaError_t launch_policy(PolicyArgs &a, cudaStream_t stream) {
    if (a.n <= kVeryFew) return launch_policy_kernel<kVeryFew / kE, true, SUMS>(a, stream);
    if (a.n <= kFew) return launch_policy_kernel<kFew / kE, true, SUMS>(a, stream);
    cudaError_t e = launch_ex(policy_count_kernel<SUMS>, dim3(unsigned(a.chunks)), dim3(kChunkThreads), 0, stream, 1, true, a);
    if (e != cudaSuccess) return e;
    a.counted = a.chunks > kInline;
    if (a.counted) {
        e = launch_ex(policy_norm_kernel, dim3(unsigned((a.chunks + 1023) / 1024)), dim3(kChunkThreads), 0, stream, 1, true, a);
        if (e != cudaSuccess) return e;
    }
    e = launch_policy_kernel<kChunkThreads, false, SUMS>(a, stream);
    if (e != cudaSuccess) return e;
    return launch_ex(policy_stats_kernel, dim3(1), dim3(kChunkThreads), 0, stream, 1, true, a);
}

}  // namespace
}  // namespace darb

using namespace darb;

extern "C" {

darb_status_t darb_policy_loss_work(int64_t tokens, int64_t *bytes) {
    DARB_TRACE("darb_policy_loss_work");
    if (bytes == nullptr || tokens < 0) return DARB_ERR_INVALID_ARG;
    if (tokens > kMaxTokens) return DARB_ERR_UNSUPPORTED;
    *bytes = policy_work(tokens);
    return DARB_OK;
}

darb_status_t darb_policy_loss(int64_t tokens, int64_t sequences, const float *logprob, const float *old_logprob,
                               const float *ref_logprob, const float *entropy, const uint8_t *mask, const float *advantage,
                               const int64_t *offsets, double clip_low, double clip_high, double kl_coef,
                               double entropy_coef, darb_per_t ratio, darb_per_t mean, float *stats, float *d_logprob,
                               float *d_entropy, void *work, cudaStream_t stream) {
    DARB_TRACE("darb_policy_loss");
    if (tokens < 0 || sequences < 0 || stats == nullptr || offsets == nullptr) return DARB_ERR_INVALID_ARG;
    if ((ratio != DARB_PER_TOKEN && ratio != DARB_PER_SEQUENCE) || (mean != DARB_PER_TOKEN && mean != DARB_PER_SEQUENCE)) return DARB_ERR_INVALID_ARG;
    // (the kernels get the coefficients in 32 bits)
    if (!(clip_low >= 0.0 && clip_low <= 1.0) || !(clip_high >= 0.0) || !std::isfinite(float(kl_coef)) || !std::isfinite(float(entropy_coef)))
        return DARB_ERR_INVALID_ARG;
    if (tokens > 0 && (logprob == nullptr || old_logprob == nullptr || d_logprob == nullptr)) return DARB_ERR_INVALID_ARG;
    if (sequences > 0 && advantage == nullptr) return DARB_ERR_INVALID_ARG;
    if (tokens > 0 && ((kl_coef != 0.0 && ref_logprob == nullptr) || (entropy == nullptr && (entropy_coef != 0.0 || d_entropy != nullptr))))
        return DARB_ERR_INVALID_ARG;
    if (tokens > kMaxTokens || sequences > kMaxTokens) return DARB_ERR_UNSUPPORTED;
    for (const void *p : {static_cast<const void *>(logprob), static_cast<const void *>(old_logprob), static_cast<const void *>(ref_logprob),
                          static_cast<const void *>(entropy), static_cast<const void *>(advantage), static_cast<const void *>(stats),
                          static_cast<const void *>(d_logprob), static_cast<const void *>(d_entropy)})
        if (!aligned_to(p, 4)) return DARB_ERR_INVALID_ARG;
    if (!aligned_to(offsets, 8) || !aligned_to(work, 16)) return DARB_ERR_INVALID_ARG;
    const int64_t need = policy_work(tokens), v = tokens * 4;
    const Range ins[] = {{logprob, v}, {old_logprob, v}, {ref_logprob, v}, {entropy, v}, {mask, tokens}, {advantage, sequences * 4}, {offsets, (sequences + 1) * 8}};
    const Range outs[] = {{stats, kStats * 4}, {d_logprob, v}, {d_entropy, v}, {work, need}};
    if (!outputs_apart(outs, ins)) return DARB_ERR_INVALID_ARG;

    PolicyArgs a = {};
    a.logprob = logprob, a.old = old_logprob, a.ref = ref_logprob, a.entropy = entropy, a.advantage = advantage;
    a.mask = mask, a.offsets = offsets, a.stats = stats, a.d_logprob = d_logprob, a.d_entropy = d_entropy;
    a.n = tokens, a.sequences = sequences, a.chunks = chunks_of(tokens);
    a.log_low = std::log1p(-clip_low), a.log_high = std::log1p(clip_high);
    split_border(a.log_low, a.low);
    split_border(a.log_high, a.high);
    a.used_low = float(1.0 - clip_low), a.used_high = float(1.0 + clip_high);
    a.kl_coef = float(kl_coef), a.entropy_coef = float(entropy_coef);
    a.per_sequence = mean == DARB_PER_SEQUENCE;
    a.vector = aligned_to(mask, 8);
    for (const float *p : {logprob, old_logprob, ref_logprob, entropy, static_cast<const float *>(d_logprob), static_cast<const float *>(d_entropy)})
        a.vector = a.vector && aligned_to(p, 16);
    return enqueue([&] {
        void *mine = nullptr;
        if (need > 0 && work == nullptr) {
            const cudaError_t e = stream_alloc(&mine, size_t(need), stream);
            if (e != cudaSuccess) return e;
        }
        lay_work(static_cast<char *>(work != nullptr ? work : mine), tokens, a.w);
        cudaError_t e = ratio == DARB_PER_SEQUENCE ? launch_policy<true>(a, stream) : launch_policy<false>(a, stream);
        if (mine != nullptr) {
            const cudaError_t f = cudaFreeAsync(mine, stream);
            if (e == cudaSuccess) e = f;
        }
        return e;
    });
}

}  // extern "C"
