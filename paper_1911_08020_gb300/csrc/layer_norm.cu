// layer_norm.cu -- layer norm over the features of each token and its backward
// pass with the gradients of gain and offset (darb_layer_norm,
// darb_layer_norm_grad): the normalisation between the layers that this library
// multiplies, in both layouts of their activations.
//
//   xh = (x - mean) rstd,  y = xh gamma + beta
//   dx = rstd (g - sum(g) / F - xh sum(g xh) / F),  g = dy gamma
//   dgamma = sum over tokens dy xh,  dbeta = sum over tokens dy
//
// Both passes are bound by memory: x (and dy) are read once, y (or dx) written
// once, and a token stays in registers between its sums and its output.
//
// Token rows.  A row is read as granules (tokens.cuh) by the threads of a CTA,
// VPT granules a thread.  The CTAs are persistent and take rows a multiple of 8
// apart, so that all rows of a CTA start alike past a 16-byte boundary whatever
// the leading dimension: a thread then owns the same features in every row, and
// keeps their gamma and beta, and in the backward pass their sums over its
// rows, in registers.  Those sums go to scratch once at the end, one partial
// result a CTA, and a second small kernel adds them in a fixed order.  Rows
// arrive through a ring of bulk copies in shared memory: the bytes in flight do
// not depend on how many registers the threads leave for occupancy.
//
// Token columns.  A CTA takes a tile of CT tokens of a step and a share of the
// features; thread = (slot, token), so that a row of the tile is one contiguous
// run, and a thread reads kColBatch of its rows at a time.  The CTAs of a cluster
// share a tile and exchange their sums once through distributed shared memory.
// A share of one batch a thread stays in registers between the sums and the
// output; larger ones are read again, from L1 or L2.
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
cudaError_t stream_alloc(void **p, size_t bytes, cudaStream_t stream);

namespace {

struct NormArgs {
    const void *x, *dy;
    void *out;              // y or dx
    int64_t ld_x, ld_dy, ld_out;
    int64_t steps, tokens;
    int32_t features;
    const float *gamma, *beta;   // or null
    float eps;
    float *mean, *rstd;          // forward: written (or null); backward: read
    float *partial;              // backward: scratch, [partials][2][partial_width], or null
};

// Floats of one half of a partial result: the features, moved by less than a
// granule, in whole granules.
__host__ __device__ __forceinline__ int64_t partial_width(int32_t features) { return (int64_t(features) + 7 + 7) / 8 * 8; }

__device__ __forceinline__ float gamma_at(const NormArgs &a, int32_t f) { return a.gamma ? __ldg(a.gamma + f) : 1.0f; }
__device__ __forceinline__ float beta_at(const NormArgs &a, int32_t f) { return a.beta ? __ldg(a.beta + f) : 0.0f; }
__device__ __forceinline__ float inverse_root(float v) { return __fdiv_rn(1.0f, __fsqrt_rn(v)); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

constexpr int kSumWarps = 16;   // warps of a CTA that shares a sum, at most

// The sums of N values over the threads of the CTA; every thread gets them.
// buf: 2 x N x kSumWarps floats of shared memory, zeros at first; its halves are
// used in turn, so that one barrier a call is enough.
template <int N>
__device__ __forceinline__ void cta_sum(float (&v)[N], float *buf, int &turn) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    const int warps = int(blockDim.x) >> 5;
    if (warps == 1) {
        __syncwarp();
        return;
    }
    float *b = buf + turn * (N * kSumWarps);
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) b[i * kSumWarps + (threadIdx.x >> 5)] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float4 q = *reinterpret_cast<const float4 *>(b + i * kSumWarps);
        v[i] = (q.x + q.y) + (q.z + q.w);
        for (int w = 4; w < warps; w += 4) {
            const float4 p = *reinterpret_cast<const float4 *>(b + i * kSumWarps + w);
            v[i] += (p.x + p.y) + (p.z + p.w);
        }
    }
}
__device__ __forceinline__ void clear_sums(float *buf, int floats) {
    for (int i = threadIdx.x; i < floats; i += blockDim.x) buf[i] = 0.0f;
    __syncthreads();
}

// ---- token rows ----

// Rows of `n` values from `base` on, `ld` apart, as the ring copies them: of a
// row's granules those that lie in the tensor as a whole.  (The first of the
// first row and the last of the last can stick out of it; a granule that two
// rows share is copied for both, and each masks the other's values.)
template <typename T>
struct RowCopies {
    const T *base, *end;
    int64_t ld, count;
    int32_t n;
    __device__ RowCopies(const void *p, int64_t ld_, int64_t rows, int32_t n_)
        : base(static_cast<const T *>(p)), end(base + (rows - 1) * ld_ + n_), ld(ld_), count(rows), n(n_) {}
    // granules [c0, c1) of row r are copied; `first`: address of granule 0
    __device__ __forceinline__ const T *range(int64_t r, int &c0, int &c1) const {
        const T *row = base + r * ld;
        const int head = row_head<T>(row);
        const T *first = row - head;
        c1 = int(row_granules<T>(head, n));
        c0 = first < base ? 1 : 0;
        if (first + c1 * kPerGranule<T> > end) --c1;
        return first;
    }
    // Start the copy of row r into `stage`; returns its bytes.
    __device__ __forceinline__ uint32_t copy(int64_t r, unsigned char *stage, uint64_t *bar) const {
        int c0, c1;
        const T *first = range(r, c0, c1);
        if (c1 <= c0) return 0;
        bulk_g2s(stage + c0 * 16, first + c0 * kPerGranule<T>, uint32_t(c1 - c0) * 16, bar);
        return uint32_t(c1 - c0) * 16;
    }
    __device__ __forceinline__ uint32_t bytes(int64_t r) const {
        int c0, c1;
        range(r, c0, c1);
        return c1 > c0 ? uint32_t(c1 - c0) * 16 : 0;
    }
};

// The granules of a thread: for every row of a CTA at the same features.
template <typename T, int VPT>
struct Owned {
    static constexpr int V = kPerGranule<T>;
    int32_t f0;        // first feature of granule u: f0 + u * step
    int32_t step, n;
    __device__ __forceinline__ int32_t feature(int u) const { return f0 + u * step; }
    __device__ __forceinline__ bool whole(int u) const { return feature(u) >= 0 && feature(u) + V <= n; }
    __device__ __forceinline__ bool partial(int u) const { return !whole(u) && feature(u) < n; }   // (else: past the row)
    __device__ __forceinline__ bool in(int u, int e) const { return feature(u) + e >= 0 && feature(u) + e < n; }

    // The granules of a row as pairs, 0 outside the row.  `stage`: this thread's
    // granule 0 of the row as copied.
    __device__ __forceinline__ void load(const RowCopies<T> &rows, int64_t r, const unsigned char *stage, bool arrived,
                                         Pair (&v)[VPT][V / 2]) const {
        const bool inner = r >= 8 && r + 8 < rows.count;   // all its granules are copied: 8 values are 16 bytes or more
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
            if (whole(u)) {
                unpack(*reinterpret_cast<const uint4 *>(stage + u * step * int(sizeof(T))), v[u]);
            } else if (inner || !partial(u)) {
                if (partial(u)) unpack(*reinterpret_cast<const uint4 *>(stage + u * step * int(sizeof(T))), v[u]);
                clear_outside(u, v[u]);
            } else {
                unpack(load_granule<T, false>(rows.base + r * rows.ld, feature(u), n, 0.0f), v[u]);
            }
        }
        if (!arrived) v[0][0] = both(__uint_as_float(0x7FC00000u));   // a copy that never came: the row is NaN
    }
    __device__ __forceinline__ void clear_outside(int u, Pair (&v)[V / 2]) const {
        if (!partial(u)) {
#pragma unroll
            for (int e = 0; e < V / 2; ++e) v[e] = both(0.0f);
            return;
        }
#pragma unroll
        for (int e = 0; e < V; e += 2) v[e / 2] = pair(in(u, e) ? low(v[e / 2]) : 0.0f, in(u, e + 1) ? high(v[e / 2]) : 0.0f);
    }
    __device__ __forceinline__ void store(T *row, const Pair (&v)[VPT][V / 2]) const {
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
            if (whole(u)) {
                *reinterpret_cast<uint4 *>(row + feature(u)) = pack(v[u]);
            } else if (partial(u)) {
                float w[V];
#pragma unroll
                for (int e = 0; e < V; e += 2) w[e] = low(v[u][e / 2]), w[e + 1] = high(v[u][e / 2]);
                store_granule(row, feature(u), n, w);
            }
        }
    }
    // Values of a vector over the features (null: `none`), 0 outside.
    __device__ __forceinline__ void gather(const float *p, float none, Pair (&v)[VPT][V / 2]) const {
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
            if (p != nullptr && whole(u) && (reinterpret_cast<uintptr_t>(p + feature(u)) & 15) == 0) {
#pragma unroll
                for (int e = 0; e < V; e += 4) {
                    const float4 q = __ldg(reinterpret_cast<const float4 *>(p + feature(u) + e));
                    v[u][e / 2] = pair(q.x, q.y);
                    v[u][e / 2 + 1] = pair(q.z, q.w);
                }
            } else {
                const auto at = [&](int e) { return !in(u, e) ? 0.0f : p == nullptr ? none : __ldg(p + feature(u) + e); };
#pragma unroll
                for (int e = 0; e < V; e += 2) v[u][e / 2] = pair(at(e), at(e + 1));
            }
        }
    }
};

// Threads that share a row, at most.  Kernels for rows of up to kHalfThreads
// are held to the registers of which an SM has enough for two CTAs.
constexpr int kRowThreads = 512, kHalfThreads = 288;
constexpr int ctas_of(int most) { return most > kHalfThreads ? 1 : 2; }

// The mean first, then the squares about it, from registers: two sums over the
// CTA a row.  A wait that gives up (after a second, and once more so that the
// copy can land) makes the row NaN; the CTA then copies and waits no more.
//   8191 x 4096 bf16: 30 us (4.5 TB/s; 6.1 a row, and 6 us to start and drain)
//   2700 x 12288 fp32: 49 us (5.4 TB/s), 16384 x 1024 fp32: 24 us (5.6 TB/s)
template <typename T, int VPT, int STAGES, int MOST>
__global__ void __launch_bounds__(MOST, ctas_of(MOST)) norm_rows_kernel(const NormArgs a, int32_t stage_bytes) {
    constexpr int V = kPerGranule<T>, H = V / 2;
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ __align__(16) float buf[2 * kSumWarps];
    __shared__ uint64_t full[STAGES];
    const int t = threadIdx.x, threads = blockDim.x;
    if (t == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(&full[s], 1);
        fence_mbar_init();
    }
    pdl_wait_previous();
    pdl_launch_dependents();
    const int64_t stride = gridDim.x, r0 = blockIdx.x;
    if (r0 >= a.tokens) return;
    const int32_t n = a.features;
    const RowCopies<T> rows(a.x, a.ld_x, a.tokens, n);
    const auto issue = [&](int64_t r, int s) {
        mbar_arrive_expect_tx(&full[s], rows.bytes(r));
        rows.copy(r, ring + s * stage_bytes, &full[s]);
    };
    if (t == 0)
        for (int s = 0; s < STAGES; ++s)
            if (r0 + s * stride < a.tokens) issue(r0 + s * stride, s);
    const float inv_n = __fdiv_rn(1.0f, float(n));
    // all rows of this CTA start alike
    const Owned<T, VPT> own = {t * V - row_head<T>(rows.base + r0 * a.ld_x), threads * V, n};
    Pair gm[VPT][H], bt[VPT][H];
    own.gather(a.gamma, 1.0f, gm);
    own.gather(a.beta, 0.0f, bt);
    clear_sums(buf, 2 * kSumWarps);
    T *y = static_cast<T *>(a.out);
    int turn = 0, stage = 0;
    uint32_t parity = 0;
    bool arrived = true;
    for (int64_t r = r0; r < a.tokens; r += stride) {
        Pair v[VPT][H], s2 = both(0.0f);
        arrived = arrived && (mbar_wait(&full[stage], parity) || mbar_wait(&full[stage], parity));
        own.load(rows, r, ring + stage * stage_bytes + t * 16, arrived, v);
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
            for (int e = 0; e < H; ++e) s2 = add2(s2, v[u][e]);
        float s[1] = {across(s2)};
        cta_sum(s, buf, turn);   // every thread has read the stage
        if (t == 0 && arrived && r + STAGES * stride < a.tokens) issue(r + STAGES * stride, stage);
        if (++stage == STAGES) stage = 0, parity ^= 1;
        const float mean = s[0] * inv_n;
        s2 = both(0.0f);
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
#pragma unroll
            for (int e = 0; e < H; ++e) v[u][e] = add2(v[u][e], both(-mean));
            if (!own.whole(u)) own.clear_outside(u, v[u]);
#pragma unroll
            for (int e = 0; e < H; ++e) s2 = fma2(v[u][e], v[u][e], s2);
        }
        s[0] = across(s2);
        cta_sum(s, buf, turn);
        const float rstd = inverse_root(s[0] * inv_n + a.eps);
        if (t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
            for (int e = 0; e < H; ++e) v[u][e] = fma2(mul2(v[u][e], both(rstd)), gm[u][e], bt[u][e]);
        own.store(y + r * a.ld_out, v);
    }
}

// SUMS: the sums over the tokens in registers, 16 features a thread; in shared
// memory (of the thread that owns the features), 32; or none, 32.
//   8192 x 4096 bf16: 43 us with the kernel that adds the partial results (4.7
//   TB/s; 5.9 a row); x 4104, with a third fewer rows in flight: 61
//   sums in shared memory (in row_sums_kernel, which reads x and dy again):
//   1000 x 12000 bf16 37 us (50), 2700 x 12288 fp32 114 (127)
enum Sums { kNoSums, kRegisterSums, kSharedSums };

template <typename T, int VPT, int STAGES, int MOST, Sums SUMS>
__global__ void __launch_bounds__(MOST, ctas_of(MOST)) back_rows_kernel(const NormArgs a, int32_t stage_bytes) {
    constexpr int V = kPerGranule<T>, H = V / 2;
    constexpr bool REGISTERS = SUMS == kRegisterSums, SHARED = SUMS == kSharedSums;
    extern __shared__ __align__(16) unsigned char ring[];   // a stage: a row of x, a row of dy
    __shared__ __align__(16) float buf[2 * 2 * kSumWarps];
    __shared__ uint64_t full[STAGES];
    const int t = threadIdx.x, threads = blockDim.x;
    if (t == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(&full[s], 1);
        fence_mbar_init();
    }
    pdl_wait_previous();
    pdl_launch_dependents();
    const int32_t n = a.features, half = stage_bytes / 2;
    const RowCopies<T> xs(a.x, a.ld_x, a.tokens, n), ds(a.dy, a.ld_dy, a.tokens, n);
    const int64_t stride = gridDim.x, r0 = blockIdx.x;
    const auto issue = [&](int64_t r, int s) {
        mbar_arrive_expect_tx(&full[s], xs.bytes(r) + ds.bytes(r));
        xs.copy(r, ring + s * stage_bytes, &full[s]);
        ds.copy(r, ring + s * stage_bytes + half, &full[s]);
    };
    if (t == 0)
        for (int s = 0; s < STAGES; ++s)
            if (r0 + s * stride < a.tokens) issue(r0 + s * stride, s);
    const float inv_n = __fdiv_rn(1.0f, float(n));
    const Owned<T, VPT> own = {t * V - row_head<T>(xs.base + r0 * a.ld_x), threads * V, n};
    Pair gm[VPT][H], sg[REGISTERS ? VPT : 1][H], sb[REGISTERS ? VPT : 1][H];
    own.gather(a.gamma, 1.0f, gm);
    // granule g of the row: V sums for dgamma, V for dbeta, at 16 bytes a thread
    float4 *sums = reinterpret_cast<float4 *>(ring + STAGES * stage_bytes) + t;
    const auto place = [&](int u, int q) { return (u * (V / 2) + q) * threads; };   // q: V / 4 words of one sum, V / 4 of the other
    if constexpr (SHARED) {
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
            for (int q = 0; q < V / 2; ++q) sums[place(u, q)] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    if constexpr (REGISTERS) {
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
            for (int e = 0; e < H; ++e) sg[u][e] = sb[u][e] = both(0.0f);
    }
    clear_sums(buf, 2 * 2 * kSumWarps);
    T *dx = static_cast<T *>(a.out);
    int turn = 0, stage = 0;
    uint32_t parity = 0;
    bool arrived = true;
    float mean_next = 0.0f, rstd_next = 0.0f;
    if (r0 < a.tokens) mean_next = __ldg(a.mean + r0), rstd_next = __ldg(a.rstd + r0);
    for (int64_t r = r0; r < a.tokens; r += stride) {
        Pair xh[VPT][H], d[VPT][H], s0 = both(0.0f), s1 = both(0.0f);
        const float mean = mean_next, rstd = rstd_next;
        if (r + stride < a.tokens) mean_next = __ldg(a.mean + r + stride), rstd_next = __ldg(a.rstd + r + stride);
        arrived = arrived && (mbar_wait(&full[stage], parity) || mbar_wait(&full[stage], parity));
        const unsigned char *at = ring + stage * stage_bytes + t * 16;
        own.load(xs, r, at, arrived, xh);
        own.load(ds, r, at + half, arrived, d);   // 0 outside the row: adds nothing to any sum
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
            for (int e = 0; e < H; ++e) {
                xh[u][e] = mul2(add2(xh[u][e], both(-mean)), both(rstd));
                if constexpr (REGISTERS) {
                    sg[u][e] = fma2(d[u][e], xh[u][e], sg[u][e]);
                    sb[u][e] = add2(sb[u][e], d[u][e]);
                }
                if constexpr (SHARED) {
                    if (e % 2 == 0) {
                        float4 &g = sums[place(u, e / 2)], &b = sums[place(u, V / 4 + e / 2)];
                        const Pair x1 = mul2(add2(xh[u][e + 1], both(-mean)), both(rstd)), d0 = d[u][e], d1 = d[u][e + 1];
                        const Pair g0 = fma2(d0, xh[u][e], pair(g.x, g.y)), g1 = fma2(d1, x1, pair(g.z, g.w));
                        const Pair b0 = add2(d0, pair(b.x, b.y)), b1 = add2(d1, pair(b.z, b.w));
                        g = make_float4(low(g0), high(g0), low(g1), high(g1));
                        b = make_float4(low(b0), high(b0), low(b1), high(b1));
                    }
                }
                d[u][e] = mul2(d[u][e], gm[u][e]);
                s0 = add2(s0, d[u][e]);
                s1 = fma2(d[u][e], xh[u][e], s1);
            }
        float s[2] = {across(s0), across(s1)};
        cta_sum(s, buf, turn);   // every thread has read the stage
        if (t == 0 && arrived && r + STAGES * stride < a.tokens) issue(r + STAGES * stride, stage);
        if (++stage == STAGES) stage = 0, parity ^= 1;
        const float c0 = s[0] * inv_n, c1 = s[1] * inv_n;
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
            for (int e = 0; e < H; ++e)
                d[u][e] = mul2(fma2(xh[u][e], both(-c1), add2(d[u][e], both(-c0))), both(rstd));
        own.store(dx + r * a.ld_out, d);
    }
    if (SUMS != kNoSums && a.partial != nullptr) {
        // as the thread holds them: feature f at f + the head of this CTA's rows
        const int64_t width = partial_width(n);
        float *p = a.partial + r0 * 2 * width;
#pragma unroll
        for (int u = 0; u < VPT; ++u)
            if (own.feature(u) < n) {
                float4 *g = reinterpret_cast<float4 *>(p + (u * threads + t) * V), *b = reinterpret_cast<float4 *>(p + width + (u * threads + t) * V);
#pragma unroll
                for (int e = 0; e < H; e += 2) {
                    if constexpr (SHARED) {
                        g[e / 2] = sums[place(u, e / 2)];
                        b[e / 2] = sums[place(u, V / 4 + e / 2)];
                        continue;
                    }
                    if constexpr (!REGISTERS) continue;
                    g[e / 2] = make_float4(low(sg[u][e]), high(sg[u][e]), low(sg[u][e + 1]), high(sg[u][e + 1]));
                    b[e / 2] = make_float4(low(sb[u][e]), high(sb[u][e]), low(sb[u][e + 1]), high(sb[u][e + 1]));
                }
            }
    }
}

// dgamma and dbeta from the partial results: 32 features of one of them a CTA, or
// a cluster where features are few and partial results many, those shared by its
// warps, joined in order.  Where rows p of the kernel that made them start `base` +
// p * `step` bytes from a 16-byte boundary, feature f lies that many elements
// further.  2432 partial results of 200 features (16000 rows, fp32): the call takes
// 20.2 us with clusters of 8, 24.6 without; 704 of 700 features 8.9 and 7.7.
constexpr int kSumSplit = 8;

template <bool CLUSTER>
__global__ void __launch_bounds__(1024) sum_partials_kernel(const float *partial, int32_t partials, int32_t features,
                                                            uint32_t base, uint32_t step, uint32_t size, float *dgamma,
                                                            float *dbeta) {
    __shared__ float s[32][33], part[32];
    pdl_wait_previous();
    pdl_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const int split = CLUSTER ? int(cluster.num_blocks()) : 1, rank = CLUSTER ? int(cluster.block_rank()) : 0;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int32_t f0 = int32_t(blockIdx.x) / split * 32;
    const int64_t width = partial_width(features);
    const float *at = partial + blockIdx.y * width + f0 + lane;
    const auto value = [&](int32_t p) { return at[int64_t(p) * 2 * width + (((base + uint32_t(p) * step) & 15u) / size)]; };
    float v = 0.0f;
    if (f0 + lane < features)
        for (int32_t p = w + 32 * rank; p < partials; p += 32 * split) v += value(p);
    s[w][lane] = v;
    __syncthreads();
    v = warp_sum(s[lane][w]);   // of feature f0 + w
    if constexpr (!CLUSTER) {
        if (lane == 0 && f0 + w < features) (blockIdx.y ? dbeta : dgamma)[f0 + w] = v;
        return;
    }
    if (lane == 0) part[w] = v;
    cluster.sync();
    if (rank == 0 && threadIdx.x < 32) {
        v = 0.0f;
        for (int r = 0; r < split; ++r) v += cluster.map_shared_rank(part, r)[lane];
        if (f0 + lane < features) (blockIdx.y ? dbeta : dgamma)[f0 + lane] = v;
    }
    cluster.sync();   // its sums may still be read
}

// Rows of any length and alignment: a CTA a row, read again for every sum.
constexpr int kAnyThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kAnyThreads) norm_any_kernel(const NormArgs a) {
    __shared__ __align__(16) float buf[2 * kSumWarps];
    clear_sums(buf, 2 * kSumWarps);
    pdl_wait_previous();
    pdl_launch_dependents();
    const int64_t r = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + r * a.ld_x;
    T *y = static_cast<T *>(a.out) + r * a.ld_out;
    const int32_t n = a.features;
    int turn = 0;
    float s[1] = {0.0f};
    for (int32_t f = threadIdx.x; f < n; f += kAnyThreads) s[0] += widen(x[f]);
    cta_sum(s, buf, turn);
    const float mean = s[0] / float(n);
    s[0] = 0.0f;
    for (int32_t f = threadIdx.x; f < n; f += kAnyThreads) {
        const float c = widen(x[f]) - mean;
        s[0] = fmaf(c, c, s[0]);
    }
    cta_sum(s, buf, turn);
    const float rstd = inverse_root(s[0] / float(n) + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    for (int32_t f = threadIdx.x; f < n; f += kAnyThreads)
        y[f] = narrow<T>(fmaf((widen(x[f]) - mean) * rstd, gamma_at(a, f), beta_at(a, f)));
}

template <typename T>
__global__ void __launch_bounds__(kAnyThreads) back_any_kernel(const NormArgs a) {
    __shared__ __align__(16) float buf[2 * 2 * kSumWarps];
    clear_sums(buf, 2 * 2 * kSumWarps);
    pdl_wait_previous();
    pdl_launch_dependents();
    const int64_t r = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + r * a.ld_x, *dy = static_cast<const T *>(a.dy) + r * a.ld_dy;
    T *dx = static_cast<T *>(a.out) + r * a.ld_out;
    const int32_t n = a.features;
    const float mean = a.mean[r], rstd = a.rstd[r];
    int turn = 0;
    float s[2] = {0.0f, 0.0f};
    for (int32_t f = threadIdx.x; f < n; f += kAnyThreads) {
        const float g = widen(dy[f]) * gamma_at(a, f);
        s[0] += g;
        s[1] = fmaf(g, (widen(x[f]) - mean) * rstd, s[1]);
    }
    cta_sum(s, buf, turn);
    const float c0 = s[0] / float(n), c1 = s[1] / float(n);
    for (int32_t f = threadIdx.x; f < n; f += kAnyThreads) {
        const float xh = (widen(x[f]) - mean) * rstd;
        dx[f] = narrow<T>(rstd * (widen(dy[f]) * gamma_at(a, f) - c0 - xh * c1));
    }
}

// The sums over the tokens p, p + partials, ... of token rows that start alike,
// one partial result a blockIdx.y (a multiple of 8 in all): a thread a granule,
// for rows too long to sum where dx is made.  Runs before dx is written: dx may
// be dy.
template <typename T>
__global__ void __launch_bounds__(kAnyThreads) row_sums_kernel(const NormArgs a) {
    constexpr int V = kPerGranule<T>, H = V / 2, U = 4;
    pdl_wait_previous();
    pdl_launch_dependents();
    const int32_t n = a.features;
    const int64_t r0 = blockIdx.y, stride = gridDim.y;
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    const int head = row_head<T>(x + r0 * a.ld_x);
    const int32_t g = int32_t(blockIdx.x) * kAnyThreads + int32_t(threadIdx.x), f = g * V - head;
    if (f >= n) return;
    Pair sg[H], sb[H];
#pragma unroll
    for (int e = 0; e < H; ++e) sg[e] = sb[e] = both(0.0f);
    for (int64_t r = r0; r < a.tokens; r += U * stride) {
        uint4 qx[U], qd[U];
        float mean[U], rstd[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = r + u * stride;
            const bool in = at < a.tokens;
            qx[u] = in ? load_granule(x + at * a.ld_x, f, n, 0.0f) : make_uint4(0, 0, 0, 0);
            qd[u] = in ? load_granule(dy + at * a.ld_dy, f, n, 0.0f) : make_uint4(0, 0, 0, 0);   // 0 adds nothing
            mean[u] = in ? __ldg(a.mean + at) : 0.0f;
            rstd[u] = in ? __ldg(a.rstd + at) : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Pair xv[H], d[H];
            unpack(qx[u], xv);
            unpack(qd[u], d);
#pragma unroll
            for (int e = 0; e < H; ++e) {
                sg[e] = fma2(d[e], mul2(add2(xv[e], both(-mean[u])), both(rstd[u])), sg[e]);
                sb[e] = add2(sb[e], d[e]);
            }
        }
    }
    float *p = a.partial + r0 * 2 * partial_width(n);
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (f + e >= 0 && f + e < n) {
            p[f + e] = e & 1 ? high(sg[e / 2]) : low(sg[e / 2]);
            p[partial_width(n) + f + e] = e & 1 ? high(sb[e / 2]) : low(sb[e / 2]);
        }
}

// The same for rows that do not start alike: a thread a feature.  40000 x 300 fp32: the
// call takes 154 us, 8192 x 4096 bf16 115.
template <typename T>
__global__ void __launch_bounds__(kAnyThreads) any_sums_kernel(const NormArgs a) {
    pdl_wait_previous();
    pdl_launch_dependents();
    const int32_t f = int32_t(blockIdx.x) * kAnyThreads + int32_t(threadIdx.x), n = a.features;
    if (f >= n) return;
    const T *x = static_cast<const T *>(a.x) + f, *dy = static_cast<const T *>(a.dy) + f;
    float sg = 0.0f, sb = 0.0f;
    // (blocks of 128 tokens first, so that no chain of additions is long)
    const int64_t stride = gridDim.y;
    for (int64_t r0 = blockIdx.y; r0 < a.tokens; r0 += 128 * stride) {
        float bg = 0.0f, bb = 0.0f;
        const int64_t end = min(a.tokens, r0 + 128 * stride);
#pragma unroll 8
        for (int64_t r = r0; r < end; r += stride) {
            const float d = widen(dy[r * a.ld_dy]);
            bg = fmaf(d, (widen(x[r * a.ld_x]) - __ldg(a.mean + r)) * __ldg(a.rstd + r), bg);
            bb += d;
        }
        sg += bg;
        sb += bb;
    }
    float *p = a.partial + int64_t(blockIdx.y) * 2 * partial_width(n);
    p[f] = sg;
    p[partial_width(n) + f] = sb;
}

// ---- narrow token rows ----
//
// Rows of at most 32 granules: LANES lanes of a warp own a row, one granule
// each, so a warp takes 32 / LANES rows at a time; the next rows are loaded while
// these are summed.  Rows of a lane group are a multiple of 8 apart, as above.
// 16384 x 64 fp32: 3.8 us forward (a CTA a row took 15), 8.4 backward (27).
constexpr int kNarrowThreads = 256;

template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

template <typename T, int LANES>
__global__ void __launch_bounds__(kNarrowThreads) norm_narrow_kernel(const NormArgs a) {
    constexpr int V = kPerGranule<T>, H = V / 2, GROUPS = kNarrowThreads / LANES;
    pdl_wait_previous();
    pdl_launch_dependents();
    const int32_t n = a.features;
    const float inv_n = __fdiv_rn(1.0f, float(n));
    const int64_t stride = int64_t(gridDim.x) * GROUPS, r0 = int64_t(blockIdx.x) * GROUPS + threadIdx.x / LANES;
    const T *x = static_cast<const T *>(a.x);
    T *y = static_cast<T *>(a.out);
    const Owned<T, 1> own = {int32_t(threadIdx.x % LANES) * V - row_head<T>(x + r0 * a.ld_x), 0, n};
    Pair gm[1][H], bt[1][H];
    own.gather(a.gamma, 1.0f, gm);
    own.gather(a.beta, 0.0f, bt);
    const int64_t rounds = (a.tokens - 1) / stride + 1;   // the same for all lanes of a warp
    const auto fetch = [&](int64_t r) {
        return r < a.tokens ? load_granule<T, false>(x + r * a.ld_x, own.f0, n, 0.0f) : make_uint4(0, 0, 0, 0);
    };
    uint4 next = fetch(r0);
    int64_t r = r0;
    for (int64_t i = 0; i < rounds; ++i, r += stride) {
        Pair v[1][H];
        unpack(next, v[0]);
        if (i + 1 < rounds) next = fetch(r + stride);
        Pair s = v[0][0];
#pragma unroll
        for (int e = 1; e < H; ++e) s = add2(s, v[0][e]);
        const float mean = lanes_sum<LANES>(across(s)) * inv_n;
#pragma unroll
        for (int e = 0; e < H; ++e) v[0][e] = add2(v[0][e], both(-mean));
        if (!own.whole(0)) own.clear_outside(0, v[0]);
        s = mul2(v[0][0], v[0][0]);
#pragma unroll
        for (int e = 1; e < H; ++e) s = fma2(v[0][e], v[0][e], s);
        const float rstd = inverse_root(lanes_sum<LANES>(across(s)) * inv_n + a.eps);
        if (r < a.tokens) {
            if (threadIdx.x % LANES == 0) {
                if (a.mean) a.mean[r] = mean;
                if (a.rstd) a.rstd[r] = rstd;
            }
#pragma unroll
            for (int e = 0; e < H; ++e) v[0][e] = fma2(mul2(v[0][e], both(rstd)), gm[0][e], bt[0][e]);
            own.store(y + r * a.ld_out, v);
        }
    }
}

template <typename T, int LANES>
__global__ void __launch_bounds__(kNarrowThreads) back_narrow_kernel(const NormArgs a) {
    constexpr int V = kPerGranule<T>, H = V / 2, GROUPS = kNarrowThreads / LANES;
    __shared__ float sums[2][LANES * V];   // of the CTA's rows
    pdl_wait_previous();
    pdl_launch_dependents();
    const int32_t n = a.features;
    const float inv_n = __fdiv_rn(1.0f, float(n));
    const int group = threadIdx.x / LANES;
    const int64_t stride = int64_t(gridDim.x) * GROUPS, r0 = int64_t(blockIdx.x) * GROUPS + group;
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    T *dx = static_cast<T *>(a.out);
    const Owned<T, 1> own = {int32_t(threadIdx.x % LANES) * V - row_head<T>(x + r0 * a.ld_x), 0, n};
    Pair gm[1][H], sg[H], sb[H];
    own.gather(a.gamma, 1.0f, gm);
#pragma unroll
    for (int e = 0; e < H; ++e) sg[e] = sb[e] = both(0.0f);
    const int64_t rounds = (a.tokens - 1) / stride + 1;
    uint4 nx, nd;
    float mean_next, rstd_next;
    const auto fetch = [&](int64_t r) {
        const bool in = r < a.tokens;
        nx = in ? load_granule(x + r * a.ld_x, own.f0, n, 0.0f) : make_uint4(0, 0, 0, 0);
        nd = in ? load_granule<T, false>(dy + r * a.ld_dy, own.f0, n, 0.0f) : make_uint4(0, 0, 0, 0);   // 0 adds nothing
        mean_next = in ? __ldg(a.mean + r) : 0.0f;
        rstd_next = in ? __ldg(a.rstd + r) : 0.0f;
    };
    fetch(r0);
    int64_t r = r0;
    for (int64_t i = 0; i < rounds; ++i, r += stride) {
        Pair xh[H], d[1][H], s0 = both(0.0f), s1 = both(0.0f);
        const float mean = mean_next, rstd = rstd_next;
        unpack(nx, xh);
        unpack(nd, d[0]);
        if (i + 1 < rounds) fetch(r + stride);
#pragma unroll
        for (int e = 0; e < H; ++e) {
            xh[e] = mul2(add2(xh[e], both(-mean)), both(rstd));
            sg[e] = fma2(d[0][e], xh[e], sg[e]);
            sb[e] = add2(sb[e], d[0][e]);
            d[0][e] = mul2(d[0][e], gm[0][e]);
            s0 = add2(s0, d[0][e]);
            s1 = fma2(d[0][e], xh[e], s1);
        }
        const float c0 = lanes_sum<LANES>(across(s0)) * inv_n, c1 = lanes_sum<LANES>(across(s1)) * inv_n;
        if (r < a.tokens) {
#pragma unroll
            for (int e = 0; e < H; ++e) d[0][e] = mul2(fma2(xh[e], both(-c1), add2(d[0][e], both(-c0))), both(rstd));
            own.store(dx + r * a.ld_out, d);
        }
    }
    if (a.partial == nullptr) return;
    // the groups' sums, one after the other: a fixed order
    for (int i = threadIdx.x; i < 2 * LANES * V; i += kNarrowThreads) (&sums[0][0])[i] = 0.0f;
    __syncthreads();
    for (int k = 0; k < GROUPS; ++k) {
        if (group == k) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (own.in(0, e)) {
                    sums[0][own.f0 + e] += e & 1 ? high(sg[e / 2]) : low(sg[e / 2]);
                    sums[1][own.f0 + e] += e & 1 ? high(sb[e / 2]) : low(sb[e / 2]);
                }
        }
        __syncthreads();
    }
    float *p = a.partial + int64_t(blockIdx.x) * 2 * partial_width(n);
    for (int i = threadIdx.x; i < n; i += kNarrowThreads) p[i] = sums[0][i], p[partial_width(n) + i] = sums[1][i];
}

// ---- token columns ----

constexpr int kColThreads = 512;
constexpr int kColWarps = kColThreads / 32;
constexpr int kColBatch = 8;
constexpr int kColSplit = 8;   // CTAs that share a tile, at most

// The rows of a thread: features f0 + slot + i * SLOTS, in batches.
template <typename T, int CT>
struct ColShare {
    static constexpr int SLOTS = kColThreads / CT, U = kColBatch;
    int32_t first, end;   // features of the thread: first, first + SLOTS, ... below end
    __device__ __forceinline__ int count() const { return first < end ? (end - first + SLOTS - 1) / SLOTS : 0; }
    __device__ __forceinline__ int32_t feature(int batch, int u) const { return first + (batch * U + u) * SLOTS; }
    __device__ __forceinline__ bool full(int batch) const { return feature(batch, U - 1) < end; }
    // A batch's values of x (row f at x + f * ld; 0 past the end).
    __device__ __forceinline__ void load(const T *x, int64_t ld, int batch, float (&v)[U]) const {
        const T *p = x + int64_t(feature(batch, 0)) * ld;
        const int64_t stride = SLOTS * ld;
        if (full(batch)) {
#pragma unroll
            for (int u = 0; u < U; ++u, p += stride) v[u] = widen(*p);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u, p += stride) v[u] = feature(batch, u) < end ? widen(*p) : 0.0f;
        }
    }
    // The same of a vector over the features; null: `none`.
    __device__ __forceinline__ void load(const float *g, float none, int batch, float (&v)[U]) const {
        const float *p = g + feature(batch, 0);
        if (g == nullptr) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = none;
        } else if (full(batch)) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = __ldg(p + u * SLOTS);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = feature(batch, u) < end ? __ldg(p + u * SLOTS) : 0.0f;
        }
    }
    __device__ __forceinline__ void store(T *y, int64_t ld, int batch, const float (&v)[U]) const {
        T *p = y + int64_t(feature(batch, 0)) * ld;
        const int64_t stride = SLOTS * ld;
        if (full(batch)) {
#pragma unroll
            for (int u = 0; u < U; ++u, p += stride) *p = narrow<T>(v[u]);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u, p += stride)
                if (feature(batch, u) < end) *p = narrow<T>(v[u]);
        }
    }
};

// Latency and instructions, not memory: 1500 x 20 fp32 5.5 us, 35 steps of it
// 8.9; 60 x 10852 x 26 fp32 53 us (2.6 TB/s).
template <typename T, int CT>
__global__ void __launch_bounds__(kColThreads) norm_columns_kernel(const NormArgs a, int32_t tiles) {
    using Share = ColShare<T, CT>;
    constexpr int SLOTS = Share::SLOTS, U = Share::U;
    __shared__ float p_mean[SLOTS][CT + 1], p_m2[SLOTS][CT + 1];
    __shared__ float2 s_part[CT], s_stat[CT];   // (mean, centred squares) of this CTA; (mean, rstd) of the token
    pdl_wait_previous();
    pdl_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const int split = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = threadIdx.x % CT, slot = threadIdx.x / CT;
    const int64_t tile = blockIdx.x / split, step = tile / tiles, c = (tile % tiles) * CT + col;
    const bool in = c < a.tokens;
    const int32_t n = a.features;
    const auto start = [&](int q) { return int32_t(int64_t(n) * q / split); };
    const int32_t f0 = start(rank), f1 = start(rank + 1);
    const Share share = {f0 + slot, f1};
    // (past the last token: the last one's values, for nobody)
    const T *x = static_cast<const T *>(a.x) + step * n * a.ld_x + (in ? c : a.tokens - 1);
    T *y = static_cast<T *>(a.out) + step * n * a.ld_out + c;
    const int rows = share.count(), batches = (rows + U - 1) / U;
    // mean and centred squares of the thread's rows, a batch at a time joined to those before
    float v[U], mean = 0.0f, m2 = 0.0f;
    for (int b = 0; b < batches; ++b) {
        share.load(x, a.ld_x, b, v);
        const int have = min(U, rows - b * U);
        float s = 0.0f, q = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) s += v[u];   // 0 past the end
        const float bm = have == U ? s * (1.0f / U) : s / float(have);
        if (have == U) {
#pragma unroll
            for (int u = 0; u < U; ++u) q = fmaf(v[u] - bm, v[u] - bm, q);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) q = u < have ? fmaf(v[u] - bm, v[u] - bm, q) : q;
        }
        const float part = __fdividef(float(have), float(b * U + have)), d = bm - mean;
        mean = fmaf(d, part, mean);
        m2 += q + d * d * (float(b * U) * part);
    }
    p_mean[slot][col] = mean;
    p_m2[slot][col] = m2;
    __syncthreads();
    // a warp joins the slots of a column: the mean first, then the squares about it
    for (int k = warp; k < CT; k += kColWarps) {
        const int32_t m = f1 - f0;
        float sum = 0.0f;
        for (int s = lane; s < SLOTS; s += 32) sum = fmaf(float(s < m ? (m - s + SLOTS - 1) / SLOTS : 0), p_mean[s][k], sum);
        const float all = m > 0 ? warp_sum(sum) / float(m) : 0.0f;
        float q = 0.0f;
        for (int s = lane; s < SLOTS; s += 32) {
            const float d = p_mean[s][k] - all;
            if (s < m) q += fmaf(d * d, float((m - s + SLOTS - 1) / SLOTS), p_m2[s][k]);
        }
        q = warp_sum(q);
        if (lane == 0) s_part[k] = make_float2(all, q);
    }
    if (split > 1) cluster.sync();
    else __syncthreads();
    if (threadIdx.x < CT) {
        float sum = 0.0f, q = 0.0f;
        float2 parts[kColSplit];
#pragma unroll
        for (int r = 0; r < kColSplit; ++r)
            if (r < split) {
                parts[r] = *cluster.map_shared_rank(&s_part[threadIdx.x], r);
                sum = fmaf(parts[r].x, float(start(r + 1) - start(r)), sum);
            }
        const float all = sum / float(n);
#pragma unroll
        for (int r = 0; r < kColSplit; ++r)
            if (r < split) {
                const float d = parts[r].x - all;
                q += fmaf(d * d, float(start(r + 1) - start(r)), parts[r].y);
            }
        const float rstd = inverse_root(q / float(n) + a.eps);
        s_stat[threadIdx.x] = make_float2(all, rstd);
        if (rank == 0 && in) {   // slot 0
            if (a.mean) a.mean[step * a.tokens + c] = all;
            if (a.rstd) a.rstd[step * a.tokens + c] = rstd;
        }
    }
    __syncthreads();
    const float2 stat = s_stat[col];
    for (int b = 0; b < batches; ++b) {
        float gm[U], bt[U];
        if (batches > 1) share.load(x, a.ld_x, b, v);
        share.load(a.gamma, 1.0f, b, gm);
        share.load(a.beta, 0.0f, b, bt);
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = fmaf((v[u] - stat.x) * stat.y, gm[u], bt[u]);
        if (in) share.store(y, a.ld_out, b, v);
    }
    if (split > 1) cluster.sync();   // its sums may still be read
}

// Sums over the CT lanes of a tile of N values a lane, N a power of two: in each
// step a lane hands half of its values to the lane across and adds what it gets
// to the other half, so that N values cost about N shuffles.  Afterwards v[0],
// v[1], ... (N / CT of them, one at least) are the sums of values first, first +
// 1, ...; returns first.
template <int CT, int N>
__device__ __forceinline__ int reduce_scatter(float (&v)[N]) {
    int first = 0, m = N;
#pragma unroll
    for (int o = CT / 2; o > 0; o >>= 1) {
        const bool upper = (threadIdx.x & o) != 0;
        if (m > 1) {
            m /= 2;
#pragma unroll
            for (int i = 0; i < N / 2; ++i)
                if (i < m) {
                    const float mine = upper ? v[i + m] : v[i], other = upper ? v[i] : v[i + m];
                    v[i] = mine + __shfl_xor_sync(0xFFFFFFFFu, other, o);
                }
            first += upper ? m : 0;
        } else {
            v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], o);
        }
    }
    return first;
}

// 35 x 1500 x 20 fp32 10.0 us with the kernel that adds the partial results;
// 60 x 10852 x 26 fp32 81 us (2.5 TB/s).
template <typename T, int CT>
__global__ void __launch_bounds__(kColThreads) back_columns_kernel(const NormArgs a, int32_t tiles) {
    using Share = ColShare<T, CT>;
    constexpr int SLOTS = Share::SLOTS, U = Share::U;
    __shared__ float p_g[SLOTS][CT + 1], p_gx[SLOTS][CT + 1];
    __shared__ float2 s_part[CT], s_sum[CT];   // sums of (g, g xh): of this CTA, and of the token over F
    pdl_wait_previous();
    pdl_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const int split = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = threadIdx.x % CT, slot = threadIdx.x / CT;
    const int64_t tile = blockIdx.x / split, step = tile / tiles, c = (tile % tiles) * CT + col;
    const bool in = c < a.tokens;
    const int32_t n = a.features, f0 = int32_t(int64_t(n) * rank / split), f1 = int32_t(int64_t(n) * (rank + 1) / split);
    const Share share = {f0 + slot, f1};
    // (past the last token: the last one's values, whose dy counts as 0)
    const int64_t cc = in ? c : a.tokens - 1;
    const T *x = static_cast<const T *>(a.x) + step * n * a.ld_x + cc, *dy = static_cast<const T *>(a.dy) + step * n * a.ld_dy + cc;
    T *dx = static_cast<T *>(a.out) + step * n * a.ld_out + c;
    const float mean = a.mean[step * a.tokens + cc], rstd = a.rstd[step * a.tokens + cc];
    // (as many batches in every thread: the sums over the lanes need all of them)
    const int batches = (f1 - f0 + SLOTS * U - 1) / (SLOTS * U);
    float xv[U], dv[U], gm[U], sg = 0.0f, sgx = 0.0f;
    for (int b = 0; b < batches; ++b) {
        share.load(x, a.ld_x, b, xv);
        share.load(dy, a.ld_dy, b, dv);   // 0 past the end: adds nothing
        share.load(a.gamma, 1.0f, b, gm);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            xv[u] = (xv[u] - mean) * rstd;
            if (!in) dv[u] = 0.0f;
            const float g = dv[u] * gm[u];
            sg += g;
            sgx = fmaf(g, xv[u], sgx);
        }
        if (a.partial != nullptr) {
            // the features' sums over this tile's tokens, one partial result a tile
            float w[2 * U];
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = dv[u] * xv[u], w[U + u] = dv[u];
            const int first = reduce_scatter<CT>(w);
            float *p = a.partial + tile * 2 * partial_width(n);
#pragma unroll
            for (int i = 0; i < 2 * U / (CT < 2 * U ? CT : 2 * U); ++i) {
                const int k = first + i;
                const int32_t f = share.feature(b, k % U);
                if (f < f1) p[(k < U ? 0 : partial_width(n)) + f] = w[i];
            }
        }
    }
    p_g[slot][col] = sg;
    p_gx[slot][col] = sgx;
    __syncthreads();
    for (int k = warp; k < CT; k += kColWarps) {
        float s0 = 0.0f, s1 = 0.0f;
        for (int s = lane; s < SLOTS; s += 32) s0 += p_g[s][k], s1 += p_gx[s][k];
        s0 = warp_sum(s0), s1 = warp_sum(s1);
        if (lane == 0) s_part[k] = make_float2(s0, s1);
    }
    if (split > 1) cluster.sync();
    else __syncthreads();
    if (threadIdx.x < CT) {
        float s0 = 0.0f, s1 = 0.0f;
        float2 parts[kColSplit];
#pragma unroll
        for (int r = 0; r < kColSplit; ++r)
            if (r < split) parts[r] = *cluster.map_shared_rank(&s_part[threadIdx.x], r);
#pragma unroll
        for (int r = 0; r < kColSplit; ++r)
            if (r < split) s0 += parts[r].x, s1 += parts[r].y;
        s_sum[threadIdx.x] = make_float2(s0 / float(n), s1 / float(n));
    }
    __syncthreads();
    const float2 sum = s_sum[col];
    for (int b = 0; b < batches; ++b) {
        if (batches > 1) {
            share.load(x, a.ld_x, b, xv);
            share.load(dy, a.ld_dy, b, dv);
            share.load(a.gamma, 1.0f, b, gm);
#pragma unroll
            for (int u = 0; u < U; ++u) xv[u] = (xv[u] - mean) * rstd;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) dv[u] = rstd * (dv[u] * gm[u] - sum.x - xv[u] * sum.y);
        if (in) share.store(dx, a.ld_out, b, dv);
    }
    if (split > 1) cluster.sync();   // its sums may still be read
}

__global__ void zero_kernel(float *a, float *b, int32_t n) {
    pdl_wait_previous();
    pdl_launch_dependents();
    const int32_t i = int32_t(blockIdx.x) * 256 + int32_t(threadIdx.x);
    if (i < n) a[i] = 0.0f, b[i] = 0.0f;
}

// ---- choice of kernels ----

// Granules of a row, at most: one more where rows can start past a boundary.
template <typename T>
int64_t most_granules(const void *p, int64_t ld, int64_t rows, int64_t features) {
    const bool aligned = aligned_to(p, 16) && (rows == 1 || ld * int64_t(sizeof(T)) % 16 == 0);
    return row_granules<T>(aligned ? 0 : kPerGranule<T> - 1, features);
}

// How a persistent row kernel runs: the threads of a CTA (0: the row is too
// long for it), the CTAs (a multiple of 8, so that the rows of one start
// alike), and a stage of its ring.
struct RowPlan {
    int threads;
    int64_t grid;
    int32_t stage_bytes;
    size_t smem;
};
template <typename Kernel>
RowPlan row_plan(Kernel kernel, int64_t granules, int vpt, int most, int copies, int stages, int64_t rows, int granule_sums = 0) {
    RowPlan p = {};
    const int64_t threads = ((granules + vpt - 1) / vpt + 31) / 32 * 32;
    if (threads > most) return p;
    p.stage_bytes = int32_t(granules) * 16 * copies;
    const size_t smem = size_t(p.stage_bytes) * stages + size_t(threads) * vpt * granule_sums;
    p.smem = smem;
    // (the kernel's own shared memory counts against the limit that needs no asking)
    if (allow_smem(kernel, smem + 1024) != cudaSuccess) return p;
    const int64_t per_sm = per_device(reinterpret_cast<const void *>(kernel), int64_t(threads) << 32 | int64_t(smem), [&]() -> long long {
        int n = 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, int(threads), smem) != cudaSuccess) {
            cudaGetLastError();
            n = 0;
        }
        return n;
    });
    if (per_sm <= 0) return p;
    p.threads = int(threads);
    p.grid = std::min<int64_t>(std::max<int64_t>(8, per_sm * sm_count() / 8 * 8), (rows + 7) / 8 * 8);
    return p;
}

// Rows of up to 32 granules: calls f with the lanes of a row as a constant and
// the grid; cudaErrorNotSupported for longer rows.
template <typename F>
cudaError_t narrow_rows(const NormArgs &a, int64_t granules, F f) {
    if (granules > 32) return cudaErrorNotSupported;
    const int lanes = granules > 16 ? 32 : granules > 8 ? 16 : 8;
    const int64_t want = (a.tokens * lanes + kNarrowThreads - 1) / kNarrowThreads;
    const dim3 grid(unsigned(std::min<int64_t>(want, 4 * int64_t(sm_count()))));
    if (lanes == 32) return f(std::integral_constant<int, 32>(), grid);
    if (lanes == 16) return f(std::integral_constant<int, 16>(), grid);
    return f(std::integral_constant<int, 8>(), grid);
}

// Whether rows of `a` and `b` start alike past a 16-byte boundary.
bool alike(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t rows, size_t es) {
    return ((reinterpret_cast<uintptr_t>(a) - reinterpret_cast<uintptr_t>(b)) & 15) == 0 &&
           (rows == 1 || (lda - ldb) * int64_t(es) % 16 == 0);
}

// Tokens of a tile of token columns: 32, or fewer where there are fewer, and
// where wider tiles would leave SMs idle, down to the 32 bytes that memory
// moves at a time.
int col_tile(int64_t steps, int64_t tokens, size_t es) {
    const int sms = sm_count();
    int ct = 32;
    while (ct > 4 && (tokens <= ct / 2 || (ct * int(es) > 32 && steps * ((tokens + ct / 2 - 1) / (ct / 2)) * kColSplit <= sms)))
        ct /= 2;
    return ct;
}

// Calls f with the tile width as a constant, the tiles of a step and the CTAs
// that share a tile.
template <typename T, typename F>
cudaError_t with_col_tile(const NormArgs &a, F f) {
    const int ct = col_tile(a.steps, a.tokens, sizeof(T));
    const int64_t tiles = (a.tokens + ct - 1) / ct, all = tiles * a.steps;
    // The split with the least time, while each thread keeps half a batch of features
    // (1500 x 20: 5.5 us; with a quarter of one 6.7, with a whole one 6.0): waves of
    // clusters, two CTAs an SM, each with a fixed part and its rows, in units of a row of
    // 32 tokens (8 ns).  CTAs that share an SM are slower: 64 x 300 x 99 bf16 on 256 CTAs
    // 8.2 us, on 512 14.7; 35 x 1500 x 20 fp32 on 140 8.9, on 280 10.4; 60 x 10852 x 26 on
    // 240 53, on 480 60.  (The backward kernel and other tiles have as much room.)
    const ClusterRoom room = cluster_room(norm_columns_kernel<T, 32>, kColThreads, 0);
    static_assert(kColSplit == 8, "the clusters that room is known of");
    const auto cost = [&](int i) {
        const int64_t waves = (all + room.of[i] - 1) / room.of[i];
        const double rows = double(a.features >> i) * ct / 32;
        return double(waves) * (500 + (2 * all > room.of[i] ? 325 + 1.25 * rows : rows));
    };
    int best = 0;
    for (int i = 1; i < 4; ++i)
        if (a.features >> i >= kColBatch / 2 * kColThreads / ct && cost(i) < cost(best)) best = i;
    const int split = 1 << best;
    if (all * split > INT32_MAX) return cudaErrorNotSupported;
    const dim3 grid(unsigned(all * split));
    if (ct == 32) return f(std::integral_constant<int, 32>(), grid, unsigned(split), int32_t(tiles));
    if (ct == 16) return f(std::integral_constant<int, 16>(), grid, unsigned(split), int32_t(tiles));
    if (ct == 8) return f(std::integral_constant<int, 8>(), grid, unsigned(split), int32_t(tiles));
    return f(std::integral_constant<int, 4>(), grid, unsigned(split), int32_t(tiles));
}

template <typename T>
cudaError_t launch_norm(const NormArgs &a, darb_layout_t layout, cudaStream_t stream) {
    if (layout == DARB_TOKEN_COLUMNS)
        return with_col_tile<T>(a, [&](auto ct, dim3 grid, unsigned split, int32_t tiles) {
            return launch_ex(norm_columns_kernel<T, ct.value>, grid, dim3(kColThreads), 0, stream, split, true, a, tiles);
        });
    if (alike(a.x, a.ld_x, a.out, a.ld_out, a.tokens, sizeof(T))) {
        // 32 features a thread
        constexpr int VPT = sizeof(T) == 2 ? 4 : 8;
        const int64_t granules = most_granules<T>(a.x, a.ld_x, a.tokens, a.features);
        cudaError_t e = narrow_rows(a, granules, [&](auto lanes, dim3 grid) {
            return launch_ex(norm_narrow_kernel<T, lanes.value>, grid, dim3(kNarrowThreads), 0, stream, 1, true, a);
        });
        const auto rows = [&](auto kernel, int vpt, int most, int stages) {
            if (e != cudaErrorNotSupported) return;
            const RowPlan p = row_plan(kernel, granules, vpt, most, 1, stages, a.tokens);
            if (p.threads > 0)
                e = launch_ex(kernel, dim3(unsigned(p.grid)), dim3(p.threads), size_t(p.stage_bytes) * stages, stream, 1, true, a,
                              p.stage_bytes);
        };
        // 16 features a thread, while that leaves enough rows at a time on an SM.  bf16, with 16
        // and with 32: up to 160 threads 19531 x 1536 27.6 and 36.1 us, 12000 x 2500 33.1 and 41.1,
        // 11718 x 2560 28.0 and 33.6; from 192 on 11160 x 2688 35.0 and 32.7, 10190 x 2944
        // 32.2 and 30.6, 9375 x 3200 39.0 and 34.9, 7324 x 4096 31.2 and 27.8; but 300 x 4096 3.3
        // and 4.0.  fp32: 8000 x 4096 43 and 48.
        const bool wide = sizeof(T) == 4 || a.tokens <= 2 * int64_t(sm_count());
        rows(norm_rows_kernel<T, VPT / 2, 3, kHalfThreads>, VPT / 2, wide ? kHalfThreads : 160, 3);
        rows(norm_rows_kernel<T, VPT, 3, 256>, VPT, 256, 3);
        rows(norm_rows_kernel<T, VPT, 3, kRowThreads>, VPT, kRowThreads, 3);
        if (e != cudaErrorNotSupported) return e;
    }
    return launch_ex(norm_any_kernel<T>, dim3(unsigned(a.tokens)), dim3(kAnyThreads), 0, stream, 1, true, a);
}

// Partial results of the sums over the tokens, at most (of any kernel).
int64_t most_partials(darb_layout_t layout, int64_t steps, int64_t tokens) {
    if (layout == DARB_TOKEN_COLUMNS && tokens == 1)   // may be taken as rows
        return std::max(steps, most_partials(DARB_TOKEN_ROWS, 1, steps));
    if (layout == DARB_TOKEN_COLUMNS) {
        const int64_t ct = std::min(col_tile(steps, tokens, 2), col_tile(steps, tokens, 4));
        return steps * ((tokens + ct - 1) / ct);
    }
    return std::min<int64_t>((tokens + 63) / 64 * 64, int64_t(sm_count()) * 32);
}

template <typename T>
cudaError_t launch_back(const NormArgs &a, darb_layout_t layout, float *dgamma, float *dbeta, cudaStream_t stream) {
    cudaError_t e = cudaSuccess;
    int64_t partials = 0;
    uint32_t base = 0, step = 0;   // of the partial results' rows, in bytes
    if (layout == DARB_TOKEN_COLUMNS) {
        e = with_col_tile<T>(a, [&](auto ct, dim3 grid, unsigned split, int32_t tiles) {
            partials = a.steps * tiles;
            return launch_ex(back_columns_kernel<T, ct.value>, grid, dim3(kColThreads), 0, stream, split, true, a, tiles);
        });
    } else {
        const bool same = alike(a.x, a.ld_x, a.out, a.ld_out, a.tokens, sizeof(T)) &&
                          alike(a.x, a.ld_x, a.dy, a.ld_dy, a.tokens, sizeof(T));
        // 16 features a thread, whose sums it keeps; 32 where the sums are a kernel of their own
        constexpr int VPT = sizeof(T) == 2 ? 2 : 4;
        const int64_t granules = most_granules<T>(a.x, a.ld_x, a.tokens, a.features);
        const auto shifted = [&] {   // partial results as the threads of aligned granules hold them
            base = uint32_t(reinterpret_cast<uintptr_t>(a.x));
            step = uint32_t(a.ld_x * int64_t(sizeof(T)));
        };
        e = cudaErrorNotSupported;
        if (same)
            e = narrow_rows(a, granules, [&](auto lanes, dim3 grid) {
                partials = grid.x;
                return launch_ex(back_narrow_kernel<T, lanes.value>, grid, dim3(kNarrowThreads), 0, stream, 1, true, a);
            });
        const auto rows = [&](auto kernel, int vpt, int most, int stages) {
            if (!same || e != cudaErrorNotSupported) return;
            const RowPlan p = row_plan(kernel, granules, vpt, most, 2, stages, a.tokens);
            if (p.threads == 0) return;
            partials = p.grid;
            shifted();
            e = launch_ex(kernel, dim3(unsigned(p.grid)), dim3(p.threads), size_t(p.stage_bytes) * stages, stream, 1, true, a,
                          p.stage_bytes);
        };
        rows(back_rows_kernel<T, VPT, 3, 256, kRegisterSums>, VPT, 256, 3);
        rows(back_rows_kernel<T, VPT, 3, kHalfThreads, kRegisterSums>, VPT, kHalfThreads, 3);
        rows(back_rows_kernel<T, VPT, 3, kRowThreads, kRegisterSums>, VPT, kRowThreads, 3);
        if (same && e == cudaErrorNotSupported && a.partial != nullptr) {
            // a stage of x and dy next to the sums: two where they fit
            constexpr int STAGES = sizeof(T) == 2 ? 2 : 1;
            const auto kernel = back_rows_kernel<T, 2 * VPT, STAGES, kRowThreads, kSharedSums>;
            const RowPlan p = row_plan(kernel, granules, 2 * VPT, kRowThreads, 2, STAGES, a.tokens, kPerGranule<T> * 8);
            if (p.threads > 0) {
                partials = p.grid;
                shifted();
                e = launch_ex(kernel, dim3(unsigned(p.grid)), dim3(p.threads), p.smem, stream, 1, true, a, p.stage_bytes);
            }
        }
        if (same && e == cudaErrorNotSupported) {
            const auto kernel = back_rows_kernel<T, 2 * VPT, 2, kRowThreads, kNoSums>;
            const RowPlan p = row_plan(kernel, granules, 2 * VPT, kRowThreads, 2, 2, a.tokens);
            if (p.threads > 0) {
                e = cudaSuccess;
                if (a.partial != nullptr) {
                    const int64_t tiles = (granules + kAnyThreads - 1) / kAnyThreads;
                    partials = std::min((a.tokens + 7) / 8 * 8, std::max<int64_t>(8, 6 * int64_t(sm_count()) / tiles / 8 * 8));
                    e = launch_ex(row_sums_kernel<T>, dim3(unsigned(tiles), unsigned(partials)), dim3(kAnyThreads), 0, stream, 1, true, a);
                }
                if (e == cudaSuccess)
                    e = launch_ex(kernel, dim3(unsigned(p.grid)), dim3(p.threads), size_t(p.stage_bytes) * 2, stream, 1, true, a,
                                  p.stage_bytes);
            }
        }
        if (e == cudaErrorNotSupported) {
            e = cudaSuccess;
            if (a.partial != nullptr) {
                // (256 tokens each, 64 of them at least: neither kernel's chains of additions get long)
                partials = std::min({a.tokens, std::max<int64_t>(64, a.tokens / 256), most_partials(layout, a.steps, a.tokens)});
                e = launch_ex(any_sums_kernel<T>, dim3(unsigned((a.features + kAnyThreads - 1) / kAnyThreads), unsigned(partials)),
                              dim3(kAnyThreads), 0, stream, 1, true, a);
            }
            if (e == cudaSuccess)
                e = launch_ex(back_any_kernel<T>, dim3(unsigned(a.tokens)), dim3(kAnyThreads), 0, stream, 1, true, a);
        }
    }
    if (e == cudaSuccess && a.partial != nullptr) {
        const unsigned blocks = unsigned((a.features + 31) / 32);
        unsigned split = 1;
        if (partials > 1024)
            while (split < kSumSplit && partials > 512 * int64_t(split) && 2 * blocks * split < unsigned(sm_count())) split *= 2;
        e = launch_ex(split > 1 ? sum_partials_kernel<true> : sum_partials_kernel<false>, dim3(blocks * split, 2), dim3(1024), 0,
                      stream, split, true, static_cast<const float *>(a.partial), int32_t(partials), a.features, base, step,
                      uint32_t(sizeof(T)), dgamma, dbeta);
    }
    return e;
}

// The scratch of the backward pass: its partial results.
darb_status_t work_bytes(darb_layout_t layout, int64_t steps, int64_t tokens, int64_t features, int64_t *bytes) {
    return enqueue([&] {
        *bytes = most_partials(layout, steps, tokens) * 2 * partial_width(int32_t(features)) * int64_t(sizeof(float));
        return cudaSuccess;
    });
}

constexpr int64_t kMaxNormFeatures = int64_t(1) << 24;   // below 2^24 a count is exact in fp32

// The checks of sizes and strides that both directions share.
darb_status_t check_norm(darb_dtype_t dtype, darb_layout_t layout, int64_t steps, int64_t tokens, int64_t features) {
    if (!token_dtype(dtype) || !token_layout(layout) || steps < 0 || tokens < 0 || features <= 0) return DARB_ERR_INVALID_ARG;
    if (layout == DARB_TOKEN_ROWS && steps != 1) return DARB_ERR_INVALID_ARG;
    if (tokens > kMaxTokens || steps > kMaxTokens || features > kMaxNormFeatures) return DARB_ERR_UNSUPPORTED;
    return DARB_OK;
}
// One token a step, its features one after the other: a row a step.
bool is_rows(darb_layout_t layout, int64_t tokens, int64_t ld0, int64_t ld1, int64_t ld2) {
    return layout == DARB_TOKEN_COLUMNS && tokens == 1 && ld0 == 1 && ld1 == 1 && ld2 == 1;
}
void as_rows(NormArgs &a, darb_layout_t &layout) {
    layout = DARB_TOKEN_ROWS;
    a.tokens = a.steps;
    a.steps = 1;
    a.ld_x = a.ld_dy = a.ld_out = a.features;
}
bool good_ld(darb_layout_t layout, int64_t tokens, int64_t features, int64_t ld) {
    return ld >= (layout == DARB_TOKEN_ROWS ? features : tokens);
}

}  // namespace
}  // namespace darb

using namespace darb;

extern "C" {

darb_status_t darb_layer_norm(const void *x, darb_dtype_t dtype, darb_layout_t layout, int64_t steps, int64_t tokens,
                              int64_t features, int64_t ld_x, const float *gamma, const float *beta, float eps, void *y,
                              int64_t ld_y, float *mean, float *rstd, cudaStream_t stream) {
    DARB_TRACE("darb_layer_norm");
    darb_status_t st = check_norm(dtype, layout, steps, tokens, features);
    if (st != DARB_OK) return st;
    if (!(eps >= 0.0f) || !good_ld(layout, tokens, features, ld_x) || !good_ld(layout, tokens, features, ld_y))
        return DARB_ERR_INVALID_ARG;
    if (steps * tokens == 0) return DARB_OK;
    const size_t es = dtype_size(dtype);
    if (x == nullptr || y == nullptr || !aligned_to(x, es) || !aligned_to(y, es) || !aligned_to(gamma, 4) ||
        !aligned_to(beta, 4) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return DARB_ERR_INVALID_ARG;
    for (const int64_t ld : {ld_x, ld_y})
        if (token_span(layout, steps, tokens, features, ld) < 0) return DARB_ERR_UNSUPPORTED;
    const bool in_place = x == y && ld_x == ld_y;
    const int64_t all = steps * tokens;
    const Range outs[] = {token_range(y, layout, steps, tokens, features, ld_y, es), {mean, all * 4}, {rstd, all * 4}};
    const Range ins[] = {token_range(in_place ? nullptr : x, layout, steps, tokens, features, ld_x, es), {gamma, features * 4}, {beta, features * 4}};
    if (!outputs_apart(outs, ins)) return DARB_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = x, a.out = y, a.ld_x = ld_x, a.ld_out = ld_y, a.steps = steps, a.tokens = tokens, a.features = int32_t(features);
    a.gamma = gamma, a.beta = beta, a.eps = eps, a.mean = mean, a.rstd = rstd;
    if (is_rows(layout, tokens, ld_x, ld_y, 1)) as_rows(a, layout);
    return enqueue([&] { return dtype == DARB_BF16 ? launch_norm<__nv_bfloat16>(a, layout, stream) : launch_norm<float>(a, layout, stream); });
}

darb_status_t darb_layer_norm_grad_work(darb_layout_t layout, int64_t steps, int64_t tokens, int64_t features, int64_t *bytes) {
    DARB_TRACE("darb_layer_norm_grad_work");
    if (bytes == nullptr) return DARB_ERR_INVALID_ARG;
    const darb_status_t st = check_norm(DARB_F32, layout, steps, tokens, features);
    if (st != DARB_OK) return st;
    // (sizes that no call takes, whose scratch need not fit 64 bits)
    if (token_span(layout, steps, tokens, features, layout == DARB_TOKEN_ROWS ? features : tokens) < 0) return DARB_ERR_UNSUPPORTED;
    return work_bytes(layout, steps, tokens, features, bytes);
}

darb_status_t darb_layer_norm_grad(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, darb_dtype_t dtype,
                                   darb_layout_t layout, int64_t steps, int64_t tokens, int64_t features,
                                   const float *gamma, const float *mean, const float *rstd, void *dx, int64_t ld_dx,
                                   float *dgamma, float *dbeta, void *work, cudaStream_t stream) {
    DARB_TRACE("darb_layer_norm_grad");
    darb_status_t st = check_norm(dtype, layout, steps, tokens, features);
    if (st != DARB_OK) return st;
    if (!good_ld(layout, tokens, features, ld_dy) || !good_ld(layout, tokens, features, ld_x) ||
        !good_ld(layout, tokens, features, ld_dx) || (dgamma == nullptr) != (dbeta == nullptr) || !aligned_to(dgamma, 4) ||
        !aligned_to(dbeta, 4))
        return DARB_ERR_INVALID_ARG;
    if (steps * tokens == 0) {
        if (dgamma == nullptr) return DARB_OK;
        if (ranges_overlap(dgamma, features * 4, dbeta, features * 4)) return DARB_ERR_INVALID_ARG;
        return enqueue([&] {
            return launch_ex(zero_kernel, dim3(unsigned((features + 255) / 256)), dim3(256), 0, stream, 1, true, dgamma, dbeta,
                             int32_t(features));
        });
    }
    const size_t es = dtype_size(dtype);
    if (dy == nullptr || x == nullptr || dx == nullptr || mean == nullptr || rstd == nullptr || !aligned_to(dy, es) ||
        !aligned_to(x, es) || !aligned_to(dx, es) || !aligned_to(gamma, 4) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return DARB_ERR_INVALID_ARG;
    if (dgamma != nullptr && !aligned_to(work, 16)) return DARB_ERR_INVALID_ARG;
    for (const int64_t ld : {ld_dy, ld_x, ld_dx})
        if (token_span(layout, steps, tokens, features, ld) < 0) return DARB_ERR_UNSUPPORTED;
    const bool in_place = dx == dy && ld_dx == ld_dy;
    const int64_t all = steps * tokens;
    int64_t scratch = 0;
    st = work_bytes(layout, steps, tokens, features, &scratch);
    if (st != DARB_OK) return st;
    const Range outs[] = {token_range(dx, layout, steps, tokens, features, ld_dx, es), {dgamma, features * 4}, {dbeta, features * 4},
                          {dgamma ? work : nullptr, scratch}};
    const Range ins[] = {token_range(in_place ? nullptr : dy, layout, steps, tokens, features, ld_dy, es),
                         token_range(x, layout, steps, tokens, features, ld_x, es), {gamma, features * 4}, {mean, all * 4}, {rstd, all * 4}};
    if (!outputs_apart(outs, ins)) return DARB_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = x, a.dy = dy, a.out = dx, a.ld_x = ld_x, a.ld_dy = ld_dy, a.ld_out = ld_dx;
    a.steps = steps, a.tokens = tokens, a.features = int32_t(features), a.gamma = gamma;
    a.mean = const_cast<float *>(mean), a.rstd = const_cast<float *>(rstd);
    a.partial = dgamma ? static_cast<float *>(work) : nullptr;
    if (is_rows(layout, tokens, ld_x, ld_dy, ld_dx)) as_rows(a, layout);
    const bool borrow = dgamma != nullptr && work == nullptr;
    return enqueue([&] {
        cudaError_t e = cudaSuccess;
        if (borrow) {
            e = stream_alloc(reinterpret_cast<void **>(&a.partial), size_t(scratch), stream);
            if (e != cudaSuccess) return e;
        }
        e = dtype == DARB_BF16 ? launch_back<__nv_bfloat16>(a, layout, dgamma, dbeta, stream)
                               : launch_back<float>(a, layout, dgamma, dbeta, stream);
        if (borrow) {
            const cudaError_t f = cudaFreeAsync(a.partial, stream);
            if (e == cudaSuccess) e = f;
        }
        return e;
    });
}

}  // extern "C"
