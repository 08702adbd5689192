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
// Token rows.  A row is read as granules (tokens.cuh).  A group of threads
// (GROUP) owns a row, VPT granules a thread; the CTAs are persistent and take
// rows a multiple of 8 apart, so that all rows of a group start alike past a
// 16-byte boundary whatever the leading dimension: a thread then owns the same
// features in every row, and keeps their gamma and beta, and in the backward
// pass their sums over its rows, in registers.  Those sums go to scratch once
// at the end, one partial result a group, and a second small kernel adds them
// in a fixed order.
//
// Token columns.  A CTA takes 32 tokens of a step and a share of the features,
// lane = token; the CTAs of a cluster share a tile and exchange their sums
// through distributed shared memory.
#include "launch.cuh"
#include "tma.cuh"
#include "tokens.cuh"
#include "trace.h"

#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

namespace cg = cooperative_groups;

namespace darb {

int sm_count();

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
    float *partial;              // backward: scratch, [partials][2][features], or null
};

__device__ __forceinline__ float gamma_at(const NormArgs &a, int32_t f) { return a.gamma ? __ldg(a.gamma + f) : 1.0f; }
__device__ __forceinline__ float beta_at(const NormArgs &a, int32_t f) { return a.beta ? __ldg(a.beta + f) : 0.0f; }
__device__ __forceinline__ float inverse_root(float v) { return __fdiv_rn(1.0f, __fsqrt_rn(v)); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// The sums of N values over the threads of a group (a warp, or the CTA); every
// thread gets them.  buf: 2 x N x 32 floats of shared memory, its halves used
// in turn so that one barrier a call is enough.
template <int GROUP, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float *buf, int &turn) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    if constexpr (GROUP > 32) {
        constexpr int W = GROUP / 32;
        float *b = buf + (turn & 1) * (N * 32);
        turn ^= 1;
        const int lane = threadIdx.x & 31;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) b[i * 32 + (threadIdx.x >> 5)] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = warp_sum(lane < W ? b[i * 32 + lane] : 0.0f);
    }
}

// ---- token rows ----

template <int GROUP>
struct RowsOf {
    static constexpr int kPerCta = GROUP == 32 ? 8 : 1;   // rows at a time
    static constexpr int kThreads = GROUP * kPerCta;
};

template <typename T, int GROUP, int VPT>
__global__ void __launch_bounds__(RowsOf<GROUP>::kThreads) norm_rows_kernel(const NormArgs a) {
    constexpr int V = kPerGranule<T>, PER = RowsOf<GROUP>::kPerCta;
    __shared__ float buf[2 * 32];
    pdl_wait_previous();
    pdl_launch_dependents();
    const int t = threadIdx.x % GROUP;
    const int32_t n = a.features;
    const float inv_n = __fdiv_rn(1.0f, float(n));
    int turn = 0;
    const int64_t stride = int64_t(gridDim.x) * PER;
    int64_t r = int64_t(blockIdx.x) * PER + threadIdx.x / GROUP;
    if (r >= a.tokens) return;
    const T *x = static_cast<const T *>(a.x);
    T *y = static_cast<T *>(a.out);
    const int head = row_head<T>(x + r * a.ld_x);   // of every row of this group
    float gm[VPT][V], bt[VPT][V];
#pragma unroll
    for (int u = 0; u < VPT; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int32_t f = (u * GROUP + t) * V - head + e;
            const bool in = f >= 0 && f < n;
            gm[u][e] = in ? gamma_at(a, f) : 0.0f;
            bt[u][e] = in ? beta_at(a, f) : 0.0f;
        }
    uint4 next[VPT];
#pragma unroll
    for (int u = 0; u < VPT; ++u)
        next[u] = load_granule<T, false>(x + r * a.ld_x, (u * GROUP + t) * V - head, n, 0.0f);
    for (; r < a.tokens; r += stride) {
        float v[VPT][V];
#pragma unroll
        for (int u = 0; u < VPT; ++u) unpack(next[u], v[u]);
        if (r + stride < a.tokens) {
#pragma unroll
            for (int u = 0; u < VPT; ++u)
                next[u] = load_granule<T, false>(x + (r + stride) * a.ld_x, (u * GROUP + t) * V - head, n, 0.0f);
        }
        float s[1] = {0.0f};
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] += v[u][e];   // 0 outside the row
        group_sum<GROUP>(s, buf, turn);
        const float mean = s[0] * inv_n;
        s[0] = 0.0f;
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int32_t f = (u * GROUP + t) * V - head + e;
                const float c = v[u][e] - mean;
                v[u][e] = c;
                s[0] += f >= 0 && f < n ? c * c : 0.0f;
            }
        group_sum<GROUP>(s, buf, turn);
        const float rstd = inverse_root(s[0] * inv_n + a.eps);
        if (t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[u][e] = fmaf(v[u][e] * rstd, gm[u][e], bt[u][e]);
            store_granule(y + r * a.ld_out, (u * GROUP + t) * V - head, n, v[u]);
        }
    }
}

template <typename T, int GROUP, int VPT>
__global__ void __launch_bounds__(RowsOf<GROUP>::kThreads) back_rows_kernel(const NormArgs a) {
    constexpr int V = kPerGranule<T>, PER = RowsOf<GROUP>::kPerCta;
    __shared__ float buf[2 * 2 * 32];
    pdl_wait_previous();
    pdl_launch_dependents();
    const int t = threadIdx.x % GROUP;
    const int32_t n = a.features;
    const float inv_n = __fdiv_rn(1.0f, float(n));
    int turn = 0;
    const int64_t stride = int64_t(gridDim.x) * PER;
    const int64_t group = int64_t(blockIdx.x) * PER + threadIdx.x / GROUP;
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    T *dx = static_cast<T *>(a.out);
    const int head = row_head<T>(x + group * a.ld_x);
    float gm[VPT][V], sg[VPT][V], sb[VPT][V];
#pragma unroll
    for (int u = 0; u < VPT; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int32_t f = (u * GROUP + t) * V - head + e;
            gm[u][e] = f >= 0 && f < n ? gamma_at(a, f) : 0.0f;
            sg[u][e] = sb[u][e] = 0.0f;
        }
    uint4 nx[VPT], nd[VPT];
    float mean_next = 0.0f, rstd_next = 0.0f;
    const auto fetch = [&](int64_t r) {
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
            nx[u] = load_granule<T>(x + r * a.ld_x, (u * GROUP + t) * V - head, n, 0.0f);
            nd[u] = load_granule<T, false>(dy + r * a.ld_dy, (u * GROUP + t) * V - head, n, 0.0f);
        }
        mean_next = __ldg(a.mean + r);
        rstd_next = __ldg(a.rstd + r);
    };
    if (group < a.tokens) fetch(group);
    for (int64_t r = group; r < a.tokens; r += stride) {
        float xh[VPT][V], d[VPT][V];
        const float mean = mean_next, rstd = rstd_next;
#pragma unroll
        for (int u = 0; u < VPT; ++u) unpack(nx[u], xh[u]), unpack(nd[u], d[u]);
        if (r + stride < a.tokens) fetch(r + stride);
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int32_t f = (u * GROUP + t) * V - head + e;
                xh[u][e] = f >= 0 && f < n ? (xh[u][e] - mean) * rstd : 0.0f;
                sg[u][e] = fmaf(d[u][e], xh[u][e], sg[u][e]);
                sb[u][e] += d[u][e];
                d[u][e] *= gm[u][e];
                s[0] += d[u][e];
                s[1] = fmaf(d[u][e], xh[u][e], s[1]);
            }
        group_sum<GROUP>(s, buf, turn);
        const float c0 = s[0] * inv_n, c1 = s[1] * inv_n;
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
#pragma unroll
            for (int e = 0; e < V; ++e) d[u][e] = rstd * (d[u][e] - c0 - xh[u][e] * c1);
            store_granule(dx + r * a.ld_out, (u * GROUP + t) * V - head, n, d[u]);
        }
    }
    if (a.partial != nullptr) {
        float *p = a.partial + group * 2 * int64_t(n);
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int32_t f = (u * GROUP + t) * V - head + e;
                if (f >= 0 && f < n) p[f] = sg[u][e], p[n + f] = sb[u][e];
            }
    }
}

// out[i] = sum over p of partial[p][i], i in [0, 2F): 32 values a CTA, the
// partial results shared by its warps, joined in order.
__global__ void __launch_bounds__(1024) sum_partials_kernel(const float *partial, int32_t partials, int32_t features,
                                                            float *dgamma, float *dbeta) {
    __shared__ float s[32][33];
    pdl_wait_previous();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t width = 2 * int64_t(features), i = int64_t(blockIdx.x) * 32 + lane;
    float v = 0.0f;
    if (i < width)
        for (int32_t p = w; p < partials; p += 32) v += partial[p * width + i];
    s[w][lane] = v;
    __syncthreads();
    v = warp_sum(s[lane][w]);   // of value blockIdx.x * 32 + w
    const int64_t j = int64_t(blockIdx.x) * 32 + w;
    if (lane == 0 && j < width) (j < features ? dgamma + j : dbeta + (j - features))[0] = v;
}

// Rows of any length and alignment: a CTA a row, read again for every sum.
constexpr int kAnyThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kAnyThreads) norm_any_kernel(const NormArgs a) {
    __shared__ float buf[2 * 32];
    pdl_wait_previous();
    pdl_launch_dependents();
    const int64_t r = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + r * a.ld_x;
    T *y = static_cast<T *>(a.out) + r * a.ld_out;
    const int32_t n = a.features;
    int turn = 0;
    float s[1] = {0.0f};
    for (int32_t f = threadIdx.x; f < n; f += kAnyThreads) s[0] += widen(x[f]);
    group_sum<kAnyThreads>(s, buf, turn);
    const float mean = s[0] / float(n);
    s[0] = 0.0f;
    for (int32_t f = threadIdx.x; f < n; f += kAnyThreads) {
        const float c = widen(x[f]) - mean;
        s[0] = fmaf(c, c, s[0]);
    }
    group_sum<kAnyThreads>(s, buf, turn);
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
    __shared__ float buf[2 * 2 * 32];
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
    group_sum<kAnyThreads>(s, buf, turn);
    const float c0 = s[0] / float(n), c1 = s[1] / float(n);
    for (int32_t f = threadIdx.x; f < n; f += kAnyThreads) {
        const float xh = (widen(x[f]) - mean) * rstd;
        dx[f] = narrow<T>(rstd * (widen(dy[f]) * gamma_at(a, f) - c0 - xh * c1));
    }
}

// The sums over the tokens p, p + partials, ... of token rows, one partial
// result a blockIdx.y; a thread a feature.  Runs before dx is written: dx may
// be dy.
template <typename T>
__global__ void __launch_bounds__(kAnyThreads) row_sums_kernel(const NormArgs a) {
    pdl_wait_previous();
    pdl_launch_dependents();
    const int32_t f = int32_t(blockIdx.x) * kAnyThreads + int32_t(threadIdx.x), n = a.features;
    if (f >= n) return;
    const T *x = static_cast<const T *>(a.x) + f, *dy = static_cast<const T *>(a.dy) + f;
    float sg = 0.0f, sb = 0.0f;
    for (int64_t r = blockIdx.y; r < a.tokens; r += gridDim.y) {
        const float d = widen(dy[r * a.ld_dy]);
        sg = fmaf(d, (widen(x[r * a.ld_x]) - __ldg(a.mean + r)) * __ldg(a.rstd + r), sg);
        sb += d;
    }
    float *p = a.partial + int64_t(blockIdx.y) * 2 * n;
    p[f] = sg;
    p[n + f] = sb;
}

// ---- token columns ----

constexpr int kColThreads = 1024;   // 32 tokens x 32 slots
constexpr int kColWarps = kColThreads / 32;
constexpr int kColSplit = 8;        // CTAs that share a tile, at most

// Sums of N values over the slots of a column and the CTAs of the cluster, for
// the column of the thread's lane.  part: [N][32][33], sum: [N][32] floats of
// shared memory.
template <int N>
__device__ __forceinline__ void column_sum(float (&v)[N], float (*part)[32][33], float (*sum)[32], cg::cluster_group &cluster) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int split = int(cluster.num_blocks());
#pragma unroll
    for (int i = 0; i < N; ++i) part[i][warp][lane] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float s = warp_sum(part[i][lane][warp]);   // of column `warp`
        if (lane == 0) sum[i][warp] = s;
    }
    if (split > 1) cluster.sync();
    else __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float s = 0.0f;
        if (split > 1) {
            for (int q = 0; q < split; ++q) s += cluster.map_shared_rank(&sum[i][0], q)[lane];
        } else {
            s = sum[i][lane];
        }
        v[i] = s;
    }
    if (split > 1) cluster.sync();   // the sums may be written again, or the CTA leave
}

template <typename T>
__global__ void __launch_bounds__(kColThreads) norm_columns_kernel(const NormArgs a, int32_t tiles) {
    __shared__ float part[1][32][33], sum[1][32];
    pdl_wait_previous();
    pdl_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const int split = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const int lane = threadIdx.x & 31, slot = threadIdx.x >> 5;
    const int64_t tile = blockIdx.x / split, step = tile / tiles, c = (tile % tiles) * 32 + lane;
    const bool in = c < a.tokens;
    const int32_t n = a.features, f0 = int32_t(int64_t(n) * rank / split), f1 = int32_t(int64_t(n) * (rank + 1) / split);
    const T *x = static_cast<const T *>(a.x) + step * n * a.ld_x + c;
    T *y = static_cast<T *>(a.out) + step * n * a.ld_out + c;
    float s[1] = {0.0f};
    if (in)
        for (int32_t f = f0 + slot; f < f1; f += kColWarps) s[0] += widen(x[f * a.ld_x]);
    column_sum(s, part, sum, cluster);
    const float mean = s[0] / float(n);
    s[0] = 0.0f;
    if (in)
        for (int32_t f = f0 + slot; f < f1; f += kColWarps) {
            const float d = widen(x[f * a.ld_x]) - mean;
            s[0] = fmaf(d, d, s[0]);
        }
    column_sum(s, part, sum, cluster);
    const float rstd = inverse_root(s[0] / float(n) + a.eps);
    if (!in) return;
    if (rank == 0 && slot == 0) {
        if (a.mean) a.mean[step * a.tokens + c] = mean;
        if (a.rstd) a.rstd[step * a.tokens + c] = rstd;
    }
    for (int32_t f = f0 + slot; f < f1; f += kColWarps)
        y[f * a.ld_out] = narrow<T>(fmaf((widen(x[f * a.ld_x]) - mean) * rstd, gamma_at(a, f), beta_at(a, f)));
}

template <typename T>
__global__ void __launch_bounds__(kColThreads) back_columns_kernel(const NormArgs a, int32_t tiles) {
    __shared__ float part[2][32][33], sum[2][32];
    pdl_wait_previous();
    pdl_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const int split = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const int lane = threadIdx.x & 31, slot = threadIdx.x >> 5;
    const int64_t tile = blockIdx.x / split, step = tile / tiles, c = (tile % tiles) * 32 + lane;
    const bool in = c < a.tokens;
    const int32_t n = a.features, f0 = int32_t(int64_t(n) * rank / split), f1 = int32_t(int64_t(n) * (rank + 1) / split);
    const T *x = static_cast<const T *>(a.x) + step * n * a.ld_x + c, *dy = static_cast<const T *>(a.dy) + step * n * a.ld_dy + c;
    T *dx = static_cast<T *>(a.out) + step * n * a.ld_out + c;
    const float mean = in ? a.mean[step * a.tokens + c] : 0.0f, rstd = in ? a.rstd[step * a.tokens + c] : 0.0f;
    float s[2] = {0.0f, 0.0f};
    for (int32_t f = f0 + slot; f < f1; f += kColWarps) {
        const float d = in ? widen(dy[f * a.ld_dy]) : 0.0f, xh = in ? (widen(x[f * a.ld_x]) - mean) * rstd : 0.0f;
        if (a.partial != nullptr) {
            // the feature's sums over this tile's tokens, one partial result a tile
            const float sg = warp_sum(d * xh), sb = warp_sum(d);
            if (lane == 0) {
                float *p = a.partial + tile * 2 * n;
                p[f] = sg;
                p[n + f] = sb;
            }
        }
        const float g = d * gamma_at(a, f);
        s[0] += g;
        s[1] = fmaf(g, xh, s[1]);
    }
    column_sum(s, part, sum, cluster);
    if (!in) return;
    const float c0 = s[0] / float(n), c1 = s[1] / float(n);
    for (int32_t f = f0 + slot; f < f1; f += kColWarps) {
        const float xh = (widen(x[f * a.ld_x]) - mean) * rstd;
        dx[f * a.ld_out] = narrow<T>(rstd * (widen(dy[f * a.ld_dy]) * gamma_at(a, f) - c0 - xh * c1));
    }
}

__global__ void zero_kernel(float *a, float *b, int32_t n) {
    pdl_wait_previous();
    pdl_launch_dependents();
    const int32_t i = int32_t(blockIdx.x) * 256 + int32_t(threadIdx.x);
    if (i < n) a[i] = 0.0f, b[i] = 0.0f;
}

// ---- choice of kernels ----

// Threads that share a row of token rows, and granules a thread: the fewest
// threads that hold the row at `most` granules a thread (0: none do).
template <typename T>
int row_group(int64_t features, int most) {
    const int64_t granules = row_granules<T>(kPerGranule<T> - 1, features);   // at the worst alignment
    for (int g = 32; g <= 1024; g *= 2)
        if (granules <= int64_t(g) * most) return g;
    return 0;
}

// The CTAs of the persistent row kernels: a multiple of 8, so that the rows of
// a group start alike.
int64_t row_grid(int64_t rows, int per_cta, int ctas_per_sm) {
    const int64_t want = (rows + per_cta - 1) / per_cta;
    const int64_t most = std::max<int64_t>(8, int64_t(sm_count()) * ctas_per_sm / 8 * 8);
    return std::min(most, (want + 7) / 8 * 8);
}

// Whether rows of `a` and `b` start alike past a 16-byte boundary.
bool alike(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t rows, size_t es) {
    return ((reinterpret_cast<uintptr_t>(a) - reinterpret_cast<uintptr_t>(b)) & 15) == 0 &&
           (rows == 1 || (lda - ldb) * int64_t(es) % 16 == 0);
}

template <typename T, int GROUP, int VPT>
cudaError_t launch_norm_group(const NormArgs &a, cudaStream_t stream) {
    using R = RowsOf<GROUP>;
    const int64_t grid = row_grid(a.tokens, R::kPerCta, std::max(1, 1536 / R::kThreads));
    return launch_ex(norm_rows_kernel<T, GROUP, VPT>, dim3(unsigned(grid)), dim3(R::kThreads), 0, stream, 1, true, a);
}
template <typename T>
constexpr int kNormVpt = sizeof(T) == 2 ? 2 : 4;

template <typename T>
cudaError_t launch_norm(const NormArgs &a, darb_layout_t layout, cudaStream_t stream) {
    constexpr int VPT = kNormVpt<T>;
    if (layout == DARB_TOKEN_COLUMNS) {
        const int64_t tiles = (a.tokens + 31) / 32, all = tiles * a.steps;
        int split = 1;
        while (split < kColSplit && all * split < sm_count() && a.features / (2 * split) >= 64) split *= 2;
        if (all * split > INT32_MAX) return cudaErrorNotSupported;
        return launch_ex(norm_columns_kernel<T>, dim3(unsigned(all * split)), dim3(kColThreads), 0, stream,
                         unsigned(split), true, a, int32_t(tiles));
    }
    const int group = alike(a.x, a.ld_x, a.out, a.ld_out, a.tokens, sizeof(T)) ? row_group<T>(a.features, VPT) : 0;
    switch (group) {
        case 32: return launch_norm_group<T, 32, VPT>(a, stream);
        case 64: return launch_norm_group<T, 64, VPT>(a, stream);
        case 128: return launch_norm_group<T, 128, VPT>(a, stream);
        case 256: return launch_norm_group<T, 256, VPT>(a, stream);
        case 512: return launch_norm_group<T, 512, VPT>(a, stream);
        case 1024: return launch_norm_group<T, 1024, VPT>(a, stream);
        default: break;
    }
    return launch_ex(norm_any_kernel<T>, dim3(unsigned(a.tokens)), dim3(kAnyThreads), 0, stream, 1, true, a);
}

// Partial results of the sums over the tokens, at most (of any kernel).
int64_t most_partials(darb_layout_t layout, int64_t steps, int64_t tokens) {
    if (layout == DARB_TOKEN_COLUMNS) return steps * ((tokens + 31) / 32);
    return std::min<int64_t>((tokens + 63) / 64 * 64, int64_t(sm_count()) * 32);
}

template <typename T, int GROUP, int VPT>
cudaError_t launch_back_group(const NormArgs &a, int64_t *partials, cudaStream_t stream) {
    using R = RowsOf<GROUP>;
    const int64_t grid = row_grid(a.tokens, R::kPerCta, std::max(1, 1024 / R::kThreads));
    *partials = grid * R::kPerCta;
    return launch_ex(back_rows_kernel<T, GROUP, VPT>, dim3(unsigned(grid)), dim3(R::kThreads), 0, stream, 1, true, a);
}

template <typename T>
cudaError_t launch_back(const NormArgs &a, darb_layout_t layout, float *dgamma, float *dbeta, cudaStream_t stream) {
    constexpr int VPT = sizeof(T) == 2 ? 1 : 2;
    cudaError_t e = cudaSuccess;
    int64_t partials = 0;
    if (layout == DARB_TOKEN_COLUMNS) {
        const int64_t tiles = (a.tokens + 31) / 32, all = tiles * a.steps;
        int split = 1;
        while (split < kColSplit && all * split < sm_count() && a.features / (2 * split) >= 64) split *= 2;
        if (all * split > INT32_MAX) return cudaErrorNotSupported;
        partials = all;
        e = launch_ex(back_columns_kernel<T>, dim3(unsigned(all * split)), dim3(kColThreads), 0, stream,
                      unsigned(split), true, a, int32_t(tiles));
    } else {
        const bool same = alike(a.x, a.ld_x, a.out, a.ld_out, a.tokens, sizeof(T)) &&
                          alike(a.x, a.ld_x, a.dy, a.ld_dy, a.tokens, sizeof(T));
        switch (same ? row_group<T>(a.features, VPT) : 0) {
            case 32: e = launch_back_group<T, 32, VPT>(a, &partials, stream); break;
            case 64: e = launch_back_group<T, 64, VPT>(a, &partials, stream); break;
            case 128: e = launch_back_group<T, 128, VPT>(a, &partials, stream); break;
            case 256: e = launch_back_group<T, 256, VPT>(a, &partials, stream); break;
            case 512: e = launch_back_group<T, 512, VPT>(a, &partials, stream); break;
            case 1024: e = launch_back_group<T, 1024, VPT>(a, &partials, stream); break;
            default:
                if (a.partial != nullptr) {
                    partials = std::min<int64_t>(a.tokens, std::min<int64_t>(64, most_partials(layout, a.steps, a.tokens)));
                    e = launch_ex(row_sums_kernel<T>, dim3(unsigned((a.features + kAnyThreads - 1) / kAnyThreads), unsigned(partials)),
                                  dim3(kAnyThreads), 0, stream, 1, true, a);
                }
                if (e == cudaSuccess)
                    e = launch_ex(back_any_kernel<T>, dim3(unsigned(a.tokens)), dim3(kAnyThreads), 0, stream, 1, true, a);
                break;
        }
    }
    if (e == cudaSuccess && a.partial != nullptr)
        e = launch_ex(sum_partials_kernel, dim3(unsigned((2 * int64_t(a.features) + 31) / 32)), dim3(1024), 0, stream, 1, true,
                      static_cast<const float *>(a.partial), int32_t(partials), a.features, dgamma, dbeta);
    return e;
}

darb_status_t status_of(cudaError_t e) {
    if (e == cudaSuccess) return DARB_OK;
    cudaGetLastError();
    return e == cudaErrorNotSupported ? DARB_ERR_UNSUPPORTED : DARB_ERR_CUDA;
}

constexpr int64_t kMaxNormFeatures = int64_t(1) << 24;   // below 2^24 a count is exact in fp32

// The checks of sizes and strides that both directions share.
darb_status_t check_norm(darb_dtype_t dtype, darb_layout_t layout, int64_t steps, int64_t tokens, int64_t features) {
    if (!token_dtype(dtype) || !token_layout(layout) || steps < 0 || tokens < 0 || features <= 0) return DARB_ERR_INVALID_ARG;
    if (layout == DARB_TOKEN_ROWS && steps != 1) return DARB_ERR_INVALID_ARG;
    if (tokens > kMaxTokens || steps > kMaxTokens || features > kMaxNormFeatures) return DARB_ERR_UNSUPPORTED;
    return DARB_OK;
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
    const int64_t nx = token_span(layout, steps, tokens, features, ld_x), ny = token_span(layout, steps, tokens, features, ld_y);
    if (nx < 0 || ny < 0) return DARB_ERR_UNSUPPORTED;
    const bool in_place = x == y && ld_x == ld_y;
    const int64_t all = steps * tokens;
    const Range outs[] = {{y, ny * int64_t(es)}, {mean, all * 4}, {rstd, all * 4}};
    const Range ins[] = {{in_place ? nullptr : x, nx * int64_t(es)}, {gamma, features * 4}, {beta, features * 4}};
    if (!outputs_apart(outs, ins)) return DARB_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = x, a.out = y, a.ld_x = ld_x, a.ld_out = ld_y, a.steps = steps, a.tokens = tokens, a.features = int32_t(features);
    a.gamma = gamma, a.beta = beta, a.eps = eps, a.mean = mean, a.rstd = rstd;
    return status_of(dtype == DARB_BF16 ? launch_norm<__nv_bfloat16>(a, layout, stream) : launch_norm<float>(a, layout, stream));
}

darb_status_t darb_layer_norm_grad_work(darb_layout_t layout, int64_t steps, int64_t tokens, int64_t features, int64_t *bytes) {
    DARB_TRACE("darb_layer_norm_grad_work");
    if (bytes == nullptr) return DARB_ERR_INVALID_ARG;
    const darb_status_t st = check_norm(DARB_F32, layout, steps, tokens, features);
    if (st != DARB_OK) return st == DARB_ERR_UNSUPPORTED ? st : DARB_ERR_INVALID_ARG;
    *bytes = most_partials(layout, steps, tokens) * 2 * features * 4;
    return DARB_OK;
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
        return status_of(launch_ex(zero_kernel, dim3(unsigned((features + 255) / 256)), dim3(256), 0, stream, 1, true, dgamma,
                                   dbeta, int32_t(features)));
    }
    const size_t es = dtype_size(dtype);
    if (dy == nullptr || x == nullptr || dx == nullptr || mean == nullptr || rstd == nullptr || !aligned_to(dy, es) ||
        !aligned_to(x, es) || !aligned_to(dx, es) || !aligned_to(gamma, 4) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return DARB_ERR_INVALID_ARG;
    if (dgamma != nullptr && (work == nullptr || !aligned_to(work, 16))) return DARB_ERR_INVALID_ARG;
    const int64_t nd = token_span(layout, steps, tokens, features, ld_dy), nx = token_span(layout, steps, tokens, features, ld_x),
                  no = token_span(layout, steps, tokens, features, ld_dx);
    if (nd < 0 || nx < 0 || no < 0) return DARB_ERR_UNSUPPORTED;
    const bool in_place = dx == dy && ld_dx == ld_dy;
    const int64_t all = steps * tokens;
    const Range outs[] = {{dx, no * int64_t(es)}, {dgamma, features * 4}, {dbeta, features * 4},
                          {dgamma ? work : nullptr, most_partials(layout, steps, tokens) * 8 * features}};
    const Range ins[] = {{in_place ? nullptr : dy, nd * int64_t(es)}, {x, nx * int64_t(es)}, {gamma, features * 4},
                         {mean, all * 4}, {rstd, all * 4}};
    if (!outputs_apart(outs, ins)) return DARB_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = x, a.dy = dy, a.out = dx, a.ld_x = ld_x, a.ld_dy = ld_dy, a.ld_out = ld_dx;
    a.steps = steps, a.tokens = tokens, a.features = int32_t(features), a.gamma = gamma;
    a.mean = const_cast<float *>(mean), a.rstd = const_cast<float *>(rstd);
    a.partial = dgamma ? static_cast<float *>(work) : nullptr;
    return status_of(dtype == DARB_BF16 ? launch_back<__nv_bfloat16>(a, layout, dgamma, dbeta, stream)
                                        : launch_back<float>(a, layout, dgamma, dbeta, stream));
}

}  // extern "C"
