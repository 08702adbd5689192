// muon.cu -- updates of weight matrices whose momentum is orthogonalised by
// Newton-Schulz products (darb_muon_create, darb_muon_step), next to darb_adamw_step.
//
//   m = beta m + (1 - beta) g',  u = (1 - beta) g' + beta m,  X = u / (|u| + eps),
//   five times  A = X X^T,  B = b A + c A A,  X = a X + B X,
//   p = p (1 - lr decay) - lr 0.2 sqrt(max(rows, cols)) X.
// With n the shorter side the products are n x n over the longer side, n x n over n,
// and n x n x the longer side.  A tall matrix takes X^T X from the right; it stays as
// it lies, because the tensor cores read either operand along either axis.  Both
// squares are symmetric: the tiles on and below the diagonal are computed and written
// twice.
//
// Operands are fp16 (11 bits; bf16's 8 would leave 1 % of X wrong).  What the bits cost
// is largest on the diagonal of A and B, whose elements outweigh the others: it is kept
// in fp32, out of the products,
//   B_ij = b A_ij + c (S_ij + (d_i + d_j) A_ij),  S = A' A' (A' without its diagonal d),
//   D_i = a + b d_i + c (S_ii + d_i^2),  X = D X + B' X,
// and X itself is held as a sum of two fp16 numbers, of which D takes both.  One product
// of the leading parts leaves X off by 5e-4 .. 1e-3 of itself (in norm), which is what
// gradients in bf16 (2^-9 each) are given; gradients in fp32 get the three products
// of both parts (A, B and X as two numbers each), as near as fp32 products come (1e-5).
// Powers of two keep all numbers in fp16's range: |X| < 2 goes in as 2^15 X, |A| < 2 as
// 2^15 A, |B'| < 4 as 2^14 B'.
//
// One launch a product for all matrices of the plan.  A CTA walks the tiles that the
// plan's schedule gives it (longest first, to the CTA that is done first): one warp
// copies boxes of 64 x 64 numbers (TMA, 128-byte swizzle), one issues tcgen05.mma
// into one of two accumulators in tensor memory, four write the tile before.
#include "launch.cuh"
#include "tcgen05.cuh"
#include "tma.cuh"
#include "tokens.cuh"
#include "trace.h"

#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <functional>
#include <mutex>
#include <new>
#include <queue>
#include <unordered_set>
#include <vector>

namespace darb {

int sm_count();

namespace {

constexpr int kIterations = 5;
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr int kPointers = 448;              // gradients of a launch
constexpr int kParts = 304;                 // CTAs of a matrix in the elementwise kernels, at most
constexpr int kPartElems = 4096;            // elements of one, at least
constexpr int kElemThreads = 256;
constexpr int64_t kMaxSide = 32768;         // rows and columns: elements fit 32 bits

constexpr int kBM = 128, kBK = 64;          // rows of a tile; depth of a stage
constexpr int kBox = 64 * 64 * 2;           // bytes of a box
constexpr int kGemmThreads = 192;           // copies, products, four warps that write
constexpr float kScaleX = 32768.0f, kScaleB = 16384.0f;

// One matrix of a plan.
struct alignas(128) Matrix {
    CUtensorMap x[2][2], a[2], b[2];        // [buffer][part], [part]
    __half *xp[2][2], *ap[2], *bp[2];
    float *p, *m;
    __nv_bfloat16 *copy;
    double *partial;                        // sums of squares of the elementwise kernels' CTAs
    float *d, *D;                           // the diagonals of A and of a I + B
    int32_t rows, cols, n;                  // n: the shorter side
    int32_t ldx, lda;                       // of the fp16 numbers
    int32_t tall, parts, part_elems;
    float size;                             // 0.2 sqrt(max(rows, cols))
};
struct Part {
    int32_t matrix, part;
};
struct Tile {
    int32_t matrix, row, col;               // first row and column
};

struct StepArgs {
    const Matrix *matrices;
    const Part *parts;
    int32_t *active;                        // per matrix: has a gradient in this step
    const float *grad_scale;
    int32_t *status;
    float beta, rest, eps, decay, lr;       // rest: 1 - beta; decay: 1 - lr decay
    int32_t nesterov;
};
struct GradArgs {
    const void *p[kPointers];
    int32_t first, count;                   // matrices
};

__device__ __forceinline__ bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// ---- momentum, norm, and the start of X ----

__device__ __forceinline__ float direction(const StepArgs &a, float g, float m) { return a.nesterov ? a.rest * g + a.beta * m : m; }

// Elements [e0, e1) of a matrix, four at a time where `vector`: f(index, count).
template <typename F>
__device__ __forceinline__ void each_quad(int64_t e0, int64_t e1, F f) {
    for (int64_t e = e0 + int64_t(threadIdx.x) * 4; e < e1; e += kElemThreads * 4) f(int(e), int(e1 - e < 4 ? e1 - e : 4));
}

template <typename G>
__device__ __forceinline__ void load4(const G *p, int e, int count, bool vector, float (&v)[4]) {
    if (vector && count == 4) {
        if constexpr (sizeof(G) == 4) {
            const float4 q = *reinterpret_cast<const float4 *>(p + e);
            v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
        } else {
            const uint2 q = *reinterpret_cast<const uint2 *>(p + e);
            const float2 x = widen2(q.x), y = widen2(q.y);
            v[0] = x.x, v[1] = x.y, v[2] = y.x, v[3] = y.y;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < count ? widen(p[e + i]) : 0.0f;
}

__device__ __forceinline__ double block_total(double v) {
    __shared__ double part[kElemThreads / 32];
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < kElemThreads / 32; ++w) v += part[w];
    return v;
}

template <typename G>
__global__ void __launch_bounds__(kElemThreads) momentum_kernel(const StepArgs a, const __grid_constant__ GradArgs grads) {
    pdl_launch_dependents();
    const Part part = a.parts[blockIdx.x];
    const Matrix &x = a.matrices[part.matrix];
    const G *g = static_cast<const G *>(grads.p[part.matrix - grads.first]);
    pdl_wait_previous();
    if (part.part == 0 && threadIdx.x == 0) a.active[part.matrix] = g != nullptr;
    if (g == nullptr) return;
    const float scale = a.grad_scale != nullptr ? *a.grad_scale : 1.0f;
    const int64_t all = int64_t(x.rows) * x.cols, e0 = int64_t(part.part) * x.part_elems, e1 = min(e0 + x.part_elems, all);
    const bool vector = aligned16(x.m) && (reinterpret_cast<uintptr_t>(g) & (4 * sizeof(G) - 1)) == 0;
    float *const m = x.m;
    double sum = 0.0;
    each_quad(e0, e1, [&](int e, int count) {
        float gv[4], mv[4], top = 0.0f, squares = 0.0f;
        load4(g, e, count, vector, gv);
        load4(m, e, count, vector, mv);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            gv[i] *= scale;
            mv[i] = mv[i] * a.beta + gv[i] * a.rest;
            gv[i] = direction(a, gv[i], mv[i]);
            top = fmaxf(top, fabsf(gv[i]));
            squares = fmaf(gv[i], gv[i], squares);
        }
        if (vector && count == 4) {
            *reinterpret_cast<float4 *>(m + e) = make_float4(mv[0], mv[1], mv[2], mv[3]);
        } else {
            for (int i = 0; i < count; ++i) m[e + i] = mv[i];
        }
        // squares that 32 bits do not hold
        if (top > 1e15f || (top < 1e-15f && top > 0.0f)) {
            double s = 0.0;
            for (int i = 0; i < 4; ++i) s += double(gv[i]) * gv[i];
            sum += s;
        } else {
            sum += double(squares);
        }
    });
    sum = block_total(sum);
    if (threadIdx.x == 0) x.partial[part.part] = sum;
}

// v as the sum of two fp16 numbers
__device__ __forceinline__ void split(float v, __half &hi, __half &lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(v - __half2float(hi));
}

template <typename G>
__global__ void __launch_bounds__(kElemThreads) start_kernel(const StepArgs a, const __grid_constant__ GradArgs grads) {
    pdl_launch_dependents();
    const Part part = a.parts[blockIdx.x];
    const Matrix &x = a.matrices[part.matrix];
    const G *g = static_cast<const G *>(grads.p[part.matrix - grads.first]);
    pdl_wait_previous();
    if (g == nullptr) return;
    double sum = 0.0;
    for (int i = threadIdx.x; i < x.parts; i += kElemThreads) sum += x.partial[i];
    sum = block_total(sum);
    const float norm = float(sqrt(sum)) + a.eps, scale = a.grad_scale != nullptr ? *a.grad_scale : 1.0f;
    const int64_t all = int64_t(x.rows) * x.cols, e0 = int64_t(part.part) * x.part_elems, e1 = min(e0 + x.part_elems, all);
    const bool vector = aligned16(x.m) && (reinterpret_cast<uintptr_t>(g) & (4 * sizeof(G) - 1)) == 0;
    const float *const m = x.m;
    __half *const hi = x.xp[0][0], *const lo = x.xp[0][1];
    const int cols = x.cols;
    const bool quads = cols % 4 == 0;
    each_quad(e0, e1, [&](int e, int count) {
        float gv[4], mv[4];
        load4(g, e, count, vector, gv);
        load4(m, e, count, vector, mv);
        alignas(8) __half h[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) split(direction(a, gv[i] * scale, mv[i]) / norm * kScaleX, h[i], l[i]);
        int row = e / cols, col = e - row * cols;
        if (quads) {   // (then count is 4: parts are multiples of 4 elements)
            const int64_t at = int64_t(row) * x.ldx + col;
            *reinterpret_cast<uint2 *>(hi + at) = *reinterpret_cast<const uint2 *>(h);
            *reinterpret_cast<uint2 *>(lo + at) = *reinterpret_cast<const uint2 *>(l);
            return;
        }
        for (int i = 0; i < count; ++i) {
            const int64_t at = int64_t(row) * x.ldx + col;
            hi[at] = h[i], lo[at] = l[i];
            if (++col == cols) col = 0, ++row;
        }
    });
}

// ---- products ----

enum Op : int { kGram, kSquare, kApply };

// Instruction descriptor of tcgen05.mma kind::f16 with fp16 A and B and an fp32
// accumulator.
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool a_mn, bool b_mn) {
    return (1u << 4) | (uint32_t(a_mn) << 15) | (uint32_t(b_mn) << 16) | (uint32_t(N >> 3) << 17) | (uint32_t(M >> 4) << 24);
}

template <int P, int BN>
struct Geo {
    static constexpr int kParts = P == 1 ? 1 : 2;                 // fp16 numbers of an operand
    static constexpr int kABytes = kBM / 64 * kBox, kBBytes = BN / 64 * kBox;
    static constexpr int kStage = kParts * (kABytes + kBBytes);
    static constexpr int kStages = (220 * 1024) / kStage < 6 ? (220 * 1024) / kStage : 6;
    static constexpr size_t kSmem = 2048 + size_t(kStages) * kStage;
};

// The product's operands of a matrix, and how they lie.
struct Operands {
    const CUtensorMap *a, *b;   // [part]
    bool a_mn, b_mn;            // contiguous along the tile, not along the depth
    int depth;
};
template <int OP>
__device__ __forceinline__ Operands operands(const Matrix &x, int buf) {
    const int longer = x.tall ? x.rows : x.cols;
    if (OP == kGram) return {x.x[buf], x.x[buf], x.tall != 0, x.tall != 0, longer};
    if (OP == kSquare) return {x.a, x.a, false, false, x.n};
    return x.tall ? Operands{x.x[buf], x.b, false, false, x.n} : Operands{x.b, x.x[buf], false, true, x.n};
}

// 32 numbers of a row, 16 bytes at a time
__device__ __forceinline__ void store32(__half *p, const __half (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(v)[i];
}
__device__ __forceinline__ void load32(const __half *p, __half (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<uint4 *>(v)[i] = reinterpret_cast<const uint4 *>(p)[i];
}

// What becomes of 32 columns from j0 on of row i of a product.
template <int P, int OP>
__device__ __forceinline__ void finish(const StepArgs &s, const Matrix &x, int buf, bool last, int i, int j0, const uint32_t (&acc)[32]) {
    constexpr bool two = P == 3;
    if (OP != kApply) {
        const int n = x.n;
        if (i >= n || j0 > i) return;
        __half *const hi = OP == kGram ? x.ap[0] : x.bp[0], *const lo = OP == kGram ? x.ap[1] : x.bp[1];
        const int64_t at = int64_t(i) * x.lda + j0;
        const float di = OP == kSquare ? x.d[i] : 0.0f;
        alignas(16) __half ah[32], al[32];
        if (OP == kSquare) {
            load32(x.ap[0] + at, ah);
            if (two) load32(x.ap[1] + at, al);
        }
        alignas(16) __half h[32], l[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const int j = j0 + e;
            const float raw = __uint_as_float(acc[e]);
            float v = raw * (1.0f / kScaleX);
            if (OP == kSquare) {
                const float sq = raw * (1.0f / (kScaleX * kScaleX));
                const float old = (__half2float(ah[e]) + (two ? __half2float(al[e]) : 0.0f)) * (1.0f / kScaleX);
                const float dj = j <= i ? x.d[j] : 0.0f;
                v = (kB * old + kC * fmaf(di + dj, old, sq)) * kScaleB;
                if (j == i) x.D[i] = kA + kB * di + kC * fmaf(di, di, sq);
            } else if (j == i) {
                x.d[i] = raw * (1.0f / (kScaleX * kScaleX));
            }
            split(v, h[e], l[e]);
            if (j < i) {   // across the diagonal: neighbouring lanes are neighbouring places
                hi[int64_t(j) * x.lda + i] = h[e];
                if (two) lo[int64_t(j) * x.lda + i] = l[e];
            }
        }
        if (j0 + 31 < i) {
            store32(hi + at, h);
            if (two) store32(lo + at, l);
        } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                if (j0 + e >= i) continue;
                hi[at + e] = h[e];
                if (two) lo[at + e] = l[e];
            }
        }
        return;
    }
    if (i >= x.rows || j0 >= x.cols) return;
    const int64_t at = int64_t(i) * x.ldx + j0;   // (rows are as long as a multiple of 64 numbers)
    const float Di = x.tall ? 0.0f : x.D[i];
    alignas(16) __half h[32], l[32];
    load32(x.xp[buf][0] + at, h);
    load32(x.xp[buf][1] + at, l);
    float v[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) {
        const int j = min(j0 + e, x.cols - 1);
        const float D = x.tall ? x.D[j] : Di;
        v[e] = fmaf(D, (__half2float(h[e]) + __half2float(l[e])) * (1.0f / kScaleX), __uint_as_float(acc[e]) * (1.0f / (kScaleX * kScaleB)));
    }
    if (!last) {
#pragma unroll
        for (int e = 0; e < 32; ++e) split(v[e] * kScaleX, h[e], l[e]);
        store32(x.xp[buf ^ 1][0] + at, h);
        store32(x.xp[buf ^ 1][1] + at, l);
        return;
    }
    const float size = s.lr * x.size;
    const int64_t to = int64_t(i) * x.cols + j0;
    float *const p = x.p + to;
    __nv_bfloat16 *const copy = x.copy != nullptr ? x.copy + to : nullptr;
    if (j0 + 32 <= x.cols && x.cols % 4 == 0 && aligned16(x.p) && (reinterpret_cast<uintptr_t>(x.copy) & 7) == 0) {
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
            float4 q = *reinterpret_cast<float4 *>(p + e);
            q = make_float4(q.x * s.decay - size * v[e], q.y * s.decay - size * v[e + 1], q.z * s.decay - size * v[e + 2],
                            q.w * s.decay - size * v[e + 3]);
            *reinterpret_cast<float4 *>(p + e) = q;
            if (copy != nullptr) {
                const __nv_bfloat162 c0 = __floats2bfloat162_rn(q.x, q.y), c1 = __floats2bfloat162_rn(q.z, q.w);
                *reinterpret_cast<uint2 *>(copy + e) = make_uint2(*reinterpret_cast<const uint32_t *>(&c0), *reinterpret_cast<const uint32_t *>(&c1));
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 32; ++e) {
        if (j0 + e >= x.cols) continue;
        const float q = p[e] * s.decay - size * v[e];
        p[e] = q;
        if (copy != nullptr) copy[e] = __float2bfloat16_rn(q);
    }
}

// A tensor map that the host has copied to the device, before the first copy by it.
__device__ __forceinline__ void acquire_map(const CUtensorMap *map) {
    asm volatile("fence.proxy.tensormap::generic.acquire.sys [%0], 128;" ::"l"(map) : "memory");
}

// The tiles of CTA b are tiles[first[b]] .. tiles[first[b + 1] - 1].
template <int P, int BN, int OP>
__global__ void __launch_bounds__(kGemmThreads, 1) product_kernel(const StepArgs s, const Tile *tiles, const int32_t *first, int buf, int last) {
    using G = Geo<P, BN>;
    constexpr int NS = G::kStages, NP = G::kParts;
    extern __shared__ unsigned char sm_raw[];
    unsigned char *const sm = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(sm_raw) + 1023) & ~uintptr_t(1023));
    uint64_t *const full = reinterpret_cast<uint64_t *>(sm), *const empty = full + NS, *const ready = empty + NS, *const read = ready + 2,
                    *const done = read + 2;
    uint32_t *const s_tmem = reinterpret_cast<uint32_t *>(done + 1);
    unsigned char *const stages = sm + 1024;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr uint32_t kColumns = 2 * BN;

    pdl_launch_dependents();
    if (tid == 0) {
        for (int i = 0; i < NS; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&ready[i], 1), mbar_init(&read[i], 4);
        mbar_init(done, 1);
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(s_tmem, kColumns);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *s_tmem;
    const int t0 = first[blockIdx.x], t1 = first[blockIdx.x + 1];
    bool ok = true;
    pdl_wait_previous();

    if (warp == 0) {
        if (lane == 0) {
            fence_proxy_async_global();
            int stage = 0;
            uint32_t parity = 0;
            int64_t issued = 0;
            int known = -1;   // the matrix of the last tile
            for (int t = t0; t < t1 && ok; ++t) {
                const Tile tile = tiles[t];
                const Matrix &x = s.matrices[tile.matrix];
                if (!s.active[tile.matrix]) continue;
                const Operands o = operands<OP>(x, buf);
                if (tile.matrix != known) {
                    for (int q = 0; q < NP; ++q) acquire_map(&o.a[q]), acquire_map(&o.b[q]);
                    known = tile.matrix;
                }
                for (int k = 0; k < o.depth; k += kBK, ++issued) {
                    if (issued >= NS && !mbar_wait(&empty[stage], parity ^ 1u)) {
                        ok = false;
                        break;
                    }
                    mbar_arrive_expect_tx(&full[stage], G::kStage);
                    unsigned char *to = stages + stage * G::kStage;
#pragma unroll
                    for (int q = 0; q < NP; ++q)
                        for (int b = 0; b < kBM; b += 64, to += kBox)
                            tensor2d_g2s(to, &o.a[q], o.a_mn ? tile.row + b : k, o.a_mn ? k : tile.row + b, &full[stage]);
#pragma unroll
                    for (int q = 0; q < NP; ++q)
                        for (int b = 0; b < BN; b += 64, to += kBox)
                            tensor2d_g2s(to, &o.b[q], o.b_mn ? tile.col + b : k, o.b_mn ? k : tile.col + b, &full[stage]);
                    if (++stage == NS) stage = 0, parity ^= 1u;
                }
            }
            if (!ok) {   // what is still on its way lands before the CTA leaves
                for (int64_t i = issued > NS ? issued - NS : 0; i < issued; ++i) mbar_wait(&full[i % NS], uint32_t(i / NS) & 1u);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            int stage = 0, used = 0;
            uint32_t parity = 0;
            for (int t = t0; t < t1 && ok; ++t) {
                const Tile tile = tiles[t];
                const Matrix &x = s.matrices[tile.matrix];
                if (!s.active[tile.matrix]) continue;
                const Operands o = operands<OP>(x, buf);
                const uint32_t idesc = idesc_f16(kBM, BN, o.a_mn, o.b_mn);
                // along the depth: rows of 128 bytes; along the tile: boxes of 64 columns, 8 deep atoms one after the other
                const uint32_t a_lbo = o.a_mn ? kBox : 16, b_lbo = o.b_mn ? kBox : 16;
                const uint32_t a_step = (o.a_mn ? 2048 : 32) >> 4, b_step = (o.b_mn ? 2048 : 32) >> 4;
                const int half = used & 1;
                if (used >= 2 && !mbar_wait(&read[half], uint32_t(used / 2 - 1) & 1u)) {
                    ok = false;
                    break;
                }
                tc_fence_after_sync();
                const uint32_t d = tmem + half * BN;
                for (int k = 0; k < o.depth; k += kBK) {
                    if (!mbar_wait(&full[stage], parity)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after_sync();
                    const uint32_t sa = smem_addr(stages + stage * G::kStage), sb = sa + NP * G::kABytes;
                    const uint64_t ah = smem_desc(sa, a_lbo, 1024, kLayoutSw128), bh = smem_desc(sb, b_lbo, 1024, kLayoutSw128);
                    const uint64_t al = ah + (G::kABytes >> 4), bl = bh + (G::kBBytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < kBK / 16; ++kk) {
                        const uint64_t ao = kk * a_step, bo = kk * b_step;
                        mma_bf16(d, ah + ao, bh + bo, idesc, (k | kk) != 0);
                        if (P == 3) {
                            mma_bf16(d, ah + ao, bl + bo, idesc, 1u);
                            mma_bf16(d, al + ao, bh + bo, idesc, 1u);
                        }
                    }
                    mma_commit(&empty[stage]);
                    if (++stage == NS) stage = 0, parity ^= 1u;
                }
                mma_commit(&ready[half]);
                ++used;
            }
            mma_commit(done);
            if (!mbar_wait(done, 0)) ok = false;   // no product is in flight when the memory is given back
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3;
        int used = 0;
        for (int t = t0; t < t1; ++t) {
            const Tile tile = tiles[t];
            const Matrix &x = s.matrices[tile.matrix];
            if (!s.active[tile.matrix]) continue;
            const int half = used & 1;
            if (!__all_sync(~0u, mbar_wait(&ready[half], uint32_t(used / 2) & 1u))) {
                ok = false;
                break;
            }
            tc_fence_after_sync();
            const uint32_t at = tmem + half * BN + (uint32_t(quarter * 32) << 16);
            const int i = tile.row + quarter * 32 + lane;
#pragma unroll 1
            for (int c = 0; c < BN; c += 32) {
                uint32_t acc[32];
                tmem_ld32(at + c, acc);
                tmem_ld_wait();
                if (c + 32 == BN) {   // the accumulator has been read
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&read[half]);
                }
                finish<P, OP>(s, x, buf, last != 0, i, tile.col + c, acc);
            }
            ++used;
        }
    }
    if (!ok) atomicOr(s.status, kStatusTimeout);
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, kColumns);
    }
}

// ---- host ----

// The tiles of one product of all matrices, given to CTAs.
struct Schedule {
    std::vector<Tile> tiles;
    std::vector<int32_t> first;
    int bn = 0;
    int64_t longest = 0;
    int64_t o_tiles = 0, o_first = 0;   // in the plan's memory
    int32_t ctas() const { return int32_t(first.size()) - 1; }
};

// A tile costs its depth (in stages), for the width of its columns and for what a
// stage and a tile cost at any width.
int64_t tile_cost(int64_t depth, int bn) { return (depth + kBK - 1) / kBK * (bn + 32) + 6 * (bn + 32); }

Schedule make_schedule(const std::vector<Matrix> &all, Op op, int bn, int ctas) {
    struct Item {
        int64_t cost;
        Tile tile;
    };
    std::vector<Item> items;
    for (size_t t = 0; t < all.size(); ++t) {
        const Matrix &x = all[t];
        if (x.n == 0) continue;
        const int rows = op == kApply ? x.rows : x.n, cols = op == kApply ? x.cols : x.n;
        const int64_t depth = op == kGram ? std::max(x.rows, x.cols) : x.n, cost = tile_cost(depth, bn);
        for (int col = 0; col < cols; col += bn)
            for (int row = 0; row < rows; row += kBM)
                if (op == kApply || col < row + kBM) items.push_back({cost, {int32_t(t), row, col}});
    }
    std::stable_sort(items.begin(), items.end(), [](const Item &a, const Item &b) { return a.cost > b.cost; });
    Schedule s;
    s.bn = bn;
    ctas = int(std::min<int64_t>(ctas, int64_t(items.size())));
    std::vector<std::vector<Tile>> mine(ctas);
    using Load = std::pair<int64_t, int>;
    std::priority_queue<Load, std::vector<Load>, std::greater<Load>> queue;
    for (int c = 0; c < ctas; ++c) queue.push({0, c});
    for (const Item &i : items) {
        Load l = queue.top();
        queue.pop();
        mine[l.second].push_back(i.tile);
        l.first += i.cost;
        s.longest = std::max(s.longest, l.first);
        queue.push(l);
    }
    s.first.push_back(0);
    for (const auto &m : mine) {
        s.tiles.insert(s.tiles.end(), m.begin(), m.end());
        s.first.push_back(int32_t(s.tiles.size()));
    }
    return s;
}

template <int P, int BN, int OP>
cudaError_t launch_product(const StepArgs &s, const Tile *tiles, const int32_t *first, int ctas, int buf, bool last, cudaStream_t stream) {
    const auto kernel = product_kernel<P, BN, OP>;
    const cudaError_t e = allow_smem(kernel, Geo<P, BN>::kSmem);
    if (e != cudaSuccess) return e;
    return launch_ex(kernel, dim3(unsigned(ctas)), dim3(kGemmThreads), Geo<P, BN>::kSmem, stream, 1, true, s, tiles, first, buf, int(last));
}
template <int OP>
cudaError_t launch_product(const StepArgs &s, const Schedule &sch, const char *memory, bool three, int buf, bool last, cudaStream_t stream) {
    const Tile *tiles = reinterpret_cast<const Tile *>(memory + sch.o_tiles);
    const int32_t *first = reinterpret_cast<const int32_t *>(memory + sch.o_first);
    const int ctas = sch.ctas();
    if (sch.bn == 256)
        return three ? launch_product<3, 256, OP>(s, tiles, first, ctas, buf, last, stream) : launch_product<1, 256, OP>(s, tiles, first, ctas, buf, last, stream);
    return three ? launch_product<3, 128, OP>(s, tiles, first, ctas, buf, last, stream) : launch_product<1, 128, OP>(s, tiles, first, ctas, buf, last, stream);
}

bool encode_map(CUtensorMap &map, const void *base, int64_t rows, int64_t cols, int64_t ld) {
    const auto encode = tensor_map_encoder();
    if (encode == nullptr) return false;
    const cuuint64_t dims[2] = {cuuint64_t(cols), cuuint64_t(rows)}, strides[1] = {cuuint64_t(ld * 2)};
    const cuuint32_t box[2] = {64, 64}, step[2] = {1, 1};
    return encode(&map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace darb

using namespace darb;

struct darb_muon_s {
    std::vector<darb::Matrix> matrices;
    std::vector<int64_t> first_part;    // of every matrix, and the number of all
    std::vector<darb::Range> written;   // all buffers that a step writes, in order of address, none twice
    darb_dtype_t gtype = DARB_F32;
    void *dmem = nullptr;
    const darb::Matrix *d_matrices = nullptr;
    const darb::Part *d_parts = nullptr;
    int32_t *d_active = nullptr, *d_status = nullptr;
    darb::Schedule schedules[3];
};

namespace {

std::mutex g_plans_mu;
std::unordered_set<const darb_muon_s *> g_plans;

bool live_plan(const darb_muon_s *p) {
    std::lock_guard<std::mutex> lk(g_plans_mu);
    return p != nullptr && g_plans.count(p) != 0;
}

bool meets_written(const darb_muon_s &plan, const void *p, int64_t bytes) {
    const auto after = std::upper_bound(plan.written.begin(), plan.written.end(), p,
                                        [](const void *q, const Range &r) { return std::less<const void *>()(q, r.p); });
    if (after != plan.written.end() && ranges_overlap(after->p, after->bytes, p, bytes)) return true;
    return after != plan.written.begin() && ranges_overlap((after - 1)->p, (after - 1)->bytes, p, bytes);
}

darb_status_t build_plan(darb_muon_s *plan, int32_t n, const int64_t *rows, const int64_t *cols, float *const *params, float *const *m,
                         void *const *copies, cudaStream_t stream) {
    std::vector<Range> &all = plan->written;
    for (int32_t i = 0; i < n; ++i) {
        if (rows[i] < 0 || cols[i] < 0) return DARB_ERR_INVALID_ARG;
        Matrix x = {};
        if (rows[i] > 0 && cols[i] > 0) {
            if (rows[i] > kMaxSide || cols[i] > kMaxSide) return DARB_ERR_UNSUPPORTED;
            x.rows = int32_t(rows[i]), x.cols = int32_t(cols[i]);
            x.n = std::min(x.rows, x.cols), x.tall = x.rows > x.cols;
            x.p = params[i], x.m = m[i], x.copy = copies != nullptr ? static_cast<__nv_bfloat16 *>(copies[i]) : nullptr;
            if (x.p == nullptr || x.m == nullptr || !aligned_to(x.p, 4) || !aligned_to(x.m, 4) || !aligned_to(x.copy, 2)) return DARB_ERR_INVALID_ARG;
            const int64_t e = rows[i] * cols[i];
            all.push_back({x.p, e * 4});
            all.push_back({x.m, e * 4});
            if (x.copy != nullptr) all.push_back({x.copy, e * 2});
        }
        plan->matrices.push_back(x);
    }
    std::sort(all.begin(), all.end(), [](const Range &a, const Range &b) { return std::less<const void *>()(a.p, b.p); });
    for (size_t i = 1; i < all.size(); ++i)
        if (ranges_overlap(all[i - 1].p, all[i - 1].bytes, all[i].p, all[i].bytes)) return DARB_ERR_INVALID_ARG;
    std::vector<Part> parts;
    for (int32_t i = 0; i < n; ++i) {
        Matrix &x = plan->matrices[i];
        plan->first_part.push_back(int64_t(parts.size()));
        if (x.n == 0) continue;
        const int64_t e = int64_t(x.rows) * x.cols, want = std::min<int64_t>(kParts, (e + kPartElems - 1) / kPartElems);
        x.part_elems = int32_t(((e + want - 1) / want + 3) / 4 * 4);
        x.parts = int32_t((e + x.part_elems - 1) / x.part_elems);
        x.ldx = (x.cols + 63) / 64 * 64;
        x.lda = (x.n + 63) / 64 * 64;
        x.size = float(0.2 * std::sqrt(double(std::max(x.rows, x.cols))));
        for (int32_t p = 0; p < x.parts; ++p) parts.push_back({i, p});
    }
    plan->first_part.push_back(int64_t(parts.size()));
    if (parts.empty()) return DARB_OK;
    const char *fail = std::getenv("DARB_FAIL_ALLOC");   // test hook, as for the library's other allocations
    if (fail != nullptr && fail[0] == '1') return DARB_ERR_OOM;
    const int sms = sm_count();
    for (int op = kGram; op <= kApply; ++op) {
        // the width whose busiest CTA has least to do
        Schedule wide = make_schedule(plan->matrices, Op(op), 256, sms), narrow = make_schedule(plan->matrices, Op(op), 128, sms);
        plan->schedules[op] = wide.longest <= narrow.longest ? std::move(wide) : std::move(narrow);
    }
    // the tables, then the numbers of every matrix
    int64_t size = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t at = size;
        size += (bytes + 1023) / 1024 * 1024;
        return at;
    };
    const int64_t o_status = take(4), o_active = take(n * 4), o_parts = take(int64_t(parts.size() * sizeof(Part))), o_matrices = take(int64_t(n * sizeof(Matrix)));
    for (Schedule &s : plan->schedules) {
        s.o_tiles = take(int64_t(s.tiles.size() * sizeof(Tile)));
        s.o_first = take(int64_t(s.first.size() * 4));
    }
    const auto places = [&](char *base) {
        for (Matrix &x : plan->matrices) {
            if (x.n == 0) continue;
            const int64_t xb = int64_t(x.rows) * x.ldx * 2, ab = int64_t(x.n) * x.lda * 2;
            for (auto &buf : x.xp)
                for (__half *&p : buf) p = reinterpret_cast<__half *>(base + take(xb));
            for (__half *&p : x.ap) p = reinterpret_cast<__half *>(base + take(ab));
            for (__half *&p : x.bp) p = reinterpret_cast<__half *>(base + take(ab));
            x.d = reinterpret_cast<float *>(base + take(int64_t(x.lda) * 4));
            x.D = reinterpret_cast<float *>(base + take(int64_t(x.lda) * 4));
            x.partial = reinterpret_cast<double *>(base + take(x.parts * 8));
        }
    };
    const int64_t o_numbers = size;
    places(nullptr);
    cudaError_t e = cudaMalloc(&plan->dmem, size_t(size));
    if (e != cudaSuccess) {
        cudaGetLastError();
        plan->dmem = nullptr;
        return e == cudaErrorMemoryAllocation ? DARB_ERR_OOM : DARB_ERR_CUDA;
    }
    char *d = static_cast<char *>(plan->dmem);
    size = o_numbers;
    places(d);
    for (Matrix &x : plan->matrices) {
        if (x.n == 0) continue;
        for (int b = 0; b < 2; ++b)
            for (int q = 0; q < 2; ++q)
                if (!encode_map(x.x[b][q], x.xp[b][q], x.rows, x.cols, x.ldx)) return DARB_ERR_CUDA;
        for (int q = 0; q < 2; ++q)
            if (!encode_map(x.a[q], x.ap[q], x.n, x.n, x.lda) || !encode_map(x.b[q], x.bp[q], x.n, x.n, x.lda)) return DARB_ERR_CUDA;
    }
    plan->d_status = reinterpret_cast<int32_t *>(d + o_status);
    plan->d_active = reinterpret_cast<int32_t *>(d + o_active);
    plan->d_parts = reinterpret_cast<const Part *>(d + o_parts);
    plan->d_matrices = reinterpret_cast<const Matrix *>(d + o_matrices);
    // zeros: the diagonals of A and B are never written
    e = cudaMemsetAsync(d, 0, size_t(size), stream);
    const auto copy = [&](int64_t at, const void *from, size_t bytes) {
        if (e == cudaSuccess) e = cudaMemcpyAsync(d + at, from, bytes, cudaMemcpyHostToDevice, stream);
    };
    copy(o_parts, parts.data(), parts.size() * sizeof(Part));
    copy(o_matrices, plan->matrices.data(), plan->matrices.size() * sizeof(Matrix));
    for (const Schedule &s : plan->schedules) {
        copy(s.o_tiles, s.tiles.data(), s.tiles.size() * sizeof(Tile));
        copy(s.o_first, s.first.data(), s.first.size() * 4);
    }
    // the tables leave with this call, and steps may come on any stream
    const cudaError_t w = cudaStreamSynchronize(stream);
    if (e == cudaSuccess && w == cudaSuccess) return DARB_OK;
    cudaGetLastError();
    return DARB_ERR_CUDA;
}

void free_plan(darb_muon_s *plan) {
    if (plan->dmem != nullptr) cudaFree(plan->dmem);
    delete plan;
}

template <typename G>
cudaError_t launch_step(const darb_muon_s &plan, StepArgs s, const void *const *grads, cudaStream_t stream) {
    const int32_t n = int32_t(plan.matrices.size());
    for (int kernel = 0; kernel < 2; ++kernel) {
        for (int32_t i0 = 0; i0 < n; i0 += kPointers) {
            const int32_t i1 = std::min(n, i0 + kPointers);
            const int64_t parts = plan.first_part[i1] - plan.first_part[i0];
            if (parts == 0) continue;
            GradArgs g = {};
            g.first = i0, g.count = i1 - i0;
            for (int32_t i = i0; i < i1; ++i) g.p[i - i0] = grads[i];
            s.parts = plan.d_parts + plan.first_part[i0];
            const cudaError_t e = launch_ex(kernel == 0 ? momentum_kernel<G> : start_kernel<G>, dim3(unsigned(parts)), dim3(kElemThreads), 0, stream, 1, true, s, g);
            if (e != cudaSuccess) return e;
        }
    }
    const bool three = sizeof(G) == 4;
    const char *memory = static_cast<const char *>(plan.dmem);
    for (int k = 0; k < kIterations; ++k) {
        const int buf = k & 1;
        const bool last = k == kIterations - 1;
        cudaError_t e = launch_product<kGram>(s, plan.schedules[kGram], memory, three, buf, last, stream);
        if (e == cudaSuccess) e = launch_product<kSquare>(s, plan.schedules[kSquare], memory, three, buf, last, stream);
        if (e == cudaSuccess) e = launch_product<kApply>(s, plan.schedules[kApply], memory, three, buf, last, stream);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

extern "C" {

darb_status_t darb_muon_create(int32_t n, const int64_t *rows, const int64_t *cols, float *const *params, float *const *m, void *const *copies,
                               darb_dtype_t gtype, darb_muon_t *out, cudaStream_t stream) {
    DARB_TRACE("darb_muon_create");
    if (out == nullptr) return DARB_ERR_INVALID_ARG;
    *out = nullptr;
    if (n <= 0 || rows == nullptr || cols == nullptr || params == nullptr || m == nullptr || !token_dtype(gtype)) return DARB_ERR_INVALID_ARG;
    darb_muon_s *plan = new (std::nothrow) darb_muon_s();
    if (plan == nullptr) return DARB_ERR_OOM;
    plan->gtype = gtype;
    darb_status_t st;
    try {
        st = build_plan(plan, n, rows, cols, params, m, copies, stream);
        if (st == DARB_OK) {
            std::lock_guard<std::mutex> lk(g_plans_mu);
            g_plans.insert(plan);
        }
    } catch (...) {   // std::bad_alloc, or a vector asked for more than it can hold
        st = DARB_ERR_OOM;
    }
    if (st != DARB_OK) {
        free_plan(plan);
        return st;
    }
    *out = plan;
    return DARB_OK;
}

darb_status_t darb_muon_step(darb_muon_t plan, const void *const *grads, const float *grad_scale, double lr, double beta, double weight_decay,
                             double eps, int nesterov, cudaStream_t stream) {
    DARB_TRACE("darb_muon_step");
    if (!live_plan(plan) || grads == nullptr || !aligned_to(grad_scale, 4)) return DARB_ERR_INVALID_ARG;
    if (!(lr >= 0.0 && std::isfinite(lr)) || !(beta >= 0.0 && beta < 1.0) || !(eps > 0.0 && std::isfinite(eps)) ||
        !(weight_decay >= 0.0 && std::isfinite(weight_decay)))
        return DARB_ERR_INVALID_ARG;
    if (grad_scale != nullptr && meets_written(*plan, grad_scale, 4)) return DARB_ERR_INVALID_ARG;
    const size_t es = dtype_size(plan->gtype);
    bool any = false;
    for (size_t i = 0; i < plan->matrices.size(); ++i) {
        const Matrix &x = plan->matrices[i];
        if (grads[i] == nullptr || x.n == 0) continue;
        any = true;
        if (!aligned_to(grads[i], es) || meets_written(*plan, grads[i], int64_t(x.rows) * x.cols * int64_t(es))) return DARB_ERR_INVALID_ARG;
    }
    if (!any) return DARB_OK;
    StepArgs s = {};
    s.matrices = plan->d_matrices;
    s.active = plan->d_active;
    s.grad_scale = grad_scale;
    s.status = plan->d_status;
    s.beta = float(beta), s.rest = float(1.0 - beta), s.eps = float(eps);
    s.decay = float(1.0 - lr * weight_decay), s.lr = float(lr);
    s.nesterov = nesterov != 0;
    return enqueue([&] {
        return plan->gtype == DARB_BF16 ? launch_step<__nv_bfloat16>(*plan, s, grads, stream) : launch_step<float>(*plan, s, grads, stream);
    });
}

darb_status_t darb_muon_sync_status(darb_muon_t plan, cudaStream_t stream) {
    DARB_TRACE("darb_muon_sync_status");
    if (!live_plan(plan)) return DARB_ERR_INVALID_ARG;
    if (plan->d_status == nullptr) return DARB_OK;   // nothing to update
    int32_t bits = 0;
    cudaError_t e = cudaMemcpyAsync(&bits, plan->d_status, 4, cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaMemsetAsync(plan->d_status, 0, 4, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return DARB_ERR_CUDA;
    }
    return bits & kStatusTimeout ? DARB_ERR_TIMEOUT : DARB_OK;
}

darb_status_t darb_muon_destroy(darb_muon_t plan) {
    DARB_TRACE("darb_muon_destroy");
    if (plan == nullptr) return DARB_OK;
    {
        std::lock_guard<std::mutex> lk(g_plans_mu);
        if (g_plans.erase(plan) == 0) return DARB_ERR_INVALID_ARG;
    }
    free_plan(plan);
    return DARB_OK;
}

}  // extern "C"
