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
// One launch a product for all matrices of the plan.  A CTA, or a pair of them, walks
// the tiles that the plan's schedule gives it (longest first, to whoever is done first):
// one warp copies boxes of 64 x 64 numbers (TMA, 128-byte swizzle), one issues tcgen05.mma
// into one of two accumulators in tensor memory, eight write the tile before.
//
// What bounds it: the tensor cores where matrices are large.  A CTA alone is bound by its
// shared memory instead (a stage of 128 x 256 x 64 writes 48 KB and reads 48 KB in what are
// 512 clocks of products); a pair shares the columns' half of the operands and writes 32.
// 4096 x 9216 and 4096 x 4096 with bf16 gradients, 4.0e12 operations: 2.8 ms, of which 0.2
// are the elementwise kernels and 2.6 products at 1.55 PFLOP/s (a plain library product's
// burst is 1.95).  Two of 6000 x 3000 and 1500 x 1500 with fp32 gradients, 3 x 1.95e12: 4.1 ms,
// 1.4 PFLOP/s.
// Small matrices are bound by the 17 launches, of which each waits for a chain of
// copies, products and stores: three of 600 x 301 and 128 x 500 take 165 us.
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
constexpr int kParts = 608;                 // CTAs of the elementwise kernels, about: four an SM, one wave
constexpr int kPartElems = 4096;            // elements of one, at least
constexpr int64_t kMaxPart = 1 << 28;
constexpr int kElemThreads = 256;
constexpr int kUnroll = 4;                  // times four elements of a thread whose loads are on their way together
constexpr int64_t kMaxSide = 32768;         // rows and columns: elements fit 32 bits

constexpr int kBM = 128, kBK = 64;          // rows of a tile; depth of a stage
constexpr int kBox = 64 * 64 * 2;           // bytes of a box
constexpr int kWriters = 8;                  // warps that write a product
constexpr int kGemmThreads = 32 * (2 + kWriters);   // copies, products, writing
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
    int32_t shift;                          // e / cols = e * reciprocal >> shift for e < 2^31
    uint64_t reciprocal;
    float size;                             // 0.2 sqrt(max(rows, cols))
};
struct Part {
    int32_t matrix, part;
};
// A tile of a product, or one of the parts of its depth that several CTAs take.
struct Tile {
    int32_t matrix, row, col;               // first row and column
    int32_t width;                          // columns
    int32_t k0, k1;                         // depth
    int32_t slot, parts;                    // where the parts' sums go (slot + part), and how many there are
    int32_t part, pad[3];
};

struct StepArgs {
    const Matrix *matrices;
    const Part *parts;
    int32_t *active;                        // per matrix: has a gradient in this step
    const float *grad_scale;
    int32_t *status;
    float *partial;                         // sums of parts of tiles
    int32_t *arrived;                       // per slot: parts that are done, 0 between steps (the momentum kernel sets it so)
    int32_t slots;
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

// Elements e .. e + 4 of those before `end`.
template <typename G>
__device__ __forceinline__ void load4(const G *p, int64_t e, int64_t end, bool vector, float (&v)[4]) {
    if (vector && e + 4 <= end) {
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
    for (int i = 0; i < 4; ++i) v[i] = e + i < end ? widen(p[e + i]) : 0.0f;
}
__device__ __forceinline__ void store4(float *p, int64_t e, int64_t end, bool vector, const float (&v)[4]) {
    if (vector && e + 4 <= end) {
        *reinterpret_cast<float4 *>(p + e) = make_float4(v[0], v[1], v[2], v[3]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (e + i < end) p[e + i] = v[i];
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
    if (blockIdx.x == 0)   // (a step whose waits gave up may have left some)
        for (int i = threadIdx.x; i < a.slots; i += kElemThreads) a.arrived[i] = 0;
    if (g == nullptr) return;
    const float scale = a.grad_scale != nullptr ? *a.grad_scale : 1.0f;
    const int64_t all = int64_t(x.rows) * x.cols, e0 = int64_t(part.part) * x.part_elems, e1 = min(e0 + x.part_elems, all);
    const bool vector = aligned16(x.m) && (reinterpret_cast<uintptr_t>(g) & (4 * sizeof(G) - 1)) == 0;
    float *const m = x.m;
    double sum = 0.0;
    for (int64_t b0 = e0 + int64_t(threadIdx.x) * 4; b0 < e1; b0 += kUnroll * kElemThreads * 4) {
        float gv[kUnroll][4], mv[kUnroll][4];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t e = b0 + u * kElemThreads * 4;
            load4(g, e, e1, vector, gv[u]);
            load4(m, e, e1, vector, mv[u]);
        }
        float top = 0.0f, squares = 0.0f;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t e = b0 + u * kElemThreads * 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float gs = gv[u][i] * scale;
                mv[u][i] = mv[u][i] * a.beta + gs * a.rest;
                gv[u][i] = direction(a, gs, mv[u][i]);
                top = fmaxf(top, fabsf(gv[u][i]));
                squares = fmaf(gv[u][i], gv[u][i], squares);
            }
            store4(m, e, e1, vector, mv[u]);
        }
        // squares that 32 bits do not hold
        if (top > 1e15f || (top < 1e-15f && top > 0.0f)) {
            double d = 0.0;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) d += double(gv[u][i]) * gv[u][i];
            sum += d;
        } else {
            sum += double(squares);
        }
    }
    sum = block_total(sum);
    if (threadIdx.x == 0) x.partial[part.part] = sum;
}

// v as the sum of two fp16 numbers
__device__ __forceinline__ void split(float v, __half &hi, __half &lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(v - __half2float(hi));
}

template <typename G>
__global__ void __launch_bounds__(kElemThreads, 4) start_kernel(const StepArgs a, const __grid_constant__ GradArgs grads) {
    pdl_launch_dependents();
    const Part part = a.parts[blockIdx.x];
    const Matrix &x = a.matrices[part.matrix];
    const G *g = static_cast<const G *>(grads.p[part.matrix - grads.first]);
    pdl_wait_previous();
    if (g == nullptr) return;
    double sum = 0.0;
    const int parts = x.parts;
    const double *const partial = x.partial;
#pragma unroll 8
    for (int i = threadIdx.x; i < parts; i += kElemThreads) sum += partial[i];
    sum = block_total(sum);
    const double root = sqrt(sum);
    const float norm = float(root) + a.eps, scale = a.grad_scale != nullptr ? *a.grad_scale : 1.0f;
    // (numbers that 32 bits hold may have a norm that they do not)
    const float factor = norm < INFINITY ? kScaleX / norm : float(double(kScaleX) / (root + double(a.eps)));
    const bool divide = !(factor < INFINITY);   // (a norm too small for its reciprocal)
    const int64_t all = int64_t(x.rows) * x.cols, e0 = int64_t(part.part) * x.part_elems, e1 = min(e0 + x.part_elems, all);
    const bool vector = aligned16(x.m) && (reinterpret_cast<uintptr_t>(g) & (4 * sizeof(G) - 1)) == 0;
    const float *const m = x.m;
    __half *const hi = x.xp[0][0], *const lo = x.xp[0][1];
    const int cols = x.cols, ldx = x.ldx, shift = x.shift;
    const uint64_t reciprocal = x.reciprocal;
    const bool quads = cols % 4 == 0;
    for (int64_t b0 = e0 + int64_t(threadIdx.x) * 4; b0 < e1; b0 += kUnroll * kElemThreads * 4) {
        float gv[kUnroll][4], mv[kUnroll][4];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t e = b0 + u * kElemThreads * 4;
            load4(g, e, e1, vector, gv[u]);
            load4(m, e, e1, vector, mv[u]);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t e = b0 + u * kElemThreads * 4;
            if (e >= e1) break;
            alignas(8) __half h[4], l[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float d = direction(a, gv[u][i] * scale, mv[u][i]);
                split(divide ? d / norm * kScaleX : d * factor, h[i], l[i]);
            }
            int row = int(uint64_t(e) * reciprocal >> shift), col = int(e) - row * cols;
            if (quads) {   // (then all four are there: parts are multiples of 4 elements)
                const int64_t at = int64_t(row) * ldx + col;
                *reinterpret_cast<uint2 *>(hi + at) = *reinterpret_cast<const uint2 *>(h);
                *reinterpret_cast<uint2 *>(lo + at) = *reinterpret_cast<const uint2 *>(l);
                continue;
            }
            for (int i = 0; i < 4 && e + i < e1; ++i) {
                const int64_t at = int64_t(row) * ldx + col;
                hi[at] = h[i], lo[at] = l[i];
                if (++col == cols) col = 0, ++row;
            }
        }
    }
}

// ---- products ----

enum Op : int { kGram, kSquare, kApply, kLast };   // kLast: the last kApply, which updates the parameters

// Instruction descriptor of tcgen05.mma kind::f16 with fp16 A and B and an fp32
// accumulator.
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool a_mn, bool b_mn) {
    return (1u << 4) | (uint32_t(a_mn) << 15) | (uint32_t(b_mn) << 16) | (uint32_t(N >> 3) << 17) | (uint32_t(M >> 4) << 24);
}

// P: products of fp16 numbers that make one of the operands.  BN: columns of a tile.
// CG: CTAs of a tile, each with 128 of its rows; a pair reads half of the columns each,
// which halves what the copies write to a shared memory.
template <int P, int BN, int CG>
struct Geo {
    static constexpr int kParts = P == 1 ? 1 : 2;                 // fp16 numbers of an operand
    static constexpr int kABytes = kBM / 64 * kBox, kBBytes = BN / CG / 64 * kBox;
    static constexpr int kStage = kParts * (kABytes + kBBytes);
    static constexpr int kTurn = kWriters * 32 * 32 * 4;          // 32 rows x 32 columns of each writing warp
    static constexpr int kFit = (227 * 1024 - 2048 - kTurn) / kStage;
    static constexpr int kStages = kFit < 6 ? kFit : 6;
    static constexpr size_t kSmem = 2048 + size_t(kStages) * kStage + kTurn;
};

// tcgen05 for one CTA or a pair.
template <int CG>
__device__ __forceinline__ void pair_alloc(uint32_t *dst, uint32_t ncols) {
    if (CG == 1) {
        tmem_alloc(dst, ncols);
        tmem_relinquish();
        return;
    }
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(dst)), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
template <int CG>
__device__ __forceinline__ void pair_dealloc(uint32_t taddr, uint32_t ncols) {
    if (CG == 1) tmem_dealloc(taddr, ncols);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
template <int CG>
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    if (CG == 1) {
        mma_bf16(d, a, b, idesc, acc);   // (the type is the descriptor's)
        return;
    }
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
// Arrive on `bar` (of both CTAs) when every product issued so far is complete.
template <int CG>
__device__ __forceinline__ void pair_commit(uint64_t *bar) {
    if (CG == 1) mma_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)),
                     "h"(uint16_t(3))
                     : "memory");
}
// A box into this CTA's shared memory that completes on a barrier of the pair's first CTA.
template <int CG>
__device__ __forceinline__ void pair_copy(void *dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_addr(dst)),
                     "l"(map), "r"(x), "r"(y), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                         smem_addr(dst)),
                     "l"(map), "r"(x), "r"(y), "r"(bar)
                     : "memory");
}
__device__ __forceinline__ uint32_t shared_of(const void *p, uint32_t rank) {
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_addr(p)), "r"(rank));
    return to;
}
__device__ __forceinline__ void pair_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

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

// A warp has 32 rows x 32 columns of a product as the numbers of a row in each lane; it
// turns them through shared memory, so that four lanes share a row, eight neighbouring
// columns each, and 8 rows of 64 bytes of fp16 are read or written at once.  The 16
// bytes c of row r stand at c ^ (r % 8).
struct Turn {
    float4 *at;   // 32 x 8

    __device__ __forceinline__ void put(int lane, const uint32_t (&v)[32]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            at[lane * 8 + (i ^ (lane & 7))] =
                make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
    }
    __device__ __forceinline__ void get(int row, int oct, float (&v)[8]) const {
        const float4 x = at[row * 8 + ((2 * oct) ^ (row & 7))], y = at[row * 8 + ((2 * oct + 1) ^ (row & 7))];
        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
    }
    __device__ __forceinline__ void set(int row, int oct, const float (&v)[8]) const {
        at[row * 8 + ((2 * oct) ^ (row & 7))] = make_float4(v[0], v[1], v[2], v[3]);
        at[row * 8 + ((2 * oct + 1) ^ (row & 7))] = make_float4(v[4], v[5], v[6], v[7]);
    }
    __device__ __forceinline__ float one(int row, int col) const {
        return reinterpret_cast<const float *>(&at[row * 8 + ((col >> 2) ^ (row & 7))])[col & 3];
    }
};

__device__ __forceinline__ void halves(const uint4 &q, float (&v)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
}
// Eight numbers as the sums of two fp16 numbers.
__device__ __forceinline__ void split8(const float (&v)[8], uint4 &hi, uint4 &lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 a = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        const float2 f = __half22float2(a);
        const __half2 b = __floats2half2_rn(v[2 * i] - f.x, v[2 * i + 1] - f.y);
        h[i] = *reinterpret_cast<const uint32_t *>(&a), l[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]), lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// What the writing of a product needs to know of a matrix, in registers: after a store
// whatever lies in memory would have to be read again.
struct Target {
    const __half *in_hi, *in_lo;   // A or X
    __half *out_hi, *out_lo;       // A, B or X
    const float *row, *col;        // the diagonal by rows and by columns, or null
    float *diagonal;               // of the result, or null
    float *p;
    __nv_bfloat16 *copy;
    int32_t rows, cols, ld;
    float size;
    bool vector;                   // parameters four at a time
};
template <int OP>
__device__ __forceinline__ Target target(const StepArgs &s, const Matrix &x, int buf) {
    Target t = {};
    if (OP == kGram || OP == kSquare) {
        t.in_hi = x.ap[0], t.in_lo = x.ap[1];
        t.out_hi = OP == kGram ? x.ap[0] : x.bp[0], t.out_lo = OP == kGram ? x.ap[1] : x.bp[1];
        if (OP == kSquare) t.row = t.col = x.d;
        t.diagonal = OP == kGram ? x.d : x.D;
        t.rows = t.cols = x.n, t.ld = x.lda;
        return t;
    }
    t.in_hi = x.xp[buf][0], t.in_lo = x.xp[buf][1], t.out_hi = x.xp[buf ^ 1][0], t.out_lo = x.xp[buf ^ 1][1];
    if (x.tall) t.col = x.D;
    else t.row = x.D;
    t.rows = x.rows, t.cols = x.cols, t.ld = x.ldx;
    t.p = x.p, t.copy = x.copy, t.size = s.lr * x.size;
    t.vector = x.cols % 4 == 0 && aligned16(x.p) && (reinterpret_cast<uintptr_t>(x.copy) & 7) == 0;
    return t;
}

// What rows i0 .. i0 + 32 and columns j0 .. j0 + 32 of a product are put together with.
// All of it is loaded before the first store: no load can be moved over a store that
// might meet it, and waiting for each in turn would take longer than the product.
template <int P, int OP>
struct Loads {
    uint4 hi[4], lo[4];
    float di[4], dj[8];              // of the diagonal: of this lane's rows, of its columns
    float p[OP == kLast ? 32 : 1];   // parameters: of this lane's rows and columns, or (unaligned) of column `lane`

    __device__ __forceinline__ void get(const Target &x, int i0, int j0) {
        constexpr bool two = P == 3, apply = OP == kApply || OP == kLast;
        const int lane = threadIdx.x & 31, oct = lane & 3, sub = lane >> 2;
        const int rows = x.rows, cols = x.cols, ld = x.ld;
        if (OP == kGram || i0 >= rows || j0 >= cols || (!apply && j0 > i0 + 31)) return;
        const int j = j0 + 8 * oct;   // this lane's columns (rows are as long as a multiple of 64 numbers)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = min(i0 + 8 * q + sub, rows - 1);
            hi[q] = *reinterpret_cast<const uint4 *>(x.in_hi + int64_t(i) * ld + j);
            if (apply || two) lo[q] = *reinterpret_cast<const uint4 *>(x.in_lo + int64_t(i) * ld + j);
        }
        if (x.row != nullptr) {
#pragma unroll
            for (int q = 0; q < 4; ++q) di[q] = x.row[min(i0 + 8 * q + sub, rows - 1)];
        }
        if (x.col != nullptr) {   // (as long as a row, and 0 past its end)
            const float4 d0 = reinterpret_cast<const float4 *>(x.col + j)[0], d1 = reinterpret_cast<const float4 *>(x.col + j)[1];
            dj[0] = d0.x, dj[1] = d0.y, dj[2] = d0.z, dj[3] = d0.w, dj[4] = d1.x, dj[5] = d1.y, dj[6] = d1.z, dj[7] = d1.w;
        }
        if (OP == kLast && x.vector) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float *from = x.p + int64_t(min(i0 + 8 * q + sub, rows - 1)) * cols;
                const float4 p0 = *reinterpret_cast<const float4 *>(from + min(j, cols - 4)), p1 = *reinterpret_cast<const float4 *>(from + min(j + 4, cols - 4));
                float *const to = p + (OP == kLast ? 8 * q : 0);
                to[0] = p0.x, to[1] = p0.y, to[2] = p0.z, to[3] = p0.w, to[4] = p1.x, to[5] = p1.y, to[6] = p1.z, to[7] = p1.w;
            }
        } else if (OP == kLast) {
#pragma unroll
            for (int r = 0; r < 32; ++r) p[OP == kLast ? r : 0] = x.p[int64_t(min(i0 + r, rows - 1)) * cols + min(j0 + lane, cols - 1)];
        }
    }
};

// What becomes of them, `v` being a row of the product in each lane.
template <int P, int OP>
__device__ __forceinline__ void finish(const float decay, const Target &x, const Loads<P, OP> &in, int i0, int j0, const uint32_t (&v)[32], const Turn &turn) {
    constexpr bool two = P == 3, apply = OP == kApply || OP == kLast;
    const int lane = threadIdx.x & 31, oct = lane & 3, sub = lane >> 2;
    const int rows = x.rows, cols = x.cols, ld = x.ld;
    if (i0 >= rows || j0 >= cols || (!apply && j0 > i0 + 31)) return;
    const int j = j0 + 8 * oct;   // this lane's columns after the turn
    const uint4 (&hi)[4] = in.hi, (&lo)[4] = in.lo;
    const float (&di)[4] = in.di, (&dj)[8] = in.dj;
    turn.put(lane, v);
    __syncwarp();

    if (!apply) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = i0 + 8 * q + sub;
            float r[8], w[8];
            turn.get(8 * q + sub, oct, r);
            if (i < rows) {
                if (OP == kSquare) {
                    float old[8], more[8];
                    halves(hi[q], old);
                    if (two) halves(lo[q], more);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float sq = r[e] * (1.0f / (kScaleX * kScaleX)), A = (two ? old[e] + more[e] : old[e]) * (1.0f / kScaleX);
                        w[e] = (kB * A + kC * fmaf(di[q] + dj[e], A, sq)) * kScaleB;
                        if (j + e == i) x.diagonal[i] = kA + kB * di[q] + kC * fmaf(di[q], di[q], sq);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        w[e] = r[e] * (1.0f / kScaleX);
                        if (j + e == i) x.diagonal[i] = r[e] * (1.0f / (kScaleX * kScaleX));
                    }
                }
                uint4 h, l;
                split8(w, h, l);
                const int64_t at = int64_t(i) * ld + j;
                if (j + 8 <= i) {
                    *reinterpret_cast<uint4 *>(x.out_hi + at) = h;
                    if (two) *reinterpret_cast<uint4 *>(x.out_lo + at) = l;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (j + e >= i) continue;
                        __half a, b;
                        split(w[e], a, b);
                        x.out_hi[at + e] = a;
                        if (two) x.out_lo[at + e] = b;
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = 0.0f;
            }
            turn.set(8 * q + sub, oct, w);
        }
        __syncwarp();
        // across the diagonal: a lane has two rows of half of the columns
        const int i = i0 + 2 * (lane & 15);
#pragma unroll 4
        for (int c = lane >> 4; c < 32; c += 2) {
            const int jj = j0 + c;
            if (jj >= cols || i >= rows || jj > i) continue;
            const float v0 = turn.one(2 * (lane & 15), c), v1 = turn.one(2 * (lane & 15) + 1, c);
            const __half2 h = __floats2half2_rn(v0, v1);
            const float2 f = __half22float2(h);
            const __half2 l = __floats2half2_rn(v0 - f.x, v1 - f.y);
            const int64_t at = int64_t(jj) * ld + i;
            if (jj < i && i + 1 < rows) {
                *reinterpret_cast<__half2 *>(x.out_hi + at) = h;
                if (two) *reinterpret_cast<__half2 *>(x.out_lo + at) = l;
            } else {
                if (jj < i) {
                    x.out_hi[at] = __low2half(h);
                    if (two) x.out_lo[at] = __low2half(l);
                }
                if (jj < i + 1 && i + 1 < rows) {
                    x.out_hi[at + 1] = __high2half(h);
                    if (two) x.out_lo[at + 1] = __high2half(l);
                }
            }
        }
        __syncwarp();
        return;
    }

    const bool by_col = x.col != nullptr;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int i = i0 + 8 * q + sub;
        if (i >= rows) continue;
        float r[8], a[8], b[8];
        turn.get(8 * q + sub, oct, r);
        halves(hi[q], a);
        halves(lo[q], b);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            r[e] = fmaf(by_col ? dj[e] : di[q], (a[e] + b[e]) * (1.0f / kScaleX), r[e] * (1.0f / (kScaleX * kScaleB)));
        if (OP == kApply) {
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] *= kScaleX;
            uint4 h, l;
            split8(r, h, l);
            const int64_t at = int64_t(i) * ld + j;
            *reinterpret_cast<uint4 *>(x.out_hi + at) = h;
            *reinterpret_cast<uint4 *>(x.out_lo + at) = l;
        } else if (!x.vector) {
            turn.set(8 * q + sub, oct, r);
        } else {
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                if (j + h >= cols) continue;
                const int64_t at = int64_t(i) * cols + j + h;
                float c[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) c[e] = in.p[OP == kLast ? 8 * q + h + e : 0] * decay - x.size * r[h + e];
                *reinterpret_cast<float4 *>(x.p + at) = make_float4(c[0], c[1], c[2], c[3]);
                if (x.copy != nullptr) {
                    const __nv_bfloat162 b0 = __floats2bfloat162_rn(c[0], c[1]), b1 = __floats2bfloat162_rn(c[2], c[3]);
                    *reinterpret_cast<uint2 *>(x.copy + at) = make_uint2(*reinterpret_cast<const uint32_t *>(&b0), *reinterpret_cast<const uint32_t *>(&b1));
                }
            }
        }
    }
    __syncwarp();
    if (OP == kLast && !x.vector) {
#pragma unroll
        for (int r = 0; r < 32; ++r) {
            if (i0 + r >= rows || j0 + lane >= cols) continue;
            const int64_t at = int64_t(i0 + r) * cols + j0 + lane;
            const float v = in.p[OP == kLast ? r : 0] * decay - x.size * turn.one(r, lane);
            x.p[at] = v;
            if (x.copy != nullptr) x.copy[at] = __float2bfloat16_rn(v);
        }
        __syncwarp();
    }
}

// A tensor map that the host has copied to the device, before the first copy by it.
__device__ __forceinline__ void acquire_map(const CUtensorMap *map) {
    asm volatile("fence.proxy.tensormap::generic.acquire.sys [%0], 128;" ::"l"(map) : "memory");
}

// The writing warps among themselves.
__device__ __forceinline__ void writers_meet() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kWriters) : "memory"); }

// The tiles of CTA (or pair) b are tiles[first[b]] .. tiles[first[b + 1] - 1].
template <int P, int BN, int CG, int OP>
__global__ void __launch_bounds__(kGemmThreads, 1) product_kernel(const StepArgs s, const Tile *tiles, const int32_t *first, int buf) {
    using G = Geo<P, BN, CG>;
    constexpr int NS = G::kStages, NP = G::kParts;
    extern __shared__ unsigned char sm_raw[];
    unsigned char *const sm = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(sm_raw) + 1023) & ~uintptr_t(1023));
    uint64_t *const full = reinterpret_cast<uint64_t *>(sm), *const empty = full + NS, *const ready = empty + NS, *const read = ready + 2,
                    *const done = read + 2;
    uint32_t *const s_tmem = reinterpret_cast<uint32_t *>(done + 1);
    volatile uint32_t *const s_last = s_tmem + 1;
    unsigned char *const stages = sm + 1024;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = CG == 2 ? int(blockIdx.x) & 1 : 0, unit = CG == 2 ? int(blockIdx.x) >> 1 : int(blockIdx.x);
    constexpr uint32_t kColumns = 2 * BN;

    pdl_launch_dependents();
    if (tid == 0) {
        for (int i = 0; i < NS; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&ready[i], 1), mbar_init(&read[i], kWriters * CG);
        mbar_init(done, 1);
        fence_mbar_init();
    }
    if (warp == 1) pair_alloc<CG>(s_tmem, kColumns);
    tc_fence_before_sync();
    __syncthreads();
    if (CG == 2) pair_meet();   // the other CTA's barriers stand before anything arrives there
    tc_fence_after_sync();
    const uint32_t tmem = *s_tmem;
    // (the plan's tables do not change: what a CTA begins with is fetched while the kernel before ends)
    const int t0 = first[unit], t1 = first[unit + 1];
    bool ok = true;
    int known = -1;   // the matrix whose maps the copying thread has at hand
    if (tid == 0 && t0 < t1) {
        known = tiles[t0].matrix;
        const Operands o = operands<OP>(s.matrices[known], buf);
        for (int q = 0; q < NP; ++q) {
            acquire_map(&o.a[q]), acquire_map(&o.b[q]);
            prefetch_tensormap(&o.a[q]), prefetch_tensormap(&o.b[q]);
        }
    }
    pdl_wait_previous();

    if (warp == 0) {
        if (lane == 0) {
            fence_proxy_async_global();
            int stage = 0;
            uint32_t parity = 0;
            int64_t issued = 0;
            for (int t = t0; t < t1 && ok; ++t) {
                const Tile tile = tiles[t];
                const Matrix &x = s.matrices[tile.matrix];
                if (!s.active[tile.matrix]) continue;
                const Operands o = operands<OP>(x, buf);
                const bool wide = CG == 1 || tile.width == BN;   // (else half of the columns)
                const int row = tile.row + rank * kBM, col = tile.col + rank * (wide ? BN / CG : BN / CG / 2);
                if (tile.matrix != known) {
                    for (int q = 0; q < NP; ++q) acquire_map(&o.a[q]), acquire_map(&o.b[q]);
                    known = tile.matrix;
                }
                for (int k = tile.k0; k < tile.k1; k += kBK, ++issued) {
                    if (issued >= NS && !mbar_wait(&empty[stage], parity ^ 1u)) {
                        ok = false;
                        break;
                    }
                    // the first CTA's barrier counts the bytes of both
                    if (rank == 0) mbar_arrive_expect_tx(&full[stage], wide ? CG * G::kStage : CG * NP * (G::kABytes + G::kBBytes / 2));
                    const uint32_t bar = CG == 2 ? shared_of(&full[stage], 0) : smem_addr(&full[stage]);
                    unsigned char *to = stages + stage * G::kStage;
#pragma unroll
                    for (int q = 0; q < NP; ++q)
                        for (int b = 0; b < kBM; b += 64, to += kBox)
                            pair_copy<CG>(to, &o.a[q], o.a_mn ? row + b : k, o.a_mn ? k : row + b, bar);
#pragma unroll
                    for (int q = 0; q < NP; ++q)
#pragma unroll
                        for (int b = 0; b < BN / CG; b += 64, to += kBox)
                            if (wide || b < BN / CG / 2) pair_copy<CG>(to, &o.b[q], o.b_mn ? col + b : k, o.b_mn ? k : col + b, bar);
                    if (++stage == NS) stage = 0, parity ^= 1u;
                }
            }
            // what is still on its way lands before the CTA leaves (in the second CTA: when the pair's products have
            // been waited for, at the end)
            if (!ok && rank == 0)
                for (int64_t i = issued > NS ? issued - NS : 0; i < issued; ++i) mbar_wait(&full[i % NS], uint32_t(i / NS) & 1u);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            int stage = 0, used = 0;
            uint32_t parity = 0;
            for (int t = t0; t < t1 && ok; ++t) {
                const Tile tile = tiles[t];
                const Matrix &x = s.matrices[tile.matrix];
                if (!s.active[tile.matrix]) continue;
                const Operands o = operands<OP>(x, buf);
                const uint32_t idesc = idesc_f16(CG * kBM, CG == 1 ? BN : tile.width, o.a_mn, o.b_mn);
                // along the depth: rows of 128 bytes; along the tile: boxes of 64 columns, 8 deep atoms one after the other
                const uint32_t a_lbo = o.a_mn ? kBox : 16, b_lbo = o.b_mn ? kBox : 16;
                const uint32_t a_step = (o.a_mn ? 2048 : 32) >> 4, b_step = (o.b_mn ? 2048 : 32) >> 4;
                const int half = used & 1;
                if (used >= 2 && !mbar_wait_acq_cluster(&read[half], uint32_t(used / 2 - 1) & 1u)) {
                    ok = false;
                    break;
                }
                tc_fence_after_sync();
                const uint32_t d = tmem + half * BN;
                for (int k = tile.k0; k < tile.k1; k += kBK) {
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
                        pair_mma<CG>(d, ah + ao, bh + bo, idesc, (k - tile.k0 | kk) != 0);
                        if (P == 3) {
                            pair_mma<CG>(d, ah + ao, bl + bo, idesc, 1u);
                            pair_mma<CG>(d, al + ao, bh + bo, idesc, 1u);
                        }
                    }
                    pair_commit<CG>(&empty[stage]);
                    if (++stage == NS) stage = 0, parity ^= 1u;
                }
                pair_commit<CG>(&ready[half]);
                ++used;
            }
            pair_commit<CG>(done);
        }
        // no product is in flight when the memory is given back
        if (lane == 0 && rank == 0 && !mbar_wait(done, 0)) ok = false;
        __syncwarp();
    } else {
        // two warps for each quarter of the accumulator's rows, with half of the columns each
        const int quarter = warp & 3;
        const Turn turn = {reinterpret_cast<float4 *>(stages + NS * G::kStage) + (warp - 2) * (32 * 8)};
        int used = 0;
        for (int t = t0; t < t1; ++t) {
            const Tile tile = tiles[t];
            const Matrix &x = s.matrices[tile.matrix];
            if (!s.active[tile.matrix]) continue;
            const int half = used & 1, i0 = tile.row + rank * kBM + quarter * 32, columns = CG == 1 ? BN / 2 : tile.width / 2, c0 = warp < 6 ? 0 : columns;
            const Target to = target<OP>(s, x, buf);
            const bool whole = OP != kGram || CG == 2 || tile.parts == 1;
            Loads<P, OP> in;
            if (whole) in.get(to, i0, tile.col + c0);   // (while the product is made)
            const bool here = __all_sync(~0u, mbar_wait(&ready[half], uint32_t(used / 2) & 1u));
            if (!here) {
                ok = false;
                if (OP != kGram || CG == 2) break;   // (else the other warps wait for this one below)
            }
            tc_fence_after_sync();
            const uint32_t at = tmem + half * BN + (uint32_t(quarter * 32) << 16);
            // the sums of a part: a column's rows side by side
            float *const mine = s.partial + (int64_t(tile.slot) * BN + c0) * kBM + quarter * 32 + lane;
#pragma unroll 1
            for (int c = 0; c < columns && here; c += 32) {
                uint32_t v[32];
                tmem_ld32(at + c0 + c, v);
                tmem_ld_wait();
                if (whole) {
                    if (c > 0) in.get(to, i0, tile.col + c0 + c);
                    finish<P, OP>(s.decay, to, in, i0, tile.col + c0 + c, v, turn);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) mine[(int64_t(tile.part) * BN + c + e) * kBM] = __uint_as_float(v[e]);
                }
            }
            // the accumulator has been read
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (CG == 1) mbar_arrive(&read[half]);
                else asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(shared_of(&read[half], 0)) : "memory");
            }
            ++used;
            if (whole) continue;
            // whoever is done last adds the parts up, in their order
            __threadfence();
            writers_meet();
            if (warp == 2 && lane == 0) {
                const bool last = atomicAdd(s.arrived + tile.slot, 1) == tile.parts - 1;
                if (last) s.arrived[tile.slot] = 0;
                *s_last = last;
            }
            writers_meet();
            if (!*s_last) continue;
            __threadfence();
#pragma unroll 1
            for (int c = 0; c < columns; c += 32) {
                if (i0 >= to.rows || tile.col + c0 + c > i0 + 31) continue;   // (nothing is made of these)
                float sum[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) sum[e] = __ldcg(mine + int64_t(c + e) * kBM);
#pragma unroll 1
                for (int q = 1; q < tile.parts; ++q)
#pragma unroll
                    for (int e = 0; e < 32; ++e) sum[e] += __ldcg(mine + (int64_t(q) * BN + c + e) * kBM);
                uint32_t v[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(sum[e]);
                finish<P, OP>(s.decay, to, in, i0, tile.col + c0 + c, v, turn);
            }
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    // (A pair's second CTA issues none: from its start this would be a wait for the whole launch, not for a tile.)
    if (CG == 2 && rank == 1 && warp == 1) {
        if (lane == 0 && !mbar_wait(done, 0)) ok = false;
        __syncwarp();
    }
    if (!ok) atomicOr(s.status, kStatusTimeout);
    if (CG == 2) pair_meet();   // neither CTA leaves while the other may reach into it
    if (warp == 1) {
        tc_fence_after_sync();
        pair_dealloc<CG>(tmem, kColumns);
    }
}

// ---- host ----

// The tiles of one product of all matrices, given to CTAs.
struct Schedule {
    std::vector<Tile> tiles;
    std::vector<int32_t> first;
    int bn = 0;
    int64_t longest = 0;
    int64_t slots = 0;                  // of parts of tiles
    int64_t o_tiles = 0, o_first = 0;   // in the plan's memory
    int32_t units() const { return int32_t(first.size()) - 1; }
};

// The forms of a product: tiles of 256 x 256 by pairs of CTAs (256 x 128 where that
// evens out what the pairs have to do), or of 128 x 128 or 64 by one.
struct Form {
    int bm, bn, cg;
};
constexpr Form kForms[] = {{256, 256, 2}, {128, 128, 1}, {128, 64, 1}};

// Clocks of a tile, about: a stage by what it moves through shared memory and the
// products that it feeds (measured), and what a tile waits for at its ends.
int64_t tile_cost(int64_t depth, bool three, int cg, int width) {
    const int64_t stages = (depth + kBK - 1) / kBK;
    if (cg == 2) return width == 256 ? stages * (three ? 1600 : 560) + 5000 : stages * (three ? 950 : 400) + 3500;
    return width == 128 ? stages * (three ? 1350 : 600) + 3500 : stages * (three ? 950 : 420) + 2500;
}

struct Item {
    int64_t cost, depth;
    Tile tile;
    int64_t unit = 0;
};

// Items, the longest first, each to the unit that is done first; the longest load.
int64_t assign(std::vector<Item> &items, int units, std::vector<int64_t> &load) {
    std::stable_sort(items.begin(), items.end(), [](const Item &a, const Item &b) { return a.cost > b.cost; });
    load.assign(units, 0);
    using Load = std::pair<int64_t, int>;
    std::priority_queue<Load, std::vector<Load>, std::greater<Load>> queue;
    for (int c = 0; c < units; ++c) queue.push({0, c});
    int64_t longest = 0;
    for (Item &i : items) {
        Load l = queue.top();
        queue.pop();
        i.unit = l.second;
        load[l.second] = l.first += i.cost;
        longest = std::max(longest, l.first);
        queue.push(l);
    }
    return longest;
}

// Few tiles are divided along their depth until there is one part for every unit, or
// none has more than twelve stages (parts of five cost more than they save: three of 600 x
// 301 170 us against 164); the slots that this takes.
int64_t divide(std::vector<Item> &items, bool three, const Form &form, int units) {
    std::vector<int64_t> parts(items.size(), 1);
    const auto stages = [&](size_t i) { return (items[i].depth + kBK - 1) / kBK; };
    for (int64_t total = int64_t(items.size()); total < units; ++total) {
        size_t most = 0;
        for (size_t i = 1; i < items.size(); ++i)
            if (stages(i) * parts[most] > stages(most) * parts[i]) most = i;
        if (stages(most) <= 12 * parts[most]) break;
        ++parts[most];
    }
    std::vector<Item> all;
    int64_t slots = 0;
    for (size_t i = 0; i < items.size(); ++i) {
        const int64_t n = parts[i], each = (stages(i) + n - 1) / n * kBK;
        const int64_t used = (items[i].depth + each - 1) / each;
        for (int64_t q = 0; q < used; ++q) {
            Item part = items[i];
            part.tile.k0 = int32_t(q * each), part.tile.k1 = int32_t(std::min(part.depth, (q + 1) * each));
            if (used > 1) part.tile.slot = int32_t(slots), part.tile.parts = int32_t(used), part.tile.part = int32_t(q);
            // (what the last part does more is about what a tile waits for at its end)
            part.cost = tile_cost(part.tile.k1 - part.tile.k0, three, form.cg, form.bn) + (used > 1 ? 4000 + 300 * used : 0);
            all.push_back(part);
        }
        if (used > 1) slots += used;
    }
    items = std::move(all);
    return slots;
}

Schedule make_schedule(const std::vector<Matrix> &all, Op op, const Form &form, bool three, int units) {
    std::vector<Item> items;
    for (size_t t = 0; t < all.size(); ++t) {
        const Matrix &x = all[t];
        if (x.n == 0) continue;
        const int rows = op == kApply ? x.rows : x.n, cols = op == kApply ? x.cols : x.n;
        const int64_t depth = op == kGram ? std::max(x.rows, x.cols) : x.n;
        for (int col = 0; col < cols; col += form.bn)
            for (int row = 0; row < rows; row += form.bm)
                if (op == kApply || col < row + form.bm)
                    items.push_back({tile_cost(depth, three, form.cg, form.bn), depth, {int32_t(t), row, col, form.bn, 0, int32_t(depth), 0, 1, 0, {}}});
    }
    Schedule s;
    s.bn = form.bn;
    if (op == kGram && form.cg == 1 && int64_t(items.size()) < units) s.slots = divide(items, three, form, units);
    const int most = units;
    std::vector<int64_t> load;
    auto shared = [&] { return int(std::min<int64_t>(most, int64_t(items.size()))); };
    s.longest = assign(items, shared(), load);
    // the last tiles of the busiest pairs in halves, as long as that helps
    for (int64_t tries = 0; form.cg == 2 && tries < 16 && tries * int64_t(items.size()) < 200000; ++tries) {
        std::vector<Item> next;
        std::vector<char> halved(load.size(), 0);
        for (auto i = items.rbegin(); i != items.rend(); ++i) {   // the shortest first
            const int cols = op == kApply ? all[i->tile.matrix].cols : all[i->tile.matrix].n;
            const bool busy = load[i->unit] * 100 > s.longest * 98 && !halved[i->unit] && i->tile.width == 256;
            if (!busy) {
                next.push_back(*i);
                continue;
            }
            halved[i->unit] = 1;
            for (int h = 0; h < 256; h += 128) {
                Item half = *i;
                half.cost = tile_cost(i->depth, three, 2, 128);
                half.tile.col += h, half.tile.width = 128;
                if (half.tile.col < cols && (op == kApply || half.tile.col < half.tile.row + form.bm)) next.push_back(half);
            }
        }
        if (std::find(halved.begin(), halved.end(), 1) == halved.end()) break;
        std::vector<int64_t> next_load;
        const int64_t longest = assign(next, int(std::min<int64_t>(most, int64_t(next.size()))), next_load);
        if (longest >= s.longest) break;
        items = std::move(next), load = std::move(next_load), s.longest = longest;
    }
    std::vector<std::vector<Tile>> mine(load.size());
    for (const Item &i : items) mine[i.unit].push_back(i.tile);
    s.first.push_back(0);
    for (const auto &m : mine) {
        s.tiles.insert(s.tiles.end(), m.begin(), m.end());
        s.first.push_back(int32_t(s.tiles.size()));
    }
    return s;
}

template <int P, int BN, int CG, int OP>
cudaError_t launch_product(const StepArgs &s, const Schedule &sch, const char *memory, int buf, cudaStream_t stream) {
    const auto kernel = product_kernel<P, BN, CG, OP>;
    constexpr size_t smem = Geo<P, BN, CG>::kSmem;
    const cudaError_t e = allow_smem(kernel, smem);
    if (e != cudaSuccess) return e;
    return launch_ex(kernel, dim3(unsigned(CG * sch.units())), dim3(kGemmThreads), smem, stream, CG, true, s, reinterpret_cast<const Tile *>(memory + sch.o_tiles),
                     reinterpret_cast<const int32_t *>(memory + sch.o_first), buf);
}
template <int OP>
cudaError_t launch_product(const StepArgs &s, const Schedule &sch, const char *memory, bool three, int buf, cudaStream_t stream) {
    if (sch.bn == 256) return three ? launch_product<3, 256, 2, OP>(s, sch, memory, buf, stream) : launch_product<1, 256, 2, OP>(s, sch, memory, buf, stream);
    if (sch.bn == 128) return three ? launch_product<3, 128, 1, OP>(s, sch, memory, buf, stream) : launch_product<1, 128, 1, OP>(s, sch, memory, buf, stream);
    return three ? launch_product<3, 64, 1, OP>(s, sch, memory, buf, stream) : launch_product<1, 64, 1, OP>(s, sch, memory, buf, stream);
}

// Pairs of CTAs that the device holds at a time.
int pair_room(bool three) {
    const auto kernel1 = product_kernel<1, 256, 2, kApply>;
    const auto kernel3 = product_kernel<3, 256, 2, kApply>;
    const size_t smem = three ? Geo<3, 256, 2>::kSmem : Geo<1, 256, 2>::kSmem;
    if ((three ? allow_smem(kernel3, smem) : allow_smem(kernel1, smem)) != cudaSuccess) return 1;
    return cluster_room(three ? kernel3 : kernel1, kGemmThreads, smem).of[1];
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
    int32_t *d_active = nullptr, *d_status = nullptr, *d_arrived = nullptr;
    float *d_partial = nullptr;
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
    // as many elements for every CTA, whatever the matrices' sizes (4096 x 9216 and 4096 x 4096
    // with bf16 gradients: 93 and 111 us; 304 CTAs of each matrix 109 and 125, 1216 in all 94 and 116)
    int64_t elements = 0;
    for (const Matrix &x : plan->matrices) elements += int64_t(x.rows) * x.cols;
    const int64_t each = (std::max<int64_t>(kPartElems, elements / kParts) + 3) / 4 * 4;
    for (int32_t i = 0; i < n; ++i) {
        Matrix &x = plan->matrices[i];
        plan->first_part.push_back(int64_t(parts.size()));
        if (x.n == 0) continue;
        const int64_t e = int64_t(x.rows) * x.cols;
        x.part_elems = int32_t(std::min<int64_t>(each, kMaxPart));
        x.parts = int32_t((e + x.part_elems - 1) / x.part_elems);
        x.ldx = (x.cols + 63) / 64 * 64;
        x.lda = (x.n + 63) / 64 * 64;
        int bits = 0;
        while ((int64_t(1) << bits) < x.cols) ++bits;
        x.shift = 31 + bits;
        x.reciprocal = ((uint64_t(1) << x.shift) + x.cols - 1) / x.cols;
        x.size = float(0.2 * std::sqrt(double(std::max(x.rows, x.cols))));
        for (int32_t p = 0; p < x.parts; ++p) parts.push_back({i, p});
    }
    plan->first_part.push_back(int64_t(parts.size()));
    if (parts.empty()) return DARB_OK;
    const char *fail = std::getenv("DARB_FAIL_ALLOC");   // test hook, as for the library's other allocations
    if (fail != nullptr && fail[0] == '1') return DARB_ERR_OOM;
    const bool three = plan->gtype == DARB_F32;
    const int sms = sm_count(), pairs = pair_room(three);
    for (int op = kGram; op <= kApply; ++op) {
        // the form whose busiest CTA has least to do
        for (const Form &f : kForms) {
            Schedule s = make_schedule(plan->matrices, Op(op), f, three, f.cg == 2 ? pairs : sms);
            if (plan->schedules[op].bn == 0 || s.longest < plan->schedules[op].longest) plan->schedules[op] = std::move(s);
        }
    }
    // the tables, then the numbers of every matrix
    int64_t size = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t at = size;
        size += (bytes + 1023) / 1024 * 1024;
        return at;
    };
    const int64_t o_status = take(4), o_active = take(n * 4), o_parts = take(int64_t(parts.size() * sizeof(Part))), o_matrices = take(int64_t(n * sizeof(Matrix)));
    const Schedule &gram = plan->schedules[kGram];
    const int64_t o_arrived = take(gram.slots * 4), o_partial = take(gram.slots * gram.bn * kBM * 4);
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
    plan->d_arrived = reinterpret_cast<int32_t *>(d + o_arrived);
    plan->d_partial = reinterpret_cast<float *>(d + o_partial);
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
        cudaError_t e = launch_product<kGram>(s, plan.schedules[kGram], memory, three, buf, stream);
        if (e == cudaSuccess) e = launch_product<kSquare>(s, plan.schedules[kSquare], memory, three, buf, stream);
        if (e == cudaSuccess)
            e = k + 1 < kIterations ? launch_product<kApply>(s, plan.schedules[kApply], memory, three, buf, stream)
                                    : launch_product<kLast>(s, plan.schedules[kApply], memory, three, buf, stream);
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
    // (what counts is what the kernels get: an eps that 32 bits round to 0 would make 0 / 0 of zero gradients)
    if (!(lr >= 0.0 && std::isfinite(float(lr))) || !(beta >= 0.0 && beta < 1.0) || !(float(eps) > 0.0f && std::isfinite(float(eps))) ||
        !(weight_decay >= 0.0 && std::isfinite(float(1.0 - lr * weight_decay))))
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
    s.partial = plan->d_partial, s.arrived = plan->d_arrived, s.slots = int32_t(plan->schedules[kGram].slots);
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
