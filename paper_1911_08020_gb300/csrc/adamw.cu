// adamw.cu -- one AdamW step over all tensors of a model in one launch
// (darb_adamw_create, darb_adamw_step): the update of the dense weights between
// two re-encodes of the prune-retrain loop (Sec. 4), with the moments in fp32
// or in 8 bits.
//
//   g' = g * scale,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = p (1 - lr wd) - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every operation is one IEEE fp32 operation in this order (no contraction), so
// the results do not depend on how the compiler or a vector width groups them.
//
// States in 8 bits.  Blocks of 256 elements share an fp32 scale (largest
// magnitude / 448); the moment m and the root r = sqrt(v) are held as e4m3 codes
// (3 bits of fraction).  The root is held instead of v because its range is half
// as wide in powers of two.  A moment moves by a thousandth a step and codes are
// up to an eighth apart: rounding to the nearest code would undo every step, so
// a value goes to the code above it with the probability that keeps its mean.
// The random numbers are a mix of the element's number and the step's seed, the
// same on every run.  A root that is not zero keeps a code that is not zero, so
// that no update is divided by eps alone.
//
// The step is bound by memory (28 bytes an element with fp32 gradients and
// states).  The unit of work is a chunk of kChunkElems consecutive elements of
// one tensor, so that tensors of any sizes share the machine evenly; which chunk
// of which tensor is looked up in a table made with the plan.  A warp takes a
// whole block of 256, 8 elements a lane, so that a block's maximum is one
// reduction.
#include "launch.cuh"
#include "tma.cuh"
#include "tokens.cuh"
#include "trace.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdlib>
#include <functional>
#include <mutex>
#include <new>
#include <unordered_set>
#include <vector>

namespace darb {

int sm_count();

namespace {

constexpr int kBlock = DARB_ADAMW_BLOCK;
constexpr int kAdamThreads = 256;
constexpr int kChunkElems = 2048;
constexpr int kPerLane = kBlock / 32;
constexpr int kGradPointers = 448;   // tensors of a launch: the pointers fit in 4 KB of arguments
static_assert(kChunkElems % (kAdamThreads * kPerLane) == 0, "whole blocks of every warp in a chunk");

struct Tensor {
    float *p;
    void *m, *v;              // fp32, or e4m3 codes of m and of sqrt(v)
    float *m_scale, *v_scale; // one for each block of 256; null with fp32 states
    __nv_bfloat16 *copy;      // the parameter rounded, or null
    int64_t n;
    int64_t first;            // number of the tensor's first element among all (whole blocks a tensor)
};
struct Chunk {
    int32_t tensor, chunk;
};

struct StepArgs {
    const Tensor *tensors;
    const Chunk *chunks;
    const float *grad_scale;   // or null
    int32_t *status;           // the plan's, of waits that gave up
    float b1, c1, b2, c2;      // c = 1 - b
    float decay, step_size, root_scale, eps;
    uint32_t key;
    int32_t first_tensor;
    const void *grads[kGradPointers];
};

// What a step multiplies by, twice each for pairs.
struct Factors {
    Pair b1, c1, b2, c2, decay, step, root_scale, eps, grad_scale;
    __device__ explicit Factors(const StepArgs &a, float scale)
        : b1(both(a.b1)), c1(both(a.c1)), b2(both(a.b2)), c2(both(a.c2)), decay(both(a.decay)), step(both(-a.step_size)),
          root_scale(both(a.root_scale)), eps(both(a.eps)), grad_scale(both(scale)) {}
};

// A pair's sum in two scalar additions: the assembler contracts a paired product
// and a paired sum into one rounding, whatever is asked of it.
__device__ __forceinline__ Pair plus(Pair a, Pair b) { return pair(__fadd_rn(low(a), low(b)), __fadd_rn(high(a), high(b))); }

__device__ __forceinline__ void update(Pair &p, Pair g, Pair &m, Pair &v, Pair &root, const Factors &k) {
    g = mul2(g, k.grad_scale);
    m = plus(mul2(m, k.b1), mul2(g, k.c1));
    v = plus(mul2(v, k.b2), mul2(mul2(g, g), k.c2));
    root = pair(__fsqrt_rn(low(v)), __fsqrt_rn(high(v)));
    const Pair denom = plus(mul2(root, k.root_scale), k.eps), num = mul2(m, k.step);   // (the step is negative here)
    p = plus(mul2(p, k.decay), pair(__fdiv_rn(low(num), low(denom)), __fdiv_rn(high(num), high(denom))));
}

// Elements i .. i + 8 of a tensor as fp32 (VEC: i is a multiple of 8 and the
// tensor 16-byte aligned; else zeros from n on).
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T *t, int64_t i, int64_t n, Pair (&v)[4]) {
    if (VEC) {
        if constexpr (sizeof(T) == 4) {
            Pair lo[2], hi[2];
            unpack(*reinterpret_cast<const uint4 *>(t + i), lo);
            unpack(*reinterpret_cast<const uint4 *>(t + i + 4), hi);
            v[0] = lo[0], v[1] = lo[1], v[2] = hi[0], v[3] = hi[1];
        } else {
            unpack(*reinterpret_cast<const uint4 *>(t + i), v);
        }
    } else {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = i + e < n ? widen(t[i + e]) : 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = pair(w[2 * e], w[2 * e + 1]);
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T *t, int64_t i, int64_t n, const Pair (&v)[4]) {
    if (VEC) {
        if constexpr (sizeof(T) == 4) {
            const Pair lo[2] = {v[0], v[1]}, hi[2] = {v[2], v[3]};
            *reinterpret_cast<uint4 *>(t + i) = pack(lo);
            *reinterpret_cast<uint4 *>(t + i + 4) = pack(hi);
        } else {
            *reinterpret_cast<uint4 *>(t + i) = pack(v);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < n) t[i + e] = narrow<T>(e & 1 ? high(v[e / 2]) : low(v[e / 2]));
    }
}

// e4m3 codes to fp32 (exact), two at a time.
__device__ __forceinline__ Pair decode2(uint16_t codes) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(codes));
    float lo, hi;
    asm("{\n .reg .b16 x, y;\n mov.b32 {x, y}, %2;\n cvt.f32.f16 %0, x;\n cvt.f32.f16 %1, y;\n}" : "=f"(lo), "=f"(hi) : "r"(h));
    return pair(lo, hi);
}
// The code of a value that codes have, or of NaN.
__device__ __forceinline__ uint32_t encode(float v) {
    uint16_t c;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(0.0f), "f"(v));
    return c & 0xFFu;
}
template <bool VEC>
__device__ __forceinline__ void load_codes(const uint8_t *t, int64_t i, int64_t n, float scale, Pair (&v)[4]) {
    uint32_t w[2] = {0, 0};
    if (VEC) {
        const uint2 q = *reinterpret_cast<const uint2 *>(t + i);
        w[0] = q.x, w[1] = q.y;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < n) w[e >> 2] |= uint32_t(t[i + e]) << (8 * (e & 3));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = mul2(decode2(uint16_t(w[e >> 1] >> (16 * (e & 1)))), both(scale));
}
template <bool VEC>
__device__ __forceinline__ void store_codes(uint8_t *t, int64_t i, int64_t n, const uint32_t (&c)[2]) {
    if (VEC) {
        *reinterpret_cast<uint2 *>(t + i) = make_uint2(c[0], c[1]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < n) t[i + e] = uint8_t(c[e / 4] >> (8 * (e & 3)));
    }
}

// Two random numbers of 16 bits for element `number` of a step, from
// number * kNumberFactor + key.
constexpr uint32_t kNumberFactor = 0x9E3779B1u;
__device__ __forceinline__ uint32_t noise_of(uint32_t z) {
    z = (z ^ (z >> 15)) * 0x6A09E667u;
    z = (z ^ (z >> 13)) * 0xBB67AE85u;
    return z ^ (z >> 16);
}

// The code of a (at most 448, but for rounding; not negative, not NaN): the code
// below or the one above it, above with the probability of its distance from the
// lower one.  noise: 16 random bits times 16, plus 8.  Adding it to a value's
// bits carries into the three bits of fraction that a code keeps as often as
// the bits below them say.  Below 2^-6 the codes are 2^-9 apart, as they are from
// 2^-6 to 2^-5, so smaller values are moved there; and halved, which makes the
// exponent field of both kinds the code's own but for the different bias.
__device__ __forceinline__ uint32_t random_code(float a, uint32_t noise) {
    if (a < 0x1p-6f) a = fmaf(a, 0.5f, 0x1p-7f);   // (a + 2^-6) / 2, rounded as the sum is
    return min((__float_as_uint(a) + (noise - (120u << 23))) >> 20, 126u);
}

// The scale of a block whose largest magnitude is `top`, and its inverse (0
// where the scale would not be normal: the block's codes are 0).
__device__ __forceinline__ float block_scale(float top, float &inverse) {
    const float scale = __fmul_rn(top, float(1.0 / 448.0));
    inverse = scale >= FLT_MIN ? __fdiv_rn(1.0f, scale) : 0.0f;
    return scale;
}

// The largest magnitude over a block (NaN if there is one): magnitudes order as
// their bits, NaN above all.
__device__ __forceinline__ float block_top(const Pair (&v)[4]) {
    float top = max_nan(fabsf(low(v[0])), fabsf(high(v[0])));
#pragma unroll
    for (int e = 1; e < 4; ++e) top = max_nan(top, max_nan(fabsf(low(v[e])), fabsf(high(v[e]))));
    return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top) & 0x7FFFFFFFu));
}

// Bytes b of four words, in one.
template <int B>
__device__ __forceinline__ uint32_t bytes_of(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
    return __byte_perm(__byte_perm(w0, w1, B | (B + 4) << 4), __byte_perm(w2, w3, B | (B + 4) << 4), 0x5410);
}

// The codes of a lane's 8 elements of a block, given the inverse scales.  z0:
// of the first element's noise; the last four elements are GAP further.  FINITE:
// no infinity or NaN in the block.
template <int GAP, bool FINITE>
__device__ __forceinline__ void encode_lane(const Pair (&m)[4], const Pair (&root)[4], float mi, float ri, uint32_t z0, uint32_t (&mc)[2],
                                            uint32_t (&rc)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float x[4], y[4];
        uint32_t cm[4], cr[4];
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            const Pair xm = mul2(m[2 * h + e / 2], both(mi)), xr = mul2(root[2 * h + e / 2], both(ri));
            x[e] = low(xm), x[e + 1] = high(xm);
            y[e] = low(xr), y[e + 1] = high(xr);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t z = noise_of(z0 + uint32_t(4 * h + e + h * GAP) * kNumberFactor);
            cm[e] = random_code(fabsf(x[e]), ((z >> 12) & 0xFFFF0u) | 8u);
            cr[e] = random_code(y[e], (z * 16u + 8u) & 0xFFFFFu);
            if (!FINITE) {   // the scale is an infinity or NaN, and every element of the block with it
                if (x[e] != x[e]) cm[e] = encode(x[e]);
                if (y[e] != y[e]) cr[e] = encode(y[e]);
            }
        }
        const uint32_t sign = bytes_of<3>(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
        mc[h] = bytes_of<0>(cm[0], cm[1], cm[2], cm[3]) | (sign & 0x80808080u);
        rc[h] = bytes_of<0>(cr[0], cr[1], cr[2], cr[3]);
        // a zero byte: a root that is not zero has the least code, 2^-9
        if (((rc[h] - 0x01010101u) & ~rc[h] & 0x80808080u) != 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float r = e & 1 ? high(root[2 * h + e / 2]) : low(root[2 * h + e / 2]);
                if (r > 0.0f && cr[e] == 0) rc[h] |= 1u << (8 * e);
            }
        }
    }
}

// The codes and scales of a block's new m and roots: 8 of its elements a lane,
// whose numbers are first, first + 1, ..., the last four GAP further.
template <int GAP>
__device__ __forceinline__ void encode_block(const Pair (&m)[4], const Pair (&root)[4], uint32_t first, uint32_t key, uint32_t (&mc)[2],
                                             uint32_t (&rc)[2], float &ms, float &rs) {
    float mi, ri;
    const float m_top = block_top(m), r_top = block_top(root);
    ms = block_scale(m_top, mi), rs = block_scale(r_top, ri);
    const uint32_t z0 = first * kNumberFactor + key;
    if (m_top < INFINITY && r_top < INFINITY) encode_lane<GAP, true>(m, root, mi, ri, z0, mc, rc);   // the same for the warp
    else encode_lane<GAP, false>(m, root, mi, ri, z0, mc, rc);
}

template <typename G, bool CODES, bool VEC>
__device__ __forceinline__ void step8(const Tensor &t, const G *grad, int64_t i, const Factors &k, uint32_t key) {
    Pair p[4], g[4], m[4], v[4], root[4];
    const int64_t block = i / kBlock;
    load8<VEC>(t.p, i, t.n, p);
    load8<VEC>(grad, i, t.n, g);
    if constexpr (CODES) {
        load_codes<VEC>(static_cast<const uint8_t *>(t.m), i, t.n, t.m_scale[block], m);
        load_codes<VEC>(static_cast<const uint8_t *>(t.v), i, t.n, t.v_scale[block], v);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = mul2(v[e], v[e]);
    } else {
        load8<VEC>(static_cast<const float *>(t.m), i, t.n, m);
        load8<VEC>(static_cast<const float *>(t.v), i, t.n, v);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) update(p[e], g[e], m[e], v[e], root[e], k);
    store8<VEC>(t.p, i, t.n, p);
    if (t.copy != nullptr) store8<VEC>(t.copy, i, t.n, p);
    if constexpr (CODES) {
        if (!VEC) {   // elements past the end are no part of the block
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[e] = pair(i + 2 * e < t.n ? low(m[e]) : 0.0f, i + 2 * e + 1 < t.n ? high(m[e]) : 0.0f);
                root[e] = pair(i + 2 * e < t.n ? low(root[e]) : 0.0f, i + 2 * e + 1 < t.n ? high(root[e]) : 0.0f);
            }
        }
        uint32_t mc[2], rc[2];
        float ms, rs;
        encode_block<0>(m, root, uint32_t(t.first) + uint32_t(i), key, mc, rc, ms, rs);
        store_codes<VEC>(static_cast<uint8_t *>(t.m), i, t.n, mc);
        store_codes<VEC>(static_cast<uint8_t *>(t.v), i, t.n, rc);
        if ((threadIdx.x & 31) == 0 && block * kBlock < t.n) {
            t.m_scale[block] = ms;
            t.v_scale[block] = rs;
        }
    } else {
        store8<VEC>(static_cast<float *>(t.m), i, t.n, m);
        store8<VEC>(static_cast<float *>(t.v), i, t.n, v);
    }
}

// Whether whole blocks of a tensor can be read and written 16 (codes: 8) bytes at a time.
template <bool CODES>
__device__ __forceinline__ bool is_aligned(const Tensor &t, const void *grad) {
    return ((reinterpret_cast<uintptr_t>(t.p) | reinterpret_cast<uintptr_t>(grad) | reinterpret_cast<uintptr_t>(t.copy)) & 15) == 0 &&
           ((reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v)) & (CODES ? 7 : 15)) == 0;
}

// A warp's share of a chunk, straight from memory: one block of 256 at a time,
// whole and aligned, or element by element.
template <typename G, bool CODES>
__device__ __forceinline__ void step_chunk(const Tensor &t, const G *grad, int64_t start, int warp, const Factors &k, uint32_t key) {
    const int64_t end = t.n - start < kChunkElems ? t.n : start + kChunkElems;
    const bool aligned = is_aligned<CODES>(t, grad);
    for (int64_t b = start + int64_t(warp) * kBlock; b < end; b += kAdamThreads / 32 * kBlock) {
        const int64_t i = b + (threadIdx.x & 31) * kPerLane;
        if (aligned && b + kBlock <= t.n) step8<G, CODES, true>(t, grad, i, k, key);
        else step8<G, CODES, false>(t, grad, i < t.n ? i : t.n, k, key);
    }
}

// States in fp32: a CTA a chunk.  66 M parameters with fp32 gradients and bf16
// copies: 283 us, 7.0 TB/s.
template <typename G>
__global__ void __launch_bounds__(kAdamThreads, 4) adamw_kernel(const __grid_constant__ StepArgs a) {
    const Chunk c = a.chunks[blockIdx.x];   // the tables are the plan's: complete before any step
    const Tensor t = a.tensors[c.tensor];
    const G *grad = static_cast<const G *>(a.grads[c.tensor - a.first_tensor]);
    pdl_wait_previous();
    pdl_launch_dependents();
    if (grad == nullptr) return;   // a tensor without a gradient stays as it is
    const Factors k(a, a.grad_scale ? *a.grad_scale : 1.0f);
    step_chunk<G, false>(t, grad, int64_t(c.chunk) * kChunkElems, threadIdx.x >> 5, k, a.key);
}

// States in codes.  An element takes some 90 instructions for its 18 bytes, so
// the loads have to run ahead of the arithmetic: persistent CTAs, whose last
// warp copies chunk after chunk into a ring of stages (whole aligned chunks;
// others are left where they are), and whose 8 other warps take a block each.
// 54.5 M parameters with bf16 gradients and copies: 174 us (5.0 TB/s; the same
// arithmetic on loads of its own 234), bound by the issue of instructions.
constexpr int kStages = 4;
template <typename G>
struct Stage {
    alignas(16) float p[kChunkElems];
    alignas(16) G g[kChunkElems];
    alignas(16) uint8_t m[kChunkElems], v[kChunkElems];
    alignas(16) float m_scale[kChunkElems / kBlock], v_scale[kChunkElems / kBlock];
    alignas(16) Tensor t;
    const G *grad;
    int64_t start;
    int32_t staged;
};

// Four consecutive elements from shared memory.
__device__ __forceinline__ void quad(const float *p, Pair &a, Pair &b) {
    Pair v[2];
    unpack(*reinterpret_cast<const uint4 *>(p), v);
    a = v[0], b = v[1];
}
__device__ __forceinline__ void quad(const __nv_bfloat16 *p, Pair &a, Pair &b) {
    const uint2 q = *reinterpret_cast<const uint2 *>(p);
    const float2 x = widen2(q.x), y = widen2(q.y);
    a = pair(x.x, x.y), b = pair(y.x, y.y);
}
__device__ __forceinline__ void quad(const uint8_t *p, float scale, Pair &a, Pair &b) {
    const uint32_t q = *reinterpret_cast<const uint32_t *>(p);
    a = mul2(decode2(uint16_t(q)), both(scale)), b = mul2(decode2(uint16_t(q >> 16)), both(scale));
}

template <typename G>
__global__ void __launch_bounds__(kAdamThreads + 32, 2) adamw_codes_kernel(const __grid_constant__ StepArgs a, int32_t chunks) {
    extern __shared__ __align__(16) unsigned char smem[];
    Stage<G> *ring = reinterpret_cast<Stage<G> *>(smem);
    __shared__ uint64_t full[kStages], empty[kStages];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], kAdamThreads / 32);
        }
        fence_mbar_init();
    }
    __syncthreads();
    pdl_wait_previous();
    pdl_launch_dependents();
    int stage = 0;
    uint32_t parity = 0;
    if (warp == kAdamThreads / 32) {
        if (lane != 0) return;
        for (int32_t c = blockIdx.x, it = 0; c < chunks; c += gridDim.x, ++it) {
            const Chunk ch = a.chunks[c];
            const Tensor t = a.tensors[ch.tensor];
            const G *grad = static_cast<const G *>(a.grads[ch.tensor - a.first_tensor]);
            const int64_t start = int64_t(ch.chunk) * kChunkElems, block = start / kBlock;
            if (it >= kStages && !mbar_wait(&empty[stage], parity ^ 1)) {
                atomicOr(a.status, kStatusTimeout);
                return;   // (every copy so far has been waited for, or will be by the other warps)
            }
            Stage<G> &s = ring[stage];
            s.t = t;
            s.grad = grad;
            s.start = start;
            s.staged = grad != nullptr && start + kChunkElems <= t.n && is_aligned<true>(t, grad) &&
                       ((reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v) | reinterpret_cast<uintptr_t>(t.m_scale) |
                         reinterpret_cast<uintptr_t>(t.v_scale)) & 15) == 0;
            if (s.staged) {
                mbar_arrive_expect_tx(&full[stage], sizeof(s.p) + sizeof(s.g) + sizeof(s.m) + sizeof(s.v) + sizeof(s.m_scale) + sizeof(s.v_scale));
                bulk_g2s(s.p, t.p + start, sizeof(s.p), &full[stage]);
                bulk_g2s(s.g, grad + start, sizeof(s.g), &full[stage]);
                bulk_g2s(s.m, static_cast<const uint8_t *>(t.m) + start, sizeof(s.m), &full[stage]);
                bulk_g2s(s.v, static_cast<const uint8_t *>(t.v) + start, sizeof(s.v), &full[stage]);
                bulk_g2s(s.m_scale, t.m_scale + block, sizeof(s.m_scale), &full[stage]);
                bulk_g2s(s.v_scale, t.v_scale + block, sizeof(s.v_scale), &full[stage]);
            } else {
                mbar_arrive(&full[stage]);
            }
            if (++stage == kStages) stage = 0, parity ^= 1;
        }
        return;
    }
    const Factors k(a, a.grad_scale ? *a.grad_scale : 1.0f);
    static_assert(kChunkElems == kAdamThreads / 32 * kBlock, "a block a warp");
    for (int32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        if (!mbar_wait(&full[stage], parity)) {   // a copy that never came
            if (lane == 0) atomicOr(a.status, kStatusTimeout);
            mbar_wait(&full[stage], parity);      // one more second for it to land before the CTA leaves
            return;
        }
        const Stage<G> &s = ring[stage];
        if (s.staged) {
            // a lane has 4 elements of either half of the block
            const int at = warp * kBlock + 4 * lane;
            Pair p[4], g[4], m[4], v[4], root[4];
            const float m_scale = s.m_scale[warp], v_scale = s.v_scale[warp];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                quad(s.p + at + 128 * h, p[2 * h], p[2 * h + 1]);
                quad(s.g + at + 128 * h, g[2 * h], g[2 * h + 1]);
                quad(s.m + at + 128 * h, m_scale, m[2 * h], m[2 * h + 1]);
                quad(s.v + at + 128 * h, v_scale, v[2 * h], v[2 * h + 1]);
            }
            const int64_t i = s.start + at, block = s.start / kBlock + warp;
            float *tp = s.t.p + i;
            __nv_bfloat16 *tc = s.t.copy;
            uint8_t *tm = static_cast<uint8_t *>(s.t.m) + i, *tv = static_cast<uint8_t *>(s.t.v) + i;
            float *tms = s.t.m_scale + block, *tvs = s.t.v_scale + block;
            const uint32_t first = uint32_t(s.t.first) + uint32_t(i);
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[stage]);   // the warp has read its part
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = mul2(v[e], v[e]);
                update(p[e], g[e], m[e], v[e], root[e], k);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Pair q[2] = {p[2 * h], p[2 * h + 1]};
                *reinterpret_cast<uint4 *>(tp + 128 * h) = pack(q);
                if (tc != nullptr) {
                    const __nv_bfloat162 x = __floats2bfloat162_rn(low(q[0]), high(q[0])), y = __floats2bfloat162_rn(low(q[1]), high(q[1]));
                    *reinterpret_cast<uint2 *>(tc + i + 128 * h) =
                        make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y));
                }
            }
            uint32_t mc[2], rc[2];
            float ms, rs;
            encode_block<124>(m, root, first, a.key, mc, rc, ms, rs);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                *reinterpret_cast<uint32_t *>(tm + 128 * h) = mc[h];
                *reinterpret_cast<uint32_t *>(tv + 128 * h) = rc[h];
            }
            if (lane == 0) *tms = ms, *tvs = rs;
        } else {
            const Tensor t = s.t;
            const G *grad = s.grad;
            const int64_t start = s.start;
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[stage]);
            if (grad != nullptr) step_chunk<G, true>(t, grad, start, warp, k, a.key);
        }
        if (++stage == kStages) stage = 0, parity ^= 1;
    }
}

template <typename G>
cudaError_t launch_step(const StepArgs &a, bool codes, int64_t chunks, cudaStream_t stream) {
    if (!codes) return launch_ex(adamw_kernel<G>, dim3(unsigned(chunks)), dim3(kAdamThreads), 0, stream, 1, true, a);
    const auto kernel = adamw_codes_kernel<G>;
    constexpr size_t smem = kStages * sizeof(Stage<G>);
    const cudaError_t e = allow_smem(kernel, smem + 1024);
    if (e != cudaSuccess) return e;
    const int64_t per_sm = per_device(reinterpret_cast<const void *>(kernel), 0, [&]() -> long long {
        int n = 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kAdamThreads + 32, smem) != cudaSuccess) cudaGetLastError();
        return std::max(n, 1);
    });
    return launch_ex(kernel, dim3(unsigned(std::min(chunks, per_sm * sm_count()))), dim3(kAdamThreads + 32), smem, stream, 1, true, a,
                     int32_t(chunks));
}

}  // namespace
}  // namespace darb

using namespace darb;

struct darb_adamw_s {
    std::vector<darb::Tensor> tensors;
    std::vector<int64_t> first_chunk;   // of every tensor, and the number of all
    std::vector<darb::Range> written;   // all buffers that a step writes, in order of address, none twice
    darb_dtype_t gtype = DARB_F32;
    bool codes = false;
    void *dmem = nullptr;
    const darb::Tensor *d_tensors = nullptr;
    const darb::Chunk *d_chunks = nullptr;
    int32_t *d_status = nullptr;
};

namespace {

std::mutex g_plans_mu;
std::unordered_set<const darb_adamw_s *> g_plans;

bool live_plan(const darb_adamw_s *p) {
    std::lock_guard<std::mutex> lk(g_plans_mu);
    return p != nullptr && g_plans.count(p) != 0;
}

// The buffers that a step writes of a tensor, each with its bytes.
std::vector<Range> written(const Tensor &t, bool codes) {
    const int64_t blocks = (t.n + kBlock - 1) / kBlock, state = codes ? t.n : t.n * 4;
    return {{t.p, t.n * 4}, {t.m, state}, {t.v, state}, {t.m_scale, blocks * 4}, {t.v_scale, blocks * 4}, {t.copy, t.n * 2}};
}

// Whether the bytes from p on meet one of the plan's buffers.
bool meets_written(const darb_adamw_s &plan, const void *p, int64_t bytes) {
    const auto after = std::upper_bound(plan.written.begin(), plan.written.end(), p,
                                        [](const void *q, const Range &r) { return std::less<const void *>()(q, r.p); });
    if (after != plan.written.end() && ranges_overlap(after->p, after->bytes, p, bytes)) return true;
    return after != plan.written.begin() && ranges_overlap((after - 1)->p, (after - 1)->bytes, p, bytes);
}

darb_status_t build_plan(darb_adamw_s *plan, int32_t n, const int64_t *numel, float *const *params, void *const *m,
                         void *const *v, float *const *m_scale, float *const *v_scale, void *const *copies,
                         cudaStream_t stream) {
    std::vector<Chunk> chunks;
    std::vector<Range> &all = plan->written;
    int64_t first = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (numel[i] < 0) return DARB_ERR_INVALID_ARG;
        if (numel[i] > kMaxSpan) return DARB_ERR_UNSUPPORTED;
        Tensor t = {};
        t.n = numel[i];
        t.first = first;
        t.p = params[i];
        t.m = m[i];
        t.v = v[i];
        if (plan->codes) {
            t.m_scale = m_scale[i];
            t.v_scale = v_scale[i];
        }
        if (copies != nullptr) t.copy = static_cast<__nv_bfloat16 *>(copies[i]);
        if (t.n > 0) {
            if (t.p == nullptr || t.m == nullptr || t.v == nullptr ||
                (plan->codes && (t.m_scale == nullptr || t.v_scale == nullptr)))
                return DARB_ERR_INVALID_ARG;
            if (!aligned_to(t.p, 4) || !aligned_to(t.m, plan->codes ? 1 : 4) || !aligned_to(t.v, plan->codes ? 1 : 4) ||
                !aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4) || !aligned_to(t.copy, 2))
                return DARB_ERR_INVALID_ARG;
            for (const Range &r : written(t, plan->codes))
                if (r.p != nullptr) all.push_back(r);
        }
        plan->first_chunk.push_back(int64_t(chunks.size()));
        const int64_t count = (t.n + kChunkElems - 1) / kChunkElems;
        if (int64_t(chunks.size()) + count > INT32_MAX) return DARB_ERR_UNSUPPORTED;
        for (int64_t c = 0; c < count; ++c) chunks.push_back({i, int32_t(c)});
        first += (t.n + kBlock - 1) / kBlock * kBlock;
        plan->tensors.push_back(t);
    }
    plan->first_chunk.push_back(int64_t(chunks.size()));
    std::sort(all.begin(), all.end(), [](const Range &a, const Range &b) { return std::less<const void *>()(a.p, b.p); });
    for (size_t i = 1; i < all.size(); ++i)
        if (ranges_overlap(all[i - 1].p, all[i - 1].bytes, all[i].p, all[i].bytes)) return DARB_ERR_INVALID_ARG;
    if (chunks.empty()) return DARB_OK;
    const char *fail = std::getenv("DARB_FAIL_ALLOC");   // test hook, as for the library's other allocations
    if (fail != nullptr && fail[0] == '1') return DARB_ERR_OOM;
    // the status word, the tensors, the chunks
    const size_t o_tensors = 256, o_chunks = o_tensors + (plan->tensors.size() * sizeof(Tensor) + 255) / 256 * 256;
    const cudaError_t e = cudaMalloc(&plan->dmem, o_chunks + chunks.size() * sizeof(Chunk));
    if (e != cudaSuccess) {
        cudaGetLastError();
        plan->dmem = nullptr;
        return e == cudaErrorMemoryAllocation ? DARB_ERR_OOM : DARB_ERR_CUDA;
    }
    char *d = static_cast<char *>(plan->dmem);
    plan->d_status = reinterpret_cast<int32_t *>(d);
    plan->d_tensors = reinterpret_cast<const Tensor *>(d + o_tensors);
    plan->d_chunks = reinterpret_cast<const Chunk *>(d + o_chunks);
    cudaError_t c = cudaMemsetAsync(d, 0, 4, stream);
    if (c == cudaSuccess)
        c = cudaMemcpyAsync(d + o_tensors, plan->tensors.data(), plan->tensors.size() * sizeof(Tensor), cudaMemcpyHostToDevice, stream);
    if (c == cudaSuccess)
        c = cudaMemcpyAsync(d + o_chunks, chunks.data(), chunks.size() * sizeof(Chunk), cudaMemcpyHostToDevice, stream);
    // the chunks leave with this call, and steps may come on any stream
    const cudaError_t w = cudaStreamSynchronize(stream);
    if (c == cudaSuccess && w == cudaSuccess) return DARB_OK;
    cudaGetLastError();
    return DARB_ERR_CUDA;
}

void free_plan(darb_adamw_s *plan) {
    if (plan->dmem != nullptr) cudaFree(plan->dmem);
    delete plan;
}

}  // namespace

extern "C" {

darb_status_t darb_adamw_create(int32_t n, const int64_t *numel, float *const *params, void *const *m, void *const *v,
                                float *const *m_scale, float *const *v_scale, void *const *copies, darb_dtype_t gtype,
                                darb_adamw_t *out, cudaStream_t stream) {
    DARB_TRACE("darb_adamw_create");
    if (out == nullptr) return DARB_ERR_INVALID_ARG;
    *out = nullptr;
    if (n <= 0 || numel == nullptr || params == nullptr || m == nullptr || v == nullptr ||
        (m_scale == nullptr) != (v_scale == nullptr) || !token_dtype(gtype))
        return DARB_ERR_INVALID_ARG;
    darb_adamw_s *plan = new (std::nothrow) darb_adamw_s();
    if (plan == nullptr) return DARB_ERR_OOM;
    plan->gtype = gtype;
    plan->codes = m_scale != nullptr;
    darb_status_t st;
    try {
        st = build_plan(plan, n, numel, params, m, v, m_scale, v_scale, copies, stream);
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

darb_status_t darb_adamw_step(darb_adamw_t plan, const void *const *grads, const float *grad_scale, int64_t step,
                              uint64_t seed, double lr, double beta1, double beta2, double eps, double weight_decay,
                              cudaStream_t stream) {
    DARB_TRACE("darb_adamw_step");
    if (!live_plan(plan) || grads == nullptr || step < 1 || !aligned_to(grad_scale, 4)) return DARB_ERR_INVALID_ARG;
    if (!(lr >= 0.0 && std::isfinite(lr)) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) ||
        !(eps >= 0.0 && std::isfinite(eps)) || !(weight_decay >= 0.0 && std::isfinite(weight_decay)))
        return DARB_ERR_INVALID_ARG;
    if (grad_scale != nullptr && meets_written(*plan, grad_scale, 4)) return DARB_ERR_INVALID_ARG;
    const size_t es = dtype_size(plan->gtype);
    const int32_t n = int32_t(plan->tensors.size());
    for (int32_t i = 0; i < n; ++i) {
        const Tensor &t = plan->tensors[i];
        if (grads[i] == nullptr || t.n == 0) continue;
        if (!aligned_to(grads[i], es) || meets_written(*plan, grads[i], t.n * int64_t(es))) return DARB_ERR_INVALID_ARG;
    }
    StepArgs a;
    a.tensors = plan->d_tensors;
    a.grad_scale = grad_scale;
    a.status = plan->d_status;
    a.b1 = float(beta1), a.c1 = float(1.0 - beta1), a.b2 = float(beta2), a.c2 = float(1.0 - beta2);
    a.decay = float(1.0 - lr * weight_decay);
    a.step_size = float(lr / (1.0 - std::pow(beta1, double(step))));
    a.root_scale = float(1.0 / std::sqrt(1.0 - std::pow(beta2, double(step))));
    a.eps = float(eps);
    a.key = uint32_t((seed * 0x9E3779B97F4A7C15ull) >> 32);
    for (int32_t t0 = 0; t0 < n; t0 += kGradPointers) {
        const int32_t t1 = std::min(n, t0 + kGradPointers);
        const int64_t chunks = plan->first_chunk[t1] - plan->first_chunk[t0];
        if (chunks == 0) continue;
        a.chunks = plan->d_chunks + plan->first_chunk[t0];
        a.first_tensor = t0;
        for (int32_t i = t0; i < t1; ++i) a.grads[i - t0] = grads[i];
        const darb_status_t st = enqueue([&] {
            return plan->gtype == DARB_BF16 ? launch_step<__nv_bfloat16>(a, plan->codes, chunks, stream)
                                            : launch_step<float>(a, plan->codes, chunks, stream);
        });
        if (st != DARB_OK) return st;
    }
    return DARB_OK;
}

darb_status_t darb_adamw_sync_status(darb_adamw_t plan, cudaStream_t stream) {
    DARB_TRACE("darb_adamw_sync_status");
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

darb_status_t darb_adamw_destroy(darb_adamw_t plan) {
    DARB_TRACE("darb_adamw_destroy");
    if (plan == nullptr) return DARB_OK;
    {
        std::lock_guard<std::mutex> lk(g_plans_mu);
        if (g_plans.erase(plan) == 0) return DARB_ERR_INVALID_ARG;
    }
    free_plan(plan);
    return DARB_OK;
}

}  // extern "C"
