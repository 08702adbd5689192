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
// The step is bound by memory (28 bytes an element with fp32 gradients and states):
// a CTA takes one chunk of kChunkElems consecutive elements of one tensor, so
// that tensors of any sizes share the machine evenly; which chunk of which
// tensor is looked up in a table made with the plan.  A warp takes a whole
// block of 256, 8 elements a lane, so that a block's maximum is one reduction.
#include "launch.cuh"
#include "tma.cuh"
#include "tokens.cuh"
#include "trace.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdlib>
#include <mutex>
#include <new>
#include <unordered_set>
#include <vector>

namespace darb {
namespace {

constexpr int kBlock = DARB_ADAMW_BLOCK;
constexpr int kAdamThreads = 256;
constexpr int kChunkElems = 4096;
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
__device__ __forceinline__ void store_codes(uint8_t *t, int64_t i, int64_t n, const uint32_t (&c)[8]) {
    const uint32_t lo = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, hi = c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24;
    if (VEC) {
        *reinterpret_cast<uint2 *>(t + i) = make_uint2(lo, hi);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < n) t[i + e] = uint8_t(c[e]);
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

// The code of |x| (at most 448, but for rounding; not NaN): the code below or
// the one above it, above with the probability of its distance from the lower
// one.  noise: 16 random bits times 16, plus 8.  Adding it to a value's bits
// carries into the three bits of fraction that a code keeps as often as the
// bits below them say; below 2^-6 the codes are 2^-9 apart, as they are from
// 2^-6 to 2^-5, so smaller values are moved there and back.
__device__ __forceinline__ uint32_t random_code(float x, uint32_t noise) {
    const float a = fabsf(x);
    const bool small = a < 0x1p-6f;
    const uint32_t bits = __float_as_uint(__fadd_rn(a, small ? 0x1p-6f : 0.0f)) + noise;
    // fp32 exponents count from 127 and codes' from 7: 120 << 3; a moved value is 1 << 3 too high
    return min((bits >> 20) - (small ? 968u : 960u), 126u);
}

// The scale of a block whose largest magnitude has the bits `top`, and its
// inverse (0 where the scale would not be normal: the block's codes are 0).
__device__ __forceinline__ float block_scale(uint32_t top, float &inverse) {
    const float scale = __fmul_rn(__uint_as_float(top), float(1.0 / 448.0));
    inverse = scale >= FLT_MIN ? __fdiv_rn(1.0f, scale) : 0.0f;
    return scale;
}

// The largest magnitude's bits over a block (magnitudes order as their bits,
// NaN above all).
__device__ __forceinline__ uint32_t block_top(const Pair (&v)[4]) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        top = max(top, max(__float_as_uint(low(v[e])) & 0x7FFFFFFFu, __float_as_uint(high(v[e])) & 0x7FFFFFFFu));
    return __reduce_max_sync(0xFFFFFFFFu, top);
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
        float mi, ri;
        const uint32_t m_top = block_top(m), r_top = block_top(root);
        const float ms = block_scale(m_top, mi), rs = block_scale(r_top, ri);
        const uint32_t first = (uint32_t(t.first) + uint32_t(i)) * kNumberFactor + key;
        uint32_t mc[8], rc[8];
        if (max(m_top, r_top) < 0x7F800000u) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const Pair xm = mul2(m[e / 2], both(mi)), xr = mul2(root[e / 2], both(ri));
                const float x = e & 1 ? high(xm) : low(xm), y = e & 1 ? high(xr) : low(xr), r = e & 1 ? high(root[e / 2]) : low(root[e / 2]);
                const uint32_t z = noise_of(first + uint32_t(e) * kNumberFactor);
                mc[e] = random_code(x, ((z >> 12) & 0xFFFF0u) | 8u) | (__float_as_uint(x) >> 24 & 0x80u);
                const uint32_t c = random_code(y, (z * 16u + 8u) & 0xFFFFFu);
                rc[e] = r > 0.0f ? max(c, 1u) : c;   // the least code is 2^-9
            }
        } else {
            // an infinity or NaN: the scale is one too, and every element with it
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = __fmul_rn(e & 1 ? high(m[e / 2]) : low(m[e / 2]), mi), r = e & 1 ? high(root[e / 2]) : low(root[e / 2]);
                const float y = __fmul_rn(r, ri);
                const uint32_t z = noise_of(first + uint32_t(e) * kNumberFactor);
                mc[e] = x != x ? encode(x) : random_code(x, ((z >> 12) & 0xFFFF0u) | 8u) | (__float_as_uint(x) >> 24 & 0x80u);
                const uint32_t c = y != y ? encode(y) : random_code(y, (z * 16u + 8u) & 0xFFFFFu);
                rc[e] = r > 0.0f ? max(c, 1u) : c;
            }
        }
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

template <typename G, bool CODES>
__global__ void __launch_bounds__(kAdamThreads, 4) adamw_kernel(const __grid_constant__ StepArgs a) {
    const Chunk c = a.chunks[blockIdx.x];   // the tables are the plan's: complete before any step
    const Tensor t = a.tensors[c.tensor];
    const G *grad = static_cast<const G *>(a.grads[c.tensor - a.first_tensor]);
    pdl_wait_previous();
    pdl_launch_dependents();
    if (grad == nullptr) return;   // a tensor without a gradient stays as it is
    const Factors k(a, a.grad_scale ? *a.grad_scale : 1.0f);
    const bool aligned = ((reinterpret_cast<uintptr_t>(t.p) | reinterpret_cast<uintptr_t>(grad) |
                           reinterpret_cast<uintptr_t>(t.copy)) & 15) == 0 &&
                         ((reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v)) & (CODES ? 7 : 15)) == 0;
    const int64_t start = int64_t(c.chunk) * kChunkElems;
    const int64_t end = t.n - start < kChunkElems ? t.n : start + kChunkElems;
    for (int64_t i = start + int64_t(threadIdx.x) * kPerLane; i - (threadIdx.x & 31) * kPerLane < end;
         i += kAdamThreads * kPerLane) {
        // a warp takes one block of 256: whole and aligned, or element by element
        const int64_t block_end = i - (threadIdx.x & 31) * kPerLane + kBlock;
        if (aligned && block_end <= t.n) step8<G, CODES, true>(t, grad, i, k, a.key);
        else step8<G, CODES, false>(t, grad, i < t.n ? i : t.n, k, a.key);
    }
}

}  // namespace
}  // namespace darb

using namespace darb;

struct darb_adamw_s {
    std::vector<darb::Tensor> tensors;
    std::vector<int64_t> first_chunk;   // of every tensor, and the number of all
    darb_dtype_t gtype = DARB_F32;
    bool codes = false;
    void *dmem = nullptr;
    const darb::Tensor *d_tensors = nullptr;
    const darb::Chunk *d_chunks = nullptr;
};

namespace {

std::mutex g_plans_mu;
std::unordered_set<const darb_adamw_s *> g_plans;

bool live_plan(const darb_adamw_s *p) {
    std::lock_guard<std::mutex> lk(g_plans_mu);
    return p != nullptr && g_plans.count(p) != 0;
}

// One past the buffers that tensor i writes, each with its bytes.
std::vector<Range> written(const Tensor &t, bool codes) {
    const int64_t blocks = (t.n + kBlock - 1) / kBlock, state = codes ? t.n : t.n * 4;
    return {{t.p, t.n * 4}, {t.m, state}, {t.v, state}, {t.m_scale, blocks * 4}, {t.v_scale, blocks * 4}, {t.copy, t.n * 2}};
}

darb_status_t build_plan(darb_adamw_s *plan, int32_t n, const int64_t *numel, float *const *params, void *const *m,
                         void *const *v, float *const *m_scale, float *const *v_scale, void *const *copies,
                         cudaStream_t stream) {
    std::vector<Chunk> chunks;
    std::vector<Range> all;
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
    std::sort(all.begin(), all.end(), [](const Range &a, const Range &b) { return a.p < b.p; });
    for (size_t i = 1; i < all.size(); ++i)
        if (ranges_overlap(all[i - 1].p, all[i - 1].bytes, all[i].p, all[i].bytes)) return DARB_ERR_INVALID_ARG;
    if (chunks.empty()) return DARB_OK;
    const char *fail = std::getenv("DARB_FAIL_ALLOC");   // test hook, as for the library's other allocations
    if (fail != nullptr && fail[0] == '1') return DARB_ERR_OOM;
    const size_t o_chunks = (plan->tensors.size() * sizeof(Tensor) + 255) / 256 * 256;
    const cudaError_t e = cudaMalloc(&plan->dmem, o_chunks + chunks.size() * sizeof(Chunk));
    if (e != cudaSuccess) {
        cudaGetLastError();
        plan->dmem = nullptr;
        return e == cudaErrorMemoryAllocation ? DARB_ERR_OOM : DARB_ERR_CUDA;
    }
    char *d = static_cast<char *>(plan->dmem);
    plan->d_tensors = reinterpret_cast<const Tensor *>(d);
    plan->d_chunks = reinterpret_cast<const Chunk *>(d + o_chunks);
    cudaError_t c = cudaMemcpyAsync(d, plan->tensors.data(), plan->tensors.size() * sizeof(Tensor), cudaMemcpyHostToDevice, stream);
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
    } catch (const std::bad_alloc &) {
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
    const size_t es = dtype_size(plan->gtype);
    const int32_t n = int32_t(plan->tensors.size());
    for (int32_t i = 0; i < n; ++i) {
        const Tensor &t = plan->tensors[i];
        if (grads[i] == nullptr || t.n == 0) continue;
        if (!aligned_to(grads[i], es)) return DARB_ERR_INVALID_ARG;
        const int64_t state = plan->codes ? t.n : t.n * 4, g = t.n * int64_t(es);
        if (ranges_overlap(grads[i], g, t.p, t.n * 4) || ranges_overlap(grads[i], g, t.m, state) ||
            ranges_overlap(grads[i], g, t.v, state) || ranges_overlap(grads[i], g, t.copy, t.n * 2))
            return DARB_ERR_INVALID_ARG;
    }
    StepArgs a;
    a.tensors = plan->d_tensors;
    a.grad_scale = grad_scale;
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
        const auto kernel = plan->gtype == DARB_BF16 ? (plan->codes ? adamw_kernel<__nv_bfloat16, true> : adamw_kernel<__nv_bfloat16, false>)
                                                     : (plan->codes ? adamw_kernel<float, true> : adamw_kernel<float, false>);
        if (launch_ex(kernel, dim3(unsigned(chunks)), dim3(kAdamThreads), 0, stream, 1, true, a) != cudaSuccess) {
            cudaGetLastError();
            return DARB_ERR_CUDA;
        }
    }
    return DARB_OK;
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
