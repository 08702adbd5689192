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

__device__ __forceinline__ void update(float &p, float g, float &m, float &v, float &root, const StepArgs &a) {
    m = __fadd_rn(__fmul_rn(m, a.b1), __fmul_rn(g, a.c1));
    v = __fadd_rn(__fmul_rn(v, a.b2), __fmul_rn(__fmul_rn(g, g), a.c2));
    root = __fsqrt_rn(v);
    const float denom = __fadd_rn(__fmul_rn(root, a.root_scale), a.eps);
    p = __fsub_rn(__fmul_rn(p, a.decay), __fdiv_rn(__fmul_rn(m, a.step_size), denom));
}

// Elements i .. i + 8 of a tensor as fp32 (VEC: i is a multiple of 8 and the
// tensor 16-byte aligned; else zeros from n on).
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T *t, int64_t i, int64_t n, float (&v)[8]) {
    if (VEC) {
        if constexpr (sizeof(T) == 4) {
            const uint4 lo = *reinterpret_cast<const uint4 *>(t + i), hi = *reinterpret_cast<const uint4 *>(t + i + 4);
            v[0] = __uint_as_float(lo.x), v[1] = __uint_as_float(lo.y), v[2] = __uint_as_float(lo.z), v[3] = __uint_as_float(lo.w);
            v[4] = __uint_as_float(hi.x), v[5] = __uint_as_float(hi.y), v[6] = __uint_as_float(hi.z), v[7] = __uint_as_float(hi.w);
        } else {
            unpack(*reinterpret_cast<const uint4 *>(t + i), v);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = i + e < n ? widen(t[i + e]) : 0.0f;
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T *t, int64_t i, int64_t n, const float (&v)[8]) {
    if (VEC) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(t + i) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>(t + i + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint4 *>(t + i) = pack(v);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < n) t[i + e] = narrow<T>(v[e]);
    }
}

// e4m3 codes to fp32 (exact), two at a time.
__device__ __forceinline__ float2 decode2(uint16_t codes) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(codes));
    float2 f;
    asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %2;\n cvt.f32.f16 %0, lo;\n cvt.f32.f16 %1, hi;\n}"
        : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}
__device__ __forceinline__ uint16_t encode2(float lo, float hi) {   // values that codes have
    uint16_t c;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(hi), "f"(lo));
    return c;
}
template <bool VEC>
__device__ __forceinline__ void load_codes(const uint8_t *t, int64_t i, int64_t n, float scale, float (&v)[8]) {
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
    for (int e = 0; e < 8; e += 2) {
        const float2 f = decode2(uint16_t(w[e >> 2] >> (8 * (e & 3))));
        v[e] = __fmul_rn(f.x, scale);
        v[e + 1] = __fmul_rn(f.y, scale);
    }
}
template <bool VEC>
__device__ __forceinline__ void store_codes(uint8_t *t, int64_t i, int64_t n, const float (&c)[8]) {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
        w[h] = uint32_t(encode2(c[4 * h], c[4 * h + 1])) | uint32_t(encode2(c[4 * h + 2], c[4 * h + 3])) << 16;
    if (VEC) {
        *reinterpret_cast<uint2 *>(t + i) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < n) t[i + e] = uint8_t(w[e >> 2] >> (8 * (e & 3)));
    }
}

// Two random numbers of 16 bits for element `number` of a step.
__device__ __forceinline__ uint32_t noise_of(uint32_t number, uint32_t key) {
    uint32_t z = number * 0x9E3779B1u + key;
    z = (z ^ (z >> 15)) * 0x6A09E667u;
    z = (z ^ (z >> 13)) * 0xBB67AE85u;
    return z ^ (z >> 16);
}

// x (at most 448 in magnitude, but for rounding) to the value of a code next to
// it, away from zero with the probability of its distance from the other one.
__device__ __forceinline__ float random_code(float x, uint32_t noise16) {
    const float a = fabsf(x);
    // below 2^-6 the codes are 2^-9 apart, as they are from 2^-6 to 2^-5
    const float shift = a < 0x1p-6f ? 0x1p-6f : 0.0f;
    const uint32_t bits = (__float_as_uint(__fadd_rn(a, shift)) + (noise16 << 4) + 8u) & 0xFFF00000u;
    const float c = fminf(__fsub_rn(__uint_as_float(bits), shift), 448.0f);
    return copysignf(a == a ? c : a, x);
}

// The scale of a block from the lanes' values, and its inverse (0 where the
// block's values are below the smallest normal scale: their codes are 0).
__device__ __forceinline__ float block_scale(const float (&v)[8], float &inverse) {
    // magnitudes order as their bits, NaN above all
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    const float scale = __fmul_rn(__uint_as_float(top), float(1.0 / 448.0));
    inverse = scale >= FLT_MIN ? __fdiv_rn(1.0f, scale) : 0.0f;
    return scale;
}

template <typename G, bool CODES, bool VEC>
__device__ __forceinline__ void step8(const Tensor &t, const G *grad, int64_t i, float grad_scale, const StepArgs &a) {
    float p[8], g[8], m[8], v[8], root[8];
    const int64_t block = i / kBlock;
    load8<VEC>(t.p, i, t.n, p);
    load8<VEC>(grad, i, t.n, g);
    if constexpr (CODES) {
        load_codes<VEC>(static_cast<const uint8_t *>(t.m), i, t.n, t.m_scale[block], m);
        load_codes<VEC>(static_cast<const uint8_t *>(t.v), i, t.n, t.v_scale[block], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], v[e]);
    } else {
        load8<VEC>(static_cast<const float *>(t.m), i, t.n, m);
        load8<VEC>(static_cast<const float *>(t.v), i, t.n, v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) update(p[e], __fmul_rn(g[e], grad_scale), m[e], v[e], root[e], a);
    store8<VEC>(t.p, i, t.n, p);
    if (t.copy != nullptr) store8<VEC>(t.copy, i, t.n, p);
    if constexpr (CODES) {
        if (!VEC) {   // elements past the end are no part of the block
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i + e >= t.n) m[e] = root[e] = 0.0f;
        }
        float mi, ri;
        const float ms = block_scale(m, mi), rs = block_scale(root, ri);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t z = noise_of(uint32_t(t.first + i) + e, a.key);
            m[e] = random_code(__fmul_rn(m[e], mi), z >> 16);
            const float c = random_code(__fmul_rn(root[e], ri), z & 0xFFFFu);
            root[e] = root[e] > 0.0f && c == 0.0f ? 0x1p-9f : c;
        }
        store_codes<VEC>(static_cast<uint8_t *>(t.m), i, t.n, m);
        store_codes<VEC>(static_cast<uint8_t *>(t.v), i, t.n, root);
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
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ StepArgs a) {
    const Chunk c = a.chunks[blockIdx.x];   // the tables are the plan's: complete before any step
    const Tensor t = a.tensors[c.tensor];
    const G *grad = static_cast<const G *>(a.grads[c.tensor - a.first_tensor]);
    pdl_wait_previous();
    pdl_launch_dependents();
    if (grad == nullptr) return;   // a tensor without a gradient stays as it is
    const float grad_scale = a.grad_scale ? *a.grad_scale : 1.0f;
    const bool aligned = ((reinterpret_cast<uintptr_t>(t.p) | reinterpret_cast<uintptr_t>(grad) |
                           reinterpret_cast<uintptr_t>(t.copy)) & 15) == 0 &&
                         ((reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v)) & (CODES ? 7 : 15)) == 0;
    const int64_t start = int64_t(c.chunk) * kChunkElems;
    const int64_t end = t.n - start < kChunkElems ? t.n : start + kChunkElems;
    for (int64_t i = start + int64_t(threadIdx.x) * kPerLane; i - (threadIdx.x & 31) * kPerLane < end;
         i += kAdamThreads * kPerLane) {
        // a warp takes one block of 256: whole and aligned, or element by element
        const int64_t block_end = i - (threadIdx.x & 31) * kPerLane + kBlock;
        if (aligned && block_end <= t.n) step8<G, CODES, true>(t, grad, i, grad_scale, a);
        else step8<G, CODES, false>(t, grad, i < t.n ? i : t.n, grad_scale, a);
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
