// tokens.cuh -- pieces shared by the kernels that work on token activations
// (log probabilities, layer norm, optimizer): 16-byte loads and stores of fp32
// or bf16 values widened to fp32, packed fp32 arithmetic, the base-2
// exponential, NaN-keeping maxima, and the host's argument checks.
//
// A row of F values starts at any element-aligned address.  The kernels cut it
// into "granules", the 16-byte aligned words of memory that overlap it: granule
// i covers elements [i*V - head, i*V - head + V) with V = 16 / element size and
// head = the elements by which the row starts past a 16-byte boundary.  Only
// the first and the last granule can be partial, and those are read and
// written element by element, so that no byte outside the row is touched.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <new>

#include "darb.h"

namespace darb {

template <typename T>
constexpr int kPerGranule = 16 / int(sizeof(T));

// ---- values ----
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// The two bf16 halves of a word, widened (exact).
__device__ __forceinline__ float2 widen2(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}

__device__ __forceinline__ void unpack(const uint4 &q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x), v[1] = __uint_as_float(q.y), v[2] = __uint_as_float(q.z), v[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack(const uint4 &q, float (&v)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = widen2(w[i]);
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ uint4 pack(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- granules of a row of n values ----
template <typename T>
__host__ __device__ __forceinline__ int row_head(const void *row) {
    return int((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
}
template <typename T>
__host__ __device__ __forceinline__ int64_t row_granules(int head, int64_t n) {
    return (head + n + kPerGranule<T> - 1) / kPerGranule<T>;
}

// Elements j0 .. j0 + V of a row (j0 = granule * V - head, so that row + j0 is
// 16-byte aligned), `fill` outside [0, n).  (Not through the read-only path: the
// kernel ahead may write the row while this one is resident.)
template <typename T>
__device__ __forceinline__ uint4 load_granule(const T *row, int64_t j0, int64_t n, float fill) {
    constexpr int V = kPerGranule<T>;
    if (j0 >= 0 && j0 + V <= n) {
        return *reinterpret_cast<const uint4 *>(row + j0);
    }
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = j0 + e >= 0 && j0 + e < n ? widen(row[j0 + e]) : fill;
    return pack(v);
}
template <typename T>
__device__ __forceinline__ void store_granule(T *row, int64_t j0, int64_t n, const float (&v)[kPerGranule<T>]) {
    constexpr int V = kPerGranule<T>;
    if (j0 >= 0 && j0 + V <= n) {
        *reinterpret_cast<uint4 *>(row + j0) = pack(v);
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (j0 + e >= 0 && j0 + e < n) row[j0 + e] = narrow<T>(v[e]);
}

// ---- arithmetic ----
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// 2^x (one instruction, results below 2^-126 are 0).
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// max that returns NaN if either operand is one.
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// Two fp32 values in a register pair; an operation on pairs is one instruction,
// each half of it one IEEE operation.  But the assembler contracts a product and the
// sum that it goes into to one rounding, whatever is asked of it: where the two
// roundings matter, the sum is two scalar additions.
struct Pair {
    unsigned long long bits;
};
__device__ __forceinline__ Pair pair(float x, float y) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p.bits) : "f"(x), "f"(y));
    return p;
}
__device__ __forceinline__ Pair both(float v) { return pair(v, v); }
__device__ __forceinline__ float low(Pair p) { return __uint_as_float(uint32_t(p.bits)); }
__device__ __forceinline__ float high(Pair p) { return __uint_as_float(uint32_t(p.bits >> 32)); }
__device__ __forceinline__ float across(Pair p) { return low(p) + high(p); }
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits));
    return r;
}

// A granule as pairs, and back.
__device__ __forceinline__ void unpack(const uint4 &q, Pair (&v)[2]) {
    v[0].bits = uint64_t(q.x) | uint64_t(q.y) << 32;
    v[1].bits = uint64_t(q.z) | uint64_t(q.w) << 32;
}
__device__ __forceinline__ void unpack(const uint4 &q, Pair (&v)[4]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = widen2(w[i]);
        v[i] = pair(f.x, f.y);
    }
}
__device__ __forceinline__ uint4 pack(const Pair (&v)[2]) {
    return make_uint4(uint32_t(v[0].bits), uint32_t(v[0].bits >> 32), uint32_t(v[1].bits), uint32_t(v[1].bits >> 32));
}
__device__ __forceinline__ uint4 pack(const Pair (&v)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(low(v[i]), high(v[i]));
        w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- host side ----

// The status of what `launch` returns (a cudaError_t).  No exception leaves a C
// entry: the tables of kernel attributes can run out of host memory.
template <typename F>
darb_status_t enqueue(F launch) noexcept {
    cudaError_t e;
    try {
        e = launch();
    } catch (const std::bad_alloc &) {
        return DARB_ERR_OOM;
    } catch (...) {
        return DARB_ERR_CUDA;
    }
    if (e == cudaSuccess) return DARB_OK;
    cudaGetLastError();
    if (e == cudaErrorMemoryAllocation) return DARB_ERR_OOM;
    return e == cudaErrorNotSupported ? DARB_ERR_UNSUPPORTED : DARB_ERR_CUDA;
}

inline bool token_dtype(darb_dtype_t t) { return t == DARB_F32 || t == DARB_BF16; }
inline bool token_layout(darb_layout_t l) { return l == DARB_TOKEN_ROWS || l == DARB_TOKEN_COLUMNS; }
inline size_t dtype_size(darb_dtype_t t) { return t == DARB_BF16 ? 2 : 4; }
inline bool aligned_to(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// The most tokens, features or steps of a call, and the most elements that one
// of its buffers may span (so that no index or size leaves its type).
constexpr int64_t kMaxTokens = int64_t(1) << 27;
constexpr int64_t kMaxFeatures = int64_t(1) << 30;
constexpr int64_t kMaxSpan = int64_t(1) << 48;

// The elements from the first to past the last of `tokens` x `features` values
// (of `steps` matrices of token columns, one after the other, features `ld`
// apart); -1 if that is above kMaxSpan.
inline int64_t token_span(darb_layout_t l, int64_t steps, int64_t tokens, int64_t features, int64_t ld) {
    if (tokens <= 0 || steps <= 0 || features <= 0) return 0;
    const __int128 n = l == DARB_TOKEN_ROWS ? static_cast<__int128>(tokens - 1) * ld + features
                                            : (static_cast<__int128>(steps) * features - 1) * ld + tokens;
    return n > kMaxSpan ? -1 : static_cast<int64_t>(n);
}

inline bool ranges_overlap(const void *a, int64_t abytes, const void *b, int64_t bbytes) {
    if (a == nullptr || b == nullptr || abytes <= 0 || bbytes <= 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + static_cast<uintptr_t>(bbytes) && y < x + static_cast<uintptr_t>(abytes);
}

// One buffer of a call, for the check that no output meets another buffer: `bytes`
// from the first to past the last; of a matrix, lines of `width` bytes `pitch` apart.
struct Range {
    const void *p;
    int64_t bytes;
    int64_t pitch = 0, width = 0;
};
// Activations whose span (token_span) has been found to be allowed.
inline Range token_range(const void *p, darb_layout_t l, int64_t steps, int64_t tokens, int64_t features, int64_t ld, size_t es) {
    const int64_t size = static_cast<int64_t>(es), bytes = token_span(l, steps, tokens, features, ld) * size;
    const int64_t lines = l == DARB_TOKEN_ROWS ? tokens : steps * features;
    if (lines < 2) return {p, bytes};
    return {p, bytes, ld * size, (l == DARB_TOKEN_ROWS ? features : tokens) * size};
}
// Whether two buffers share a byte.  Lines of one pitch, or a run and lines, lie side by
// side where either fits between the other's lines (slices of one wide buffer);
// different pitches are told apart by their first and last bytes alone.
inline bool buffers_overlap(const Range &a, const Range &b) {
    if (!ranges_overlap(a.p, a.bytes, b.p, b.bytes)) return false;
    const int64_t pitch = a.pitch > b.pitch ? a.pitch : b.pitch;
    if (pitch == 0 || (a.pitch != b.pitch && a.pitch != 0 && b.pitch != 0)) return true;
    const int64_t wa = a.pitch ? a.width : a.bytes, wb = b.pitch ? b.width : b.bytes;
    int64_t d = static_cast<int64_t>(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)) % pitch;   // of b's lines past a's
    if (d < 0) d += pitch;
    return d < wa || d + wb > pitch;
}
template <int NO, int NI>
inline bool outputs_apart(const Range (&outs)[NO], const Range (&ins)[NI]) {
    for (int o = 0; o < NO; ++o) {
        for (int i = 0; i < NI; ++i)
            if (buffers_overlap(outs[o], ins[i])) return false;
        for (int p = 0; p < o; ++p)
            if (buffers_overlap(outs[o], outs[p])) return false;
    }
    return true;
}

}  // namespace darb
