// scan.cu -- a gated linear recurrence over whole sequences (darb_gated_scan) and
// its backward pass (darb_gated_scan_grad): the recurrent layer whose gates are one
// product of all steps, next to the LSTM and GRU sequences, whose gates need the
// step before.
//
//   a_t = sigmoid(gate_t) (or gate_t itself),  u_t = (1 - a_t) x_t (or x_t),
//   h_t = a_t h_(t-1) + u_t.
// Backward, from the last step to the first, with c what flows to a step from the
// one after it:
//   g_t = dh_t + c,  d_x_t = g_t (1 - a_t) (or g_t),
//   d_gate_t = g_t (h_(t-1) - x_t) a_t (1 - a_t)   (without the x_t where it is not
//   coupled, without a (1 - a) where the gate is a value),  c = a_t g_t.
// In c that is a recurrence of the same form, c_t = a_t c_(t+1) + a_t dh_t, so one
// kernel does both; the backward pass walks the steps with negative strides.
//
// Steps are maps h -> A h + H, and maps compose: (A2, H2) after (A1, H1) is
// (A2 A1, A2 H1 + H2).  A thread takes 16 elements -- 4 steps of 4 neighbouring
// channels, or 16 steps of one -- composes its steps' maps, and learns the state
// before them from the threads (of the CTA, of the cluster) that have the steps
// before.  Then it runs its steps again from registers.  Inputs are read once and
// outputs written once, with no scratch and no waiting on other CTAs but at the
// cluster's barrier; the order of all sums is fixed by the sizes.
//
// What bounds it: memory (12 bytes an element in fp32, 24 backward).  Everything
// else follows from keeping loads in flight: time is split over the 8 warps of a CTA
// and, where the channels alone do not fill the GPU, over the 2 to 8 CTAs of a
// cluster; a thread's next 16 elements are on their way while it works on these.
#include "launch.cuh"
#include "tma.cuh"
#include "tokens.cuh"
#include "trace.h"

#include <algorithm>

namespace darb {

int sm_count();

namespace {

constexpr int kScanThreads = 256;
constexpr int kScanWarps = kScanThreads / 32;
constexpr int kElems = 16;          // elements of a thread in a round
constexpr int kMaxCluster = 8;
constexpr int kNarrow = 8;          // fewer contiguous channels than this: runs of steps go through shared memory
constexpr int kRun = kScanWarps * kElems;   // steps of a CTA in a round there

// The element (outer o, step t, inner i) of a tensor is at o * ld + t * step + i.
struct Operand {
    const void *p;
    int64_t ld, step;
};

struct ScanArgs {
    Operand gate, x, dh, before;   // dh and the states before each step: backward only
    Operand out[2];                // h; or d_gate and d_x
    const float *first;            // the carry before the first step walked (h0; d_last), or null: 0
    const float *h0;               // backward: the state before step 0, or null: 0
    float *last;                   // the carry after the last step walked (h_last; d_h0), or null
    int64_t steps, channels;       // channels: outer x inner
    int32_t outer, inner;
    int32_t groups_log;            // warps that share a channel, each with steps of its own
    int32_t coupled;
};

// V neighbouring elements as they lie in memory.
template <typename T, int V>
struct Word;
template <>
struct Word<float, 4> {
    float4 w;
    __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w; }
    __device__ __forceinline__ void set(const float (&v)[4]) { w = make_float4(v[0], v[1], v[2], v[3]); }
};
template <>
struct Word<__nv_bfloat16, 4> {
    uint2 w;
    __device__ __forceinline__ void get(float (&v)[4]) const {
        const float2 a = widen2(w.x), b = widen2(w.y);
        v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
    }
    __device__ __forceinline__ void set(const float (&v)[4]) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
        w = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
    }
};
template <typename T>
struct Word<T, 1> {
    T w;
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = widen(w); }
    __device__ __forceinline__ void set(const float (&v)[1]) { w = narrow<T>(v[0]); }
};

// a and 1 - a from a gate, each to the last places of its own (a sigmoid near 1
// leaves its distance from 1 exact); +-inf give exactly 1 and 0.
template <bool LOGITS>
__device__ __forceinline__ void open_gate(float gate, float &a, float &rest) {
    if (LOGITS) {
        const float e = exp2_fast(-kLog2e * fabsf(gate));
        const float near = __fdividef(1.0f, 1.0f + e), far = e * near;
        const bool up = gate >= 0.0f;
        a = up ? near : far;
        rest = up ? far : near;
    } else {
        a = gate;
        rest = 1.0f - gate;
    }
}

// The state after a map, from the one before.  Nothing comes of a state of 0, even
// where the product of gates above 1 has overflown.
__device__ __forceinline__ float through(float A, float H, float c) { return c == 0.0f ? H : fmaf(A, c, H); }

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_meet() {
    cluster_arrive();
    cluster_wait();
}
__device__ __forceinline__ void store_remote(float *here, uint32_t rank, float v) {
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_addr(here)), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(v) : "memory");
}

// STAGED: fewer than kNarrow channels lie together, so that a warp's loads would
// touch a sector for every lane.  There a CTA takes 32 / inner rows of kRun steps
// each, read and written along the rows, and turns them through shared memory (rows
// `inner` floats longer than their steps: a warp's 32 channels hit 32 banks).
template <typename T, bool BACK, int V, bool STAGED, bool LOGITS>
__global__ void __launch_bounds__(kScanThreads, BACK ? 1 : 2)
scan_kernel(const ScanArgs s, const int cluster) {
    constexpr int S = kElems / V;          // steps of a thread in a round
    constexpr int IN = BACK ? 4 : 2;       // tensors read
    constexpr int OUT = BACK ? 2 : 1;
    constexpr int W = 32 * V;
    using Raw = Word<T, V>;
    __shared__ float s_A[2][kScanWarps][W], s_H[2][kScanWarps][W];
    __shared__ float s_rA[2][kMaxCluster][W], s_rH[2][kMaxCluster][W];
    __shared__ float s_start[W];
    extern __shared__ float s_tile[];

    pdl_launch_dependents();
    if (cluster > 1) cluster_arrive();   // (the others' shared memory is there once they run)
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tg = 1 << s.groups_log, group = warp & (tg - 1), ct = warp >> s.groups_log;
    const int rank = cluster > 1 ? int(blockIdx.x) % cluster : 0;
    const int64_t tile = blockIdx.x / unsigned(cluster);
    const int64_t steps = s.steps;
    const int L = tg * S;
    const int inner = s.inner;
    const int rows = STAGED ? 32 / inner : 0;                  // rows of a tile
    const int run = kRun * inner, pitch = run + inner;

    // the thread's channels
    int64_t c;
    bool valid;
    if (STAGED) {
        c = tile * (rows * inner) + lane;
        valid = lane < rows * inner && c < s.channels;
    } else {
        c = ((tile * (kScanWarps >> s.groups_log) + ct) * 32 + lane) * V;
        valid = c < s.channels;
    }
    const int64_t co = valid ? c / inner : 0, ci = valid ? c - co * inner : 0;
    // (lanes past the rows' channels read the first one's steps and write none)
    const bool staged = STAGED && lane < rows * inner;
    const int row0 = staged ? lane / inner : 0, rowi = staged ? lane - row0 * inner : 0;

    const Operand *const ins[4] = {&s.gate, &s.x, &s.dh, &s.before};
    const T *in[IN];
    T *out[OUT];
#pragma unroll
    for (int k = 0; k < IN; ++k) in[k] = static_cast<const T *>(ins[k]->p) + (STAGED ? 0 : co * ins[k]->ld + ci);
#pragma unroll
    for (int k = 0; k < OUT; ++k) out[k] = static_cast<T *>(const_cast<void *>(s.out[k].p)) + (STAGED ? 0 : co * s.out[k].ld + ci);

    Raw raw[IN][S];      // not STAGED: the thread's steps; STAGED: elements of the tile, 256 apart
    auto load = [&](int64_t round) {
        const int64_t first = (round * cluster + rank) * L;
        if (STAGED) {
#pragma unroll
            for (int j = 0; j < S; ++j) {
                const int e = tid + j * kScanThreads;
                const int r = inner == 1 ? e / kRun : e / run, q = e - r * run;
                const int tl = inner == 1 ? q : q / inner, i = q - tl * inner;
                const int64_t t = first + tl, o = tile * rows + r;
                const bool on = r < rows && o < s.outer && t < steps;
#pragma unroll
                for (int k = 0; k < IN; ++k) {
                    const float zero[V] = {};
                    raw[k][j].set(zero);
                    if (!on || (BACK && k == 3 && t == steps - 1)) continue;   // (before step 0: state0)
                    raw[k][j] = *reinterpret_cast<const Raw *>(in[k] + o * ins[k]->ld + t * ins[k]->step + i);
                }
            }
            return;
        }
        const int64_t t0 = first + group * S;
#pragma unroll
        for (int j = 0; j < S; ++j) {
            const int64_t t = t0 + j;
#pragma unroll
            for (int k = 0; k < IN; ++k) {
                const float zero[V] = {};
                raw[k][j].set(zero);
                if (valid && t < steps - (BACK && k == 3 ? 1 : 0))
                    raw[k][j] = *reinterpret_cast<const Raw *>(in[k] + t * ins[k]->step);
            }
        }
    };

    pdl_wait_previous();
    load(0);
    float carry[V], state0[V];   // state0: backward, the state before step 0, in 32 bits
#pragma unroll
    for (int v = 0; v < V; ++v) {
        carry[v] = valid && s.first != nullptr ? s.first[c + v] : 0.0f;
        state0[v] = BACK && valid && s.h0 != nullptr ? s.h0[c + v] : 0.0f;
    }

    if (cluster > 1) cluster_wait();
    const int64_t rounds = (steps + int64_t(cluster) * L - 1) / (int64_t(cluster) * L);
    for (int64_t round = 0; round < rounds; ++round) {
        const int64_t t0 = (round * cluster + rank) * L + group * S;
        const int buf = int(round & 1);
        float *const at = s_tile + row0 * pitch + group * S * inner + rowi;   // STAGED: the thread's first step in the tile
        const int plane = rows * pitch;
        if (STAGED) {
            if (round > 0) __syncthreads();   // the tile has been written out
#pragma unroll
            for (int j = 0; j < S; ++j) {
                const int e = tid + j * kScanThreads;
                const int r = inner == 1 ? e / kRun : e / run, q = e - r * run;
                if (r < rows) {
#pragma unroll
                    for (int k = 0; k < IN; ++k) {
                        float v[V];
                        raw[k][j].get(v);
                        s_tile[k * plane + r * pitch + q] = v[0];
                    }
                }
            }
            __syncthreads();
        }

        // the maps of the steps.  Forward: p = u.  Backward: p = dh, q = what g is
        // multiplied by in d_gate, rest in d_x
        float a[S][V], p[S][V], q[BACK ? S : 1][V], rest[BACK ? S : 1][V];
        float A[V], H[V];
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = 1.0f, H[v] = 0.0f;
#pragma unroll
        for (int j = 0; j < S; ++j) {
            float gate[V], x[V], dh[V], hp[V];
            if (STAGED) {
                gate[0] = at[j * inner], x[0] = at[plane + j * inner];
                if (BACK) dh[0] = at[2 * plane + j * inner], hp[0] = at[3 * plane + j * inner];
            } else {
                raw[0][j].get(gate);
                raw[1][j].get(x);
                if (BACK) {
                    raw[IN - 2][j].get(dh);
                    raw[IN - 1][j].get(hp);
                }
            }
            const bool on = t0 + j < steps;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float r;
                open_gate<LOGITS>(gate[v], a[j][v], r);
                if (BACK) {
                    const float h = t0 + j == steps - 1 ? state0[v] : hp[v];
                    const float slope = LOGITS ? a[j][v] * r : 1.0f;
                    q[j][v] = (s.coupled ? h - x[v] : h) * slope;
                    rest[j][v] = s.coupled ? r : 1.0f;
                    p[j][v] = dh[v];
                } else {
                    p[j][v] = s.coupled ? r * x[v] : x[v];
                }
                if (!on) a[j][v] = 1.0f, p[j][v] = 0.0f;
                H[v] = BACK ? a[j][v] * (H[v] + p[j][v]) : fmaf(a[j][v], H[v], p[j][v]);
                A[v] *= a[j][v];
            }
        }
        if (round + 1 < rounds) load(round + 1);

        // the carry into the thread's steps
        float in_c[V];
        if (tg > 1 || cluster > 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) s_A[buf][warp][v * 32 + lane] = A[v], s_H[buf][warp][v * 32 + lane] = H[v];
            __syncthreads();
            const int w0 = warp & ~(tg - 1);   // the first warp of these channels
            if (cluster > 1) {
                // the map of all steps of this CTA, to every CTA: a warp folds one of the V channels of a lane
                const int v = warp % V;
                float CA = 1.0f, CH = 0.0f;
                for (int w = 0; w < kScanWarps; ++w) {
                    const float wa = s_A[buf][w][v * 32 + lane];
                    CH = through(wa, s_H[buf][w][v * 32 + lane], CH);
                    CA *= wa;
                }
                for (int k = warp / V; k < cluster; k += kScanWarps / V) {
                    store_remote(&s_rA[buf][rank][v * 32 + lane], k, CA);
                    store_remote(&s_rH[buf][rank][v * 32 + lane], k, CH);
                }
                cluster_meet();   // (the slots of a round are written again two meetings later)
                if (warp == 0) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        for (int k = 0; k < cluster; ++k) {
                            if (k == rank) s_start[v * 32 + lane] = carry[v];
                            carry[v] = through(s_rA[buf][k][v * 32 + lane], s_rH[buf][k][v * 32 + lane], carry[v]);
                        }
                    }
                }
                __syncthreads();
#pragma unroll
                for (int v = 0; v < V; ++v) in_c[v] = s_start[v * 32 + lane];
                for (int w = 0; w < group; ++w)
#pragma unroll
                    for (int v = 0; v < V; ++v) in_c[v] = through(s_A[buf][w][v * 32 + lane], s_H[buf][w][v * 32 + lane], in_c[v]);
            } else {
                for (int w = 0; w < tg; ++w) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (w == group) in_c[v] = carry[v];
                        carry[v] = through(s_A[buf][w0 + w][v * 32 + lane], s_H[buf][w0 + w][v * 32 + lane], carry[v]);
                    }
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) in_c[v] = carry[v], carry[v] = through(A[v], H[v], carry[v]);
        }

        // the steps again, from that carry
#pragma unroll
        for (int j = 0; j < S; ++j) {
            const int64_t t = t0 + j;
            float o0[V], o1[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (BACK) {
                    const float g = p[j][v] + in_c[v];
                    o0[v] = g * q[j][v];
                    o1[v] = g * rest[j][v];
                    in_c[v] = a[j][v] * g;
                } else {
                    in_c[v] = fmaf(a[j][v], in_c[v], p[j][v]);
                    o0[v] = in_c[v];
                }
            }
            if (STAGED) {
                if (staged) {
                    at[j * inner] = o0[0];
                    if (BACK) at[plane + j * inner] = o1[0];
                }
            } else if (valid && t < steps) {
                Raw w;
                w.set(o0);
                *reinterpret_cast<Raw *>(out[0] + t * s.out[0].step) = w;
                if (BACK) {
                    w.set(o1);
                    *reinterpret_cast<Raw *>(out[OUT - 1] + t * s.out[1].step) = w;
                }
            }
        }
        if (STAGED) {
            __syncthreads();
            const int64_t first = (round * cluster + rank) * L;
#pragma unroll 4
            for (int j = 0; j < S; ++j) {
                const int e = tid + j * kScanThreads;
                const int r = inner == 1 ? e / kRun : e / run, q1 = e - r * run;
                const int tl = inner == 1 ? q1 : q1 / inner, i = q1 - tl * inner;
                const int64_t t = first + tl, o = tile * rows + r;
                if (r < rows && o < s.outer && t < steps) {
#pragma unroll
                    for (int k = 0; k < OUT; ++k)
                        out[k][o * s.out[k].ld + t * s.out[k].step + i] = narrow<T>(s_tile[k * plane + r * pitch + q1]);
                }
            }
        }
    }
    if (s.last != nullptr && valid && rank == 0 && (cluster > 1 ? warp == 0 : group == 0)) {
#pragma unroll
        for (int v = 0; v < V; ++v) s.last[c + v] = carry[v];
    }
}

// ---- host ----

template <typename T, bool BACK, int V, bool STAGED, bool LOGITS>
cudaError_t launch_scan_kernel(ScanArgs &s, cudaStream_t stream) {
    constexpr int S = kElems / V;
    const auto kernel = scan_kernel<T, BACK, V, STAGED, LOGITS>;
    int64_t tiles;
    size_t smem = 0;
    if (STAGED) {
        const int rows = 32 / s.inner;
        s.groups_log = 3;
        tiles = (s.outer + rows - 1) / rows;
        smem = size_t(BACK ? 4 : 2) * rows * (kRun + 1) * s.inner * sizeof(float);
        const cudaError_t e = allow_smem(kernel, size_t(BACK ? 4 : 2) * 32 * (kRun + 1) * sizeof(float) + 48 * 1024);
        if (e != cudaSuccess) return e;
    } else {
        // warps of one channel as far as the steps go round, the others take channels of their own
        s.groups_log = 0;
        while (s.groups_log < 3 && (int64_t(S) << s.groups_log) < s.steps) ++s.groups_log;
        const int64_t per = int64_t(32 * V) * (kScanWarps >> s.groups_log);
        tiles = (s.channels + per - 1) / per;
    }
    // time over a cluster's CTAs while the GPU has room for three of them an SM
    int cluster = 1;
    while (cluster < kMaxCluster && tiles * cluster * 2 <= int64_t(3) * sm_count() && (int64_t(S) << s.groups_log) * cluster < s.steps)
        cluster *= 2;
    if (tiles * cluster > INT32_MAX) return cudaErrorNotSupported;
    return launch_ex(kernel, dim3(unsigned(tiles * cluster)), dim3(kScanThreads), smem, stream, unsigned(cluster), true, s, cluster);
}

template <typename T, bool BACK>
cudaError_t launch_scan(ScanArgs &s, bool logits, bool vector, cudaStream_t stream) {
    if (vector)
        return logits ? launch_scan_kernel<T, BACK, 4, false, true>(s, stream) : launch_scan_kernel<T, BACK, 4, false, false>(s, stream);
    if (s.inner < kNarrow)
        return logits ? launch_scan_kernel<T, BACK, 1, true, true>(s, stream) : launch_scan_kernel<T, BACK, 1, true, false>(s, stream);
    return logits ? launch_scan_kernel<T, BACK, 1, false, true>(s, stream) : launch_scan_kernel<T, BACK, 1, false, false>(s, stream);
}

struct Shape {
    int64_t outer, steps, inner;
};

// Whether an element's place is its own, and the bytes that it may take: INVALID_ARG,
// UNSUPPORTED or OK.
darb_status_t check_operand(const Operand &o, const Shape &n, size_t es) {
    if (o.p == nullptr || !aligned_to(o.p, es) || o.ld < 0 || o.step < 0) return DARB_ERR_INVALID_ARG;
    const __int128 ld = n.outer > 1 ? o.ld : 0, step = n.steps > 1 ? o.step : 0;
    const __int128 rows = (n.steps - 1) * step + n.inner, cols = (n.outer - 1) * ld + n.inner;
    const bool steps_inside = (n.steps == 1 || step >= n.inner) && (n.outer == 1 || ld >= rows);
    const bool outer_inside = (n.outer == 1 || ld >= n.inner) && (n.steps == 1 || step >= cols);
    if (!steps_inside && !outer_inside) return DARB_ERR_INVALID_ARG;
    return (n.outer - 1) * ld + rows > kMaxSpan ? DARB_ERR_UNSUPPORTED : DARB_OK;
}

// The bytes of an operand as lines of one pitch, where it is that regular.
Range operand_range(const Operand &o, const Shape &n, size_t es) {
    const int64_t size = int64_t(es), ld = n.outer > 1 ? o.ld : 0, step = n.steps > 1 ? o.step : 0;
    const int64_t bytes = ((n.outer - 1) * ld + (n.steps - 1) * step + n.inner) * size;
    if (n.outer == 1 && n.steps == 1) return {o.p, bytes};
    if (n.outer == 1 || (n.steps > 1 && ld == n.steps * step)) return {o.p, bytes, step * size, n.inner * size};
    if (n.steps == 1 || step == n.outer * ld) return {o.p, bytes, ld * size, n.inner * size};
    if (step == n.inner) return {o.p, bytes, ld * size, n.steps * n.inner * size};
    return {o.p, bytes};
}

bool vectors(const Operand &o, const Shape &n, size_t es) {
    return aligned_to(o.p, 4 * es) && (n.outer == 1 || o.ld % 4 == 0) && (n.steps == 1 || o.step % 4 == 0);
}

bool same(const Operand &a, const Operand &b) { return a.p == b.p && a.ld == b.ld && a.step == b.step; }

Operand reversed(const Operand &o, int64_t last, size_t es) {
    return {static_cast<const char *>(o.p) + last * o.step * int64_t(es), o.ld, -o.step};
}

// What both calls ask of their sizes; OK with *nothing set where there is nothing to do.
darb_status_t check_shape(darb_dtype_t dtype, darb_gates_t gates, const Shape &n, bool *nothing) {
    if (!token_dtype(dtype) || (gates != DARB_GATES_LOGITS && gates != DARB_GATES_VALUES)) return DARB_ERR_INVALID_ARG;
    if (n.outer < 0 || n.steps < 0 || n.inner < 0) return DARB_ERR_INVALID_ARG;
    *nothing = n.outer == 0 || n.inner == 0;
    if (n.outer > kMaxFeatures || n.inner > kMaxFeatures || n.steps > kMaxFeatures || n.outer * n.inner > kMaxFeatures) return DARB_ERR_UNSUPPORTED;
    return DARB_OK;
}

// No steps: the carry goes through as it is.
darb_status_t pass_on(const float *first, float *last, int64_t channels, cudaStream_t stream) {
    if (last == nullptr || last == first) return DARB_OK;
    return enqueue([&] {
        return first != nullptr ? cudaMemcpyAsync(last, first, size_t(channels) * 4, cudaMemcpyDeviceToDevice, stream)
                                : cudaMemsetAsync(last, 0, size_t(channels) * 4, stream);
    });
}

}  // namespace
}  // namespace darb

using namespace darb;

extern "C" {

darb_status_t darb_gated_scan(const void *gate, int64_t ld_gate, int64_t step_gate, const void *x, int64_t ld_x,
                              int64_t step_x, darb_dtype_t dtype, darb_gates_t gates, int coupled, int64_t outer,
                              int64_t steps, int64_t inner, const float *h0, void *h, int64_t ld_h, int64_t step_h,
                              float *h_last, cudaStream_t stream) {
    DARB_TRACE("darb_gated_scan");
    const Shape n = {outer, steps, inner};
    bool nothing = false;
    darb_status_t st = check_shape(dtype, gates, n, &nothing);
    if (st != DARB_OK || nothing) return st;
    if (!aligned_to(h0, 4) || !aligned_to(h_last, 4)) return DARB_ERR_INVALID_ARG;
    const int64_t states = outer * inner * 4;
    if (h0 != h_last && ranges_overlap(h0, states, h_last, states)) return DARB_ERR_INVALID_ARG;
    if (steps == 0) return pass_on(h0, h_last, outer * inner, stream);
    const size_t es = dtype_size(dtype);
    ScanArgs s = {};
    s.gate = {gate, ld_gate, step_gate}, s.x = {x, ld_x, step_x}, s.out[0] = {h, ld_h, step_h};
    bool vector = inner % 4 == 0;
    for (const Operand &o : {s.gate, s.x, s.out[0]}) {
        st = check_operand(o, n, es);
        if (st != DARB_OK) return st;
        vector = vector && vectors(o, n, es);
    }
    const Range outs[] = {operand_range(s.out[0], n, es), {h_last, states}};
    Range ins[] = {operand_range(s.gate, n, es), operand_range(s.x, n, es), {h0, states}};
    if (same(s.x, s.out[0])) ins[1].p = nullptr;
    if (h0 == h_last) ins[2].p = nullptr;
    if (!outputs_apart(outs, ins) || (h0 == h_last && buffers_overlap(outs[0], {h0, states}))) return DARB_ERR_INVALID_ARG;
    s.first = h0, s.last = h_last, s.steps = steps, s.channels = outer * inner;
    s.outer = int32_t(outer), s.inner = int32_t(inner), s.coupled = coupled != 0;
    const bool logits = gates == DARB_GATES_LOGITS;
    return enqueue([&] {
        return dtype == DARB_BF16 ? launch_scan<__nv_bfloat16, false>(s, logits, vector, stream) : launch_scan<float, false>(s, logits, vector, stream);
    });
}

darb_status_t darb_gated_scan_grad(const void *dh, int64_t ld_dh, int64_t step_dh, const void *gate, int64_t ld_gate,
                                   int64_t step_gate, const void *x, int64_t ld_x, int64_t step_x, const void *h,
                                   int64_t ld_h, int64_t step_h, darb_dtype_t dtype, darb_gates_t gates, int coupled,
                                   int64_t outer, int64_t steps, int64_t inner, const float *h0, const float *d_last,
                                   void *d_gate, int64_t ld_dgate, int64_t step_dgate, void *d_x, int64_t ld_dx,
                                   int64_t step_dx, float *d_h0, cudaStream_t stream) {
    DARB_TRACE("darb_gated_scan_grad");
    const Shape n = {outer, steps, inner};
    bool nothing = false;
    darb_status_t st = check_shape(dtype, gates, n, &nothing);
    if (st != DARB_OK || nothing) return st;
    if (!aligned_to(h0, 4) || !aligned_to(d_last, 4) || !aligned_to(d_h0, 4)) return DARB_ERR_INVALID_ARG;
    const int64_t states = outer * inner * 4;
    if (d_last != d_h0 && ranges_overlap(d_last, states, d_h0, states)) return DARB_ERR_INVALID_ARG;
    if (ranges_overlap(h0, states, d_h0, states)) return DARB_ERR_INVALID_ARG;
    if (steps == 0) return pass_on(d_last, d_h0, outer * inner, stream);
    const size_t es = dtype_size(dtype);
    const Operand in[4] = {{gate, ld_gate, step_gate}, {x, ld_x, step_x}, {dh, ld_dh, step_dh}, {h, ld_h, step_h}};
    const Operand out[2] = {{d_gate, ld_dgate, step_dgate}, {d_x, ld_dx, step_dx}};
    bool vector = inner % 4 == 0;
    for (const Operand &o : {in[0], in[1], in[2], in[3], out[0], out[1]}) {
        st = check_operand(o, n, es);
        if (st != DARB_OK) return st;
        vector = vector && vectors(o, n, es);
    }
    // an output may take the place of its input: d_gate the gate's, d_x that of x
    Range ins[] = {operand_range(in[0], n, es), operand_range(in[1], n, es), operand_range(in[2], n, es),
                   operand_range(in[3], n, es), {h0, states}, {d_last, states}};
    const Range outs[] = {operand_range(out[0], n, es), operand_range(out[1], n, es), {d_h0, states}};
    const Range gate_in = ins[0], x_in = ins[1];
    if (same(in[0], out[0])) ins[0].p = nullptr;
    if (same(in[1], out[1])) ins[1].p = nullptr;
    if (d_last == d_h0) ins[5].p = nullptr;
    if (!outputs_apart(outs, ins) || buffers_overlap(outs[1], gate_in) || buffers_overlap(outs[0], x_in) || buffers_overlap(outs[2], gate_in) ||
        buffers_overlap(outs[2], x_in))
        return DARB_ERR_INVALID_ARG;
    ScanArgs s = {};
    const int64_t last = steps - 1;
    s.gate = reversed(in[0], last, es), s.x = reversed(in[1], last, es), s.dh = reversed(in[2], last, es);
    s.before = reversed(in[3], last - 1, es);   // the state before each step
    s.out[0] = reversed(out[0], last, es), s.out[1] = reversed(out[1], last, es);
    s.first = d_last, s.h0 = h0, s.last = d_h0, s.steps = steps, s.channels = outer * inner;
    s.outer = int32_t(outer), s.inner = int32_t(inner), s.coupled = coupled != 0;
    const bool logits = gates == DARB_GATES_LOGITS;
    return enqueue([&] {
        return dtype == DARB_BF16 ? launch_scan<__nv_bfloat16, true>(s, logits, vector, stream) : launch_scan<float, true>(s, logits, vector, stream);
    });
}

}  // extern "C"
