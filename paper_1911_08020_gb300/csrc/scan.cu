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
// (A2 A1, A2 H1 + H2).  A thread takes a run of steps of one channel or of four
// neighbouring ones, composes its steps' maps, and learns the state before them from the
// lanes, warps and CTAs that have the steps before.  Then it runs its steps again from
// registers.  Inputs are read once and outputs written once, with no scratch; the order
// of all sums is fixed by the sizes.
//
// What bounds it is memory (12 bytes an element in fp32, 24 backward): the arithmetic
// alone, with no loads, takes 123 us where 4 x 16384 x 2048 bf16 take 172 (floor 119).
// So what counts is how many loads are on their way and how they lie:
//  * loads go to shared memory asynchronously, two rounds ahead, into places that only
//    their own thread reads, so that they cost neither registers nor barriers;
//  * time is split over lanes (shuffles), then over the 8 or 16 warps of a CTA, which hand the
//    carry on one by one without a barrier of all (a CTA barrier a round: 292 us against
//    269), then, where channels are few, over the 2 to 8 CTAs of a cluster;
//  * 128 bytes lie side by side wherever the channels allow it.
// Three kernels, by how the operands lie (form_of): channels four at a time; rows of
// consecutive steps, by aligned granules; and anything else, an element at a time, through
// shared memory where few channels lie together.
#include "launch.cuh"
#include "tma.cuh"
#include "tokens.cuh"
#include "trace.h"

#include <algorithm>
#include <type_traits>

namespace darb {

int sm_count();

namespace {

constexpr int kScanThreads = 256;
constexpr int kScanWarps = kScanThreads / 32;
constexpr int kElems = 16;          // elements of a thread in a round
constexpr int kMaxCluster = 8;
// Fewer contiguous channels than this: runs of steps go through shared memory.  fp32, us with that and without, forward
// and backward: 40000 x 1000 x 1 (unaligned) 277 and 313, 396 and 620; 30000 x 1000 x 2 393 and 287, 568 and 640;
// 100 x 20000 x 3 152 and 106, 128 and 137 (but 30000 x 1000 x 3 backward 855 and 749); x 5 977 and 438, 1422 and 922.
constexpr int kNarrow = 2, kNarrowBack = 4;
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

// Four neighbouring elements as they lie in memory.
template <typename T>
struct Word;
template <>
struct Word<float> {
    float4 w;
    __device__ __forceinline__ void get(Pair (&v)[2]) const { v[0] = pair(w.x, w.y), v[1] = pair(w.z, w.w); }
    __device__ __forceinline__ void set(const Pair (&v)[2]) { w = make_float4(low(v[0]), high(v[0]), low(v[1]), high(v[1])); }
};
template <>
struct Word<__nv_bfloat16> {
    uint2 w;
    __device__ __forceinline__ void get(Pair (&v)[2]) const {
        const float2 a = widen2(w.x), b = widen2(w.y);
        v[0] = pair(a.x, a.y), v[1] = pair(b.x, b.y);
    }
    __device__ __forceinline__ void set(const Pair (&v)[2]) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(low(v[0]), high(v[0])), b = __floats2bfloat162_rn(low(v[1]), high(v[1]));
        w = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
    }
};

// 1 / x, one instruction (off by one unit; of infinity 0).
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// a and 1 - a from a gate, neither as the other's difference from 1 where it is the smaller (a
// sigmoid near 1 keeps its distance from 1).  The exponential's argument is rounded, so that the
// smaller one is off by about |gate| 2^-24 of itself beside its last places (gates of 4 to 8: 8,
// 17 to 30: 29 of these units); +-inf give exactly 1 and 0.
template <bool LOGITS>
__device__ __forceinline__ void open_gate(float gate, float &a, float &rest) {
    if (LOGITS) {
        const float e = exp2_fast(-kLog2e * gate);
        a = reciprocal(1.0f + e);
        rest = gate >= 0.0f ? e * a : 1.0f - a;
    } else {
        a = gate;
        rest = 1.0f - gate;
    }
}

// The same of two gates.
template <bool LOGITS>
__device__ __forceinline__ void open_gates(Pair gate, Pair &a, Pair &rest) {
    if (LOGITS) {
        const Pair z = mul2(gate, both(-kLog2e)), e = pair(exp2_fast(low(z)), exp2_fast(high(z))), d = add2(e, both(1.0f));
        a = pair(reciprocal(low(d)), reciprocal(high(d)));
        const Pair near = mul2(e, a), far = fma2(a, both(-1.0f), both(1.0f));
        rest = pair(low(gate) >= 0.0f ? low(near) : low(far), high(gate) >= 0.0f ? high(near) : high(far));
    } else {
        a = gate;
        rest = fma2(a, both(-1.0f), both(1.0f));
    }
}

// The state after a map, from the one before.  Where gates may be above 1 nothing
// comes of a state of 0, even where the product of the gates has overflown.
template <bool LOGITS>
__device__ __forceinline__ float through(float A, float H, float c) { return !LOGITS && c == 0.0f ? H : fmaf(A, c, H); }
template <bool LOGITS>
__device__ __forceinline__ Pair through(Pair A, Pair H, Pair c) {
    const Pair r = fma2(A, c, H);
    return LOGITS ? r : pair(low(c) == 0.0f ? low(H) : low(r), high(c) == 0.0f ? high(H) : high(r));
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_meet() {
    cluster_arrive();
    cluster_wait();
}
__device__ __forceinline__ uint32_t remote(const void *here, uint32_t rank) {
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_addr(here)), "r"(rank));
    return to;
}
__device__ __forceinline__ void store_remote(float *here, uint32_t rank, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote(here, rank)), "f"(v) : "memory");
}
__device__ __forceinline__ void store_remote(float2 *here, uint32_t rank, float2 v) {
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(remote(here, rank)), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ void store_remote(float4 *here, uint32_t rank, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(remote(here, rank)), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
                 : "memory");
}

// Four channels as two pairs.
struct Quad {
    Pair p[2];
};
__device__ __forceinline__ Quad quad(float4 v) { return {pair(v.x, v.y), pair(v.z, v.w)}; }
__device__ __forceinline__ float4 floats(const Quad &q) { return make_float4(low(q.p[0]), high(q.p[0]), low(q.p[1]), high(q.p[1])); }
template <bool LOGITS>
__device__ __forceinline__ void state_through(const Quad &A, const Quad &H, Quad &c) {
#pragma unroll
    for (int h = 0; h < 2; ++h) c.p[h] = through<LOGITS>(A.p[h], H.p[h], c.p[h]);
}
// A map, and another after it.
template <bool LOGITS>
__device__ __forceinline__ void map_through(const Quad &A, const Quad &H, Quad &CA, Quad &CH) {
    state_through<LOGITS>(A, H, CH);
#pragma unroll
    for (int h = 0; h < 2; ++h) CA.p[h] = mul2(CA.p[h], A.p[h]);
}
// A carry goes from warp to warp, and from the last one to the first one's next round:
// a named barrier for each warp that takes one, at which the giver does not wait.  (A
// warp gives again when the carry has been round all the others, so that one place and
// one barrier do.  16 warps use the barrier of __syncthreads too, which they do without.)
template <int WARPS>
__device__ __forceinline__ void take_carry(int warp) {
    __syncwarp();
    asm volatile("bar.sync %0, 64;" ::"r"(warp + (WARPS < 16)) : "memory");
}
template <int WARPS>
__device__ __forceinline__ void give_carry(int warp) {
    __syncwarp();
    asm volatile("bar.arrive %0, 64;" ::"r"(warp + (WARPS < 16)) : "memory");
}

__device__ __forceinline__ Pair shuffle_up(Pair v, int d) {
    Pair r;
    r.bits = __shfl_up_sync(~0u, v.bits, d);
    return r;
}

// An asynchronous copy of 8 or 16 bytes to shared memory.
template <int BYTES>
__device__ __forceinline__ void cp_async_word(uint32_t dst, const void *src) {
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---- channels four at a time ----

// A round's inputs wait in shared memory, each thread's in places of its own: loads
// are on their way for two rounds without holding registers, and no barrier
// goes with them.
constexpr int kStages = 3;
constexpr int kStageBytes = 128;   // of a thread and round

// LC lanes of a warp have neighbouring channels, the other lanes later steps.
template <typename T, bool BACK, int LC, int WARPS, bool LOGITS>
__global__ void __launch_bounds__(WARPS * 32, 16 / WARPS) channel_kernel(const ScanArgs s, const int cluster) {
    constexpr int V = 4, IN = BACK ? 4 : 2, OUT = BACK ? 2 : 1;
    constexpr int S = kStageBytes / (IN * V * int(sizeof(T)));   // steps of a thread in a round
    constexpr int TL = 32 / LC, NS = kStages;
    constexpr bool kMayCluster = LC < 16;
    constexpr int kThreads = WARPS * 32;
    using Raw = Word<T>;
    constexpr int CW = kMayCluster ? WARPS : 1, CC = kMayCluster ? kMaxCluster : 1;
    __shared__ Quad s_carry[WARPS][LC], s_A[2][CW][LC], s_H[2][CW][LC];
    __shared__ float4 s_rA[2][CC][LC], s_rH[2][CC][LC];
    extern __shared__ __align__(16) unsigned char s_raw[];
    Raw *const slots = reinterpret_cast<Raw *>(s_raw) + threadIdx.x;   // [stage][tensor][step][thread]

    pdl_launch_dependents();
    if (kMayCluster && cluster > 1) cluster_arrive();   // (the others' shared memory is there once they run)
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int cl = lane % LC, tl = lane / LC;
    const int tg = 1 << s.groups_log, group = warp & (tg - 1), ct = warp >> s.groups_log;
    const int rank = kMayCluster && cluster > 1 ? int(blockIdx.x) % cluster : 0;
    const int64_t tile = blockIdx.x / unsigned(cluster);
    const int64_t steps = s.steps, stride = int64_t(tg) * (TL * S) * cluster;
    const int64_t c = ((tile * (WARPS >> s.groups_log) + ct) * LC + cl) * V;
    const bool valid = c < s.channels;
    const int64_t co = valid ? c / s.inner : 0, ci = valid ? c - co * s.inner : 0;
    const int64_t t0 = (int64_t(rank) * tg + group) * (TL * S) + tl * S;   // the thread's first step

    const Operand *const ins[4] = {&s.gate, &s.x, &s.dh, &s.before};
    const T *in[IN];     // at the first step of the next round to load
    T *out[OUT];         // at the first step of the round
#pragma unroll
    for (int k = 0; k < IN; ++k) in[k] = static_cast<const T *>(ins[k]->p) + co * ins[k]->ld + ci + t0 * ins[k]->step;
#pragma unroll
    for (int k = 0; k < OUT; ++k) out[k] = static_cast<T *>(const_cast<void *>(s.out[k].p)) + co * s.out[k].ld + ci + t0 * s.out[k].step;

    int64_t in_round[IN], out_round[OUT];
#pragma unroll
    for (int k = 0; k < IN; ++k) in_round[k] = stride * ins[k]->step;
#pragma unroll
    for (int k = 0; k < OUT; ++k) out_round[k] = stride * s.out[k].step;

    const int64_t rounds = (steps + stride - 1) / stride;
    int64_t left_to_load = valid ? steps - t0 : 0;   // steps from the first of the next round to load
    int in_slot = 0;
    auto load = [&]() {
        const uint32_t to = smem_addr(slots + in_slot * (IN * S * kThreads));
        constexpr uint32_t kWord = kThreads * sizeof(Raw);
        if (left_to_load > S) {
#pragma unroll
            for (int k = 0; k < IN; ++k) {
                const T *p = in[k];
#pragma unroll
                for (int j = 0; j < S; ++j, p += ins[k]->step) cp_async_word<sizeof(Raw)>(to + (k * S + j) * kWord, p);
            }
        } else {
#pragma unroll
            for (int k = 0; k < IN; ++k) {
                const T *p = in[k];
#pragma unroll
                for (int j = 0; j < S; ++j, p += ins[k]->step) {
                    // (no state before step 0 in memory: state0)
                    if (j < left_to_load - (BACK && k == 3 ? 1 : 0)) cp_async_word<sizeof(Raw)>(to + (k * S + j) * kWord, p);
                }
            }
        }
        cp_async_commit();
#pragma unroll
        for (int k = 0; k < IN; ++k) in[k] += in_round[k];
        left_to_load -= stride;
        in_slot = in_slot + 1 == NS ? 0 : in_slot + 1;
    };

    pdl_wait_previous();
#pragma unroll
    for (int r = 0; r < NS - 1; ++r) load();
    Quad carry = {{both(0.0f), both(0.0f)}}, state0 = carry;   // state0: backward, the state before step 0, in 32 bits
    if (valid && s.first != nullptr) carry = {pair(s.first[c], s.first[c + 1]), pair(s.first[c + 2], s.first[c + 3])};
    if (BACK && valid && s.h0 != nullptr) state0 = {pair(s.h0[c], s.h0[c + 1]), pair(s.h0[c + 2], s.h0[c + 3])};
    if (kMayCluster && cluster > 1) cluster_wait();

    int slot = 0;
    int64_t left = valid ? steps - t0 : 0;   // steps from the thread's first of the round
    for (int64_t round = 0; round < rounds; ++round, left -= stride) {
        const int buf = int(round & 1);
        load();
        cp_async_wait<NS - 1>();
        const Raw *const from = slots + slot * (IN * S * kThreads);
        slot = slot + 1 == NS ? 0 : slot + 1;

        // the maps of the steps.  Forward: p = u.  Backward: p = dh, q = what g is
        // multiplied by in d_gate, rest in d_x
        Quad a[S], p[S], q[BACK ? S : 1], rest[BACK ? S : 1];
        Quad A = {{both(1.0f), both(1.0f)}}, H = {{both(0.0f), both(0.0f)}};
        auto maps = [&](auto full) {
            constexpr bool all = decltype(full)::value;
#pragma unroll
            for (int j = 0; j < S; ++j) {
                Pair gate[2], x[2], dh[2], hp[2];
                const Raw g = from[j * kThreads], xr = from[(S + j) * kThreads];
                g.get(gate);
                xr.get(x);
                if (BACK) {
                    const Raw d = from[(2 * S + j) * kThreads], h = from[((IN - 1) * S + j) * kThreads];
                    d.get(dh);
                    h.get(hp);
                    if (!all && j == left - 1) hp[0] = state0.p[0], hp[1] = state0.p[1];
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    Pair r;
                    open_gates<LOGITS>(gate[h], a[j].p[h], r);
                    if (BACK) {
                        const Pair d = s.coupled ? fma2(x[h], both(-1.0f), hp[h]) : hp[h];
                        q[j].p[h] = LOGITS ? mul2(d, mul2(a[j].p[h], r)) : d;
                        rest[j].p[h] = s.coupled ? r : both(1.0f);
                        p[j].p[h] = dh[h];
                    } else {
                        p[j].p[h] = s.coupled ? mul2(r, x[h]) : x[h];
                    }
                    if (!all && j >= left) a[j].p[h] = both(1.0f), p[j].p[h] = both(0.0f);
                    H.p[h] = BACK ? mul2(a[j].p[h], add2(H.p[h], p[j].p[h])) : fma2(a[j].p[h], H.p[h], p[j].p[h]);
                    A.p[h] = mul2(A.p[h], a[j].p[h]);
                }
            }
        };
        if (left > S) maps(std::true_type());
        else maps(std::false_type());

        // the maps of the lanes before, then all of the warp's
        Quad Ae, He;
        if (TL > 1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int d = 1; d < TL; d <<= 1) {
                    const Pair pa = shuffle_up(A.p[h], d * LC), ph = shuffle_up(H.p[h], d * LC);
                    if (tl >= d) H.p[h] = through<LOGITS>(A.p[h], H.p[h], ph), A.p[h] = mul2(A.p[h], pa);
                }
                Ae.p[h] = shuffle_up(A.p[h], LC), He.p[h] = shuffle_up(H.p[h], LC);
                if (tl == 0) Ae.p[h] = both(1.0f), He.p[h] = both(0.0f);
            }
        }
        // the carry into the warp's steps
        Quad in_c = carry;
        const bool split = kMayCluster && cluster > 1;
        if (split) {
            if (tl == TL - 1) s_A[buf][warp][cl] = A, s_H[buf][warp][cl] = H;
            __syncthreads();
            // the map of all steps of this CTA, to every CTA
            if (warp < cluster && tl == 0) {
                Quad CA = s_A[buf][0][cl], CH = s_H[buf][0][cl];
#pragma unroll
                for (int w = 1; w < CW; ++w) map_through<LOGITS>(s_A[buf][w][cl], s_H[buf][w][cl], CA, CH);
                store_remote(&s_rA[buf][rank][cl], warp, floats(CA));
                store_remote(&s_rH[buf][rank][cl], warp, floats(CH));
            }
            cluster_meet();   // (the slots of a round are written again two meetings later)
            for (int k = 0; k < cluster; ++k) {
                if (k == rank) in_c = carry;
                state_through<LOGITS>(quad(s_rA[buf][k][cl]), quad(s_rH[buf][k][cl]), carry);
            }
            for (int w = 0; w < group; ++w) state_through<LOGITS>(s_A[buf][w][cl], s_H[buf][w][cl], in_c);
        } else if (tg > 1) {
            if (round > 0 || group > 0) {
                take_carry<WARPS>(warp);
                in_c = s_carry[warp][cl];
            }
            if (round + 1 < rounds || group < tg - 1) {
                const int next = warp - group + ((group + 1) & (tg - 1));
                if (tl == TL - 1) {
                    Quad out_c = in_c;
                    state_through<LOGITS>(A, H, out_c);
                    s_carry[next][cl] = out_c;
                }
                give_carry<WARPS>(next);
            }
        }
        if (TL > 1) state_through<LOGITS>(Ae, He, in_c);

        // the steps again, from that carry
        auto steps_again = [&](auto full) {
            constexpr bool all = decltype(full)::value;
            T *to[OUT];
#pragma unroll
            for (int k = 0; k < OUT; ++k) to[k] = out[k];
#pragma unroll
            for (int j = 0; j < S; ++j) {
                Pair o0[2], o1[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (BACK) {
                        const Pair g = add2(p[j].p[h], in_c.p[h]);
                        o0[h] = mul2(g, q[j].p[h]);
                        o1[h] = mul2(g, rest[j].p[h]);
                        in_c.p[h] = mul2(a[j].p[h], g);
                    } else {
                        o0[h] = in_c.p[h] = fma2(a[j].p[h], in_c.p[h], p[j].p[h]);
                    }
                }
                if (all || j < left) {
                    Raw w;
                    w.set(o0);
                    *reinterpret_cast<Raw *>(to[0]) = w;
                    if (BACK) {
                        w.set(o1);
                        *reinterpret_cast<Raw *>(to[OUT - 1]) = w;
                    }
                }
#pragma unroll
                for (int k = 0; k < OUT; ++k) to[k] += s.out[k].step;
            }
        };
        if (left >= S) steps_again(std::true_type());
        else steps_again(std::false_type());
#pragma unroll
        for (int k = 0; k < OUT; ++k) out[k] += out_round[k];
        // the carry out of the round, with the lanes that have its last steps
        if (tg == 1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) carry.p[h].bits = TL > 1 ? __shfl_sync(~0u, in_c.p[h].bits, (TL - 1) * LC + cl) : in_c.p[h].bits;
        }
        if (round + 1 == rounds && s.last != nullptr && valid) {
            // (split: all threads have the carry)
            if (split ? rank == 0 && warp == 0 && tl == 0 : group == tg - 1 && tl == TL - 1) {
                const float4 v = floats(split ? carry : in_c);
                s.last[c] = v.x, s.last[c + 1] = v.y, s.last[c + 2] = v.z, s.last[c + 3] = v.w;
            }
        }
    }
    cp_async_wait<0>();
}

// ---- time as the contiguous axis ----

// A row is cut into granules of 16 aligned bytes; the rows of all tensors start equally
// far past such a boundary.  Granules are numbered in the order of the walk, from
// the row's last one backward.  A thread takes J of them, 32 apart, so that a warp reads
// 512 bytes side by side; lanes are put together by shuffles, warps and CTAs as above.
template <typename T, bool BACK, bool LOGITS>
__global__ void __launch_bounds__(kScanThreads, 2) row_kernel(const ScanArgs s, const int cluster) {
    constexpr int V = kPerGranule<T>, IN = BACK ? 4 : 2, J = kStageBytes / (IN * 16), NS = kStages;
    __shared__ float2 s_map[2][kScanWarps], s_remote[2][kMaxCluster];
    __shared__ float s_carry[kScanWarps];
    extern __shared__ __align__(16) unsigned char s_raw[];
    uint4 *const slots = reinterpret_cast<uint4 *>(s_raw) + threadIdx.x;   // [stage][tensor][granule][thread]

    pdl_launch_dependents();
    if (cluster > 1) cluster_arrive();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tg = 1 << s.groups_log, group = warp & (tg - 1);
    const int rank = cluster > 1 ? int(blockIdx.x) % cluster : 0;
    const int64_t row = (blockIdx.x / unsigned(cluster)) * int64_t(kScanWarps >> s.groups_log) + (warp >> s.groups_log);
    const bool valid = row < s.channels;
    const int steps = int(s.steps);   // (2^30 at most)
    const Operand *const ins[4] = {&s.gate, &s.x, &s.dh, &s.before};
    const T *in[IN];
#pragma unroll
    for (int k = 0; k < IN; ++k) in[k] = static_cast<const T *>(ins[k]->p) + (valid ? row * ins[k]->ld : 0);
    T *const out0 = static_cast<T *>(const_cast<void *>(s.out[0].p)) + (valid ? row * s.out[0].ld : 0);
    T *const out1 = BACK ? static_cast<T *>(const_cast<void *>(s.out[1].p)) + (valid ? row * s.out[1].ld : 0) : nullptr;
    const int head = row_head<T>(in[0]);
    const int granules = valid ? int(row_granules<T>(head, steps)) : 0;
    const int most = (steps + V - 1) / V + 1;   // of any row
    const int stride = tg * (32 * J) * cluster, rounds = (most + stride - 1) / stride;
    const int w0 = (rank * tg + group) * (32 * J) + lane;
    // the first step of the thread's j-th granule in a round (`steps`: there is none)
    auto first_step = [&](int round, int j) {
        const int w = w0 + round * stride + j * 32;
        return w >= granules ? steps : (BACK ? granules - 1 - w : w) * V - head;
    };
    auto whole = [&](int t) { return t >= 0 && t <= steps - V; };
    int next = 0, in_slot = 0;   // the next round to load, and where to
    auto load = [&]() {
        const uint32_t to = smem_addr(slots + in_slot * (IN * J * kScanThreads));
        if (next < rounds) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int t = first_step(next, j);
                if (!whole(t)) continue;
#pragma unroll
                for (int k = 0; k < IN; ++k) cp_async_word<16>(to + (k * J + j) * (kScanThreads * 16), in[k] + t);
            }
        }
        cp_async_commit();
        ++next;
        in_slot = in_slot + 1 == NS ? 0 : in_slot + 1;
    };
    pdl_wait_previous();
#pragma unroll
    for (int r = 0; r < NS - 1; ++r) load();
    float carry = valid && s.first != nullptr ? s.first[row] : 0.0f;
    const float state0 = BACK && valid && s.h0 != nullptr ? s.h0[row] : 0.0f;
    if (cluster > 1) cluster_wait();

    int slot = 0;
    for (int round = 0; round < rounds; ++round) {
        const int buf = round & 1;
        // backward, the state before a warp's last granule, which another warp has
        float edge = 0.0f;
        if (BACK && lane == 31) {
            const int t = first_step(round, J - 1);
            if (t > 0 && t < steps) edge = widen(in[IN - 1][t - 1]);
        }
        load();
        cp_async_wait<NS - 1>();
        uint4 raw[IN][J];
        {
            const uint4 *const from = slots + slot * (IN * J * kScanThreads);
            slot = slot + 1 == NS ? 0 : slot + 1;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int t = first_step(round, j);
#pragma unroll
                for (int k = 0; k < IN; ++k) {
                    raw[k][j] = from[(k * J + j) * kScanThreads];
                    if (!whole(t) && t < steps) raw[k][j] = load_granule(in[k], t, steps, 0.0f);
                }
            }
        }
        float a[J][V], p[J][V], q[BACK ? J : 1][V], rest[BACK ? J : 1][V];
        float Ae[J], He[J], At[J], Ht[J];   // of the lanes before, of the 32 granules
        float CA = 1.0f, CH = 0.0f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int t = first_step(round, j);
            Pair gate[V / 2], x[V / 2];
            float dh[V], h[V];
            unpack(raw[0][j], gate);
            unpack(raw[1][j], x);
            if (BACK) {
                unpack(raw[IN - 2][j], dh);
                unpack(raw[IN - 1][j], h);
                // the states before: the last of the granule before is the next lane's
                float last[2];
                {
                    float all[V];
                    unpack(raw[IN - 1][j], all);
                    last[0] = all[V - 1];
                    unpack(raw[IN - 1][j + 1 < J ? j + 1 : j], all);
                    last[1] = all[V - 1];
                }
                const float across = __shfl_sync(~0u, last[1], 0);
                float before = __shfl_down_sync(~0u, last[0], 1);
                if (lane == 31) before = j + 1 < J ? across : edge;
#pragma unroll
                for (int e = V - 1; e > 0; --e) h[e] = t + e == 0 ? state0 : h[e - 1];
                h[0] = t == 0 ? state0 : before;
            }
#pragma unroll
            for (int e = 0; e < V; e += 2) {
                Pair ga, r;
                open_gates<LOGITS>(gate[e / 2], ga, r);
                a[j][e] = low(ga), a[j][e + 1] = high(ga);
                if (BACK) {
                    const Pair before = pair(h[e], h[e + 1]), d = s.coupled ? fma2(x[e / 2], both(-1.0f), before) : before;
                    const Pair qe = LOGITS ? mul2(d, mul2(ga, r)) : d;
                    q[j][e] = low(qe), q[j][e + 1] = high(qe);
                    rest[j][e] = s.coupled ? low(r) : 1.0f, rest[j][e + 1] = s.coupled ? high(r) : 1.0f;
                    p[j][e] = dh[e], p[j][e + 1] = dh[e + 1];
                } else {
                    const Pair u = s.coupled ? mul2(r, x[e / 2]) : x[e / 2];
                    p[j][e] = low(u), p[j][e + 1] = high(u);
                }
            }
            if (!whole(t)) {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (t + e < 0 || t >= steps - e) a[j][e] = 1.0f, p[j][e] = 0.0f;
            }
            float A = 1.0f, H = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int e = BACK ? V - 1 - i : i;
                H = BACK ? a[j][e] * (H + p[j][e]) : fmaf(a[j][e], H, p[j][e]);
                A *= a[j][e];
            }
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const float pa = __shfl_up_sync(~0u, A, d), ph = __shfl_up_sync(~0u, H, d);
                if (lane >= d) H = through<LOGITS>(A, H, ph), A *= pa;
            }
            Ae[j] = __shfl_up_sync(~0u, A, 1), He[j] = __shfl_up_sync(~0u, H, 1);
            if (lane == 0) Ae[j] = 1.0f, He[j] = 0.0f;
            At[j] = __shfl_sync(~0u, A, 31), Ht[j] = __shfl_sync(~0u, H, 31);
            CH = through<LOGITS>(At[j], Ht[j], CH);
            CA *= At[j];
        }
        float in_c = carry;
        if (cluster > 1) {
            if (lane == 0) s_map[buf][warp] = make_float2(CA, CH);
            __syncthreads();
            if (tid < cluster) {
                float2 all = make_float2(1.0f, 0.0f);
                for (int w = 0; w < kScanWarps; ++w) {
                    const float2 m = s_map[buf][w];
                    all = make_float2(all.x * m.x, through<LOGITS>(m.x, m.y, all.y));
                }
                store_remote(&s_remote[buf][rank], tid, all);
            }
            cluster_meet();   // (the slots of a round are written again two meetings later)
            for (int k = 0; k < cluster; ++k) {
                if (k == rank) in_c = carry;
                const float2 m = s_remote[buf][k];
                carry = through<LOGITS>(m.x, m.y, carry);
            }
            for (int w = 0; w < group; ++w) {
                const float2 m = s_map[buf][w];
                in_c = through<LOGITS>(m.x, m.y, in_c);
            }
        } else {
            if (tg > 1 && (round > 0 || group > 0)) {
                take_carry<kScanWarps>(warp);
                in_c = s_carry[warp];
            }
            carry = through<LOGITS>(CA, CH, in_c);
            if (tg > 1 && (round + 1 < rounds || group < tg - 1)) {
                const int next = warp - group + ((group + 1) & (tg - 1));
                if (lane == 0) s_carry[next] = carry;
                give_carry<kScanWarps>(next);
            }
        }

        // the steps again, from that carry
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int t = first_step(round, j);
            float at = through<LOGITS>(Ae[j], He[j], in_c), o0[V], o1[V];
            in_c = through<LOGITS>(At[j], Ht[j], in_c);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int e = BACK ? V - 1 - i : i;
                if (BACK) {
                    const float g = p[j][e] + at;
                    o0[e] = g * q[j][e];
                    o1[e] = g * rest[j][e];
                    at = a[j][e] * g;
                } else {
                    at = fmaf(a[j][e], at, p[j][e]);
                    o0[e] = at;
                }
            }
            if (t >= steps) continue;
            store_granule(out0, t, steps, o0);
            if (BACK) store_granule(out1, t, steps, o1);
        }
    }
    // (of the last warp's steps, or with a cluster everyone's)
    if (s.last != nullptr && valid && rank == 0 && group == tg - 1 && lane == 0) s.last[row] = carry;
    cp_async_wait<0>();
}

// ---- anything else, an element at a time ----

// STAGED: few channels lie together (kNarrow), so that a warp's loads would
// touch a sector for every lane.  There a CTA takes 32 / inner rows of kRun steps
// each, read and written along the rows, and turns them through shared memory (rows
// `inner` floats longer than their steps: a warp's 32 channels hit 32 banks).
template <typename T, bool BACK, bool STAGED, bool LOGITS>
__global__ void __launch_bounds__(kScanThreads, BACK ? 1 : 2)
strided_kernel(const ScanArgs s, const int cluster) {
    constexpr int S = kElems;              // steps of a thread in a round
    constexpr int IN = BACK ? 4 : 2;       // tensors read
    constexpr int OUT = BACK ? 2 : 1;
    __shared__ float s_A[2][kScanWarps][32], s_H[2][kScanWarps][32];
    __shared__ float s_rA[2][kMaxCluster][32], s_rH[2][kMaxCluster][32];
    __shared__ float s_start[32];
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
    // e / inner for e < 4096 and inner < 4: 65536 / inner rounded up is off by less than one
    // part in 4096 * 3 / 65536 of the quotient's unit
    const uint32_t part = STAGED ? (65536u + inner - 1) / inner : 0;
    auto over_inner = [&](int e) { return int(uint32_t(e) * part >> 16); };

    // the thread's channels
    int64_t c;
    bool valid;
    if (STAGED) {
        c = tile * (rows * inner) + lane;
        valid = lane < rows * inner && c < s.channels;
    } else {
        c = (tile * (kScanWarps >> s.groups_log) + ct) * 32 + lane;
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

    T raw[IN][S];      // not STAGED: the thread's steps; STAGED: elements of the tile, 256 apart
    auto load = [&](int64_t round) {
        const int64_t first = (round * cluster + rank) * L;
        if (STAGED) {
#pragma unroll
            for (int j = 0; j < S; ++j) {
                const int e = tid + j * kScanThreads, f = over_inner(e), r = f / kRun, i = e - f * inner;
                const int64_t t = first + f % kRun, o = tile * rows + r;
                const bool on = r < rows && o < s.outer && t < steps;
#pragma unroll
                for (int k = 0; k < IN; ++k) {
                    raw[k][j] = narrow<T>(0.0f);
                    if (!on || (BACK && k == 3 && t == steps - 1)) continue;   // (before step 0: state0)
                    raw[k][j] = in[k][o * ins[k]->ld + t * ins[k]->step + i];
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
                raw[k][j] = valid && t < steps - (BACK && k == 3 ? 1 : 0) ? in[k][t * ins[k]->step] : narrow<T>(0.0f);
            }
        }
    };

    pdl_wait_previous();
    load(0);
    float carry = valid && s.first != nullptr ? s.first[c] : 0.0f;
    const float state0 = BACK && valid && s.h0 != nullptr ? s.h0[c] : 0.0f;   // backward: the state before step 0, in 32 bits

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
                const int e = tid + j * kScanThreads, r = over_inner(e) / kRun, q = e - r * run;
                if (r < rows) {
#pragma unroll
                    for (int k = 0; k < IN; ++k) s_tile[k * plane + r * pitch + q] = widen(raw[k][j]);
                }
            }
            __syncthreads();
        }

        // the maps of the steps.  Forward: p = u.  Backward: p = dh, q = what g is
        // multiplied by in d_gate, rest in d_x
        float a[S], p[S], q[BACK ? S : 1], rest[BACK ? S : 1];
        float A = 1.0f, H = 0.0f;
#pragma unroll
        for (int j = 0; j < S; ++j) {
            float gate, x, dh = 0.0f, h = 0.0f;
            if (STAGED) {
                gate = at[j * inner], x = at[plane + j * inner];
                if (BACK) dh = at[2 * plane + j * inner], h = at[3 * plane + j * inner];
            } else {
                gate = widen(raw[0][j]), x = widen(raw[1][j]);
                if (BACK) dh = widen(raw[IN - 2][j]), h = widen(raw[IN - 1][j]);
            }
            float r;
            open_gate<LOGITS>(gate, a[j], r);
            if (BACK) {
                if (t0 + j == steps - 1) h = state0;
                const float slope = LOGITS ? a[j] * r : 1.0f;
                q[j] = (s.coupled ? h - x : h) * slope;
                rest[j] = s.coupled ? r : 1.0f;
                p[j] = dh;
            } else {
                p[j] = s.coupled ? r * x : x;
            }
            if (t0 + j >= steps) a[j] = 1.0f, p[j] = 0.0f;
            H = BACK ? a[j] * (H + p[j]) : fmaf(a[j], H, p[j]);
            A *= a[j];
        }
        if (round + 1 < rounds) load(round + 1);

        // the carry into the thread's steps
        float in_c = carry;
        if (tg > 1 || cluster > 1) {
            s_A[buf][warp][lane] = A, s_H[buf][warp][lane] = H;
            __syncthreads();
            const int w0 = warp & ~(tg - 1);   // the first warp of these channels
            if (cluster > 1) {
                // the map of all steps of this CTA, to every CTA
                float CA = 1.0f, CH = 0.0f;
                for (int w = 0; w < kScanWarps; ++w) {
                    const float wa = s_A[buf][w][lane];
                    CH = through<LOGITS>(wa, s_H[buf][w][lane], CH);
                    CA *= wa;
                }
                for (int k = warp; k < cluster; k += kScanWarps) {
                    store_remote(&s_rA[buf][rank][lane], k, CA);
                    store_remote(&s_rH[buf][rank][lane], k, CH);
                }
                cluster_meet();   // (the slots of a round are written again two meetings later)
                if (warp == 0) {
                    for (int k = 0; k < cluster; ++k) {
                        if (k == rank) s_start[lane] = carry;
                        carry = through<LOGITS>(s_rA[buf][k][lane], s_rH[buf][k][lane], carry);
                    }
                }
                __syncthreads();
                in_c = s_start[lane];
                for (int w = 0; w < group; ++w) in_c = through<LOGITS>(s_A[buf][w][lane], s_H[buf][w][lane], in_c);
            } else {
                for (int w = 0; w < tg; ++w) {
                    if (w == group) in_c = carry;
                    carry = through<LOGITS>(s_A[buf][w0 + w][lane], s_H[buf][w0 + w][lane], carry);
                }
            }
        } else {
            carry = through<LOGITS>(A, H, carry);
        }

        // the steps again, from that carry
#pragma unroll
        for (int j = 0; j < S; ++j) {
            const int64_t t = t0 + j;
            float o0, o1 = 0.0f;
            if (BACK) {
                const float g = p[j] + in_c;
                o0 = g * q[j];
                o1 = g * rest[j];
                in_c = a[j] * g;
            } else {
                o0 = in_c = fmaf(a[j], in_c, p[j]);
            }
            if (STAGED) {
                if (staged) {
                    at[j * inner] = o0;
                    if (BACK) at[plane + j * inner] = o1;
                }
            } else if (valid && t < steps) {
                out[0][t * s.out[0].step] = narrow<T>(o0);
                if (BACK) out[OUT - 1][t * s.out[1].step] = narrow<T>(o1);
            }
        }
        if (STAGED) {
            __syncthreads();
            const int64_t first = (round * cluster + rank) * L;
#pragma unroll 4
            for (int j = 0; j < S; ++j) {
                const int e = tid + j * kScanThreads, f = over_inner(e), r = f / kRun, i = e - f * inner, q1 = e - r * run;
                const int64_t t = first + f % kRun, o = tile * rows + r;
                if (r < rows && o < s.outer && t < steps) {
#pragma unroll
                    for (int k = 0; k < OUT; ++k)
                        out[k][o * s.out[k].ld + t * s.out[k].step + i] = narrow<T>(s_tile[k * plane + r * pitch + q1]);
                }
            }
        }
    }
    if (s.last != nullptr && valid && rank == 0 && (cluster > 1 ? warp == 0 : group == 0)) s.last[c] = carry;
}

// ---- host ----

// Warps that share a channel: as many as the steps go round, a warp taking `per` of
// them in a round.  The logarithm.
int groups_for(int64_t steps, int64_t per, int warps = kScanWarps) {
    int log = 0;
    while ((1 << log) < warps && (per << log) < steps) ++log;
    return log;
}
// CTAs that share channels: while the GPU holds two of `tiles` CTAs on an SM, and the
// steps go round.  (With it, without, to half and to twice as many CTAs, us: 64 rows of 20011 fp32 8.7, 11.9, 11.5, 10.9;
// 4 x 16384 x 256 bf16 52, 124, 72, 49, backward 99, 279, 154, 98; 16384 x 4 x 64 fp32 37, 102, 38, 38.)
int cluster_for(int64_t tiles, int64_t steps, int64_t per) {
    int cluster = 1;
    while (cluster < kMaxCluster && tiles * cluster <= sm_count() && per * cluster < steps) cluster *= 2;
    return cluster;
}

template <typename T, bool BACK, int LC, int WARPS, bool LOGITS>
cudaError_t launch_channels(ScanArgs &s, int64_t tiles, int cluster, cudaStream_t stream) {
    const auto kernel = channel_kernel<T, BACK, LC, WARPS, LOGITS>;
    constexpr size_t smem = size_t(kStages) * kStageBytes * WARPS * 32;
    const cudaError_t e = allow_smem(kernel, smem);
    if (e != cudaSuccess) return e;
    if (tiles * cluster > INT32_MAX) return cudaErrorNotSupported;
    return launch_ex(kernel, dim3(unsigned(tiles * cluster)), dim3(WARPS * 32), smem, stream, unsigned(cluster), true, s, cluster);
}
template <typename T, bool BACK, bool LOGITS>
cudaError_t launch_channels(ScanArgs &s, cudaStream_t stream) {
    constexpr int S = kStageBytes / ((BACK ? 4 : 2) * 4 * int(sizeof(T)));
    // How many lanes have neighbouring channels, and how many warps share a channel: the fewest
    // rounds of all CTAs one after the other, with one round's time for a CTA to begin
    // (35 steps of 1500 x 20 fp32, backward: 32 lanes 5.6 us, 8 lanes 10.6; 1000 steps of
    // 40 x 1024: 84 and 76; 100 steps of 200 x 4096 bf16: one warp 106, eight 134).  Of 64 bytes at
    // a time memory gives two thirds as much (8 lanes of bf16: 4 x 16384 x 2048 270 us, 16 lanes 172).
    int lanes = 0;
    int64_t tiles = 0, least = INT64_MAX;
    const auto consider = [&](int with, int warps, int price) {
        for (int log = 0; (1 << log) <= warps; ++log) {
            const int64_t per = int64_t(with) * 4 * (warps >> log), n = (s.channels + per - 1) / per, room = int64_t(16 / warps) * sm_count();
            const int64_t rounds = (s.steps + (int64_t(S * (32 / with)) << log) - 1) / (int64_t(S * (32 / with)) << log);
            const int64_t cost = (n + room - 1) / room * (rounds + 1) * price;
            if (cost < least) least = cost, lanes = with, tiles = n, s.groups_log = log;
        }
    };
    consider(32, kScanWarps, 2);
    if (sizeof(T) == 2) consider(16, 16, 2);
    consider(8, kScanWarps, sizeof(T) == 2 ? 3 : 2);
    // (so few channels that a cluster shares them: 8 lanes)
    if (tiles * 2 <= sm_count()) least = INT64_MAX, consider(8, kScanWarps, 2);
    if (lanes == 32) return launch_channels<T, BACK, 32, kScanWarps, LOGITS>(s, tiles, 1, stream);
    if (sizeof(T) == 2 && lanes == 16) return launch_channels<T, BACK, sizeof(T) == 2 ? 16 : 8, sizeof(T) == 2 ? 16 : kScanWarps, LOGITS>(s, tiles, 1, stream);
    const int cluster = s.groups_log < 3 ? 1 : cluster_for(tiles, s.steps, int64_t(S * 4) << s.groups_log);
    return launch_channels<T, BACK, 8, kScanWarps, LOGITS>(s, tiles, cluster, stream);
}

template <typename T, bool BACK, bool LOGITS>
cudaError_t launch_rows(ScanArgs &s, cudaStream_t stream) {
    constexpr int64_t per = 32 * (kStageBytes / ((BACK ? 4 : 2) * 16)) * kPerGranule<T>;   // steps of a warp in a round
    constexpr size_t smem = size_t(kStages) * kStageBytes * kScanThreads;
    const auto kernel = row_kernel<T, BACK, LOGITS>;
    const cudaError_t e = allow_smem(kernel, smem);
    if (e != cudaSuccess) return e;
    // warps that share a row: the fewest rounds of all CTAs one after the other, with two
    // rounds' time for a CTA to begin
    const auto tiles_of = [&](int log) { return (s.channels + (kScanWarps >> log) - 1) / (kScanWarps >> log); };
    int64_t least = INT64_MAX;
    for (int log = 0; log < 4; ++log) {
        const int64_t waves = (tiles_of(log) + 2 * sm_count() - 1) / (2 * sm_count()), rounds = (s.steps + (per << log) - 1) / (per << log);
        if (waves * (rounds + 2) < least) least = waves * (rounds + 2), s.groups_log = log;
    }
    const int64_t tiles = tiles_of(s.groups_log);
    const int cluster = s.groups_log < 3 ? 1 : cluster_for(tiles, s.steps, per << s.groups_log);
    if (tiles * cluster > INT32_MAX) return cudaErrorNotSupported;
    return launch_ex(kernel, dim3(unsigned(tiles * cluster)), dim3(kScanThreads), smem, stream, unsigned(cluster), true, s, cluster);
}

template <typename T, bool BACK, bool STAGED, bool LOGITS>
cudaError_t launch_strided(ScanArgs &s, cudaStream_t stream) {
    const auto kernel = strided_kernel<T, BACK, STAGED, LOGITS>;
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
        s.groups_log = groups_for(s.steps, kElems);
        const int64_t per = int64_t(32) * (kScanWarps >> s.groups_log);
        tiles = (s.channels + per - 1) / per;
    }
    const int cluster = s.groups_log < 3 ? 1 : cluster_for(tiles, s.steps, int64_t(kElems) << s.groups_log);
    if (tiles * cluster > INT32_MAX) return cudaErrorNotSupported;
    return launch_ex(kernel, dim3(unsigned(tiles * cluster)), dim3(kScanThreads), smem, stream, unsigned(cluster), true, s, cluster);
}

enum Form { kChannels, kRows, kStaged, kStrided };

template <typename T, bool BACK, bool LOGITS>
cudaError_t launch_scan(ScanArgs &s, Form form, cudaStream_t stream) {
    switch (form) {
        case kChannels: return launch_channels<T, BACK, LOGITS>(s, stream);
        case kRows: return launch_rows<T, BACK, LOGITS>(s, stream);
        case kStaged: return launch_strided<T, BACK, true, LOGITS>(s, stream);
        default: return launch_strided<T, BACK, false, LOGITS>(s, stream);
    }
}
template <bool BACK>
darb_status_t enqueue_scan(ScanArgs &s, darb_dtype_t dtype, bool logits, Form form, cudaStream_t stream) {
    return enqueue([&] {
        if (dtype == DARB_BF16) return logits ? launch_scan<__nv_bfloat16, BACK, true>(s, form, stream) : launch_scan<__nv_bfloat16, BACK, false>(s, form, stream);
        return logits ? launch_scan<float, BACK, true>(s, form, stream) : launch_scan<float, BACK, false>(s, form, stream);
    });
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

// The bytes of an operand as lines of one pitch, in two ways: short lines, and the long
// ones that they lie in.  Two operands share no byte if either way tells them apart
// (slices of rows side by side; rows or elements that take turns).
struct Place {
    Range fine, coarse;
};
Place place_of(const Operand &o, const Shape &n, size_t es) {
    const int64_t size = int64_t(es), ld = n.outer > 1 ? o.ld : 0, step = n.steps > 1 ? o.step : 0;
    const int64_t row = (n.steps - 1) * step + n.inner, bytes = ((n.outer - 1) * ld + row) * size;
    const Range whole = {o.p, bytes}, steps = {o.p, bytes, step * size, n.inner * size}, rows = {o.p, bytes, ld * size, row * size};
    if (n.outer == 1) return {n.steps == 1 ? whole : steps, whole};
    if (n.steps == 1) return {rows, whole};
    // rows of steps; or steps of rows
    if (ld >= row) return {ld % step == 0 ? steps : rows, rows};
    const Range columns = {o.p, bytes, ld * size, n.inner * size}, all_rows = {o.p, bytes, step * size, ((n.outer - 1) * ld + n.inner) * size};
    return {step % ld == 0 ? columns : all_rows, all_rows};
}
Place place_of(const void *p, int64_t bytes) { return {{p, bytes}, {p, bytes}}; }
bool meet(const Place &a, const Place &b) { return buffers_overlap(a.fine, b.fine) && buffers_overlap(a.coarse, b.coarse); }
template <int NO, int NI>
bool apart(const Place (&outs)[NO], const Place (&ins)[NI]) {
    for (int o = 0; o < NO; ++o) {
        for (const Place &i : ins)
            if (meet(outs[o], i)) return false;
        for (int p = 0; p < o; ++p)
            if (meet(outs[o], outs[p])) return false;
    }
    return true;
}

// Which kernel takes these operands.
template <int N>
Form form_of(const Operand (&all)[N], const Shape &n, size_t es) {
    bool vectors = n.inner % 4 == 0, rows = n.inner == 1;
    for (const Operand &o : all) {
        vectors = vectors && aligned_to(o.p, 4 * es) && (n.outer == 1 || o.ld % 4 == 0) && (n.steps == 1 || o.step % 4 == 0);
        // rows of consecutive steps, all of which start equally far past 16 bytes
        const auto past = [&](int64_t row) { return (reinterpret_cast<uintptr_t>(o.p) + uintptr_t(row * o.ld) * es) % 16; };
        const auto past0 = [&](int64_t row) { return (reinterpret_cast<uintptr_t>(all[0].p) + uintptr_t(row * all[0].ld) * es) % 16; };
        rows = rows && (n.steps == 1 || o.step == 1) && past(0) == past0(0) && (n.outer == 1 || past(1) == past0(1));
    }
    return vectors ? kChannels : rows ? kRows : n.inner < (N > 3 ? kNarrowBack : kNarrow) ? kStaged : kStrided;   // (backward: six operands)
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
    const Operand all[] = {s.gate, s.x, s.out[0]};
    for (const Operand &o : all) {
        st = check_operand(o, n, es);
        if (st != DARB_OK) return st;
    }
    const Place outs[] = {place_of(s.out[0], n, es), place_of(h_last, states)}, nowhere = place_of(nullptr, 0);
    Place ins[] = {place_of(s.gate, n, es), place_of(s.x, n, es), place_of(h0, states)};
    if (same(s.x, s.out[0])) ins[1] = nowhere;
    if (h0 == h_last) ins[2] = nowhere;
    if (!apart(outs, ins) || (h0 == h_last && meet(outs[0], place_of(h0, states)))) return DARB_ERR_INVALID_ARG;
    s.first = h0, s.last = h_last, s.steps = steps, s.channels = outer * inner;
    s.outer = int32_t(outer), s.inner = int32_t(inner), s.coupled = coupled != 0;
    return enqueue_scan<false>(s, dtype, gates == DARB_GATES_LOGITS, form_of(all, n, es), stream);
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
    const Operand all[] = {in[0], in[1], in[2], in[3], out[0], out[1]};
    for (const Operand &o : all) {
        st = check_operand(o, n, es);
        if (st != DARB_OK) return st;
    }
    // an output may take the place of its input: d_gate the gate's, d_x that of x
    Place ins[] = {place_of(in[0], n, es), place_of(in[1], n, es), place_of(in[2], n, es), place_of(in[3], n, es), place_of(h0, states), place_of(d_last, states)};
    const Place outs[] = {place_of(out[0], n, es), place_of(out[1], n, es), place_of(d_h0, states)}, nowhere = place_of(nullptr, 0);
    const Place gate_in = ins[0], x_in = ins[1];
    if (same(in[0], out[0])) ins[0] = nowhere;
    if (same(in[1], out[1])) ins[1] = nowhere;
    if (d_last == d_h0) ins[5] = nowhere;
    if (!apart(outs, ins) || meet(outs[1], gate_in) || meet(outs[0], x_in) || meet(outs[2], gate_in) ||
        meet(outs[2], x_in))
        return DARB_ERR_INVALID_ARG;
    ScanArgs s = {};
    const Form form = form_of(all, n, es);
    if (form == kRows) {
        s.gate = in[0], s.x = in[1], s.dh = in[2], s.before = in[3], s.out[0] = out[0], s.out[1] = out[1];
    } else {   // the steps are walked with negative strides
        const int64_t last = steps - 1;
        s.gate = reversed(in[0], last, es), s.x = reversed(in[1], last, es), s.dh = reversed(in[2], last, es);
        s.before = reversed(in[3], last - 1, es);   // the state before each step
        s.out[0] = reversed(out[0], last, es), s.out[1] = reversed(out[1], last, es);
    }
    s.first = d_last, s.h0 = h0, s.last = d_h0, s.steps = steps, s.channels = outer * inner;
    s.outer = int32_t(outer), s.inner = int32_t(inner), s.coupled = coupled != 0;
    return enqueue_scan<true>(s, dtype, gates == DARB_GATES_LOGITS, form, stream);
}

}  // extern "C"
