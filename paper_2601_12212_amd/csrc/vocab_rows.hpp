// One workgroup's pass over a stretch of a row of logits: what the log-probabilities (logprobs.hip) and the losses and gradients
// (distill.hip) share.
//
// A stretch is n elements from `p` on, of any alignment.  Elements up to the first multiple of 16 bytes and behind the last whole
// unit of eight are `loose`, up to 14, one to a thread; the units are read 16 bytes at a time.  A thread takes U units at a go, NT
// units apart, so that a go of the workgroup reads NT * U * 8 elements front to back.
//
// Softmax statistics.  With c = log2(e) / T a row's weights are 2^(x c - M2), M2 = fl(m c) for the largest logit m so far: one fused multiply-add
// and one exp2 an element, and since every sum refers to the M2 that was subtracted, its rounding drops out of all results.  Sums are fp32.
// Where that rounding is itself a large power (|m c| from 2^20 on, up to rows that hold nothing but masks of the type's lowest value)
// the exponent is (x - m) c.
#pragma once
#include "common.hpp"
#include "kernels.hpp"

namespace dt {

#define VR_NT 256              // threads of a workgroup
#define VR_U 4                 // units of a thread at a go
#define VR_GO (VR_NT * VR_U)   // units of a go
#define VR_GO_ELEMS (8 * VR_GO)
constexpr float LN2 = 0.69314718055994530942f, LOG2E = 1.4426950408889634074f;

template <bool BF16>
struct Elem;
template <>
struct Elem<true> {
    typedef uint16_t T;
    static __device__ __forceinline__ float get(const T *p) { return bf16_bits_to_float(*p); }
};
template <>
struct Elem<false> {
    typedef float T;
    static __device__ __forceinline__ float get(const T *p) { return *p; }
};

template <bool BF16>
struct Stretch {
    const typename Elem<BF16>::T *p;
    int n, head, units, loose;
    __device__ __forceinline__ Stretch(const void *logits, int64_t at, int count) {
        p = (const typename Elem<BF16>::T *)logits + at;
        n = count;
        const int per16 = BF16 ? 8 : 4;
        head = min((int)(-(uintptr_t)p / sizeof(*p)) & (per16 - 1), n);
        units = (n - head) >> 3;
        loose = n - 8 * units;
    }
    // where loose element i, i < loose, lies in the stretch
    __device__ __forceinline__ int loose_at(int i) const { return i < head ? i : i + 8 * units; }
    __device__ __forceinline__ int goes() const { return (units + VR_GO - 1) / VR_GO; }
};

typedef u32 Vec16 __attribute__((ext_vector_type(4)));
template <bool BF16>
struct Raw {
    Vec16 r[VR_U][BF16 ? 1 : 2];
};
// the units of go `it` of this thread; those past the end are the last unit again
template <bool BF16, bool KEEP>
__device__ __forceinline__ void go_request(const Stretch<BF16> &st, int it, Raw<BF16> &raw) {
#pragma unroll
    for (int u = 0; u < VR_U; ++u) {
        const int unit = min(it * VR_GO + u * VR_NT + (int)threadIdx.x, st.units - 1);
        const Vec16 *q = (const Vec16 *)(st.p + st.head + 8 * (int64_t)unit);
#pragma unroll
        for (int h = 0; h < (BF16 ? 1 : 2); ++h) raw.r[u][h] = KEEP ? q[h] : __builtin_nontemporal_load(q + h);
    }
    __builtin_amdgcn_sched_barrier(0);  // all on their way before anything that follows
}
// what was read, as floats; of units past the end -inf
template <bool BF16>
__device__ __forceinline__ void go_finish(const Stretch<BF16> &st, int it, const Raw<BF16> &raw, float (&x)[8 * VR_U]) {
#pragma unroll
    for (int u = 0; u < VR_U; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (BF16) {
                x[8 * u + 2 * e] = __uint_as_float(raw.r[u][0][e] << 16);
                x[8 * u + 2 * e + 1] = __uint_as_float(raw.r[u][0][e] & 0xFFFF0000u);
            } else {
                x[8 * u + e] = __uint_as_float(raw.r[u][0][e]);
                x[8 * u + 4 + e] = __uint_as_float(raw.r[u][1][e]);
            }
        }
    if ((it + 1) * VR_GO > st.units) {  // uniform
#pragma unroll
        for (int u = 0; u < VR_U; ++u) {
            const bool there = it * VR_GO + u * VR_NT + (int)threadIdx.x < st.units;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[8 * u + e] = there ? x[8 * u + e] : -INFINITY;
        }
    }
}

// Sums of a part of a row against its largest logit m: s = sum 2^(x c - M2), w = sum 2^(x c - M2) (x c - M2).
struct Sums {
    float m, s, w;
};
__device__ __forceinline__ bool plain_ref(float M2) { return fabsf(M2) < 1048576.f; }
// how far the reference lies from m c
__device__ __forceinline__ float ref_off(float m, float c) {
    const float M2 = m * c;
    return plain_ref(M2) ? fmaf(-m, c, M2) : 0.f;
}
// how far, in powers of two, sums against `from` lie below those against `to`, to >= from
__device__ __forceinline__ float ref_step(float from, float to, float c) {
    const float a = from * c, b = to * c;
    const float d = plain_ref(a) && plain_ref(b) ? a - b : from == to ? 0.f : (from - to) * c + (ref_off(from, c) - ref_off(to, c));
    return fmaxf(d, -1e4f);  // (a sum of nothing, times any power, stays nothing)
}
template <bool ENT>
__device__ __forceinline__ void sums_move(Sums &a, float to, float c) {
    const float d = ref_step(a.m, to, c), k = __builtin_amdgcn_exp2f(d);
    if (ENT) a.w = k * fmaf(a.s, d, a.w);
    a.s *= k;
    a.m = to;
}
template <bool ENT>
__device__ __forceinline__ void sums_join(Sums &a, Sums b, float c) {
    const float to = fmaxf(a.m, b.m);
    sums_move<ENT>(a, to, c);
    sums_move<ENT>(b, to, c);
    a.s += b.s;
    if (ENT) a.w += b.w;
}
// log2 of an element's weight in the row, before the sum is divided out
__device__ __forceinline__ float log2_weight(float x, float m, float c) {
    const float M2 = m * c;
    return plain_ref(M2) ? fmaf(x, c, -M2) : x == m ? 0.f : (x - m) * c;
}
template <bool ENT>
__device__ __forceinline__ void sums_add(Sums &a, const float (&x)[8 * VR_U], float mx, float c) {
    if (mx > a.m) sums_move<ENT>(a, mx, c);
    if (a.m == -INFINITY) return;
    const float M2 = a.m * c;
    if (plain_ref(M2)) {
#pragma unroll
        for (int j = 0; j < 8 * VR_U; ++j) {
            const float t = fmaf(x[j], c, -M2), e = __builtin_amdgcn_exp2f(t);
            a.s += e;
            if (ENT) a.w = fmaf(e, fmaxf(t, -1e4f), a.w);  // (0 for a weight of 0)
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8 * VR_U; ++j) {
            const float t = x[j] == a.m ? 0.f : (x[j] - a.m) * c, e = __builtin_amdgcn_exp2f(t);
            a.s += e;
            if (ENT) a.w = fmaf(e, fmaxf(t, -1e4f), a.w);
        }
    }
}
template <bool ENT>
__device__ __forceinline__ void sums_add1(Sums &a, float x, float c) {
    sums_join<ENT>(a, Sums{x, x == -INFINITY ? 0.f : 1.f, 0.f}, c);
}
__device__ __forceinline__ float max_of(const float (&x)[8 * VR_U]) {
    float mx = x[0];
#pragma unroll
    for (int j = 1; j < 8 * VR_U; ++j) mx = fmaxf(mx, x[j]);
    return mx;
}

// The sums of a workgroup's threads, in every thread.  Two barriers; `room` is the caller's.
template <bool ENT>
__device__ __forceinline__ Sums block_sums(Sums a, float c, Sums (&room)[VR_NT / 64]) {
    sums_move<ENT>(a, wave_max(a.m), c);
    a.s = wave_sum(a.s);
    if (ENT) a.w = wave_sum(a.w);
    __syncthreads();
    if (lane_id() == 0) room[threadIdx.x >> 6] = a;
    __syncthreads();
    Sums r = room[0];
#pragma unroll
    for (int i = 1; i < VR_NT / 64; ++i) sums_join<ENT>(r, room[i], c);
    return r;
}

// What a row's sums say.
struct RowStat {
    float m;     // largest logit
    float log2s; // log2 of the sum against M2 = fl(m c), or against m c
    float l;     // log sum exp((x - m) / T)
};
__device__ __forceinline__ RowStat row_stat(float m, float s, float c) {
    RowStat r;
    r.m = m;
    r.log2s = s > 0.f ? log2f(s) : -INFINITY;
    r.l = s > 0.f ? (ref_off(m, c) + r.log2s) * LN2 : -INFINITY;
    return r;
}
__device__ __forceinline__ float log_prob(float x, const RowStat &r, float c) {
    return r.m == -INFINITY ? -INFINITY : (log2_weight(x, r.m, c) - r.log2s) * LN2;
}

// How a call of n rows is cut: a part of a row, one to a workgroup, is this many goes.  Whole rows once they fill the chip with eight
// workgroups to a compute unit, else as many parts as do, of a go at least.  VR_MOST_GOES: what the shared memory of a workgroup is sized for.
constexpr int64_t VR_WORKGROUPS = 2048;
constexpr int VR_MOST_GOES = 32;
inline int vocab_part_goes(int64_t n, int V) {
    const int goes = (V + VR_GO_ELEMS - 1) / VR_GO_ELEMS;
    const int64_t parts = n < VR_WORKGROUPS ? (VR_WORKGROUPS + n - 1) / (n > 0 ? n : 1) : 1;
    const int64_t per = parts >= goes ? 1 : (goes + parts - 1) / parts;
    return (int)(per < VR_MOST_GOES ? per : VR_MOST_GOES);
}
inline int vocab_parts(int64_t n, int V) {
    const int per = vocab_part_goes(n, V) * VR_GO_ELEMS;
    return (V + per - 1) / per;
}

}  // namespace dt
