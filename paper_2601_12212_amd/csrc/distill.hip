// Rows of a draft model's logits against a teacher's best ones (forward Kullback-Leibler divergence over the teacher's entries), and
// the gradients of this loss and of log-probabilities and entropies.
//
// With q = softmax(x / T), the teacher's entries (id_i, p_i), S the set of their ids, P = sum p_i, p_t the weight of "none of them" (0 without
// DT_DISTILL_TAIL) and q_t = sum of q outside S:
//     loss     = sum_i p_i (log p_i - log q_id_i) + p_t (log p_t - log q_t)
//     d / dx_j = w / T [ (P + p_t) q_j - (j outside S: p_t q_j / q_t) - (sum of p_i with id_i = j) ]
// Both sides of q_t come from sums of their own, S's elements left out of the stream and added one by one: 1 - (sum in S) would have no digits
// left where the student is sure.  Outside S every gradient is q_j times one factor of the row, for log-probabilities and entropies q_j times a linear
// function of log q_j: one exponential an element, which is read and written once by one thread, so that a gradient may take its logits' place.
//
// Which elements belong to S a wave knows from its lanes: lane i holds where entries i and 64 + i lie (go, thread, element of the thread).
#include <algorithm>

#include "vocab_rows.hpp"

#include "exp_pair.hpp"

namespace dt {

// ---- the teacher's entries for a row ----
#define SLOTS (DT_DISTILL_K_MAX / 64)  // entries of a lane
struct TeacherHead {
    float P, rest, in_m, in_s;         // the student's sum in S
};
struct Teacher {                       // the entries, as the first wave leaves them for all
    double p[DT_DISTILL_K_MAX], lp[DT_DISTILL_K_MAX];
    float sum[DT_DISTILL_K_MAX];       // p of all entries with the same id
    float x[DT_DISTILL_K_MAX];         // the student's logits
    int id[DT_DISTILL_K_MAX];          // -1: none
    int found[512];                    // an entry for a hash of its id
    TeacherHead head;
};
struct Entries {  // of a lane: where they are worked on
    int where[SLOTS];   // go * waves + wave, -1: a loose element, -2: none
    int which[SLOTS];   // lane | element << 6
};
struct Given {  // as they were given
    int id[SLOTS];
    float val[SLOTS];
};
// The teacher's row, -1: none.
__device__ __forceinline__ int64_t teacher_row(const DistillArgs &a, int64_t r) {
    const int64_t t = a.teacher_row ? (int64_t)a.teacher_row[r] : r;
    return t < 0 || t >= a.n_teacher ? -1 : t;
}
__device__ __forceinline__ void entries_load(const DistillArgs &a, int64_t tr, Given &G) {
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        const int i = 64 * s + lane_id();
        G.id[s] = -1;
        G.val[s] = -INFINITY;
        if (i < a.k) {
            G.id[s] = a.teacher_id[tr * a.k + i];
            G.val[s] = a.teacher_val[tr * a.k + i];
        }
    }
}
template <int NT, int U, bool BF16>
__device__ __forceinline__ void entries_place(const DistillArgs &a, const Row<BF16> &row, Given &G, Entries &E) {
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        if (!(G.id[s] >= 0 && G.id[s] < a.V && G.val[s] > -INFINITY)) G.id[s] = -1;
        const Place p = place_of<BF16, NT, U>(row, max(G.id[s], 0));
        E.where[s] = G.id[s] < 0 ? -2 : p.go < 0 ? -1 : p.go * (NT / 64) + (p.thread >> 6);
        E.which[s] = (p.thread & 63) | p.elem << 6;
    }
}
// f(lane, slot, lane of the entry) for the entries at `where` (uniform), of `lane`: one after the other, the same for all lanes
template <class F>
__device__ __forceinline__ void entries_at(const DistillArgs &a, const Entries &E, int where, F f) {
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        if (s && a.k <= 64 * s) break;  // uniform
        for (u64 b = ballot(E.where[s] == where); b; b &= b - 1) {
            const int i = __builtin_ctzll(b), w = __builtin_amdgcn_readlane(E.which[s], i);
            f(w & 63, s, i);
        }
    }
}
// what lanes of a wave have left in shared memory, for its other lanes
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ double wave_sum_f64(double v) { return readlane_f64(wave_scan_incl_f64(v), 63); }
// By one wave: the entries into `t`; x: the student's logits.
__device__ __forceinline__ void teacher_probs(const DistillArgs &a, float lse, const Given &G, const float (&x)[SLOTS], Teacher &t) {
    const int lane = lane_id();
    const bool renorm = a.flags & DT_DISTILL_RENORM;
    if (renorm) {  // p_i / P does not depend on what all values share, and with the largest taken off nothing leaves the exponential's range that counts
        float most = -INFINITY;
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) most = fmaxf(most, G.id[s] >= 0 ? G.val[s] : -INFINITY);
        lse = wave_max(most);
    }
    double P = 0.0, p[SLOTS], lp[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        p[s] = lp[s] = 0.0;
        if (s && a.k <= 64 * s) break;  // uniform, as below: what is not there is not even fetched
        if (G.id[s] >= 0) {
            const float v = G.val[s], hi = v - lse, back = hi - v;
            lp[s] = (double)v - (double)lse;
            p[s] = exp_pair(hi, (v - (hi - back)) - (lse + back));
            P += p[s];
        }
    }
    P = wave_sum_f64(P);
    if (renorm && P > 0.0) {  // (1 to DT_DISTILL_K_MAX: the largest of them is 1)
        const float l0 = logf((float)P);
        const double l = (double)l0 + (P * exp_pair(-l0, 0.f) - 1.0);
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            p[s] /= P;
            lp[s] -= l;
        }
        P = 1.0;
    }
    // sums over entries with the same id
    bool first[SLOTS], twice = false;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        first[s] = G.id[s] >= 0;
        if (s && a.k <= 64 * s) break;
        t.id[64 * s + lane] = G.id[s];
        t.p[64 * s + lane] = p[s];
        t.lp[64 * s + lane] = lp[s];
        t.sum[64 * s + lane] = (float)p[s];
        t.x[64 * s + lane] = x[s];
    }
    wave_sync();
    // Every entry writes its number to a place that its id names; who finds another's there has the same id, or only the same place, and tries another.
    // (Whoever is found is done, so every turn has fewer.  All ids against all: 17 us a call of few rows with 100 entries, 7.)
    bool open[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) open[s] = G.id[s] >= 0;
    for (u32 by = 0x9E3779B1u;; by += 0x3C6EF372u) {
        bool more = false;
#pragma unroll
        for (int s = 0; s < SLOTS; ++s)
            if (open[s]) t.found[(u32)G.id[s] * by >> 23] = 64 * s + lane;
        wave_sync();
#pragma unroll
        for (int s = 0; s < SLOTS; ++s)
            if (open[s]) {
                const int other = t.found[(u32)G.id[s] * by >> 23];
                const bool same = t.id[other] == G.id[s];
                open[s] = !same;
                twice |= same && other != 64 * s + lane;
                more |= !same;
            }
        if (!ballot(more)) break;
        wave_sync();
    }
    if (ballot(twice)) {
        float sum[SLOTS];
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            sum[s] = 0.f;
            for (int j = 0; j < a.k; ++j)
                if (t.id[j] == G.id[s]) {
                    sum[s] += t.sum[j];
                    first[s] = first[s] && j >= 64 * s + lane;
                }
        }
        wave_sync();
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) t.sum[64 * s + lane] = sum[s];
    }
    // the student's elements of S, one for each id
    Sums in = {-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        if (s && a.k <= 64 * s) break;
        if (first[s]) sums_add1<false>(in, x[s], a.c);
    }
    wave_sums<false>(in, a.c);
    if (lane == 0) {
        t.head = TeacherHead{(float)P, (a.flags & DT_DISTILL_TAIL) ? (float)fmax(0.0, 1.0 - P) : 0.f, in.m, in.s};
    }
}

// ---- the loss ----
// q (a + b log2 q) of an element, q = 2^((x - m) c - log2 s)
struct Slope {
    float m, log2s, c, a, b;
};
__device__ __forceinline__ Slope slope(float m, float l, float c, float a, float b) {
    // (nothing finite in the row: every q is 0)
    return m == -INFINITY ? Slope{0.f, INFINITY, c, a, b} : Slope{m, l * LOG2E, c, a, b};
}
// a q of an element against a sum that is at hand: the factor's quotient by the sum, and not the sum's logarithm, whose roundings would be in every gradient of the row (up to
// 6e-7 of each in fp32 rows of 50,001).
__device__ __forceinline__ Slope slope_by_sum(float m, float part, float c, float a) {
    return part > 0.f ? Slope{m, ref_off(m, c), c, a * part, 0.f} : Slope{0.f, INFINITY, c, a, 0.f};
}
// What the gradients of a row with a teacher go by.  Outside S the gradient is q_j (P - p_t (1 - q_t) / q_t): q_j / q_t, which the sums outside S give, times
// P q_t - p_t q_in with q_in = 1 - q_t, a sum of its own.  Neither factor leaves fp32's range, and where a student is near its teacher only
// P and q_in, or p_t and q_t, meet, which are small and known to their last digits.
struct DistillSlope {
    Slope out, in;
    float w;
    int64_t at;
};
// From the row's sums in S and outside, by any thread.
struct RowLoss {
    RowStat st;
    float part;         // 1 / the sum over all tokens, against st.m
    float q_in, q_out;  // of the student
    Sums out;
};
__device__ __forceinline__ RowLoss row_loss(const DistillArgs &a, const TeacherHead &t, const Sums &out) {
    Sums in = {t.in_m, t.in_s, 0.f}, o = out;
    const float m = fmaxf(in.m, out.m);
    sums_move<false>(in, m, a.c);
    sums_move<false>(o, m, a.c);
    const float whole = in.s + o.s, part = whole > 0.f ? 1.f / whole : 0.f;
    RowLoss R;
    R.st = row_stat(m, whole, a.c);
    R.part = part;
    R.q_in = in.s * part;
    R.q_out = o.s * part;
    R.out = out;
    return R;
}
__device__ __forceinline__ DistillSlope loss_slope(const DistillArgs &a, float w, const TeacherHead &t, const RowLoss &R, int64_t at) {
    return DistillSlope{slope_by_sum(R.out.m, R.out.s > 0.f ? 1.f / R.out.s : 0.f, a.c, w * (t.P * R.q_out - t.rest * R.q_in)), slope_by_sum(R.st.m, R.part, a.c, w * (t.P + t.rest)), w, at};
}
// (a sum outside S that is nothing beside the largest logit still has a logarithm)
__device__ __forceinline__ float log_outside(const DistillArgs &a, const RowLoss &R) {
    return !(R.out.s > 0.f) ? -INFINITY : R.q_in < R.q_out ? log1pf(-R.q_in) : (ref_below(R.out.m, R.st.m, a.c) + log2f(R.out.s) - R.st.log2s) * LN2;
}
// one lane; in: the loss of the entries
__device__ __forceinline__ void loss_store(const DistillArgs &a, int64_t r, const TeacherHead &t, const RowLoss &R, double in) {
    const float tail = log_outside(a, R);
    if (t.rest > 0.f) in += (double)t.rest * ((double)logf(t.rest) - (double)tail);
    a.loss[r] = (float)in;
    a.stats[2 * r] = R.st.m;
    a.stats[2 * r + 1] = R.st.l;
    a.tail[r] = tail;
}
// by the first wave
__device__ __forceinline__ void loss_write(const DistillArgs &a, int64_t r, const Teacher &t, const RowLoss &R) {
    double term = 0.0;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        const int i = 64 * s + lane_id();
        if (s && a.k <= 64 * s) break;
        const double p = t.p[i];
        if (p > 0.0) term += p * (t.lp[i] - (double)log_prob(t.x[i], R.st, a.c));
    }
    term = wave_sum_f64(term);
    if (lane_id() == 0) loss_store(a, r, t.head, R, term);
}
// Where the row's sums come together elsewhere: sum p_i (log p_i - (x_i - m) / T), m the largest logit in S, to which the log-probability of m is to be added P times.
__device__ __forceinline__ double loss_in(const DistillArgs &a, const Teacher &t) {
    double term = 0.0;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        const int i = 64 * s + lane_id();
        if (s && a.k <= 64 * s) break;
        const double p = t.p[i];
        if (p > 0.0) term += p * (t.lp[i] - (t.head.in_m > -INFINITY ? ((double)t.x[i] - (double)t.head.in_m) * (double)(a.c * LN2) : -INFINITY));
    }
    return wave_sum_f64(term);
}
__device__ __forceinline__ double loss_of(const DistillArgs &a, const TeacherHead &t, double in, const RowLoss &R) {
    return t.P > 0.f && t.in_m > -INFINITY ? in - (double)t.P * (double)log_prob(t.in_m, R.st, a.c) : in;
}
__device__ __forceinline__ void row_loss_none(const DistillArgs &a, int64_t r) {
    if (threadIdx.x == 0) a.loss[r] = a.stats[2 * r] = a.stats[2 * r + 1] = a.tail[r] = 0.f;
}

// ---- gradients ----
// two gradients to the nearest bf16, ties to even (v_cvt_pk_bf16_f32): their one rounding
typedef float Pair __attribute__((ext_vector_type(2)));
typedef __bf16 PairBf16 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32 to_bf16(float lo, float hi) { return __builtin_bit_cast(u32, __builtin_convertvector((Pair{lo, hi}), PairBf16)); }
template <bool BF16>
__device__ __forceinline__ void put_elem(void *grad, int64_t at, float v) {
    if (BF16) ((uint16_t *)grad)[at] = (uint16_t)to_bf16(v, v);
    else ((float *)grad)[at] = v;
}
typedef u32 Vec16Any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef u32 Vec16Any4 __attribute__((ext_vector_type(4), aligned(4)));
template <bool BF16>
__device__ __forceinline__ void put_unit(void *grad, int64_t at, const float *g) {
    Vec16 v;
    if constexpr (BF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = to_bf16(g[2 * e], g[2 * e + 1]);
        __builtin_nontemporal_store(v, (Vec16Any2 *)((uint16_t *)grad + at));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(g[e]);
        __builtin_nontemporal_store(v, (Vec16Any4 *)((float *)grad + at));
    }
}
template <bool ENT>
__device__ __forceinline__ float slope_at(const Slope &k, float x) {
    const float t = fmaf(x - k.m, k.c, -k.log2s), q = __builtin_amdgcn_exp2f(t);
    return q * (ENT ? fmaf(k.b, fmaxf(t, -1e4f), k.a) : k.a);
}
template <bool BF16>
__device__ __forceinline__ void grad_zero(void *grad, int64_t at, int n, int nt) {
    for (int i = threadIdx.x; i < n; i += nt) put_elem<BF16>(grad, at + i, 0.f);
}
// a bit for each of the thread's elements of the go that are in S; room: the wave's
template <int NT, int U>
struct Hidden {
    u32 m[U / 4];
    bool any;  // in the wave
    __device__ __forceinline__ Hidden(const Entries &E, int it, u32 (&room)[NT * U / 4]) : any(false) {
        const int here = it * (NT / 64) + (threadIdx.x >> 6);
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) any |= ballot(E.where[s] == here) != 0;
#pragma unroll
        for (int i = 0; i < U / 4; ++i) m[i] = 0;
        if (!any) return;
        u32 *const mine = room + (threadIdx.x >> 6) * (64 * U / 4);
#pragma unroll
        for (int i = 0; i < U / 4; ++i) mine[64 * i + lane_id()] = 0;
        wave_sync();
#pragma unroll
        for (int s = 0; s < SLOTS; ++s)
            if (E.where[s] == here) {
                const int lane = E.which[s] & 63, elem = E.which[s] >> 6;
                atomicOr(&mine[64 * (elem >> 5) + lane], 1u << (elem & 31));
            }
        wave_sync();
#pragma unroll
        for (int i = 0; i < U / 4; ++i) m[i] = mine[64 * i + lane_id()];
    }
    // of units first .. first + G - 1
    template <int G>
    __device__ __forceinline__ void hide(int first, float (&x)[8 * G]) const {
        if (!any) return;  // uniform
        const u32 b = m[first / 4] >> (8 * (first % 4));
#pragma unroll
        for (int j = 0; j < 8 * G; ++j) x[j] = b >> j & 1 ? -INFINITY : x[j];
    }
};
__device__ __forceinline__ float hide_loose(const DistillArgs &a, const Entries &E, float x) {
    if (threadIdx.x >= 64) return x;
    entries_at(a, E, -1, [&](int lane, int, int) { x = lane_id() == lane ? -INFINITY : x; });
    return x;
}
// The gradients of a go, G units at once; at: where the row's gradient starts.
template <int NT, int G, bool ENT, bool BF16, int U>
__device__ __forceinline__ void put_go(const Row<BF16> &row, int it, const Slope &k, void *grad, int64_t at, const Raw<BF16, U> &raw) {
    constexpr int E = Row<BF16>::E;
#pragma unroll
    for (int first = 0; first < U; first += G) {
        float x[8 * G];
        go_take<NT, G>(row, it, raw, first, x);
#pragma unroll
        for (int i = 0; i < 8 * G / E; ++i) {
            const int unit = (it * raw.N + 8 * first / E + i) * NT + (int)threadIdx.x;
            float g[E];
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = slope_at<ENT>(k, x[E * i + e]);
            if (unit < row.units) put_unit<BF16>(grad, at + row.head + E * (int64_t)unit, g);
        }
    }
}
// A lane's entries as the gradient needs them: from what the first wave has left, or as the launch before has.
struct OwnLeft {
    const Teacher &t;
    __device__ __forceinline__ int id(int s) const { return t.id[64 * s + lane_id()]; }
    __device__ __forceinline__ float sum(int s) const { return t.sum[64 * s + lane_id()]; }
    __device__ __forceinline__ float sum_of(int s, int lane) const { return t.sum[64 * s + lane]; }
};
struct OwnLoaded {
    int ids[SLOTS];
    float sums[SLOTS];
    __device__ __forceinline__ int id(int s) const { return ids[s]; }
    __device__ __forceinline__ float sum(int s) const { return sums[s]; }
    __device__ __forceinline__ float sum_of(int s, int lane) const { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sums[s]), lane)); }
};
// Of a row with a teacher: all as if outside S, then those in S, from the lanes that have them as entries; xs: their logits.  (The stores of a wave to
// one address take effect in the order of its instructions.)
template <int NT, int G, bool BF16, int U, class Own>
__device__ __forceinline__ void distill_put_go(const DistillArgs &a, const Row<BF16> &row, int it, const Entries &E, const Own &own, const DistillSlope &d,
                                               const Raw<BF16, U> &raw, const float (&xs)[SLOTS]) {
    put_go<NT, G, false>(row, it, d.out, a.grad, d.at, raw);
    wave_sync();
    const int here = it * (NT / 64) + (threadIdx.x >> 6);
#pragma unroll
    for (int s = 0; s < SLOTS; ++s)
        if (E.where[s] == here) put_elem<BF16>(a.grad, d.at + own.id(s), slope_at<false>(d.in, xs[s]) - d.w * own.sum(s));
}
template <bool BF16, class Own>
__device__ __forceinline__ void distill_grad_loose(const DistillArgs &a, const Row<BF16> &row, const Entries &E, const Own &own, const DistillSlope &d, float x) {
    if (row.loose == 0 || threadIdx.x >= 64) return;
    float g = slope_at<false>(d.out, x);
    entries_at(a, E, -1, [&](int lane, int s, int i) { g = lane_id() == lane ? slope_at<false>(d.in, x) - d.w * own.sum_of(s, i) : g; });
    if ((int)threadIdx.x < row.loose) put_elem<BF16>(a.grad, d.at + row.loose_at(threadIdx.x), g);
}
__device__ __forceinline__ void s_elems(const Teacher &t, float (&x)[SLOTS]) {
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) x[s] = t.x[64 * s + lane_id()];
}
template <bool BF16>
__device__ __forceinline__ void s_elems(const Row<BF16> &row, const Given &G, float (&x)[SLOTS]) {
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) x[s] = G.id[s] >= 0 ? row.at(G.id[s]) : -INFINITY;
}

// ---- rows that a workgroup holds: read once ----
// Waves of a SIMD: as many as leave a thread its registers (the loss alone of 300 bf16 rows of 20,001 by 512 threads: 10.3 us at 8 with two in scratch, 9.7 at 7; of 8,000 of 12,001 by
// 256 47.9 at 8 with four in scratch, 48.2 at 7).
template <bool BF16, bool GRAD, int NT, int U>
__global__ __launch_bounds__(NT, NT == 1024 ? 4 : NT == 64 ? 5 : BF16 ? (GRAD || NT * U == 4096 ? 7 : 8) : U == 4 ? 6 : 4) void distill_held_kernel(DistillArgs a) {
    constexpr int G = 2;  // units that are worked on at once: 8,000 bf16 rows of 6,000 with the gradient in 48 us, 54 with four
    __shared__ Teacher t;
    __shared__ Sums room[NT / 64];
    __shared__ u32 marks[NT * U / 4];
    const int64_t r = blockIdx.x;
    const int64_t tr = teacher_row(a, r);
    if (tr < 0) {
        row_loss_none(a, r);
        if (GRAD) grad_zero<BF16>(a.grad, r * a.grad_stride, a.V, NT);
        return;
    }
    const bool lead = threadIdx.x < 64;
    const float lse = a.teacher_lse ? a.teacher_lse[tr] : 0.f, w = (a.grad_loss ? a.grad_loss[r] : 1.f) * a.inv_t;
    const Row<BF16> row(a.logits, r * a.row_stride, a.V);
    Given given;
    entries_load(a, tr, given);
    Raw<BF16, U> raw;
    go_request<NT, false>(row, 0, raw);
    const float xl = (int)threadIdx.x < row.loose ? row.at(row.loose_at(threadIdx.x)) : -INFINITY;
    Entries E;
    entries_place<NT, U>(a, row, given, E);
    if (lead) {
        float xs[SLOTS];
        s_elems<BF16>(row, given, xs);
        teacher_probs(a, lse, given, xs, t);
    }
    const Hidden<NT, U> hidden(E, 0, marks);
    Sums s = {-INFINITY, 0.f, 0.f};
    bool zeros = false;
#pragma unroll
    for (int u = 0; u < U; u += G) {
        float x[8 * G];
        go_take<NT, G>(row, 0, raw, u, x);
        hidden.template hide<G>(u, x);
        sums_add<false>(s, x, max_of(x), a.c, zeros);
    }
    go_keep(raw);
    if (row.loose > 0) sums_add1<false>(s, hide_loose(a, E, xl), a.c);
    s = block_sums<false, NT>(s, a.c, room);
    const RowLoss R = row_loss(a, t.head, s);
    if (lead) loss_write(a, r, t, R);
    if (GRAD) {
        const DistillSlope d = loss_slope(a, w, t.head, R, r * a.grad_stride);
        float xs[SLOTS];
        s_elems(t, xs);
        distill_put_go<NT, G>(a, row, 0, E, OwnLeft{t}, d, raw, xs);
        distill_grad_loose(a, row, E, OwnLeft{t}, d, xl);
    }
}

// ---- rows that are streamed ----
// A workgroup's sums outside S over goes first .. end - 1, and the loose elements where `loose`.
template <bool BF16, bool KEEP, int NT>
__device__ __forceinline__ Sums sums_outside(const DistillArgs &a, const Row<BF16> &row, const Entries &E, int first, int end, bool loose) {
    constexpr int U = STREAM_U;
    __shared__ u32 marks[NT * U / 4];
    Sums s = {-INFINITY, 0.f, 0.f};
    bool zeros = false;
    for (int it = first; it < end; ++it) {
        Raw<BF16, U> raw;
        go_request<NT, KEEP>(row, it, raw);
        float x[8 * U];
        go_take<NT, U>(row, it, raw, 0, x);
        Hidden<NT, U>(E, it, marks).template hide<U>(0, x);
        sums_add<false>(s, x, max_of(x), a.c, zeros);
    }
    if (loose && row.loose > 0) {
        const float xl = (int)threadIdx.x < row.loose ? row.at(row.loose_at(threadIdx.x)) : -INFINITY;
        sums_add1<false>(s, hide_loose(a, E, xl), a.c);
    }
    return s;
}
template <int NT, bool KEEP, bool BF16, class Own>
__device__ __forceinline__ void grad_goes(const DistillArgs &a, const Row<BF16> &row, const Entries &E, const Own &own, const DistillSlope &d, int first, int end,
                                          bool loose, Raw<BF16, STREAM_U> raw, const float (&xs)[SLOTS]) {
    constexpr int U = STREAM_U;
    for (int it = first; it < end; ++it) {
        if (it > first) go_request<NT, KEEP>(row, it, raw);
        go_keep(raw);
        distill_put_go<NT, 1>(a, row, it, E, own, d, raw, xs);
    }
    if (loose) {
        const float xl = (int)threadIdx.x < row.loose ? row.at(row.loose_at(threadIdx.x)) : -INFINITY;
        distill_grad_loose(a, row, E, own, d, xl);
    }
}

// Whole rows, and their gradient in a second pass over the row: from behind the L2s, which do not hold the rows of all
// workgroups (600 fp32 rows of 66,001: 309 MB are fetched for 158; 83 us, where the bytes once in and once out are 50).
template <bool BF16, bool GRAD, int NT>
__global__ __launch_bounds__(NT, NT == 1024 ? 8 : 7) void distill_stream_kernel(DistillArgs a) {
    constexpr int U = STREAM_U;
    __shared__ Teacher t;
    __shared__ Sums room[NT / 64];
    const int64_t r = blockIdx.x;
    const int64_t tr = teacher_row(a, r);
    if (tr < 0) {
        row_loss_none(a, r);
        if (GRAD) grad_zero<BF16>(a.grad, r * a.grad_stride, a.V, NT);
        return;
    }
    const bool lead = threadIdx.x < 64;
    const float lse = a.teacher_lse ? a.teacher_lse[tr] : 0.f, w = (a.grad_loss ? a.grad_loss[r] : 1.f) * a.inv_t;
    const Row<BF16> row(a.logits, r * a.row_stride, a.V);
    const int goes = row.template goes<NT, U>();
    Given G;
    Entries E;
    entries_load(a, tr, G);
    entries_place<NT, U>(a, row, G, E);
    if (lead) {
        float xs[SLOTS];
        s_elems<BF16>(row, G, xs);
        teacher_probs(a, lse, G, xs, t);
    }
    Sums s = sums_outside<BF16, GRAD, NT>(a, row, E, 0, goes, true);
    s = block_sums<false, NT>(s, a.c, room);
    const RowLoss R = row_loss(a, t.head, s);
    if (lead) loss_write(a, r, t, R);
    Raw<BF16, U> raw = {};
    if (GRAD && goes > 0) go_request<NT, false>(row, 0, raw);
    float xs[SLOTS];
    s_elems(t, xs);
    if (GRAD) grad_goes<NT, false>(a, row, E, OwnLeft{t}, loss_slope(a, w, t.head, R, r * a.grad_stride), 0, goes, true, raw, xs);
}

// What is left of a row's teacher for those who join its parts.
struct RowHead {
    TeacherHead t;
    double in;
};
// the workspace: sums of the parts (largest logit, sum), heads, entries
__device__ __forceinline__ float2 *row_sums(const DistillArgs &a, int64_t r) { return (float2 *)a.ws + r * a.parts; }
__device__ __forceinline__ RowHead *row_heads(const DistillArgs &a) { return (RowHead *)((float2 *)a.ws + a.n * a.parts); }
// of all parts, in every lane
__device__ __forceinline__ Sums parts_sums(const DistillArgs &a, int64_t r) {
    Sums s = {-INFINITY, 0.f, 0.f};
    if (lane_id() < a.parts) {
        const float2 p = row_sums(a, r)[lane_id()];
        s.m = p.x;
        s.s = p.y;
    }
    wave_sums<false>(s, a.c);
    return s;
}
__host__ __device__ __forceinline__ u32 teacher_groups(int64_t n) { return (u32)(n + 7) & ~7u; }
// Sums outside S of a part of a row, after workgroups that have the rows' teachers: a multiple of the XCDs' number, so that the next launch finds a part in
// the L2 where it was read (51 rows of 128,256 with the gradient 12.0 us, 13.8 if the next launch is three XCDs off), and the elements of S as they are left here, since it may write their gradients over them.  (The loss by the part that arrives last,
// in one launch: 127 fp32 rows of 128,256 entries 16.7 us, 15.2 so, 30 bf16 rows 8.0 and 6.8.)
template <bool BF16, bool GRAD, bool KEEP>
__global__ __launch_bounds__(STREAM_NT) void distill_part_kernel(DistillArgs a) {
    constexpr int NT = STREAM_NT, U = STREAM_U;
    __shared__ Sums room[NT / 64];
    __shared__ Teacher t;
    const u32 teachers = teacher_groups(a.n);
    const bool has_teacher = blockIdx.x < teachers;
    if (has_teacher && blockIdx.x >= a.n) return;
    const RowPart rp = has_teacher ? RowPart{blockIdx.x, a.parts} : row_part(blockIdx.x - teachers, a.parts);
    const int64_t r = rp.row;
    const int part = rp.part, first = part * a.part_goes;
    const int64_t tr = teacher_row(a, r);
    if (tr < 0) return;
    const Row<BF16> row(a.logits, r * a.row_stride, a.V);
    Given G;
    Entries E;
    entries_load(a, tr, G);
    entries_place<NT, U>(a, row, G, E);
    if (!has_teacher) {
        Sums s = sums_outside<BF16, KEEP, NT>(a, row, E, first, min(first + a.part_goes, row.template goes<NT, U>()), part == 0);
        s = block_sums<false, NT>(s, a.c, room);
        if (threadIdx.x == 0) row_sums(a, r)[part] = make_float2(s.m, s.s);
    } else {
        if (threadIdx.x >= 64) return;
        float xs[SLOTS];
        s_elems<BF16>(row, G, xs);
        teacher_probs(a, a.teacher_lse ? a.teacher_lse[tr] : 0.f, G, xs, t);
        wave_sync();
        if (GRAD) {
            float2 *const entries = a.entries + r * a.k;
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) {
                const int i = 64 * s + lane_id();
                if (i < a.k) entries[i] = make_float2(xs[s], t.sum[i]);
            }
        }
        const double in = loss_in(a, t);
        if (lane_id() == 0) row_heads(a)[r] = RowHead{t.head, in};
    }
}
// The loss of rows whose parts are there.
__global__ __launch_bounds__(64) void distill_loss_kernel(DistillArgs a) {
    const int64_t r = blockIdx.x;
    const RowHead h = row_heads(a)[r];
    const Sums out = parts_sums(a, r);
    if (teacher_row(a, r) < 0) {
        row_loss_none(a, r);
        return;
    }
    const RowLoss R = row_loss(a, h.t, out);
    if (lane_id() == 0) loss_store(a, r, h.t, R, loss_of(a, h.t, h.in, R));
}
// The loss of rows whose parts are there, and the gradient of a part.
template <bool BF16>
__global__ __launch_bounds__(STREAM_NT) void distill_join_kernel(DistillArgs a) {
    constexpr int NT = STREAM_NT, U = STREAM_U;
    const RowPart rp = row_part(blockIdx.x, a.parts);
    const int64_t r = rp.row;
    const int part = rp.part, first = part * a.part_goes;
    const int64_t tr = teacher_row(a, r);
    const Row<BF16> row(a.logits, r * a.row_stride, a.V);
    const int end = min(first + a.part_goes, row.template goes<NT, U>());
    if (tr < 0) {
        if (part == 0) row_loss_none(a, r);
        const int from = min(part * a.part_goes * STREAM_ELEMS, a.V), to = min((part + 1) * a.part_goes * STREAM_ELEMS, a.V);
        grad_zero<BF16>(a.grad, r * a.grad_stride + from, to - from, NT);
        return;
    }
    const float w = (a.grad_loss ? a.grad_loss[r] : 1.f) * a.inv_t;
    Given G;
    Entries E;
    entries_load(a, tr, G);
    OwnLoaded own;
    float xs[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        const float2 e = 64 * s + lane_id() < a.k ? a.entries[r * a.k + 64 * s + lane_id()] : make_float2(0.f, 0.f);
        xs[s] = e.x;
        own.sums[s] = e.y;
    }
    const RowHead h = row_heads(a)[r];
    Raw<BF16, U> raw = {};
    if (first < end) go_request<NT, false>(row, first, raw);
    const Sums out = parts_sums(a, r);
    entries_place<NT, U>(a, row, G, E);
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) own.ids[s] = G.id[s];
    const RowLoss R = row_loss(a, h.t, out);
    if (part == 0 && threadIdx.x == 0) loss_store(a, r, h.t, R, loss_of(a, h.t, h.in, R));
    grad_goes<NT, false>(a, row, E, own, loss_slope(a, w, h.t, R, r * a.grad_stride), first, end, part == 0, raw, xs);
}

// The gradient of a part of a row from what the loss has saved.
template <bool BF16, bool KEEP>
__global__ __launch_bounds__(STREAM_NT) void distill_grad_kernel(DistillArgs a) {
    constexpr int NT = STREAM_NT, U = STREAM_U;
    __shared__ Teacher t;
    const RowPart rp = row_part(blockIdx.x, a.parts);
    const int64_t r = rp.row;
    const int part = rp.part, first = part * a.part_goes;
    const int64_t tr = teacher_row(a, r);
    const Row<BF16> row(a.logits, r * a.row_stride, a.V);
    if (tr < 0) {
        const int from = min(part * a.part_goes * STREAM_ELEMS, a.V), to = min((part + 1) * a.part_goes * STREAM_ELEMS, a.V);
        grad_zero<BF16>(a.grad, r * a.grad_stride + from, to - from, NT);
        return;
    }
    const float lse = a.teacher_lse ? a.teacher_lse[tr] : 0.f, w = (a.grad_loss ? a.grad_loss[r] : 1.f) * a.inv_t;
    const float m = a.stats[2 * r], l = a.stats[2 * r + 1], tail = a.tail[r];
    const int end = min(first + a.part_goes, row.template goes<NT, U>());
    Given G;
    Entries E;
    entries_load(a, tr, G);
    Raw<BF16, U> raw = {};
    if (first < end) go_request<NT, KEEP>(row, first, raw);
    entries_place<NT, U>(a, row, G, E);
    // The logits of the entries that this wave is to store: no other stores them.
    float xs[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        const int go = E.where[s] / (NT / 64), wave = E.where[s] % (NT / 64);
        xs[s] = E.where[s] >= 0 && go >= first && go < end && wave == (int)(threadIdx.x >> 6) ? row.at(G.id[s]) : 0.f;
    }
    if (threadIdx.x < 64) teacher_probs(a, lse, G, xs, t);
    __syncthreads();
    const Slope out = slope(tail > -INFINITY ? m : -INFINITY, l + tail, a.c, w * (t.head.P * expf(tail) + t.head.rest * expm1f(tail)), 0.f);
    grad_goes<NT, KEEP>(a, row, E, OwnLeft{t}, DistillSlope{out, slope(m, l, a.c, w * (t.head.P + t.head.rest), 0.f), w, r * a.grad_stride}, first, end, part == 0, raw, xs);
}

// The gradient of log-probabilities and entropies: q_j (a + b log q_j) and, at the token, its own share.
//     d / dx_j = 1 / T [ g_lp (1[j = y] - q_j) - g_H q_j (log q_j + H) ]
template <bool BF16, bool ENT, bool KEEP>
__global__ __launch_bounds__(STREAM_NT) void logprob_grad_kernel(LogprobGradArgs a) {
    constexpr int NT = STREAM_NT, U = STREAM_U;
    const RowPart rp = row_part(blockIdx.x, a.parts);
    const int64_t r = rp.row, at = r * a.grad_stride;
    const int part = rp.part, first = part * a.part_goes;
    const Row<BF16> row(a.logits, r * a.row_stride, a.V);
    const int y = a.tokens ? a.tokens[r] : -1;
    const float g = y >= 0 && y < a.V && a.g_logprob ? a.g_logprob[r] * a.inv_t : 0.f;
    const float h = ENT ? a.g_entropy[r] * a.inv_t : 0.f;
    const Slope k = slope(a.stats[2 * r], a.stats[2 * r + 1], a.c, ENT ? -fmaf(h, a.entropy[r], g) : -g, -h * LN2);
    Place here = {-2, 0, 0};
    float xy = 0.f;
    if (g != 0.f) {
        here = place_of<BF16, NT, U>(row, y);
        if ((int)threadIdx.x == here.thread) xy = row.at(y);  // (before this thread stores anything)
    }
    const int end = min(first + a.part_goes, row.template goes<NT, U>());
    for (int it = first; it < end; ++it) {
        Raw<BF16, U> raw;
        go_request<NT, KEEP>(row, it, raw);
        go_keep(raw);
        put_go<NT, 1, ENT>(row, it, k, a.grad, at, raw);
        if (it == here.go && (int)threadIdx.x == here.thread) put_elem<BF16>(a.grad, at + y, slope_at<ENT>(k, xy) + g);
    }
    if (part == 0 && (int)threadIdx.x < row.loose) {
        const int i = row.loose_at(threadIdx.x);
        float d = slope_at<ENT>(k, row.at(i));
        if (here.go == -1 && (int)threadIdx.x == here.thread) d += g;
        put_elem<BF16>(a.grad, at + i, d);
    }
}

constexpr int64_t MEET_ROWS = 3 * CUS / 2, HELD_ROWS = 11 * CUS / 8;
// How rows are cut whose gradient is asked for too.  Rows of up to 131,072 bf16 entries, or half as many of fp32, fit the registers of a compute unit, a workgroup of 1,024
// threads, which then reads them once (shorter rows too, however many: 8,000 of 21,840 138 us, whole 161); while it waits, though, the compute unit has nothing else.  So: with one row to a compute unit, or many, and long ones.
// Loss and gradient, us, in parts | held | whole (read twice), bf16:
//     V = 50,001:  n = 64 10.0 | 12.4 | 15.9;  127 12.8 | 12.7 | -;  200 15.9 | 13.2 | 18.0;  300 20.2 | 24.5 | 22.1;  800 - | 49 | 43;  2,048 - | 101 | 100
//     V = 128,256: n = 64 12.8 | 20.3 | 30.4;  127 18.8 | 20.8 | -;  200 28.0 | 23.5 | 35.5;  300 39.7 | 44.1 | 44.2;  383 49.1 | 46.2 | -;  800 - | 94 | 100;  2,048 - | 198 | 246
// and fp32 rows of 50,001: n = 300 33.2 | 33.0, 383 44.3 | 35.3.
static Cut grad_cut(int64_t n, int V, bool bf16) {
    if (V >= HELD_LEAST && V <= HELD_V && launch_holds(n, 512)) return HELD;
    const Cut c = rows_cut(n, V, bf16, false, false);
    if (c == HELD || c == PARTS || V < HELD_LEAST) return c;
    const bool fits = V <= (bf16 ? 131072 : 65536);
    if (fits && (n <= CUS || (row_is_long(V, bf16) && n >= HELD_ROWS && launch_holds(n, 1024)))) return HELD;
    return n < MEET_ROWS ? PARTS : WHOLE;
}
// The loss alone: as log-probabilities (200 rows of 50,001 bf16 entries wide 9.5 us, in parts 10.5), but little more than one row to a compute unit in parts (300 rows of
// 50,001 fp32 entries 15.2 us, wide 20.5, whole 20.9; of 21,840 bf16 held 9.7, 10.3), and long rows wide (1,200 of 128,256 bf16 52 us, whole 54).
static Cut loss_cut(int64_t n, int V, bool bf16) {
    if (V > HELD_MID && V <= HELD_V && n < MEET_ROWS) return HELD;
    const Cut c = rows_cut(n, V, bf16, false, false);
    if (c == HELD || c == PARTS || V < HELD_LEAST) return c;
    if (n > CUS && n < MEET_ROWS) return PARTS;
    return n <= CUS || (row_is_long(V, bf16) && n < MANY_ROWS) ? WIDE : WHOLE;
}
template <bool BF16, bool GRAD>
static hipError_t launch_distill(const DistillArgs &a, hipStream_t st) {
    const auto held = [&](auto h) {
        constexpr int NT = decltype(h)::NT, U = decltype(h)::U;
        launch_kernel(KID_DISTILL, st, distill_held_kernel<BF16, GRAD, NT, U>, dim3((u32)a.n), dim3(NT), 0, a);
    };
    const Cut cut = GRAD ? grad_cut(a.n, a.V, BF16) : loss_cut(a.n, a.V, BF16);
    if (cut == HELD && a.V <= HELD_MID) {
        by_held_mid(a.n, a.V, held);
    } else if (cut == HELD && a.V <= HELD_V) {
        if (a.n <= CUS) held(Held<1024, 4>());
        else held(Held<512, 8>());
    } else if (cut == HELD) {
        if constexpr (GRAD) {
            if (a.V <= 65536) held(Held<1024, 8>());
            else if constexpr (BF16) held(Held<1024, 16>());
        }
    } else if (cut == PARTS) {
        const dim3 grid((u32)(a.n * a.parts) + teacher_groups(a.n));
        if (GRAD || rows_keep(a.n, a.V, BF16)) launch_kernel(KID_DISTILL, st, distill_part_kernel<BF16, GRAD, true>, grid, dim3(STREAM_NT), 0, a);
        else launch_kernel(KID_DISTILL, st, distill_part_kernel<BF16, GRAD, GRAD>, grid, dim3(STREAM_NT), 0, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if constexpr (GRAD) launch_kernel(KID_DISTILL_JOIN, st, distill_join_kernel<BF16>, dim3((u32)(a.n * a.parts)), dim3(STREAM_NT), 0, a);
        else launch_kernel(KID_DISTILL_JOIN, st, distill_loss_kernel, dim3((u32)a.n), dim3(64), 0, a);
    } else if (cut == WIDE) {
        if constexpr (!GRAD)
            launch_kernel(KID_DISTILL, st, distill_stream_kernel<BF16, false, WIDE_NT>, dim3((u32)a.n), dim3(WIDE_NT), 0, a);
    } else {
        launch_kernel(KID_DISTILL, st, distill_stream_kernel<BF16, GRAD, STREAM_NT>, dim3((u32)a.n), dim3(STREAM_NT), 0, a);
    }
    return hipGetLastError();
}

// As many as parts can be, as for logprob_workspace.
size_t distill_workspace(int64_t n, int V) {
    return (size_t)std::min(n, MEET_ROWS - 1) * (row_goes(V) * sizeof(float2) + sizeof(RowHead) + DT_DISTILL_K_MAX * sizeof(float2));
}
hipError_t distill_launch(DistillArgs a, hipStream_t st) {
    a.part_goes = part_goes(a.n, a.V);
    a.parts = row_parts(a.V, a.part_goes);
    a.entries = (float2 *)((RowHead *)((float2 *)a.ws + a.n * a.parts) + a.n);
    if (a.dtype == DT_BF16) return a.grad ? launch_distill<true, true>(a, st) : launch_distill<true, false>(a, st);
    return a.grad ? launch_distill<false, true>(a, st) : launch_distill<false, false>(a, st);
}
// Goes of a part where nothing joins the parts: one, unless that took more than the 2^32 - 1 threads of a launch.  (Workgroups that start together
// then read and write side by side: 8,192 rows of 32,000 bf16 entries 179 us, with two goes 194, four, whole rows, 198; a copy of as many bytes 167 and 190.)
static int grad_goes_of(int64_t n, int V) {
    int per = 1;
    while (n * row_parts(V, per) > ((int64_t)1 << 24) - 1) ++per;
    return per;
}
template <bool BF16>
static void launch_distill_grad(const DistillArgs &a, hipStream_t st) {
    const dim3 grid((u32)(a.n * a.parts));
    if (rows_keep(a.n, a.V, BF16)) launch_kernel(KID_ROWS_GRAD, st, distill_grad_kernel<BF16, true>, grid, dim3(STREAM_NT), 0, a);
    else launch_kernel(KID_ROWS_GRAD, st, distill_grad_kernel<BF16, false>, grid, dim3(STREAM_NT), 0, a);
}
hipError_t distill_grad_launch(DistillArgs a, hipStream_t st) {
    a.part_goes = grad_goes_of(a.n, a.V);
    a.parts = row_parts(a.V, a.part_goes);
    if (a.dtype == DT_BF16) launch_distill_grad<true>(a, st);
    else launch_distill_grad<false>(a, st);
    return hipGetLastError();
}
template <bool BF16, bool ENT>
static void launch_logprob_grad(const LogprobGradArgs &a, hipStream_t st) {
    const dim3 grid((u32)(a.n * a.parts));
    if (rows_keep(a.n, a.V, BF16)) launch_kernel(KID_ROWS_GRAD, st, logprob_grad_kernel<BF16, ENT, true>, grid, dim3(STREAM_NT), 0, a);
    else launch_kernel(KID_ROWS_GRAD, st, logprob_grad_kernel<BF16, ENT, false>, grid, dim3(STREAM_NT), 0, a);
}
hipError_t logprob_grad_launch(LogprobGradArgs a, hipStream_t st) {
    a.part_goes = grad_goes_of(a.n, a.V);
    a.parts = row_parts(a.V, a.part_goes);
    if (a.dtype == DT_BF16) a.g_entropy ? launch_logprob_grad<true, true>(a, st) : launch_logprob_grad<true, false>(a, st);
    else a.g_entropy ? launch_logprob_grad<false, true>(a, st) : launch_logprob_grad<false, false>(a, st);
    return hipGetLastError();
}

}  // namespace dt
