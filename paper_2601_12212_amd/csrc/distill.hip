// Rows of a draft model's logits against a teacher's best ones (forward Kullback-Leibler divergence over the teacher's entries), and
// the gradients of this loss and of log-probabilities and entropies.
//
// With q = softmax(x / T), the teacher's entries (id_i, p_i), S the set of their ids, P = sum p_i, p_t the weight of "none of them" (0 without
// DT_DISTILL_TAIL) and q_t = sum of q outside S:
//     loss     = sum_i p_i (log p_i - log q_id_i) + p_t (log p_t - log q_t)
//     d / dx_j = w / T [ (P + p_t) q_j - (j outside S: p_t q_j / q_t) - (sum of p_i with id_i = j) ]
// Both sides of q_t come from sums of their own, S's elements left out of the stream and added one by one: 1 - (sum in S) would have no digits
// left where the student is sure.  Outside S every gradient is q_j times one factor of the row, for log-probabilities and entropies q_j times a linear
// function of log q_j: one exponential an element, read and written once, and the few elements of S are written over at the end.
#include "vocab_rows.hpp"

namespace dt {

// ---- the teacher's entries for a row ----
struct Teacher {
    int id[DT_DISTILL_K_MAX];    // -1: none
    float p[DT_DISTILL_K_MAX], lp[DT_DISTILL_K_MAX];
    float sum[DT_DISTILL_K_MAX]; // p of all entries with this id, in the first of them; -1 in the others
    double part[VR_NT / 64];
    float P, rest;
    Sums in_s;                   // the student's elements of S
    float loss;
};
// The teacher's row, -1: none.
__device__ __forceinline__ int64_t teacher_row(const DistillArgs &a, int64_t r) {
    const int64_t t = a.teacher_row ? (int64_t)a.teacher_row[r] : r;
    return t < 0 || t >= a.n_teacher ? -1 : t;
}
__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __hiloint2double(__shfl_xor(__double2hiint(v), o, 64), __shfl_xor(__double2loint(v), o, 64));
    return v;
}
__device__ __forceinline__ double block_sum_f64(double v, double (&room)[VR_NT / 64]) {
    v = wave_sum_f64(v);
    __syncthreads();
    if (lane_id() == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    double r = room[0];
#pragma unroll
    for (int i = 1; i < VR_NT / 64; ++i) r += room[i];
    return r;
}
// Probabilities in 64 bits, since 1 - P is one of them.  Ends with a barrier.
__device__ __forceinline__ void teacher_load(const DistillArgs &a, int64_t tr, Teacher &t) {
    const int tid = threadIdx.x;
    double lp = 0.0, p = 0.0;
    if (tid < a.k) {
        const int id = a.teacher_id[tr * a.k + tid];
        const float val = a.teacher_val[tr * a.k + tid], lse = a.teacher_lse ? a.teacher_lse[tr] : 0.f;
        const bool there = id >= 0 && id < a.V && val > -INFINITY;
        if (there) {
            lp = (double)val - (double)lse;
            p = exp(lp);
        }
        t.id[tid] = there ? id : -1;
    }
    double P = block_sum_f64(p, t.part);
    if ((a.flags & DT_DISTILL_RENORM) && P > 0.0) {
        p /= P;
        lp -= log(P);
        P = 1.0;
    }
    if (tid < a.k) {
        t.p[tid] = (float)p;
        t.lp[tid] = (float)lp;
    }
    if (tid == 0) {
        t.rest = (a.flags & DT_DISTILL_TAIL) ? (float)fmax(0.0, 1.0 - P) : 0.f;
        t.P = (float)P;
    }
    __syncthreads();
    if (tid < a.k) {
        const int id = t.id[tid];
        float sum = 0.f;
        bool first = id >= 0;
        for (int j = 0; j < a.k; ++j)
            if (t.id[j] == id) {
                sum += t.p[j];
                first &= j >= tid;
            }
        t.sum[tid] = first ? sum : -1.f;
    }
    __syncthreads();
}

// ---- elements of S in a stretch: a bit for each of a thread's 32 elements of a go, and one for each loose one ----
__device__ __forceinline__ void marks_clear(u32 *marks, int goes) {
    for (int i = threadIdx.x; i <= goes * VR_NT; i += VR_NT) marks[i] = 0;
}
template <bool BF16>
__device__ __forceinline__ void mark(const Stretch<BF16> &st, u32 *marks, int at) {  // at: place in the stretch
    const int u8 = at - st.head;
    if (u8 < 0 || u8 >= 8 * st.units) {
        const int i = u8 < 0 ? at : at - 8 * st.units;
        atomicOr(&marks[st.goes() * VR_NT], 1u << i);
        return;
    }
    const int unit = u8 >> 3, it = unit / VR_GO, u = unit % VR_GO / VR_NT, t = unit % VR_NT;
    atomicOr(&marks[it * VR_NT + t], 1u << (8 * u + (u8 & 7)));
}

// The sums of a stretch without the elements of S.
template <bool BF16, bool KEEP>
__device__ __forceinline__ Sums sums_outside(const Stretch<BF16> &st, const u32 *marks, float c) {
    Sums r = {-INFINITY, 0.f, 0.f};
    const int goes = st.goes();
    for (int it = 0; it < goes; ++it) {
        Raw<BF16> raw;
        go_request<BF16, KEEP>(st, it, raw);
        float x[8 * VR_U];
        go_finish<BF16>(st, it, raw, x);
        const u32 m = marks[it * VR_NT + threadIdx.x];
        if (m) {
#pragma unroll
            for (int j = 0; j < 8 * VR_U; ++j) x[j] = m >> j & 1 ? -INFINITY : x[j];
        }
        sums_add<false>(r, x, max_of(x), c);
    }
    if ((int)threadIdx.x < st.loose && !(marks[goes * VR_NT] >> threadIdx.x & 1))
        sums_add1<false>(r, Elem<BF16>::get(st.p + st.loose_at(threadIdx.x)), c);
    return r;
}

// What both passes over a row go by.
struct RowLoss {
    RowStat st;
    float tail;       // log of the probability outside S
    float in_s, out;  // factors of q_j in S and outside, w / T in them
};
// out: the row's sums outside S; x: thread tid's element of S, if it is the first of its id.  Writes loss, stats and tail where `tell`.
__device__ __forceinline__ RowLoss row_loss(const DistillArgs &a, int64_t r, Teacher &t, Sums outside, float x, Sums (&room)[VR_NT / 64], bool tell) {
    const int tid = threadIdx.x;
    const bool mine = tid < a.k && t.id[tid] >= 0, first = mine && t.sum[tid] >= 0.f;
    Sums s = {first ? x : -INFINITY, first && x > -INFINITY ? 1.f : 0.f, 0.f};
    s = block_sums<false>(s, a.c, room);
    const float m = fmaxf(s.m, outside.m);
    sums_move<false>(s, m, a.c);
    sums_move<false>(outside, m, a.c);
    const float whole = s.s + outside.s;
    RowLoss R;
    R.st = row_stat(m, whole, a.c);
    R.tail = !(whole > 0.f) ? -INFINITY : s.s < outside.s ? log1pf(-s.s / whole) : logf(outside.s / whole);
    const float w = (a.grad_loss ? a.grad_loss[r] : 1.f) * a.inv_t;
    R.in_s = w * (t.P + t.rest);
    R.out = outside.s > 0.f ? R.in_s - w * t.rest * (whole / outside.s) : R.in_s;
    if (tell) {
        double term = 0.0;
        if (mine && t.p[tid] > 0.f) term = (double)t.p[tid] * ((double)t.lp[tid] - (double)log_prob(x, R.st, a.c));
        if (tid == 0 && t.rest > 0.f) term += (double)t.rest * ((double)logf(t.rest) - (double)R.tail);
        const double loss = block_sum_f64(term, t.part);
        if (tid == 0) {
            a.loss[r] = (float)loss;
            a.stats[2 * r] = R.st.m;
            a.stats[2 * r + 1] = R.st.l;
            a.tail[r] = R.tail;
        }
    }
    return R;
}
__device__ __forceinline__ void row_loss_none(const DistillArgs &a, int64_t r) {
    if (threadIdx.x == 0) a.loss[r] = a.stats[2 * r] = a.stats[2 * r + 1] = a.tail[r] = 0.f;
}

// ---- gradients ----
template <bool BF16>
struct Out8 {
    Vec16 r[BF16 ? 1 : 2];
};
__device__ __forceinline__ u32 to_bf16(float v) {  // to the nearest, ties to even: the one rounding of a gradient
    const u32 u = __float_as_uint(v);
    return (v != v ? 0x7FC00000u : u + 0x7FFFu + (u >> 16 & 1u)) >> 16;
}
template <bool BF16>
__device__ __forceinline__ void put_elem(void *grad, int64_t at, float v) {
    if (BF16) ((uint16_t *)grad)[at] = (uint16_t)to_bf16(v);
    else ((float *)grad)[at] = v;
}
typedef u32 Vec16Any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef u32 Vec16Any4 __attribute__((ext_vector_type(4), aligned(4)));
template <bool BF16>
__device__ __forceinline__ void put_unit(void *grad, int64_t at, const float *g) {
    if constexpr (BF16) {
        Vec16 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = to_bf16(g[2 * e]) | to_bf16(g[2 * e + 1]) << 16;
        __builtin_nontemporal_store(v, (Vec16Any2 *)((uint16_t *)grad + at));
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Vec16 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(g[4 * h + e]);
            __builtin_nontemporal_store(v, (Vec16Any4 *)((float *)grad + at + 4 * h));
        }
    }
}
// q (a + b log2 q) of an element, q = 2^((x - m) c - log2 s)
struct Slope {
    float m, log2s, c, a, b;
};
template <bool ENT>
__device__ __forceinline__ float slope_at(const Slope &k, float x) {
    const float t = fmaf(x - k.m, k.c, -k.log2s), q = __builtin_amdgcn_exp2f(t);
    return q * (ENT ? fmaf(k.b, fmaxf(t, -1e4f), k.a) : k.a);
}
__device__ __forceinline__ Slope slope(float m, float l, float c, float a, float b) {
    // (nothing finite in the row: every q is 0)
    return m == -INFINITY ? Slope{0.f, INFINITY, c, a, b} : Slope{m, l * LOG2E, c, a, b};
}
template <bool BF16, bool ENT>
__device__ __forceinline__ void grad_stretch(const Stretch<BF16> &st, const Slope &k, void *grad, int64_t at) {
    const int goes = st.goes();
    for (int it = 0; it < goes; ++it) {
        Raw<BF16> raw;
        go_request<BF16, false>(st, it, raw);
        float x[8 * VR_U];
        go_finish<BF16>(st, it, raw, x);
#pragma unroll
        for (int u = 0; u < VR_U; ++u) {
            const int unit = it * VR_GO + u * VR_NT + (int)threadIdx.x;
            float g[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = slope_at<ENT>(k, x[8 * u + e]);
            if (unit < st.units) put_unit<BF16>(grad, at + st.head + 8 * (int64_t)unit, g);
        }
    }
    if ((int)threadIdx.x < st.loose) {
        const int i = st.loose_at(threadIdx.x);
        put_elem<BF16>(grad, at + i, slope_at<ENT>(k, Elem<BF16>::get(st.p + i)));
    }
}
template <bool BF16>
__device__ __forceinline__ void grad_zero(void *grad, int64_t at, int n) {
    for (int i = threadIdx.x; i < n; i += VR_NT) put_elem<BF16>(grad, at + i, 0.f);
}

extern __shared__ __align__(16) u32 distill_marks[];

template <bool BF16>
__device__ __forceinline__ float elem_of(const void *logits, int64_t at) {
    return Elem<BF16>::get((const typename Elem<BF16>::T *)logits + at);
}
// thread tid's element of S
template <bool BF16>
__device__ __forceinline__ float s_elem(const DistillArgs &a, int64_t row, const Teacher &t) {
    const int tid = threadIdx.x;
    return tid < a.k && t.id[tid] >= 0 ? elem_of<BF16>(a.logits, row + t.id[tid]) : -INFINITY;
}
// the gradients of S's elements in [id0, id0 + n), behind the stretch's
template <bool BF16>
__device__ __forceinline__ void grad_of_s(const DistillArgs &a, int64_t r, const Teacher &t, const Slope &in_s, float x, int id0, int n) {
    const int tid = threadIdx.x;
    __syncthreads();
    if (tid < a.k && t.id[tid] >= id0 && t.id[tid] < id0 + n && t.sum[tid] >= 0.f) {
        const float w = (a.grad_loss ? a.grad_loss[r] : 1.f) * a.inv_t;
        put_elem<BF16>(a.grad, r * a.grad_stride + t.id[tid], slope_at<false>(in_s, x) - w * t.sum[tid]);
    }
}

// Loss of whole rows, one to a workgroup, and their gradient in a second pass over the row, which the caches then hold.
template <bool BF16, bool GRAD>
__global__ __launch_bounds__(VR_NT) void distill_row_kernel(DistillArgs a) {
    __shared__ Teacher t;
    __shared__ Sums room[VR_NT / 64];
    const int64_t r = blockIdx.x, row = r * a.row_stride;
    const int64_t tr = teacher_row(a, r);
    if (tr < 0) {
        row_loss_none(a, r);
        if (GRAD) grad_zero<BF16>(a.grad, r * a.grad_stride, a.V);
        return;
    }
    const Stretch<BF16> st(a.logits, row, a.V);
    marks_clear(distill_marks, st.goes());
    teacher_load(a, tr, t);
    const float x = s_elem<BF16>(a, row, t);
    if ((int)threadIdx.x < a.k && t.id[threadIdx.x] >= 0) mark<BF16>(st, distill_marks, t.id[threadIdx.x]);
    __syncthreads();
    Sums s = sums_outside<BF16, GRAD>(st, distill_marks, a.c);
    s = block_sums<false>(s, a.c, room);
    const RowLoss R = row_loss(a, r, t, s, x, room, true);
    if (GRAD) {
        grad_stretch<BF16, false>(st, slope(R.st.m, R.st.l, a.c, R.out, 0.f), a.grad, r * a.grad_stride);
        grad_of_s<BF16>(a, r, t, slope(R.st.m, R.st.l, a.c, R.in_s, 0.f), x, 0, a.V);
    }
}

// Sums outside S of a part of a row, and the elements of S in it (the next launch may write their gradients over them).
template <bool BF16>
__global__ __launch_bounds__(VR_NT) void distill_part_kernel(DistillArgs a) {
    __shared__ Sums room[VR_NT / 64];
    const int64_t r = blockIdx.x, row = r * a.row_stride;
    const int part = blockIdx.y, tid = threadIdx.x, id0 = part * a.part_elems, n = min(a.V - id0, a.part_elems);
    const int64_t tr = teacher_row(a, r);
    if (tr < 0) return;
    const Stretch<BF16> st(a.logits, row + id0, n);
    marks_clear(distill_marks, st.goes());
    __syncthreads();
    if (tid < a.k) {
        const int id = a.teacher_id[tr * a.k + tid];
        if (id >= id0 && id < id0 + n && a.teacher_val[tr * a.k + tid] > -INFINITY) {
            mark<BF16>(st, distill_marks, id - id0);
            a.s_elems[r * a.k + tid] = elem_of<BF16>(a.logits, row + id);
        }
    }
    __syncthreads();
    Sums s = sums_outside<BF16, true>(st, distill_marks, a.c);
    s = block_sums<false>(s, a.c, room);
    if (tid == 0) ((float2 *)a.ws)[r * a.parts + part] = make_float2(s.m, s.s);
}
// the parts of a row (up to 64) together, in every thread
__device__ __forceinline__ Sums join_parts(const DistillArgs &a, int64_t r) {
    Sums s = {-INFINITY, 0.f, 0.f};
    if (lane_id() < a.parts) {
        const float2 p = ((const float2 *)a.ws)[r * a.parts + lane_id()];
        s.m = p.x;
        s.s = p.y;
    }
    sums_move<false>(s, wave_max(s.m), a.c);
    s.s = wave_sum(s.s);
    return s;
}
// The loss of rows whose parts are there, and with GRAD the gradient of a part.
template <bool BF16, bool GRAD>
__global__ __launch_bounds__(VR_NT) void distill_join_kernel(DistillArgs a) {
    __shared__ Teacher t;
    __shared__ Sums room[VR_NT / 64];
    const int64_t r = blockIdx.x, row = r * a.row_stride;
    const int part = blockIdx.y, id0 = part * a.part_elems, n = GRAD ? min(a.V - id0, a.part_elems) : 0;
    const int64_t tr = teacher_row(a, r);
    if (tr < 0) {
        if (part == 0) row_loss_none(a, r);
        if (GRAD) grad_zero<BF16>(a.grad, r * a.grad_stride + id0, n);
        return;
    }
    teacher_load(a, tr, t);
    const float x = (int)threadIdx.x < a.k && t.id[threadIdx.x] >= 0 ? a.s_elems[r * a.k + threadIdx.x] : -INFINITY;
    const RowLoss R = row_loss(a, r, t, join_parts(a, r), x, room, part == 0);
    if (GRAD) {
        const Stretch<BF16> st(a.logits, row + id0, n);
        grad_stretch<BF16, false>(st, slope(R.st.m, R.st.l, a.c, R.out, 0.f), a.grad, r * a.grad_stride + id0);
        grad_of_s<BF16>(a, r, t, slope(R.st.m, R.st.l, a.c, R.in_s, 0.f), x, id0, n);
    }
}

// The gradient of a part of a row from what the loss has saved.
template <bool BF16>
__global__ __launch_bounds__(VR_NT) void distill_grad_kernel(DistillArgs a) {
    __shared__ Teacher t;
    const int64_t r = blockIdx.x, row = r * a.row_stride;
    const int id0 = blockIdx.y * a.part_elems, n = min(a.V - id0, a.part_elems);
    const int64_t tr = teacher_row(a, r);
    if (tr < 0) {
        grad_zero<BF16>(a.grad, r * a.grad_stride + id0, n);
        return;
    }
    const float m = a.stats[2 * r], l = a.stats[2 * r + 1], tail = a.tail[r];
    teacher_load(a, tr, t);
    const float x = s_elem<BF16>(a, row, t);
    const float w = (a.grad_loss ? a.grad_loss[r] : 1.f) * a.inv_t, in_s = w * (t.P + t.rest);
    const float out = tail > -INFINITY ? in_s - w * t.rest * expf(-tail) : in_s;
    const Stretch<BF16> st(a.logits, row + id0, n);
    grad_stretch<BF16, false>(st, slope(m, l, a.c, out, 0.f), a.grad, r * a.grad_stride + id0);
    grad_of_s<BF16>(a, r, t, slope(m, l, a.c, in_s, 0.f), x, id0, n);
}

// The gradient of log-probabilities and entropies: q_j (a + b log q_j) and, at the token, its own share.
//     d / dx_j = 1 / T [ g_lp (1[j = y] - q_j) - g_H q_j (log q_j + H) ]
template <bool BF16, bool ENT>
__global__ __launch_bounds__(VR_NT) void logprob_grad_kernel(LogprobGradArgs a) {
    const int64_t r = blockIdx.x, row = r * a.row_stride;
    const int id0 = blockIdx.y * a.part_elems, n = min(a.V - id0, a.part_elems);
    const int y = a.tokens ? a.tokens[r] : -1;
    const float g = y >= 0 && y < a.V && a.g_logprob ? a.g_logprob[r] * a.inv_t : 0.f;
    const float h = ENT ? a.g_entropy[r] * a.inv_t : 0.f;
    const Slope k = slope(a.stats[2 * r], a.stats[2 * r + 1], a.c, ENT ? -fmaf(h, a.entropy[r], g) : -g, -h * LN2);
    const bool here = g != 0.f && y >= id0 && y < id0 + n;
    const float x = here ? elem_of<BF16>(a.logits, row + y) : 0.f;
    const Stretch<BF16> st(a.logits, row + id0, n);
    grad_stretch<BF16, ENT>(st, k, a.grad, r * a.grad_stride + id0);
    if (here) {  // the same for all threads
        __syncthreads();
        if (threadIdx.x == 0) put_elem<BF16>(a.grad, r * a.grad_stride + y, slope_at<ENT>(k, x) + g);
    }
}

static size_t marks_bytes(int elems) { return ((size_t)(elems + VR_GO_ELEMS - 1) / VR_GO_ELEMS * VR_NT + 1) * 4; }

template <bool BF16, bool GRAD>
static hipError_t launch_distill(const DistillArgs &a, hipStream_t st) {
    if (a.parts == 1) {
        launch_kernel(KID_DISTILL, st, distill_row_kernel<BF16, GRAD>, dim3((u32)a.n), dim3(VR_NT), marks_bytes(a.V), a);
        return hipGetLastError();
    }
    launch_kernel(KID_DISTILL, st, distill_part_kernel<BF16>, dim3((u32)a.n, a.parts), dim3(VR_NT), marks_bytes(a.part_elems), a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    launch_kernel(KID_DISTILL_JOIN, st, distill_join_kernel<BF16, GRAD>, dim3((u32)a.n, GRAD ? a.parts : 1), dim3(VR_NT), 0, a);
    return hipGetLastError();
}

size_t distill_workspace(int64_t n, int V) { return (size_t)n * (vocab_parts(n, V) * sizeof(float2) + DT_DISTILL_K_MAX * sizeof(float)); }
hipError_t distill_launch(DistillArgs a, hipStream_t st) {
    a.part_elems = vocab_part_goes(a.n, a.V) * VR_GO_ELEMS;
    a.parts = vocab_parts(a.n, a.V);
    a.s_elems = (float *)((float2 *)a.ws + a.n * a.parts);
    if (a.dtype == DT_BF16) return a.grad ? launch_distill<true, true>(a, st) : launch_distill<true, false>(a, st);
    return a.grad ? launch_distill<false, true>(a, st) : launch_distill<false, false>(a, st);
}
hipError_t distill_grad_launch(DistillArgs a, hipStream_t st) {
    a.part_elems = vocab_part_goes(a.n, a.V) * VR_GO_ELEMS;
    a.parts = vocab_parts(a.n, a.V);
    const dim3 grid((u32)a.n, a.parts);
    if (a.dtype == DT_BF16) launch_kernel(KID_ROWS_GRAD, st, distill_grad_kernel<true>, grid, dim3(VR_NT), 0, a);
    else launch_kernel(KID_ROWS_GRAD, st, distill_grad_kernel<false>, grid, dim3(VR_NT), 0, a);
    return hipGetLastError();
}
template <bool BF16>
static void launch_logprob_grad(const LogprobGradArgs &a, hipStream_t st) {
    const dim3 grid((u32)a.n, a.parts);
    if (a.g_entropy) launch_kernel(KID_ROWS_GRAD, st, logprob_grad_kernel<BF16, true>, grid, dim3(VR_NT), 0, a);
    else launch_kernel(KID_ROWS_GRAD, st, logprob_grad_kernel<BF16, false>, grid, dim3(VR_NT), 0, a);
}
hipError_t logprob_grad_launch(LogprobGradArgs a, hipStream_t st) {
    a.part_elems = vocab_part_goes(a.n, a.V) * VR_GO_ELEMS;
    a.parts = vocab_parts(a.n, a.V);
    if (a.dtype == DT_BF16) launch_logprob_grad<true>(a, st);
    else launch_logprob_grad<false>(a, st);
    return hipGetLastError();
}

}  // namespace dt
