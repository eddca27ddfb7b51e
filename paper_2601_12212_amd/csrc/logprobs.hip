// Log-probabilities of given tokens, the entropy of their rows and the best alternatives: one pass over a row for its largest
// logit m, s = sum 2^(x c - M2) and w = sum 2^(x c - M2) (x c - M2) (vocab_rows.hpp), of which
//     log-probability of y = ln 2 ((y c - M2) - log2 s),   entropy = ln 2 (log2 s - w / s),
// both sums of terms of one sign.
//
// The k best: every thread leaves the largest of the 32 elements that it took at a go, as the upper half of its ordered image, in
// shared memory.  The k-th largest of the threads' own maxima bounds the k-th largest element from below, and tightly (places
// far apart in the row go to one thread); the few goes that reach it are read again, their elements that reach it listed, and the list ranked
// by counting keys of (value, id).  A list that overflows (ties, a row whose best are neighbours) gives way to a radix selection over
// the stretch, eight bits at a time, and the ties that still fit are taken in ascending id.
#include "vocab_rows.hpp"

namespace dt {

#define LP_CAP 1024  // candidates that are listed

// The k largest (value, id) keys of a stretch, out of LDS: keys[0 .. returned count), in no order.
struct TopRoom {
    u32 kth;      // 16-bit key of the bound
    u32 n;        // candidates
    u32 hist[256];
    u32 tm[VR_NT];  // the threads' largest, 16-bit keys
    u32 counts[VR_NT / 64];
    u32 prefix, need;
    u64 keys[LP_CAP];
};

__device__ __forceinline__ void top_keep(TopRoom &r, float x, int id) {
    const u32 at = atomicAdd(&r.n, 1u);
    if (at < LP_CAP) r.keys[at] = make_key(x, (u32)id);
}

// Radix selection: exactly the k best of a stretch that holds more than k candidates.  Every thread reads it element by element.
template <bool BF16>
__device__ __noinline__ void top_by_radix(TopRoom &r, const typename Elem<BF16>::T *p, int n, int id0, int k) {
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
    const u32 none = ord32(-INFINITY);
    u32 prefix = 0;
    int need = k;
    for (int shift = 24; shift >= (BF16 ? 16 : 0); shift -= 8) {
        __syncthreads();
        r.hist[tid] = 0;
        __syncthreads();
        for (int i0 = 0; i0 < n; i0 += VR_NT) {
            const int i = i0 + tid;
            const u32 key = i < n ? ord32(Elem<BF16>::get(p + i)) : none;
            const bool in = key > none && (shift == 24 || (key ^ prefix) >> (shift + 8) == 0);
            const u32 digit = key >> shift & 255u;
            // ties come by the thousand: what agrees with the wave's first lane is counted at once
            const u64 some = ballot(in);
            if (!some) continue;
            const u32 first = (u32)__builtin_amdgcn_readlane((int)digit, __builtin_ctzll(some));
            const u64 same = ballot(in && digit == first);
            if (lane == __builtin_ctzll(some)) atomicAdd(&r.hist[first], (u32)__popcll(same));
            if (in && digit != first) atomicAdd(&r.hist[digit], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            int left = need, d = 255;
            for (; d > 0 && (int)r.hist[d] < left; --d) left -= (int)r.hist[d];
            r.need = (u32)left;
            r.prefix = prefix | (u32)d << shift;
        }
        __syncthreads();
        prefix = r.prefix;
        need = (int)r.need;
    }
    // `prefix` is the k-th best's key (its upper half for bf16), `need` of the elements that have it are among the best
    if (tid == 0) r.n = 0;
    int taken = 0;
    for (int i0 = 0; i0 < n; i0 += VR_NT) {
        const int i = i0 + tid;
        const float x = i < n ? Elem<BF16>::get(p + i) : -INFINITY;
        const u32 key = BF16 ? ord32(x) >> 16 << 16 : ord32(x);
        __syncthreads();
        if (key > prefix) top_keep(r, x, id0 + i);
        const u64 tie = ballot(i < n && key == prefix && x > -INFINITY);
        if (lane == 0) r.counts[wave] = (u32)__popcll(tie);
        __syncthreads();
        int before = taken;
        for (int w = 0; w < VR_NT / 64; ++w) {
            if (w < wave) before += (int)r.counts[w];
            taken += (int)r.counts[w];
        }
        if (i < n && key == prefix && x > -INFINITY && before + (int)lanes_below(tie) < need) top_keep(r, x, id0 + i);
    }
    __syncthreads();
}

// slots [goes][NT]: 16-bit keys of the largest of every go; mine: of the thread's largest
template <bool BF16>
__device__ __forceinline__ int top_of_stretch(TopRoom &r, const Stretch<BF16> &st, const uint16_t *slots, float mine, int id0, int k) {
    const int tid = threadIdx.x;
    r.tm[tid] = ord32(mine) >> 16;
    if (tid == 0) r.n = 0;
    __syncthreads();
    if (tid < 64) {
        u32 key[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) key[q] = r.tm[q * 64 + tid];
        const u32 t = wave_kth<4>(key, k);
        if (tid == 0) r.kth = t;
    }
    __syncthreads();
    const u32 kth = r.kth;
    const float edge = key_edge(kth);
    if (tid < st.loose) {
        const int i = st.loose_at(tid);
        const float x = Elem<BF16>::get(st.p + i);
        if (x >= edge && x > -INFINITY) top_keep(r, x, id0 + i);
    }
    if (r.tm[tid] >= kth) {
        for (int it = 0, goes = st.goes(); it < goes; ++it) {
            const u32 key = slots[it * VR_NT + tid];
            if (key < kth || key <= 0x007Fu) continue;
            for (int u = 0; u < VR_U; ++u) {
                const int unit = it * VR_GO + u * VR_NT + tid;
                if (unit >= st.units) break;
                const int at = st.head + 8 * unit;
                for (int e = 0; e < 8; ++e) {
                    const float x = Elem<BF16>::get(st.p + at + e);
                    if (x >= edge && x > -INFINITY) top_keep(r, x, id0 + at + e);
                }
            }
        }
    }
    __syncthreads();
    int n = (int)r.n;
    if (n > LP_CAP) {
        top_by_radix<BF16>(r, st.p, st.n, id0, k);
        n = (int)r.n;
    }
    return n;
}

// f(rank, key) for the k best of n keys, and f(rank, 0) for ranks that have none
template <class F>
__device__ __forceinline__ void ranked(const u64 *keys, int n, int k, F f) {
    for (int i = threadIdx.x; i < n; i += VR_NT) {
        const u64 key = keys[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += keys[j] > key;
        if (rank < k) f(rank, key);
    }
    for (int i = n + (int)threadIdx.x; i < k; i += VR_NT) f(i, 0ull);
}

struct Part {  // of a row, left for logprob_join_kernel
    float m, s, w, pad;
};

// Where entry e's row starts, or -1: it has none
__device__ __forceinline__ int64_t entry_row(const LogprobArgs &a, int64_t e) {
    const int64_t b = e / a.per_seq;
    const int64_t s = a.row_of ? (int64_t)a.row_of[e] : e - b * a.per_seq;
    return s < 0 || s >= a.rows_per_seq ? -1 : (b * a.rows_per_seq + s) * a.row_stride;
}
template <bool BF16>
__device__ __forceinline__ float logit_at(const LogprobArgs &a, int64_t at) {
    return Elem<BF16>::get((const typename Elem<BF16>::T *)a.logits + at);
}
__device__ __forceinline__ void entry_none(const LogprobArgs &a, int64_t e) {
    const int tid = threadIdx.x;
    if (tid == 0) {
        if (a.logprob) a.logprob[e] = 0.f;
        if (a.entropy) a.entropy[e] = 0.f;
        a.stats[2 * e] = a.stats[2 * e + 1] = 0.f;
    }
    if (tid < a.k) {
        a.top_logprob[e * a.k + tid] = -INFINITY;
        a.top_id[e * a.k + tid] = -1;
    }
}
// thread 0: what the row's sums say
template <bool BF16>
__device__ __forceinline__ void entry_write(const LogprobArgs &a, int64_t e, int64_t at, const Sums &r, const RowStat &st) {
    a.stats[2 * e] = st.m;
    a.stats[2 * e + 1] = st.l;
    if (a.entropy) a.entropy[e] = r.s > 0.f ? (st.log2s - r.w / r.s) * LN2 : 0.f;
    if (a.logprob) {
        const int y = a.tokens[e];
        a.logprob[e] = y >= 0 && y < a.V ? log_prob(logit_at<BF16>(a, at + y), st, a.c) : 0.f;
    }
}

extern __shared__ __align__(16) unsigned char lp_lds[];

template <bool BF16, bool ENT, bool TOP>
__global__ __launch_bounds__(VR_NT) void logprob_kernel(LogprobArgs a) {
    const int64_t e = blockIdx.x;
    const int part = blockIdx.y, tid = threadIdx.x;
    __shared__ Sums s_sums[VR_NT / 64];
    TopRoom *const room = (TopRoom *)lp_lds;
    uint16_t *const slots = (uint16_t *)(room + 1);
    const int64_t at = entry_row(a, e);
    if (at < 0) {
        if (part == 0 && a.parts == 1) entry_none(a, e);
        return;
    }
    const int id0 = part * a.part_elems, n = min(a.V - id0, a.part_elems);
    const Stretch<BF16> st(a.logits, at + id0, n);
    Sums r = {-INFINITY, 0.f, 0.f};
    float mine = -INFINITY;
    const int goes = st.goes();
    for (int it = 0; it < goes; ++it) {
        Raw<BF16> raw;
        go_request<BF16, false>(st, it, raw);
        float x[8 * VR_U];
        go_finish<BF16>(st, it, raw, x);
        const float mx = max_of(x);
        if (TOP) {
            slots[it * VR_NT + tid] = (uint16_t)(ord32(mx) >> 16);
            mine = fmaxf(mine, mx);
        }
        sums_add<ENT>(r, x, mx, a.c);
    }
    if (tid < st.loose) sums_add1<ENT>(r, Elem<BF16>::get(st.p + st.loose_at(tid)), a.c);
    r = block_sums<ENT>(r, a.c, s_sums);
    if (a.parts == 1) {
        const RowStat rs = row_stat(r.m, r.s, a.c);
        if (tid == 0) entry_write<BF16>(a, e, at, r, rs);
        if (TOP) {
            const int found = top_of_stretch<BF16>(*room, st, slots, mine, id0, a.k);
            ranked(room->keys, found, a.k, [&](int rank, u64 key) {
                a.top_logprob[e * a.k + rank] = key ? log_prob(key_val(key), rs, a.c) : -INFINITY;
                a.top_id[e * a.k + rank] = key ? (int)key_idx(key) : -1;
            });
        }
    } else {
        if (tid == 0) ((Part *)a.ws)[e * a.parts + part] = Part{r.m, r.s, r.w, 0.f};
        if (TOP) {
            const int found = top_of_stretch<BF16>(*room, st, slots, mine, id0, a.k);
            u64 *const out = a.keys + (e * a.parts + part) * a.k;
            ranked(room->keys, found, a.k, [&](int rank, u64 key) { out[rank] = key; });
        }
    }
}

// The parts of a row (up to 64) together.
template <bool BF16>
__global__ __launch_bounds__(VR_NT) void logprob_join_kernel(LogprobArgs a) {
    const int64_t e = blockIdx.x;
    const int tid = threadIdx.x;
    const int64_t at = entry_row(a, e);
    if (at < 0) {
        entry_none(a, e);
        return;
    }
    u64 *const keys = (u64 *)lp_lds;
    const int n = a.parts * a.k;
    for (int i = tid; i < n; i += VR_NT) keys[i] = a.keys[e * n + i];
    Sums r = {-INFINITY, 0.f, 0.f};
    if ((tid & 63) < a.parts) {
        const Part p = ((const Part *)a.ws)[e * a.parts + (tid & 63)];
        r = Sums{p.m, p.s, p.w};
    }
    sums_move<true>(r, wave_max(r.m), a.c);
    r.s = wave_sum(r.s);
    r.w = wave_sum(r.w);
    const RowStat rs = row_stat(r.m, r.s, a.c);
    if (tid == 0) entry_write<BF16>(a, e, at, r, rs);
    if (n == 0) return;
    __syncthreads();
    int mine = 0;  // keys of nothing come last: among them the order does not matter, but every rank below k is written once
    for (int i = tid; i < n; i += VR_NT) mine += keys[i] != 0;
    __shared__ int s_n[VR_NT / 64];
    mine = wave_sum_i32(mine);
    if (lane_id() == 0) s_n[tid >> 6] = mine;
    __syncthreads();
    int found = 0;
    for (int i = 0; i < VR_NT / 64; ++i) found += s_n[i];
    for (int i = tid; i < n; i += VR_NT) {
        const u64 key = keys[i];
        if (!key) continue;
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += keys[j] > key;
        if (rank < a.k) {
            a.top_logprob[e * a.k + rank] = log_prob(key_val(key), rs, a.c);
            a.top_id[e * a.k + rank] = (int)key_idx(key);
        }
    }
    for (int i = found + tid; i < a.k; i += VR_NT) {
        a.top_logprob[e * a.k + i] = -INFINITY;
        a.top_id[e * a.k + i] = -1;
    }
}

template <bool BF16, bool ENT, bool TOP>
static hipError_t launch_rows(const LogprobArgs &a, hipStream_t st) {
    const int goes = (a.part_elems + VR_GO_ELEMS - 1) / VR_GO_ELEMS;
    const size_t lds = TOP ? sizeof(TopRoom) + (size_t)goes * VR_NT * 2 : 0;
    launch_kernel(KID_LOGPROBS, st, logprob_kernel<BF16, ENT, TOP>, dim3((u32)a.n, a.parts), dim3(VR_NT), lds, a);
    return hipGetLastError();
}
template <bool BF16>
static hipError_t launch_type(const LogprobArgs &a, hipStream_t st) {
    hipError_t e;
    if (a.entropy) e = a.k ? launch_rows<BF16, true, true>(a, st) : launch_rows<BF16, true, false>(a, st);
    else e = a.k ? launch_rows<BF16, false, true>(a, st) : launch_rows<BF16, false, false>(a, st);
    if (e != hipSuccess || a.parts == 1) return e;
    launch_kernel(KID_LOGPROBS_JOIN, st, logprob_join_kernel<BF16>, dim3((u32)a.n), dim3(VR_NT), (size_t)a.parts * a.k * 8, a);
    return hipGetLastError();
}

size_t logprob_workspace(int64_t n, int V) {
    const int64_t parts = n * vocab_parts(n, V);
    return (size_t)parts * (sizeof(Part) + DT_K_MAX * 8);
}
hipError_t logprob_launch(LogprobArgs a, hipStream_t st) {
    a.part_elems = vocab_part_goes(a.n, a.V) * VR_GO_ELEMS;
    a.parts = vocab_parts(a.n, a.V);
    a.keys = (u64 *)((Part *)a.ws + a.n * a.parts);
    return a.dtype == DT_BF16 ? launch_type<true>(a, st) : launch_type<false>(a, st);
}

}  // namespace dt
