// Log-probabilities of given tokens, the entropy of their rows and the best alternatives: one pass over a row for its largest
// logit m, s = sum 2^(x c - M2) and w = sum 2^(x c - M2) (x c - M2) (vocab_rows.hpp), of which
//     log-probability of y = ln 2 ((y c - M2) - log2 s),   entropy = ln 2 (log2 s - w / s),
// both sums of terms of one sign.
//
// The k best: the k-th largest of the threads' own maxima (16-bit keys, the upper half of the ordered image) bounds the k-th largest element
// from below, and tightly, since places far apart in the row go to one thread.  Where a row is streamed, every thread leaves the largest of the
// 32 elements of a go as such a key, a `slot`; the few slots that reach the bound are read again, their elements that reach it listed, and the list
// ranked by counting keys of (value, id).  A list that overflows (ties, a row whose best are neighbours) gives way to a radix selection over
// the row, eight bits at a time, and the ties that still fit are taken in ascending id.
#include "vocab_rows.hpp"

namespace dt {

#define NO_KEY 0x007Fu  // 16-bit key of -inf

template <int NT>
struct TopRoom {
    static constexpr int CAP = NT == 64 ? 256 : 1024, HITS = 256;
    u32 n, hits, kth, need, prefix;
    u32 tm[256];           // the threads' largest, 16-bit keys, two threads' as one where there are more
    u32 counts[NT / 64];
    u32 hit[HITS];         // slots that reach the bound
    union {
        u64 keys[CAP];     // candidates
        u32 hist[256];
    };
};

template <int NT>
__device__ __forceinline__ void top_keep(TopRoom<NT> &r, float x, int id) {
    const u32 at = atomicAdd(&r.n, 1u);
    if (at < TopRoom<NT>::CAP) r.keys[at] = make_key(x, (u32)id);
}

// Radix selection: exactly the k best of a row that holds more than k finite entries.
template <bool BF16, int NT>
__device__ __noinline__ void top_by_radix(TopRoom<NT> &r, const typename Elem<BF16>::T *p, int n, int k) {
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
    const u32 none = ord32(-INFINITY);
    u32 prefix = 0;
    int need = k;
    for (int shift = 24; shift >= (BF16 ? 16 : 0); shift -= 8) {
        __syncthreads();
        for (int i = tid; i < 256; i += NT) r.hist[i] = 0;
        __syncthreads();
        for (int i0 = 0; i0 < n; i0 += NT) {
            const int i = i0 + tid;
            const u32 key = i < n ? ord32(Elem<BF16>::get(p + i)) : none;
            const bool in = key > none && (shift == 24 || (key ^ prefix) >> (shift + 8) == 0);
            const u32 digit = key >> shift & 255u;
            // ties come by the thousand: what agrees with the first lane that counts is counted at once
            const u64 some = ballot(in);
            if (!some) continue;
            const int lead = __builtin_ctzll(some);
            const u32 first = (u32)__builtin_amdgcn_readlane((int)digit, lead);
            const u64 same = ballot(in && digit == first);
            if (lane == lead) atomicAdd(&r.hist[first], (u32)__popcll(same));
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
    __syncthreads();
    if (tid == 0) r.n = 0;
    int taken = 0;
    for (int i0 = 0; i0 < n; i0 += NT) {
        const int i = i0 + tid;
        const float x = i < n ? Elem<BF16>::get(p + i) : -INFINITY;
        const u32 key = BF16 ? ord32(x) >> 16 << 16 : ord32(x);
        const bool tied = key == prefix && x > -INFINITY;
        const u64 tie = ballot(tied);
        __syncthreads();
        if (key > prefix) top_keep(r, x, i);
        if (lane == 0) r.counts[wave] = (u32)__popcll(tie);
        __syncthreads();
        int before = taken;
        for (int w = 0; w < NT / 64; ++w) {
            if (w < wave) before += (int)r.counts[w];
            taken += (int)r.counts[w];
        }
        if (tied && before + (int)lanes_below(tie) < need) top_keep(r, x, i);
    }
    __syncthreads();
}

// The bound from the maxima in tm (256, or the lanes' own with one wave), found by one wave; ends with a barrier.
template <int NT>
__device__ __forceinline__ u32 top_bound(TopRoom<NT> &r, float mine, int k) {
    if constexpr (NT == 64) {
        const u32 key[1] = {ord32(mine) >> 16};
        return wave_kth<1>(key, k);
    } else {
        if (threadIdx.x < 64) {
            u32 key[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) key[q] = r.tm[q * 64 + threadIdx.x];
            const u32 t = wave_kth<4>(key, k);
            if (threadIdx.x == 0) r.kth = t;
        }
        __syncthreads();
        return r.kth;
    }
}
// a thread's maximum among those of its place, before a barrier
template <int NT>
__device__ __forceinline__ void top_offer(TopRoom<NT> &r, float mine) {
    if (NT == 64) return;
    if (NT == 256) r.tm[threadIdx.x] = ord32(mine) >> 16;
    else atomicMax(&r.tm[threadIdx.x & 255], ord32(mine) >> 16);
}

// f(rank, key) for the k best of n keys, and f(rank, 0) for ranks that have none.  Up to 64 keys, as there are mostly, lie in the lanes of one wave, and each is
// handed to all of them.
template <int NT, class F>
__device__ __forceinline__ void ranked(const u64 *keys, int n, int k, F f) {
    if (n <= 64) {
        if (threadIdx.x >= 64) return;
        const int lane = lane_id();
        const u64 key = lane < n ? keys[lane] : 0ull;
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += readlane_u64(key, j) > key;
        if (lane < n && rank < k) f(rank, key);
        if (lane >= n && lane < k) f(lane, 0ull);
        return;
    }
    for (int i = threadIdx.x; i < n; i += NT) {
        const u64 key = keys[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += keys[j] > key;
        if (rank < k) f(rank, key);
    }
}

// Where entry e's row starts, or -1: it has none
__device__ __forceinline__ int64_t entry_row(const LogprobArgs &a, int64_t e) {
    const u32 b = (u32)e / (u32)a.per_seq;
    const int64_t s = a.row_of ? (int64_t)a.row_of[e] : e - (int64_t)b * a.per_seq;
    return s < 0 || s >= a.rows_per_seq ? -1 : (b * a.rows_per_seq + s) * a.row_stride;
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
// the given token's logit, NaN: none is given (no logit is NaN)
template <bool BF16>
__device__ __forceinline__ float token_logit(const LogprobArgs &a, int64_t e, int64_t at) {
    const int y = a.logprob ? a.tokens[e] : -1;
    return y >= 0 && y < a.V ? Elem<BF16>::get((const typename Elem<BF16>::T *)a.logits + at + y) : NAN;
}
// one thread: what the row's sums say
__device__ __forceinline__ void entry_write(const LogprobArgs &a, int64_t e, float xy, const Sums &r, const RowStat &st) {
    a.stats[2 * e] = st.m;
    a.stats[2 * e + 1] = st.l;
    if (a.entropy) a.entropy[e] = r.s > 0.f ? (st.log2s - r.w / r.s) * LN2 : 0.f;
    if (a.logprob) a.logprob[e] = xy != xy ? 0.f : log_prob(xy, st, a.c);
}
template <int NT>
__device__ __forceinline__ void alternatives_write(const LogprobArgs &a, int64_t e, const TopRoom<NT> &room, int found, const RowStat &st) {
    ranked<NT>(room.keys, found, a.k, [&](int rank, u64 key) {
        a.top_logprob[e * a.k + rank] = key ? log_prob(key_val(key), st, a.c) : -INFINITY;
        a.top_id[e * a.k + rank] = key ? (int)key_idx(key) : -1;
    });
}

// ---- rows that a workgroup holds ----
template <bool BF16, bool ENT, bool TOP, int NT, int U>
__global__ __launch_bounds__(NT, !BF16 && U == 8 ? 4 : TOP ? 6 : 8) void logprob_held_kernel(LogprobArgs a) {
    constexpr int G = U == 4 ? 4 : 2;  // units that are worked on at once
    const int64_t e = blockIdx.x;
    const int tid = threadIdx.x;
    __shared__ Sums s_sums[NT / 64];
    __shared__ TopRoom<TOP ? NT : 64> room_;
    TopRoom<NT> &room = (TopRoom<NT> &)room_;
    const int64_t at = entry_row(a, e);
    if (at < 0) {
        entry_none(a, e);
        return;
    }
    const Row<BF16> row(a.logits, at, a.V);
    Raw<BF16, U> raw;
    go_request<NT, false>(row, 0, raw);
    const float xl = tid < row.loose ? row.at(row.loose_at(tid)) : -INFINITY;
    const float xy = token_logit<BF16>(a, e, at);
    if (TOP) {
        if (tid == 0) room.n = 0;
        if (NT > 256) {
            if (tid < 256) room.tm[tid] = NO_KEY;
            __syncthreads();
        }
    }
    Sums r = {-INFINITY, 0.f, 0.f};
    float mine = xl;
    bool zeros = false;
#pragma unroll
    for (int u = 0; u < U; u += G) {
        float x[8 * G];
        go_take<NT, G>(row, 0, raw, u, x);
        const float mx = max_of(x);
        mine = fmaxf(mine, mx);
        sums_add<ENT>(r, x, mx, a.c, zeros);
    }
    go_keep(raw);
    if (row.loose > 0) sums_add1<ENT>(r, xl, a.c);  // uniform
    if (TOP) top_offer<NT>(room, mine);
    r = block_sums<ENT, NT>(r, a.c, s_sums);
    const RowStat st = row_stat(r.m, r.s, a.c);
    if (tid == NT - 1) entry_write(a, e, xy, r, st);
    if (!TOP) return;
    const float edge = key_edge(top_bound<NT>(room, mine, a.k));
    if (mine >= edge && mine > -INFINITY) {
        if (xl >= edge && xl > -INFINITY) top_keep(room, xl, row.loose_at(tid));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[8];
            go_take<NT, 1>(row, 0, raw, u, x);
            const float most = max_of(x);
            if (most >= edge && most > -INFINITY)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (x[j] >= edge && x[j] > -INFINITY) top_keep(room, x[j], row.head + 8 * (u * NT + tid) + j);
        }
    }
    __syncthreads();
    int found = (int)room.n;
    if (found > TopRoom<NT>::CAP) {
        top_by_radix<BF16, NT>(room, row.p, a.V, a.k);
        found = (int)room.n;
    }
    alternatives_write<NT>(a, e, room, found, st);
}

// ---- rows that are streamed ----
struct Part {  // of a row, left for logprob_join_kernel
    float m, s, w, pad;
};
extern __shared__ __align__(16) unsigned char lp_lds[];

// The candidates among the slots that reach the bound: slot i of the row is go i / NT, thread i % NT.  Ends with a barrier; the number found.
template <int NT, bool BF16, class Slot>
__device__ __forceinline__ int top_of_slots(TopRoom<NT> &r, const Row<BF16> &row, int k, float mine, Slot slot) {
    constexpr int U = STREAM_U;
    typedef TopRoom<NT> R;
    const int tid = threadIdx.x, goes = row.template goes<NT * U>();
    const u32 kth = top_bound<NT>(r, mine, k);
    const float edge = key_edge(kth);
    if (r.tm[tid & 255] >= kth)
        for (int it = 0; it < goes; ++it) {
            const u32 key = slot(it);
            if (key >= kth && key > NO_KEY) {
                const u32 at = atomicAdd(&r.hits, 1u);
                if (at < R::HITS) r.hit[at] = (u32)(it * NT + tid);
            }
        }
    if (tid < row.loose) {
        const int i = row.loose_at(tid);
        const float x = row.at(i);
        if (x >= edge && x > -INFINITY) top_keep(r, x, i);
    }
    __syncthreads();
    const int hits = (int)r.hits;
    if (hits <= R::HITS)
        for (int i = tid; i < hits * U; i += NT) {  // a unit to a thread
            const int s = (int)r.hit[i / U], unit = ((s / NT) * U + i % U) * NT + s % NT;
            if (unit >= row.units) continue;
            const int at = row.head + 8 * unit;
            float x[8];
            const Vec16 *q = (const Vec16 *)(row.p + at);
            const Vec16 lo = q[0], hi = BF16 ? lo : q[1];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (BF16) {
                    x[2 * j] = __uint_as_float(lo[j] << 16);
                    x[2 * j + 1] = __uint_as_float(lo[j] & 0xFFFF0000u);
                } else {
                    x[j] = __uint_as_float(lo[j]);
                    x[4 + j] = __uint_as_float(hi[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (x[j] >= edge && x[j] > -INFINITY) top_keep(r, x[j], at + j);
        }
    __syncthreads();
    if (hits <= R::HITS && (int)r.n <= R::CAP) return (int)r.n;
    top_by_radix<BF16, NT>(r, row.p, row.V, k);
    return (int)r.n;
}

// Goes of a row, from part * part_goes on: all of them (JOIN false) or a part's, for logprob_join_kernel.
template <bool BF16, bool ENT, bool TOP, bool JOIN, int NT>
__global__ __launch_bounds__(NT, 8) void logprob_stream_kernel(LogprobArgs a) {
    constexpr int U = STREAM_U;
    const RowPart rp = row_part(JOIN ? a.parts : 1);
    const int64_t e = rp.row;
    const int part = rp.part, tid = threadIdx.x;
    __shared__ Sums s_sums[NT / 64];
    TopRoom<NT> &room = *(TopRoom<NT> *)lp_lds;  // TOP && !JOIN, and behind it the slots
    uint16_t *const slots = JOIN ? a.slots + (e * a.goes) * NT + tid : (uint16_t *)(&room + 1) + tid;
    const int64_t at = entry_row(a, e);
    if (at < 0) {
        if (!JOIN) entry_none(a, e);
        return;
    }
    const Row<BF16> row(a.logits, at, a.V);
    const float xy = JOIN ? 0.f : token_logit<BF16>(a, e, at);
    if (TOP && !JOIN) {
        if (tid == 0) room.n = room.hits = 0;
        if (NT > 256) {
            if (tid < 256) room.tm[tid] = NO_KEY;
            __syncthreads();
        }
    }
    Sums r = {-INFINITY, 0.f, 0.f};
    float mine = -INFINITY;
    const int end = JOIN ? min((part + 1) * a.part_goes, row.template goes<NT * U>()) : row.template goes<NT * U>();
    bool zeros = false;
    int it = JOIN ? part * a.part_goes : 0;
    for (; it < end; ++it) {
        Raw<BF16, U> raw;
        go_request<NT, false>(row, it, raw);
        float x[8 * U];
        go_take<NT, U>(row, it, raw, 0, x);
        const float mx = max_of(x);
        if (TOP) {
            slots[it * NT] = (uint16_t)(ord32(mx) >> 16);
            mine = fmaxf(mine, mx);
        }
        sums_add<ENT>(r, x, mx, a.c, zeros);
    }
    if (part == 0 && tid < row.loose) sums_add1<ENT>(r, row.at(row.loose_at(tid)), a.c);
    if (TOP && !JOIN) top_offer<NT>(room, mine);
    r = block_sums<ENT, NT>(r, a.c, s_sums);
    if (JOIN) {
        if (tid == 0) ((Part *)a.ws)[e * a.parts + part] = Part{r.m, r.s, r.w, 0.f};
        return;
    }
    const RowStat st = row_stat(r.m, r.s, a.c);
    if (tid == NT - 1) entry_write(a, e, xy, r, st);
    if (TOP) {
        const int found = top_of_slots<NT, BF16>(room, row, a.k, mine, [&](int it) { return (u32)slots[it * NT]; });
        alternatives_write<NT>(a, e, room, found, st);
    }
}

// The parts of a row together.
template <bool BF16, bool TOP>
__global__ __launch_bounds__(STREAM_NT, 4) void logprob_join_kernel(LogprobArgs a) {
    constexpr int NT = STREAM_NT;
    const int64_t e = blockIdx.x;
    const int tid = threadIdx.x;
    TopRoom<NT> &room = *(TopRoom<NT> *)lp_lds;  // TOP, and behind it the slots
    uint16_t *const slots = (uint16_t *)(&room + 1);
    const int64_t at = entry_row(a, e);
    if (at < 0) {
        entry_none(a, e);
        return;
    }
    const Row<BF16> row(a.logits, at, a.V);
    const float xy = token_logit<BF16>(a, e, at);
    Sums r = {-INFINITY, 0.f, 0.f};
    if (lane_id() < a.parts) {
        const Part p = ((const Part *)a.ws)[e * a.parts + lane_id()];
        r = Sums{p.m, p.s, p.w};
    }
    const int goes = row.template goes<STREAM_GO>();
    if (TOP) {
        if (tid == 0) room.n = room.hits = 0;
        constexpr int MOST = (DT_VOCAB_MAX / STREAM_ELEMS * NT * 2 / 16 + NT - 1) / NT;
        const Vec16 *const from = (const Vec16 *)(a.slots + e * a.goes * NT);
        Vec16 v[MOST];
#pragma unroll
        for (int i = 0; i < MOST; ++i)
            if (i * NT + tid < goes * NT / 8) v[i] = from[i * NT + tid];
#pragma unroll
        for (int i = 0; i < MOST; ++i)
            if (i * NT + tid < goes * NT / 8) ((Vec16 *)slots)[i * NT + tid] = v[i];
    }
    wave_sums<true>(r, a.c);
    const RowStat st = row_stat(r.m, r.s, a.c);
    if (tid == NT - 1) entry_write(a, e, xy, r, st);
    if (!TOP) return;
    __syncthreads();
    u32 best = NO_KEY;
    for (int it = 0; it < goes; ++it) best = max(best, (u32)slots[it * NT + tid]);
    room.tm[tid] = best;
    __syncthreads();
    const int found = top_of_slots<NT, BF16>(room, row, a.k, 0.f, [&](int it) { return (u32)slots[it * NT + tid]; });
    alternatives_write<NT>(a, e, room, found, st);
}

template <bool BF16, bool ENT, bool TOP>
static hipError_t launch_rows(const LogprobArgs &a, hipStream_t st) {
    if (rows_held(a.V)) {
        by_held(a.V, [&](auto h) {
            constexpr int NT = decltype(h)::NT, U = decltype(h)::U;
            launch_kernel(KID_LOGPROBS, st, logprob_held_kernel<BF16, ENT, TOP, NT, U>, dim3((u32)a.n), dim3(NT), 0, a);
        });
        return hipGetLastError();
    }
    const size_t lds = TOP ? sizeof(TopRoom<STREAM_NT>) + (size_t)a.goes * STREAM_NT * 2 : 0;
    if (a.parts == 1) {
        const size_t lds4 = TOP ? sizeof(TopRoom<1024>) + (size_t)((a.V + 32767) / 32768) * 2048 : 0, lds2 = TOP ? sizeof(TopRoom<512>) + (size_t)((a.V + 16383) / 16384) * 1024 : 0;
        if (long_nt() == 256) launch_kernel(KID_LOGPROBS, st, logprob_stream_kernel<BF16, ENT, TOP, false, 256>, dim3((u32)a.n), dim3(256), lds, a);
        else if (long_nt() == 512) launch_kernel(KID_LOGPROBS, st, logprob_stream_kernel<BF16, ENT, TOP, false, 512>, dim3((u32)a.n), dim3(512), lds2, a);
        else launch_kernel(KID_LOGPROBS, st, logprob_stream_kernel<BF16, ENT, TOP, false, 1024>, dim3((u32)a.n), dim3(1024), lds4, a);
    } else {
        launch_kernel(KID_LOGPROBS, st, logprob_stream_kernel<BF16, ENT, TOP, true, STREAM_NT>, dim3((u32)(a.n * a.parts)), dim3(STREAM_NT), 0, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        launch_kernel(KID_LOGPROBS_JOIN, st, logprob_join_kernel<BF16, TOP>, dim3((u32)a.n), dim3(STREAM_NT), lds, a);
    }
    return hipGetLastError();
}
template <bool BF16>
static hipError_t launch_type(const LogprobArgs &a, hipStream_t st) {
    if (a.entropy) return a.k ? launch_rows<BF16, true, true>(a, st) : launch_rows<BF16, true, false>(a, st);
    return a.k ? launch_rows<BF16, false, true>(a, st) : launch_rows<BF16, false, false>(a, st);
}

size_t logprob_workspace(int64_t n, int V) {
    const int parts = row_parts(V, part_goes(n, V));
    if (rows_held(V) || parts == 1) return 0;
    return (size_t)n * parts * sizeof(Part) + (size_t)n * row_goes(V) * STREAM_NT * 2;
}
hipError_t logprob_launch(LogprobArgs a, hipStream_t st) {
    a.goes = row_goes(a.V);
    a.part_goes = part_goes(a.n, a.V);
    a.parts = row_parts(a.V, a.part_goes);
    a.slots = (uint16_t *)((Part *)a.ws + a.n * a.parts);
    return a.dtype == DT_BF16 ? launch_type<true>(a, st) : launch_type<false>(a, st);
}

}  // namespace dt
