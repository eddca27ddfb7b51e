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
#include <algorithm>

#include "vocab_rows.hpp"

namespace dt {

#define NO_KEY 0x007Fu  // 16-bit key of -inf

template <int NT>
struct TopRoom {
    static constexpr int CAP = NT == 64 ? 256 : 1024, HITS = 256;
    u32 n, hits, kth, need, prefix;
    u32 tm[256];           // the threads' largest, 16-bit keys, two threads' as one where there are more
    u32 counts[NT / 64];
    union {
        u32 hit[HITS];     // slots that reach the bound
        u32 hist[256];
    };
    u64 keys[CAP];         // candidates
};
// Eights of a held row with an element that reaches the bound, and whose they are.
template <int NT>
struct TopEights {
    static constexpr int CAP = NT == 64 ? 64 : 128;
    float x[CAP][8];
    u32 whose[CAP];        // thread and unit
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
        for (int j0 = 0; j0 < n; j0 += 8)  // lanes past the n-th hold 0, which is above none
#pragma unroll
            for (int j = 0; j < 8; ++j) rank += readlane_u64(key, j0 + j) > key;
        if (lane >= n) rank = lane;  // one of none, of key 0
        if (rank < k) f(rank, key);
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
// Waves of a SIMD: as many as leave a thread its registers, but a few spilled ones with TOP (8,000 bf16 rows of 12,000, k 1: 52 us at 6, 55 at 5).
template <bool BF16, bool ENT, bool TOP, int NT, int U>
__global__ __launch_bounds__(NT, NT == 1024 || (!BF16 && U == 8) ? 4 : TOP ? 6 : ENT && U == 8 ? 7 : 8) void logprob_held_kernel(LogprobArgs a) {
    constexpr int G = 2;  // units that are worked on at once: with four, registers go to scratch, and 8,000 fp32 rows of 6,000 (k 20) take 98 us for 48
    const int64_t e = blockIdx.x;
    const int tid = threadIdx.x;
    __shared__ Sums s_sums[NT / 64];
    __shared__ TopRoom<TOP ? NT : 64> room_;
    __shared__ TopEights<NT> eights;
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
        if (tid == 0) room.n = room.hits = 0;
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
    // The few eights that reach the bound go through LDS: a branch for each of a thread's elements is long code that is met for the first time
    // (one bf16 row of 21,840, k 31: 10.5 us, and 8.9 so).
    if (mine >= edge && mine > -INFINITY) {
        if (xl >= edge && xl > -INFINITY) top_keep(room, xl, row.loose_at(tid));
        u32 some = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[8];
            go_take<NT, 1>(row, 0, raw, u, x);
            const float most = max_of(x);
            some |= (u32)(most >= edge && most > -INFINITY) << u;
        }
        u32 put = atomicAdd(&room.hits, (u32)__popc(some));
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (some >> u & 1u) {
                if (put < TopEights<NT>::CAP) {
                    float x[8];
                    go_take<NT, 1>(row, 0, raw, u, x);
                    eights.whose[put] = (u32)(tid * U + u);
#pragma unroll
                    for (int j = 0; j < 8; ++j) eights.x[put][j] = x[j];
                }
                ++put;
            }
    }
    __syncthreads();
    const int hits = (int)room.hits;
    if (hits <= TopEights<NT>::CAP)
        for (int i = tid; i < 8 * hits; i += NT) {
            const float x = eights.x[i >> 3][i & 7];
            const u32 whose = eights.whose[i >> 3];
            if (x >= edge && x > -INFINITY) top_keep(room, x, id_of<NT, U>(row, 0, (int)(whose / U), 8 * (int)(whose % U) + (i & 7)));
        }
    __syncthreads();
    int found = (int)room.n;
    if (hits > TopEights<NT>::CAP || found > TopRoom<NT>::CAP) {
        top_by_radix<BF16, NT>(room, row.p, a.V, a.k);
        found = (int)room.n;
    }
    alternatives_write<NT>(a, e, room, found, st);
}

// ---- rows that are streamed ----
// A slot is the largest of a thread's elements of a go, the upper half of its ordered image: slot i of the row is that of go i / NT, thread i % NT.  Found by
// top_of_slots: the candidates among the slots that reach the bound.  each(least, hit): hit(slot) for those of a thread's whose key reaches `least`; mine: the largest of its keys.
// Ends with a barrier; the number found.
template <int NT, bool BF16, class Each>
__device__ __forceinline__ int top_of_slots(TopRoom<NT> &r, const Row<BF16> &row, int k, u32 mine, Each each) {
    constexpr int E = Row<BF16>::E, N = STREAM_U * 8 / E;
    typedef TopRoom<NT> R;
    const int tid = threadIdx.x;
    const u32 kth = top_bound<NT>(r, 0.f, k);
    const float edge = key_edge(kth);
    const u32 least = max(kth, NO_KEY + 1);
    if (mine >= least)
        each(least, [&](int slot) {
            const u32 at = atomicAdd(&r.hits, 1u);
            if (at < R::HITS) r.hit[at] = (u32)slot;
        });
    if (tid < row.loose) {
        const int i = row.loose_at(tid);
        const float x = row.at(i);
        if (x >= edge && x > -INFINITY) top_keep(r, x, i);
    }
    __syncthreads();
    const int hits = (int)r.hits;
    if (hits <= R::HITS)
        for (int i = tid; i < hits * N; i += NT) {  // a unit to a thread
            const int s = (int)r.hit[i / N], unit = ((s / NT) * N + i % N) * NT + s % NT;
            if (unit >= row.units) continue;
            const int at = row.head + E * unit;
            float x[E];
            unpack(*(const Vec16 *)(row.p + at), x);
            u32 some = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) some |= (u32)(x[j] >= edge && x[j] > -INFINITY) << j;
            for (; some; some &= some - 1) {
                const int i = at + __builtin_ctz(some);
                top_keep(r, row.at(i), i);
            }
        }
    __syncthreads();
    if (hits <= R::HITS && (int)r.n <= R::CAP) return (int)r.n;
    top_by_radix<BF16, NT>(r, row.p, row.V, k);
    return (int)r.n;
}

extern __shared__ __align__(16) unsigned char lp_lds[];

// Whole rows.  ASK: a go is asked for while the one before is worked on.
template <bool BF16, bool ENT, bool TOP, int NT, bool ASK, bool KEEP>
__global__ __launch_bounds__(NT, ASK ? 4 : 8) void logprob_stream_kernel(LogprobArgs a) {
    constexpr int U = STREAM_U;
    const int64_t e = blockIdx.x;
    const int tid = threadIdx.x;
    __shared__ Sums s_sums[NT / 64];
    TopRoom<NT> &room = *(TopRoom<NT> *)lp_lds;  // TOP, and behind it the slots
    uint16_t *const slots = (uint16_t *)(&room + 1) + tid;
    const int64_t at = entry_row(a, e);
    if (at < 0) {
        entry_none(a, e);
        return;
    }
    const Row<BF16> row(a.logits, at, a.V);
    const float xy = token_logit<BF16>(a, e, at);
    if (TOP) {
        if (tid == 0) room.n = room.hits = 0;
        if (NT > 256) {
            if (tid < 256) room.tm[tid] = NO_KEY;
            __syncthreads();
        }
    }
    Sums r = {-INFINITY, 0.f, 0.f};
    float mine = -INFINITY;
    const int goes = row.template goes<NT, U>();
    bool zeros = false;
    Raw<BF16, U> raw, next;
    if (ASK && goes > 0) go_request<NT, KEEP>(row, 0, raw);
    for (int it = 0; it < goes; ++it) {
        if (ASK) go_request<NT, KEEP>(row, min(it + 1, goes - 1), next);
        else go_request<NT, KEEP>(row, it, raw);
        float x[8 * U];
        go_take<NT, U>(row, it, raw, 0, x);
        if (ASK) raw = next;
        const float mx = max_of(x);
        if (TOP) {
            slots[it * NT] = (uint16_t)(ord32(mx) >> 16);
            mine = fmaxf(mine, mx);
        }
        sums_add<ENT>(r, x, mx, a.c, zeros);
    }
    if (tid < row.loose) sums_add1<ENT>(r, row.at(row.loose_at(tid)), a.c);
    if (TOP) top_offer<NT>(room, mine);
    r = block_sums<ENT, NT>(r, a.c, s_sums);
    const RowStat st = row_stat(r.m, r.s, a.c);
    if (tid == NT - 1) entry_write(a, e, xy, r, st);
    if (!TOP) return;
    const int found = top_of_slots<NT>(room, row, a.k, ord32(mine) >> 16, [&](u32 least, auto hit) {
        for (int it = 0; it < goes; ++it)
            if (slots[it * NT] >= least) hit(it * NT + tid);
    });
    alternatives_write<NT>(a, e, room, found, st);
}

// Parts of a row, part_goes goes each.  The slots go to the memory side four to a word.
template <bool BF16, bool ENT, bool TOP>
__global__ __launch_bounds__(STREAM_NT, 8) void logprob_parts_kernel(LogprobArgs a) {
    constexpr int NT = STREAM_NT, U = STREAM_U, WORDS = NT / 4;  // words of a go
    const RowPart rp = row_part(blockIdx.x, a.parts);
    const int64_t e = rp.row;
    const int part = rp.part, tid = threadIdx.x;
    __shared__ Sums s_sums[NT / 64];
    __shared__ TopRoom<TOP ? NT : 64> room_;
    __shared__ bool s_last;
    TopRoom<NT> &room = (TopRoom<NT> &)room_;
    const int64_t at = entry_row(a, e);
    if (at < 0) {
        if (part == 0) entry_none(a, e);
        return;
    }
    const Row<BF16> row(a.logits, at, a.V);
    u64 *const slots = a.slots + e * a.goes * WORDS;
    Sums r = {-INFINITY, 0.f, 0.f};
    const int goes = row.template goes<NT, U>(), end = min((part + 1) * a.part_goes, goes);
    bool zeros = false;
    for (int it = part * a.part_goes; it < end; ++it) {
        Raw<BF16, U> raw;
        go_request<NT, true>(row, it, raw);
        float x[8 * U];
        go_take<NT, U>(row, it, raw, 0, x);
        const float mx = max_of(x);
        if (TOP) {
            const int key = (int)(ord32(mx) >> 16);
            const u32 lo = (u32)dpp_mov<0x00, 0xf>(0, key) | (u32)dpp_mov<0x55, 0xf>(0, key) << 16;  // those of a quad
            const u32 hi = (u32)dpp_mov<0xAA, 0xf>(0, key) | (u32)dpp_mov<0xFF, 0xf>(0, key) << 16;
            if ((tid & 3) == 0) put_agent(slots + it * WORDS + tid / 4, (u64)hi << 32 | lo);
        }
        sums_add<ENT>(r, x, mx, a.c, zeros);
    }
    if (part == 0 && tid < row.loose) sums_add1<ENT>(r, row.at(row.loose_at(tid)), a.c);
    if (TOP) {
        if (tid == 0) room.n = room.hits = 0;
        drain();  // the slots are there before the barrier, and the first wave's mark comes behind it
    }
    r = block_sums<ENT, NT>(r, a.c, s_sums);
    u64 *const sums = (u64 *)a.ws + 2 * e * a.parts, *const marks = a.marks + e * a.parts;
    if (tid < 64) {
        if (tid == 0) {
            put_agent(sums + 2 * part, (u64)__float_as_uint(r.s) << 32 | __float_as_uint(r.m));
            put_agent(sums + 2 * part + 1, (u64)__float_as_uint(r.w));
        }
        const bool last = part_arrive(marks, part, a.parts, a.tag);
        if (TOP && tid == 0) s_last = last;
        if (!TOP && !last) return;
    } else if (!TOP)
        return;
    if (TOP) {
        __syncthreads();
        if (!s_last) return;
    }
    // The parts of the row together.
    const float xy = token_logit<BF16>(a, e, at);
    u64 word[4], lo = 0, hi = 0;  // of slots, the first 1,024 of the row's
    const int words = goes * WORDS;
    if (TOP) {
#pragma unroll
        for (int i = 0; i < 4; ++i) word[i] = get_agent(slots + min(i * NT + tid, words - 1));
    }
    r = Sums{-INFINITY, 0.f, 0.f};
    if (lane_id() < a.parts) {
        lo = get_agent(sums + 2 * lane_id());
        hi = get_agent(sums + 2 * lane_id() + 1);
        r = Sums{__uint_as_float((u32)lo), __uint_as_float((u32)(lo >> 32)), __uint_as_float((u32)hi)};
    }
    wave_sums<ENT>(r, a.c);
    const RowStat st = row_stat(r.m, r.s, a.c);
    if (tid == 0) entry_write(a, e, xy, r, st);
    if (tid < 64) parts_leave(marks, a.parts);
    if (!TOP) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) word[i] = i * NT + tid < words ? word[i] : NO_KEY * 0x0001000100010001ull;
    const auto key_of = [](u64 w, int j) { return (u32)(w >> 16 * j) & 0xFFFFu; };
    u32 best = NO_KEY;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) best = max(best, key_of(word[i], j));
    for (int at = 4 * NT + tid; at < words; at += NT) {
        const u64 w = get_agent(slots + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) best = max(best, key_of(w, j));
    }
    room.tm[tid] = best;
    __syncthreads();
    // (Bits first, and one body for a hit: this is code that nobody has run before the last part, and every line of it is fetched.  A branch for each of
    // a thread's sixteen keys, and for each of a unit's elements: 20 of one row of 128,256 10.3 us, 8.8 so, of 64 rows 14.6, 12.8.)
    const int found = top_of_slots<NT>(room, row, a.k, best, [&](u32 least, auto hit) {
        u32 bits = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) bits |= (u32)(key_of(word[i], j) >= least) << (4 * i + j);
        for (; bits; bits &= bits - 1) {
            const int b = __builtin_ctz(bits);
            hit(4 * ((b >> 2) * NT + tid) + (b & 3));
        }
        for (int at = 4 * NT + tid; at < words; at += NT) {
            const u64 w = get_agent(slots + at);
            for (int j = 0; j < 4; ++j)
                if (key_of(w, j) >= least) hit(4 * at + j);
        }
    });
    alternatives_write<NT>(a, e, room, found, st);
}

template <bool BF16, bool ENT, bool TOP>
static hipError_t launch_rows(const LogprobArgs &a, hipStream_t st) {
    const auto whole = [&](auto nt, auto ask, auto keep) {
        constexpr int NT = decltype(nt)::value;
        constexpr bool ASK = decltype(ask)::value, KEEP = decltype(keep)::value;
        const size_t goes = (a.V + NT * STREAM_U * 8 - 1) / (NT * STREAM_U * 8), lds = TOP ? sizeof(TopRoom<NT>) + goes * NT * 2 : 0;
        launch_kernel(KID_LOGPROBS, st, logprob_stream_kernel<BF16, ENT, TOP, NT, ASK, KEEP>, dim3((u32)a.n), dim3(NT), lds, a);
    };
    const auto held = [&](auto h) {
        constexpr int NT = decltype(h)::NT, U = decltype(h)::U;
        launch_kernel(KID_LOGPROBS, st, logprob_held_kernel<BF16, ENT, TOP, NT, U>, dim3((u32)a.n), dim3(NT), 0, a);
    };
    switch (rows_cut(a.n, a.V, BF16, a.row_of != nullptr, TOP)) {
        case HELD:
            if (a.V <= HELD_MID) by_held_mid(a.n, a.V, held);
            else held(Held<1024, 4>());
            break;
        case PARTS:
            launch_kernel(KID_LOGPROBS, st, logprob_parts_kernel<BF16, ENT, TOP>, dim3((u32)(a.n * a.parts)), dim3(STREAM_NT), 0, a);
            break;
        case WIDE:
            if (rows_keep(a.n, a.V, BF16)) whole(std::integral_constant<int, WIDE_NT>(), std::false_type(), std::true_type());
            else whole(std::integral_constant<int, WIDE_NT>(), std::false_type(), std::false_type());
            break;
        case AHEAD: whole(std::integral_constant<int, STREAM_NT>(), std::true_type(), std::false_type()); break;
        case WHOLE: whole(std::integral_constant<int, STREAM_NT>(), std::false_type(), std::false_type()); break;
    }
    return hipGetLastError();
}
template <bool BF16>
static hipError_t launch_type(const LogprobArgs &a, hipStream_t st) {
    if (a.entropy) return a.k ? launch_rows<BF16, true, true>(a, st) : launch_rows<BF16, true, false>(a, st);
    return a.k ? launch_rows<BF16, false, true>(a, st) : launch_rows<BF16, false, false>(a, st);
}

// Sums of the parts, their marks, slots: as many as parts can be, so that what suffices for a call does for one of fewer or shorter rows.
size_t logprob_workspace(int64_t n, int V) { return (size_t)std::min(n, PARTS_ROWS - 1) * row_goes(V) * (24 + STREAM_NT * 2); }
hipError_t logprob_launch(LogprobArgs a, hipStream_t st) {
    a.goes = row_goes(a.V);
    a.part_goes = part_goes(a.n, a.V);
    a.parts = row_parts(a.V, a.part_goes);
    a.marks = (u64 *)a.ws + 2 * a.n * a.parts;
    a.slots = a.marks + a.n * a.parts;
    a.tag = launch_tag();
    return a.dtype == DT_BF16 ? launch_type<true>(a, st) : launch_type<false>(a, st);
}

}  // namespace dt
