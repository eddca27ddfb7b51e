// A workgroup's pass over a row of logits: what the log-probabilities (logprobs.hip) and the losses and gradients (distill.hip) share.
//
// A row is V elements from any address.  Elements up to the first multiple of 16 bytes and behind the last whole unit of 16 bytes are `loose`, up to 14, one
// to a thread.  A thread takes 8 U elements at a go, in units NT apart, so that a go of a workgroup of NT threads reads NT * U * 8 elements front to back, and every
// load of a wave 1 KB side by side.  (Units of eight fp32 elements, 32 bytes to a lane: gradients of 2,048 rows of 32,000 108 us.)
//
// Softmax statistics.  With c = log2(e) / T a row's weights are 2^(x c - M2), M2 = fl(m c) for the largest logit m so far: one fused multiply-add
// and one exp2 an element, and since every sum refers to the M2 that was subtracted, its rounding drops out of all results.  Sums are fp32.
// Where that rounding is itself a large power (|m c| from 2^20 on, up to rows that hold nothing but masks of the type's lowest value)
// the exponent is (x - m) c.
#pragma once
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace dt {

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
struct Row {
    static constexpr int E = BF16 ? 8 : 4;  // elements of a unit
    const typename Elem<BF16>::T *p;
    int V, head, units, loose;
    __device__ __forceinline__ Row(const void *logits, int64_t at, int n) {
        p = (const typename Elem<BF16>::T *)logits + at;
        V = n;
        head = min((int)(-(uintptr_t)p / sizeof(*p)) & (E - 1), n);
        units = (n - head) / E;
        loose = n - E * units;
    }
    __device__ __forceinline__ float at(int i) const { return Elem<BF16>::get(p + i); }
    // where loose element i, i < loose, lies in the row
    __device__ __forceinline__ int loose_at(int i) const { return i < head ? i : i + E * units; }
    template <int NT, int U>
    __device__ __forceinline__ int goes() const { return (E * units + NT * U * 8 - 1) / (NT * U * 8); }
};

// Where element `id` is worked on: at go `go` (-1: a loose one) by thread `thread`, as its element `elem`.
struct Place {
    int go, thread, elem;
};
template <bool BF16, int NT, int U>
__device__ __forceinline__ Place place_of(const Row<BF16> &row, int id) {
    constexpr u32 E = Row<BF16>::E, GO = NT * U * 8 / E;  // units of a go
    const u32 at = (u32)(id - row.head);
    if (at >= E * (u32)row.units) return Place{-1, id < row.head ? id : id - (int)E * row.units, 0};
    const u32 unit = at / E, in_go = unit % GO;
    return Place{(int)(unit / GO), (int)(in_go % NT), (int)(E * (in_go / NT) + at % E)};
}
// the id of a thread's element `elem` of go `it`
template <int NT, int U, bool BF16>
__device__ __forceinline__ int id_of(const Row<BF16> &row, int it, int thread, int elem) {
    constexpr int E = Row<BF16>::E;
    return row.head + E * ((it * (U * 8 / E) + elem / E) * NT + thread) + elem % E;
}

typedef u32 Vec16 __attribute__((ext_vector_type(4)));
template <bool BF16, int U>
struct Raw {
    static constexpr int N = U * 8 / Row<BF16>::E;
    Vec16 r[N];
};
// the units of go `it` of this thread; those past the end are the last unit again (row.units > 0).  KEEP: through the caches, as other loads, or past them.
template <int NT, bool KEEP, bool BF16, int U>
__device__ __forceinline__ void go_request(const Row<BF16> &row, int it, Raw<BF16, U> &raw) {
#pragma unroll
    for (int u = 0; u < raw.N; ++u) {
        const int unit = min((it * raw.N + u) * NT + (int)threadIdx.x, row.units - 1);
        const Vec16 *q = (const Vec16 *)(row.p + row.head + row.E * (int64_t)unit);
        raw.r[u] = KEEP ? *q : __builtin_nontemporal_load(q);
    }
    __builtin_amdgcn_sched_barrier(0);  // all on their way before anything that follows
}
__device__ __forceinline__ void unpack(const Vec16 &v, float (&x)[8]) {  // bf16
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(v[e] << 16);
        x[2 * e + 1] = __uint_as_float(v[e] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(const Vec16 &v, float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(v[e]);
}
// elements 8 first .. 8 (first + G) - 1 of what was read, as floats; of units past the end -inf
template <int NT, int G, bool BF16, int U>
__device__ __forceinline__ void go_take(const Row<BF16> &row, int it, const Raw<BF16, U> &raw, int first, float (&x)[8 * G]) {
    constexpr int E = Row<BF16>::E, N = 8 * G / E;
    const int from = 8 * first / E;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        float y[E];
        unpack(raw.r[from + u], y);
#pragma unroll
        for (int e = 0; e < E; ++e) x[E * u + e] = y[e];
    }
    if ((it * raw.N + from + N) * NT > row.units) {  // uniform
        asm volatile("");  // (a branch, and not a choice for every element)
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const bool there = (it * raw.N + from + u) * NT + (int)threadIdx.x < row.units;
#pragma unroll
            for (int e = 0; e < E; ++e) x[E * u + e] = there ? x[E * u + e] : -INFINITY;
        }
    }
}

// Few logits, which the last-level cache (256 MB) is likely to hold as what has written them left them, are read through the caches; more are read past them.  Us, through |
// past: wide 128 fp32 rows of 128,256 (66 MB) 14.7 | 17.0, of 50,001 9.9 | 10.5; loss in parts 300 fp32 rows of 50,001 15.1 | 16.0, 383 of 128,256 (196 MB) 39.7 | 36.0;
// gradients of 100 bf16 rows of 128,256 10.0 | 11.3, 8,192 of 32,000 (524 MB) 185 | 179.  (A branch inside of all kernels costs more registers than it gives.)
inline bool rows_keep(int64_t n, int V, bool bf16) { return n * V <= ((int64_t)64 << 20) / (bf16 ? 2 : 4); }

// Between two passes over what was read: else the compiler keeps the first pass's floats, twice the registers of bf16 elements.  And before what is read is worked
// on and stored unit by unit: all of it has arrived then.
template <bool BF16, int U>
__device__ __forceinline__ void go_keep(Raw<BF16, U> &raw) {
#pragma unroll
    for (int u = 0; u < raw.N; ++u) asm("" : "+v"(raw.r[u]));
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
__device__ __forceinline__ float ref_below(float from, float to, float c) {
    const float a = from * c, b = to * c;
    return plain_ref(a) && plain_ref(b) ? a - b : from == to ? 0.f : (from - to) * c + (ref_off(from, c) - ref_off(to, c));
}
__device__ __forceinline__ float ref_step(float from, float to, float c) {
    return fmaxf(ref_below(from, to, c), -1e4f);  // (a sum of nothing, times any power, stays nothing)
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
// Elements into a thread's sums; mx: their largest.  A weight of 0 has an exponent of -inf, whose share of w is no number: where a wave
// comes upon one (`zeros`, the same for its lanes), w is summed with the exponents held above -1e4, from there on.  (Always so it would be an instruction more for
// every element.)
template <bool ENT, int N>
__device__ __forceinline__ void sums_add(Sums &a, const float (&x)[N], float mx, float c, bool &zeros) {
    if (mx > a.m) sums_move<ENT>(a, mx, c);
    float M2 = a.m * c;
    if (ballot(!plain_ref(M2))) {  // a wave that has met nothing finite yet, or logits out of the ordinary
        const float m = a.m == -INFINITY ? 0.f : a.m, off = -ref_off(m, c);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float t = fmaf(x[j] - m, c, off), e = __builtin_amdgcn_exp2f(t);
            a.s += e;
            if (ENT) a.w = fmaf(e, fmaxf(t, -1e4f), a.w);
        }
        return;
    }
    float s[2] = {0.f, 0.f}, w[2] = {0.f, 0.f};
    if (!ENT || !zeros) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float t = fmaf(x[j], c, -M2), e = __builtin_amdgcn_exp2f(t);
            s[j & 1] += e;
            if (ENT) w[j & 1] = fmaf(e, t, w[j & 1]);
        }
        w[0] += w[1];
        if (ENT && ballot(w[0] != w[0])) zeros = true;
    }
    if (ENT && zeros) {
        s[0] = s[1] = w[0] = 0.f;
        asm("" : "+v"(M2));
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float t = fmaf(x[j], c, -M2), e = __builtin_amdgcn_exp2f(t);
            s[j & 1] += e;
            w[0] = fmaf(e, fmaxf(t, -1e4f), w[0]);
        }
    }
    a.s += s[0] + s[1];
    if (ENT) a.w += w[0];
}
template <bool ENT>
__device__ __forceinline__ void sums_add1(Sums &a, float x, float c) {
    const float t = -ref_off(x, c), e = x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(t);  // (not 1: a sum is against M2, and so is what is read off it)
    sums_join<ENT>(a, Sums{x, e, ENT ? e * t : 0.f}, c);
}
// (v_max3_f32 by name: fmaxf makes every element a quiet number first, an instruction each)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
template <int N>
__device__ __forceinline__ float max_of(const float (&x)[N]) {
    static_assert(N % 4 == 0, "pairs");
    float p = max3(x[0], x[1], x[1]), q = max3(x[2], x[3], x[3]);
#pragma unroll
    for (int j = 4; j < N; j += 4) {
        p = max3(p, x[j], x[j + 1]);
        q = max3(q, x[j + 2], x[j + 3]);
    }
    return max3(p, q, q);
}

// the sums of a wave's lanes, in every lane
template <bool ENT>
__device__ __forceinline__ void wave_sums(Sums &a, float c) {
    sums_move<ENT>(a, wave_max(a.m), c);
    a.s = wave_sum(a.s);
    if (ENT) a.w = wave_sum(a.w);
}
// The sums of a workgroup's threads, in every thread.  `room` is written once in a kernel; the barrier is there for the caller's
// shared memory too.
template <bool ENT, int NT>
__device__ __forceinline__ Sums block_sums(Sums a, float c, Sums (&room)[NT / 64]) {
    wave_sums<ENT>(a, c);
    if (NT == 64) {
        __syncthreads();
        return a;
    }
    if (lane_id() == 0) room[threadIdx.x >> 6] = a;
    __syncthreads();
    Sums r = lane_id() < NT / 64 ? room[lane_id() % (NT / 64)] : Sums{-INFINITY, 0.f, 0.f};
    wave_sums<ENT>(r, c);
    return r;
}

// What a row's sums say.
struct RowStat {
    float m;     // largest logit
    float log2s; // log2 of the sum against its reference
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
    const float t = log2_weight(x, r.m, c);
    // (a logit next to the type's lowest leaves fp32's range times log2(e), and may not without)
    return r.m == -INFINITY ? -INFINITY : t > -INFINITY ? (t - r.log2s) * LN2 : (x - r.m) * (c * LN2);
}

// ---- parts of a row that meet in their own launch ----------------------------------------------------
// Every part leaves what it has at the memory side, then a mark, the launch's number; who then sees the marks of all parts joins them.  The part whose mark
// lands last sees them all; the one before it may as well, and does the same over again.  Nobody waits.  Marks are taken away by who has joined, for a replayed
// graph, whose launches have the same number.
// By one wave, behind what it has left there.  True: all are there.
__device__ __forceinline__ bool part_arrive(u64 *marks, int part, int parts, u64 tag) {
    drain();
    if (lane_id() == 0) put_agent(marks + part, tag);
    drain();
    return ballot(lane_id() < parts && get_agent(marks + min(lane_id(), parts - 1)) != tag) == 0ull;
}
__device__ __forceinline__ void parts_leave(u64 *marks, int parts) {
    if (lane_id() < parts) put_agent(marks + lane_id(), 0);
}

// ---- how a call of n rows is cut -------------------------------------------------------------------
// A go of a workgroup that streams reads 8,192 elements, 16 or 32 KB; with four times the threads, four times that.
constexpr int STREAM_NT = 256, WIDE_NT = 1024, STREAM_U = 4, STREAM_ELEMS = 8 * STREAM_NT * STREAM_U;
inline int row_goes(int V) { return (V + STREAM_ELEMS - 1) / STREAM_ELEMS; }
constexpr int64_t CUS = 256;
// Workgroups that hold a row in their registers: threads, and units of a thread.  f(Held<NT, U>) for n rows of V entries.  As few threads as hold the row, but while
// compute units have room more of them, each with less to do.  Us, less | more threads:
//     V = 1,900:  n = 1,000 4.6 | 6.7 (log-probabilities), 7.5 | 9.8 (loss and gradient, as all second figures here), bf16
//     V = 12,000: n = 1 4.7 | 4.6, 7.0 | 5.7;  300 6.7 | 6.4, 9.7 | 9.0;  8,000 46 | 57, 77 | 85, bf16;  n = 1 4.8 | 4.4, 7.2 | 6.0;  300 7.0 | 6.9, 10.4 | 9.4;  1,000 11.1 | 11.1, 16.9 | 20.1, fp32
//     V = 21,840: n = 64 6.2 | 6.1, 8.4 | 8.1;  300 8.8 | 8.8, 12.6 | 12.6;  1,000 14.8 | 16.4, 21.6 | 23.9, bf16;  n = 64 6.7 | 6.1, 8.8 | 8.3;  300 9.9 | 9.9, 13.8 | 16.9, fp32
template <int NT_, int U_>
struct Held {
    static constexpr int NT = NT_, U = U_;
};
constexpr int HELD_LEAST = 32, HELD_MID = 16384, HELD_V = 32768;  // (shorter rows may have no whole unit)
template <class F>
inline void by_held_mid(int64_t n, int V, F f) {
    if (V <= 2048) f(Held<64, 4>());
    else if (V <= 8192) f(Held<256, 4>());
    else if (n <= 2 * CUS) f(Held<512, 4>());
    else f(Held<256, 8>());
}
// A launch has fewer than 2^32 threads.  (Rows are fewer than 2^24: only workgroups of more than 256 come there.)
inline bool launch_holds(int64_t n, int nt) { return n * nt < (int64_t)1 << 32; }
enum Cut {
    HELD,   // a workgroup holds a row
    PARTS,  // a row is many workgroups', which meet
    WIDE,   // whole rows, 1,024 threads to each
    AHEAD,  // whole rows, 256 threads to each, a go asked for while the one before is worked on
    WHOLE   // whole rows, 256 threads to each
};
// Rows that are streamed: few are cut, so that they fill the chip; with one row to a compute unit 1,024 threads read it, if it is long; with two, 256 threads that ask ahead;
// beyond that rows are there by the thousand, and eight small workgroups to a compute unit overlap one's end with another's reading, with as few registers as that takes.
// Alternatives (best) are listed by a row's last part alone, so that parts end earlier.
// Log-probabilities of n rows of V bf16 entries, us, with no / 20 alternatives, parts | wide | ahead | whole:
//     V = 50,001:  n = 64 6.7 / 10.8 | 7.8 / 10.3 | 8.5 / 11.4 | 8.3 / 13.9;  96 7.6 / 11.9 | 8.0 / 10.6 | 8.8 / 11.4 | 11.0 / 14.2;  127 8.3 / 13.0 | 8.8 / 11.3 | 8.9 / 11.6 | 10.9 / 14.2;
//                  200 9.8 / 15.1 | 9.7 / 12.3 | 9.2 / 11.8 | 11.5 / 14.6;  500 13.8 / 21.0 | 15.3 / 18.4 | 12.5 / 15.8 | 13.8 / 17.3
//     V = 128,256: n = 64 8.5 / 12.8 | 11.4 / 14.2 | 14.7 / 17.6 | 20.4 / 24.1;  96 10.2 / 15.0 | 11.6 / 14.6 | 14.9 / 17.7 | 20.7 / 24.6;  127 12.2 / 17.3 | 11.8 / 14.9 | 15.0 / 17.7 | 21.1 / 24.9;
//                  200 15.0 / 21.4 | 12.6 / 15.6 | 15.4 / 18.4 | 21.7 / 25.4;  500 28.6 / 37.3 | 25.0 / 27.7 | 23.5 / 26.7 | 26.1 / 30.1;  2,048 83 / 106 | 84 / 93 | 90 / 97 | 83 / 90
//     V = 250,001: n = 96 13.3 / 21.7 | 19.1 / 22.6;  127 15.5 / 24.9 | 19.5 / 22.9
// A row that a workgroup could hold, V = 21,840, held | ahead or whole: n = 300 8.8 / 13.6 | 7.6 / 11.1;  8,000 85 / 121 | 69 / 85;  V = 12,000: 300 6.7 / 10.3 | 6.6 / 9.9;  8,000 46 / 67 | 52 / 63.
// some_none: rows that are named one by one, of which some are none.  Then the next workgroup has to take a place that is free: long rows, the emitted ones of 64
// sequences, 281 of 576, were 24.4 us wide, where two fit a compute unit, and 30.5 by 256 threads, where those that come to a compute unit at first stay.
constexpr int64_t PARTS_ROWS = 128, MANY_ROWS = 2048;
inline bool row_is_long(int V, bool bf16) { return (int64_t)V * (bf16 ? 2 : 4) >= 160 * 1024; }
inline Cut rows_cut(int64_t n, int V, bool bf16, bool some_none, bool best) {
    if (V < HELD_LEAST) return WHOLE;
    if (V <= HELD_MID || (V <= HELD_V && n <= CUS)) return HELD;
    if (n < (best && V <= 1 << 18 ? 80 : PARTS_ROWS)) return PARTS;
    if (n <= (row_is_long(V, bf16) ? some_none ? MANY_ROWS - 1 : CUS : 5 * CUS / 8)) return WIDE;
    return n <= 2 * CUS ? AHEAD : WHOLE;
}
// goes of a part, so that there are about eight workgroups to a compute unit; parts of a row (up to 64)
inline int part_goes(int64_t n, int V) {
    const int goes = row_goes(V);
    const int64_t parts = (8 * CUS + n - 1) / n;
    return parts >= goes ? 1 : (int)((goes + parts - 1) / parts);
}
inline int row_parts(int V, int part_goes) { return (row_goes(V) + part_goes - 1) / part_goes; }
// Launches are lines of workgroups, the parts of a row one after the other: workgroup i is part i % parts of row i / parts.
struct RowPart {
    int64_t row;
    int part;
};
__device__ __forceinline__ RowPart row_part(u32 i, int parts) {
    const u32 r = parts == 1 ? i : i / (u32)parts;
    return RowPart{(int64_t)r, (int)(i - r * (u32)parts)};
}

}  // namespace dt
