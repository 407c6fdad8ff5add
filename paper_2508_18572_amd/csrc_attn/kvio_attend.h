// kvio_attend.h -- what the attention kernels share on the device.
#pragma once

#include "kvio_attn_internal.h"

namespace kvio {

constexpr float kMinusInf = -__builtin_huge_valf();
constexpr int kTile = 32;                    // keys that a wave takes at a time
// A running maximum stays until a score passes it by this much (in powers of two): probabilities
// and their sums stay below 2^8 times the number of keys, and rescaling is rare.
constexpr float kSlack = 8.0f;
// fp16 probabilities (beside fp16 values; beside e4m3 ones a ValueUnit does as much) are taken 2^7 times as large, up to 2^15
// with the slack: steps of 2^-24 are then 2^-31 of the largest, and thousands of small ones beside a large one count.
template <bool BF16, bool E4M3> constexpr float kRaised = BF16 || E4M3 ? 0.0f : 7.0f;

// The keys of a sequence: those that any row sees, [lo, hi), and those that all see.
struct Span {
    int32_t lo, hi, whole_lo, whole_hi;
    int32_t tiles;                           // of kTile keys, at multiples of it, that hold [lo, hi)
};
// The first key that a row at `place` sees.  Places may be so far below zero that 32 bits do not hold what a window leaves.
__device__ __forceinline__ int32_t window_from(const AttendArgs &a, int place) {
    return a.window > 0 && place >= a.window ? place - a.window + 1 : 0;
}
__device__ __forceinline__ Span span_of(const AttendArgs &a, const Seq &s) {
    Span r;
    const int last = s.first + s.rows - 1;   // the last row's place
    r.hi = last + 1;
    r.lo = window_from(a, s.first);
    r.whole_lo = window_from(a, last);
    r.whole_hi = s.first + 1;
    const uint32_t lo = static_cast<uint32_t>(r.lo), hi = static_cast<uint32_t>(r.hi);      // 0 or more, where they count
    r.tiles = s.rows > 0 && r.hi > r.lo ? static_cast<int32_t>((hi + kTile - 1) / kTile - lo / kTile) : 0;
    return r;
}

// All sequences' tiles, end to end, cut into equal ranges.
struct Ranges {
    int32_t total, per_worker;
};
// `begin` (if not null): the first tile of sequence b.
__device__ __forceinline__ Ranges ranges_of(const AttendArgs &a, int lane, int b = 0, int64_t *begin = nullptr) {
    int all = 0, before = 0;
    for (int i = lane; i < a.c.num_seqs; i += 64) {
        const int t = span_of(a, seq_of(a.c, i)).tiles;
        all += t;
        before += i < b ? t : 0;
    }
    for (int by = 1; by < 64; by *= 2) {
        all += lane_xor(all, by);
        if (begin != nullptr) before += lane_xor(before, by);
    }
    if (begin != nullptr) *begin = wave_first(before);
    Ranges r;
    r.total = wave_first(all);
    r.per_worker = (r.total + a.workers - 1) / a.workers;
    if (r.per_worker < a.min_tiles) r.per_worker = a.min_tiles;
    return r;
}
// The sequence that holds tile `at` (one does), and where its tiles begin.
__device__ __forceinline__ int find_tile(const AttendArgs &a, int64_t at, int lane, int64_t *begin) {
    int64_t before = 0;
    for (int i = 0;; i += 64) {
        const int t = i + lane < a.c.num_seqs ? span_of(a, seq_of(a.c, i + lane)).tiles : 0;
        const int upto = lanes_upto(t, lane);
        const uint64_t behind = wave_ballot(before + upto > at);
        if (behind != 0) {
            const int l = __builtin_ctzll(behind);
            *begin = before + wave_read(upto, l) - wave_read(t, l);
            return i + l;
        }
        before += wave_read(upto, 63);
    }
}

// Floats into the partial results: of a worker, head and one of its two shared sequences, a row's
// sums, then its maximum and the sum of its probabilities.
__device__ __forceinline__ int64_t partial_at(const AttendArgs &a, int worker, int h, int which, int row, int dim) {
    return (((int64_t(worker) * a.c.heads + h) * 2 + which) * a.slot_rows + row) * (dim + 2);
}

__device__ __forceinline__ float lse_of(float top, float sum) {
    return sum == 0 ? kMinusInf : (top + log2_fast(sum)) * 0.69314718055994530942f;
}

// Partial results [from, to) of a row, joined by a wave in order: their maximum, sum and sums, D / 64 dims a lane.  Partial
// i has its D sums at sums(i), its maximum and sum at ends(i).  Four at a time, so that their loads
// wait for nothing; more cost more in fetching the code than they save (384 partial results of 32 rows: 32 at a time 15 us).
__device__ __forceinline__ float join_weight(float top, float now) { return top == now || top == kMinusInf ? 1.0f : exp2_fast(top - now); }
template <int D, class Sums, class Ends>
__device__ __forceinline__ void join_partials(int from, int to, int lane, Sums sums, Ends ends, float *top, float *sum, float (&acc)[D / 64]) {
    constexpr int kDims = D / 64, kAtOnce = 4;
    *top = kMinusInf, *sum = 0;
#pragma unroll
    for (int d = 0; d < kDims; ++d) acc[d] = 0;
    for (int i = from; i < to; i += kAtOnce) {
        float x[kAtOnce][kDims], its_top[kAtOnce], its_sum[kAtOnce];
        float now = *top;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int at = i + u < to ? i + u : to - 1;
            const float *o = sums(at), *e = ends(at);
            its_top[u] = e[0], its_sum[u] = e[1];
#pragma unroll
            for (int d = 0; d < kDims; ++d) x[u][d] = o[d * 64 + lane];
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) now = fmaxf(now, its_top[u]);
        const float mine = join_weight(*top, now);
        *sum *= mine;
#pragma unroll
        for (int d = 0; d < kDims; ++d) acc[d] *= mine;
        *top = now;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const float w = join_weight(its_top[u], now);
            *sum += i + u < to ? its_sum[u] * w : 0.0f;
#pragma unroll
            for (int d = 0; d < kDims; ++d) acc[d] += i + u < to ? x[u][d] * w : 0.0f;
        }
    }
}

// Rows of sequences of which no row sees a key: zeros, by one wave for a KV head.
__device__ __forceinline__ void rows_without_keys(const AttendArgs &a, int h, int lane) {
    for (int b = 0; b < a.c.num_seqs; ++b) {
        const Seq s = seq_of(a.c, b);
        if (s.rows <= 0 || s.first + s.rows > 0) continue;     // the last row's place is not below zero: it sees its own key
        for (int i = 0; i < s.rows * a.group; ++i) {
            const int token = i / a.group, qh = h * a.group + i - token * a.group;
            for (int d = lane; d < a.c.head_dim; d += 64)
                reinterpret_cast<uint16_t *>(a.out + (s.row0 + token) * a.out_stride)[int64_t(qh) * a.c.head_dim + d] = 0;
            if (a.lse != nullptr && lane == 0) a.lse[int64_t(s.row0 + token) * a.q_heads + qh] = kMinusInf;
        }
    }
}

__device__ __forceinline__ bool is_finite(float v) { return v - v == 0; }

// fp16 probabilities meet e4m3 values with these' scales, in units of a power of two that follows the largest scale so far:
// products with probabilities (up to 2^8) stay below 2^15, and far smaller scales keep their precision.  Of a wave; out^T is
// kept in that unit.
struct ValueUnit {
    float unit = 0x1p-120f, inverse = 0x1p120f;
    // `scale`: of the lane's key (0 for none).  What out^T has to be multiplied by.  A scale that is infinite or NaN becomes 0
    // (a hidden key's probability, 0, times it would be NaN) and sets `odd`: such keys' values are added on their own.
    __device__ __forceinline__ float take(float &scale, bool &odd) {
        const float size = fabsf(scale);
        odd = false;
        if (!wave_any(!(size * 0x1p-7f <= unit))) return 1.0f;
        const bool finite = is_finite(scale);
        odd = wave_any(!finite);
        if (!finite) scale = 0;
        float most = fabsf(scale);
        for (int by = 1; by < 64; by *= 2) most = fmaxf(most, lane_xor(most, by));
        if (most * 0x1p-7f <= unit) return 1.0f;
        const float before = unit;
        unit = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, most) & 0x7f800000u)) * 0x1p-6f;
        inverse = 1.0f / unit;
        return before * inverse;
    }
};

// What a code of an odd value is multiplied by to give an infinity or NaN, or to stay what it is.
__device__ __forceinline__ float odd_scale_at(const AttendArgs &a, int page, int h) {
    const float s = a.c.v_scale[page * a.c.scale_stride + h];
    return is_finite(s) ? 1.0f : s;
}

// Ones where an element of the word, two of 16 bits or four codes, is infinite or NaN.
template <bool BF16, bool E4M3>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    if constexpr (E4M3) {
        const uint32_t m = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;      // codes 0x7f and 0xff
        return (m >> 7) * 0xffu;
    } else {
        constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u;
        return ((w & kExp) == kExp ? 0xffffu : 0u) | (((w >> 16) & kExp) == kExp ? 0xffff0000u : 0u);
    }
}

// Whether any of some words has such an element.
template <bool BF16, bool E4M3>
struct NotFinite {
    uint32_t most = 0;                       // of the elements' sizes, in each half; in e4m3 a byte's top bit for each
    __device__ __forceinline__ void look(uint32_t w) {
        if constexpr (E4M3) most |= (w & 0x7f7f7f7fu) + 0x01010101u;
        else most = larger_halves(most, w & 0x7fff7fffu);
    }
    __device__ __forceinline__ bool found() const {
        constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u;
        return E4M3 ? (most & 0x80808080u) != 0 : (most & 0xffffu) >= kExp || (most >> 16) >= kExp;
    }
};

// The lowest n + 1 bits: none below 0, all from 31 on.
__device__ __forceinline__ uint32_t low_bits(int n) { return n < 0 ? 0u : n >= 31 ? ~0u : (2u << n) - 1u; }
// v where bit n of `bits` is set, else w.
__device__ __forceinline__ float where_bit(uint32_t bits, int n, float v, float w) {
    const uint32_t m = static_cast<uint32_t>(static_cast<int32_t>(bits << (31 - n)) >> 31);
    return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, v) & m) | (__builtin_bit_cast(uint32_t, w) & ~m));
}

// Element i of a row of the cache, as coded.
template <bool BF16, bool E4M3>
__device__ __forceinline__ float element(const uint8_t *p, int i) {
    if constexpr (E4M3) return e4m3_f32<false>(p[i]).x;
    const uint32_t u = reinterpret_cast<const uint16_t *>(p)[i];
    return BF16 ? bf16_lo(u) : f16_lo(u);
}

}  // namespace kvio
