// kvio_attend_steps.hip -- attention of a few new tokens to a sequence (decoding
// steps, drafted tokens): up to 64 rows of query heads and tokens to a KV head.
//
// Such calls read every cached key and value once and compute little: they are
// bound by HBM.  A wave streams 32 keys at a time of one KV head from global
// memory into registers, with no LDS but for the keys' slots and scales, and
// holds the rows as columns of both products:
//   scores^T (keys x rows) = K Q^T,  out^T (dims x rows) += V^T probabilities^T.
// The order of a sum's elements is free, so both operands of a product take
// whatever order their loads give: keys' dims go to lanes in pieces of 16
// contiguous bytes, and the scores that a lane gets are the probabilities that it
// has to bring to the second product.  V has to be brought key by key for each
// dim; a lane loads D / 16 dims of 8 keys and turns them with byte permutes,
// before codes are widened to 16 bits.
//
// Work is split over all contexts' tiles of 32 keys, laid end to end, in equal
// ranges, one to a wave, so that ragged batches load the GPU evenly.  A context that lies
// in several ranges leaves partial results (maximum, sum, out) that a second
// kernel joins in order.
#include "kvio_attend.h"

#include <algorithm>

namespace kvio {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
// Rows times query heads up to which each is joined by 16 waves: few have many partial results each.  One context of 131072
// tokens, 32 heads: 61 us, with one wave 108; 160 rows of 64 heads (5 drafts of 32 contexts): one wave 104 us, 16 174.
constexpr int kFewRows = 512;

// A wave's slots and scales of two tiles, and its rows of Q.
template <int D, int NT>
struct alignas(16) WaveLds {
    int32_t slot[2][kTile];
    float k_scale[2][kTile], v_scale[2][kTile];
    uint8_t q[16 * NT][2 * D + 16];          // 16 more, so that 16 rows' pieces lie in all banks
};

// Waves to a SIMD for which the registers last without scratch, found by compiling for more.
constexpr int occupancy(bool e4m3, int dim, int columns) {
    return dim * columns <= 64 ? 4 : dim * columns <= 128 ? 3 : dim * columns <= 256 && (dim == 64 ? columns < 4 : e4m3 || dim == 128) ? 2 : 1;
}

template <bool BF16, bool E4M3, int D, int NT>
struct Steps {
    static constexpr int kDims = D / 16;                 // dims of V to a lane
    static constexpr int kElem = E4M3 ? 1 : 2;
    static constexpr int kSteps = D / 32;                // products along a head
    static constexpr int kKWords = D * kElem / 16;       // words of K to a lane and 16 keys
    static constexpr int kVWords = kDims * kElem / 4;    // words of V to a lane and key
    // Probabilities take the cache's type; beside e4m3 values, whose scales they carry, fp16 (in bf16 their roundings were
    // the larger part of the result's error) in a ValueUnit.
    static constexpr bool kPBf16 = BF16 && !E4M3;
    // A result shows that rounding too, unless it is in bf16 and the probabilities are not: what it takes off is a second
    // probability.  Such calls wait for memory: 0 to 2% of the time (16 contexts of 16000 tokens, seven query heads to a KV
    // head: 127 us without and with it; 64 rows of heads of 64 dims: 43 -> 46 us) take the error against 64 bits from 0.0021
    // to 0.0017 of the result's norm in bf16 and from 0.00028 to 0.00021 in fp16, what rounding the result makes.
    static constexpr bool kTwice = !(E4M3 && BF16);

    struct Tile {
        uint32_t k[2][kKWords];
        uint32_t v[8][kVWords];
    };

    static __device__ __forceinline__ void load_k(const AttendArgs &a, const int32_t *slots, int h, int lane, Tile *t) {
        const int64_t seg = int64_t(D) * kElem, row = seg * a.c.heads;
        for (int i = 0; i < 2; ++i) {
            const int slot = slots[16 * i + lane % 16];
            const uint8_t *p = a.c.k_cache + (slot < 0 ? 0 : slot) * row + h * seg + lane / 16 * 16;
            for (int w = 0; w < kKWords / 4; ++w) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(p + 64 * w);
                for (int e = 0; e < 4; ++e) t->k[i][4 * w + e] = x[e];
            }
        }
    }
    static __device__ __forceinline__ void load_v(const AttendArgs &a, const int32_t *slots, int h, int lane, Tile *t) {
        const int64_t seg = int64_t(D) * kElem, row = seg * a.c.heads;
        for (int i = 0; i < 8; ++i) {
            const int slot = slots[16 * (i / 4) + lane / 16 * 4 + i % 4];
            const uint8_t *p = a.c.v_cache + (slot < 0 ? 0 : slot) * row + h * seg + lane % 16 * (kDims * kElem);
            if constexpr (kVWords == 1) t->v[i][0] = *reinterpret_cast<const uint32_t *>(p);
            else if constexpr (kVWords == 2) {
                const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
                t->v[i][0] = x.x, t->v[i][1] = x.y;
            } else {
                for (int w = 0; w < kVWords / 4; ++w) {
                    const u32x4 x = *reinterpret_cast<const u32x4 *>(p + 16 * w);
                    for (int e = 0; e < 4; ++e) t->v[i][4 * w + e] = x[e];
                }
            }
        }
    }

    // K of 16 keys for step s, as the first operand.
    static __device__ __forceinline__ u32x4 k_operand(const uint32_t *k, int s) {
        if constexpr (E4M3)
            return u32x4{e4m3_16<BF16, false>(k[2 * s]), e4m3_16<BF16, true>(k[2 * s]), e4m3_16<BF16, false>(k[2 * s + 1]), e4m3_16<BF16, true>(k[2 * s + 1])};
        else return u32x4{k[4 * s], k[4 * s + 1], k[4 * s + 2], k[4 * s + 3]};
    }
    // Bytes into a row of Q of what goes with it: the lane's piece of 8 dims.
    static __device__ __forceinline__ int q_offset(int s, int g) {
        return E4M3 ? 2 * (64 * (s / 2) + 16 * g + 8 * (s % 2)) : 2 * (32 * s + 8 * g);
    }
    // V^T of dims dt = 4 w + 0 .. 3 (e4m3) or 2 w + 0 .. 1 of each lane's share, as first operands.
    static __device__ __forceinline__ void v_operands(const Tile &t, int w, u32x4 *out) {
        for (int p = 0; p < 4; ++p) {
            const uint32_t x = t.v[2 * p][w], y = t.v[2 * p + 1][w];
            if constexpr (E4M3) {
                const uint32_t a = bytes_of(y, x, 0x05010400), b = bytes_of(y, x, 0x07030602);
                out[0][p] = e4m3_16<false, false>(a);
                out[1][p] = e4m3_16<false, true>(a);
                out[2][p] = e4m3_16<false, false>(b);
                out[3][p] = e4m3_16<false, true>(b);
            } else {
                out[0][p] = bytes_of(y, x, 0x05040100);
                out[1][p] = bytes_of(y, x, 0x07060302);
            }
        }
    }
};

// One range of tiles of one KV head to a wave.
template <bool BF16, bool E4M3, int D, int NT>
__global__ void __launch_bounds__(kThreads, occupancy(E4M3, D, NT)) attend_steps(const AttendArgs a) {
    using S = Steps<BF16, E4M3, D, NT>;
    __shared__ WaveLds<D, NT> lds[kWaves];
    const CacheArgs &c = a.c;
    const int lane = static_cast<int>(threadIdx.x) & 63, wave = wave_first(static_cast<int>(threadIdx.x) >> 6);
    const int g = lane / 16, m = lane % 16;
    WaveLds<D, NT> &keys = lds[wave];
    // The heads of a workgroup are neighbours, so that it reads tokens' rows in long pieces.
    const int head_groups = c.heads / a.heads_per_group, splits = kWaves / a.heads_per_group;
    const int blk = static_cast<int>(blockIdx.x) / head_groups;
    const int h = (static_cast<int>(blockIdx.x) - blk * head_groups) * a.heads_per_group + wave % a.heads_per_group;
    const int worker = blk * splits + wave / a.heads_per_group;

    const Ranges r = ranges_of(a, lane);
    if (worker == 0) rows_without_keys(a, h, lane);
    const int64_t begin = int64_t(worker) * r.per_worker;
    const int64_t end = begin + r.per_worker < r.total ? begin + r.per_worker : r.total;
    if (begin >= end) return;
    int64_t at = begin;
    int64_t seq_begin;                                   // where sequence b's tiles begin
    int b = find_tile(a, at, lane, &seq_begin);
    for (; at < end; ++b) {
        const Seq s = seq_of(c, b);
        const Span span = span_of(a, s);
        const int64_t seq_end = seq_begin + span.tiles;
        if (span.tiles == 0) continue;
        const int64_t stop = seq_end < end ? seq_end : end;
        const int first = static_cast<int>(at - seq_begin), n = static_cast<int>(stop - at);
        const int base0 = (span.lo / kTile + first) * kTile;     // context place of the first key
        const int rows = s.rows * a.group;

        int place[NT];                                   // of the lane's column; below any key for none
        for (int t = 0; t < NT; ++t) {
            const int row = 16 * t + m, token = static_cast<int>(div_by(static_cast<uint32_t>(row), a.group_div));
            place[t] = row < rows ? s.first + token : -1;
            const uint8_t *p = a.q + (s.row0 + token) * a.q_stride + int64_t(h * a.group + row - token * a.group) * (2 * D);
            for (int i = g; i < D / 8; i += 4)
                *reinterpret_cast<u32x4 *>(keys.q[row] + 16 * i) = row < rows ? *reinterpret_cast<const u32x4 *>(p + 16 * i) : u32x4{0, 0, 0, 0};
        }
        // A SIMD's only wave has the registers to keep Q's operands, and nobody to work while it waits for LDS: 8 drafts of 4
        // heads 43.6 us, with Q read from LDS each time 44.5; 4 of 4 with 256 dims 47.4 and 49.9; but 5 of 8 over e4m3 104 and 102.
        constexpr bool kKeepQ = occupancy(E4M3, D, NT) == 1;
        u32x4 q[kKeepQ ? NT : 1][kKeepQ ? S::kSteps : 1];
        auto q_operand = [&](int t, int s2) __attribute__((always_inline)) {
            return *reinterpret_cast<const u32x4 *>(keys.q[16 * t + m] + S::q_offset(s2, g));
        };
        if constexpr (kKeepQ) {
            wave_lds_fence();
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int s2 = 0; s2 < S::kSteps; ++s2) q[t][s2] = q_operand(t, s2);
        }
        f32x4 acc[NT][S::kDims];
        float top[NT], sum[NT];
        for (int t = 0; t < NT; ++t) {
            for (int d = 0; d < S::kDims; ++d) acc[t][d] = f32x4{0, 0, 0, 0};
            top[t] = kMinusInf;
            sum[t] = 0;
        }

        // The page of the lane's key (lanes 32 and up: of the same keys) in a tile; -2 for a key that no row sees.
        auto page_in = [&](int tile) {
            const int key = base0 + tile * kTile + (lane & 31);
            if (tile >= n || key < span.lo || key >= span.hi) return -2;
            return c.page_table[b * c.table_stride + static_cast<int>(div_by(static_cast<uint32_t>(key), c.page_div))];
        };
        float k_scale = 1, v_scale = 1;
        ValueUnit unit;
        auto put_slot = [&](int tile, int page) {        // and ask for the scales
            const int key = base0 + tile * kTile + (lane & 31);
            const bool there = page >= 0 && page < c.num_pages;
            const int j = static_cast<int>(div_by(static_cast<uint32_t>(key), c.page_div));
            if (page != -2 && !there) record_bad_page(c, b, j);
            if (lane < 32) keys.slot[tile & 1][lane] = there ? page * c.page_size + (key - j * c.page_size) : -1;
            if (E4M3) {
                k_scale = there ? c.k_scale[page * c.scale_stride + h] * a.scale_log2 : 0.0f;
                v_scale = there ? c.v_scale[page * c.scale_stride + h] : 0.0f;
            }
        };
        bool odd_scale = false;                          // in the tile whose scales were put last
        auto take_unit = [&]() {
            if constexpr (E4M3) {
                const float less = unit.take(v_scale, odd_scale);
                if (less != 1.0f)
                    for (int t = 0; t < NT; ++t)
                        for (int d = 0; d < S::kDims; ++d) acc[t][d] *= less;
            }
        };
        auto put_scales = [&](int tile) {
            take_unit();                                 // before the tile is worked on
            if (E4M3 && lane < 32) {
                keys.k_scale[tile & 1][lane] = k_scale;
                keys.v_scale[tile & 1][lane] = v_scale;
            }
        };
        // One tile; the registers of its keys and values take the next one's as soon as they are free.
        typename S::Tile x;
        auto work = [&](int tile) {
            const int base = base0 + tile * kTile;
            const int32_t *slot = keys.slot[tile & 1], *next_slot = keys.slot[(tile + 1) & 1];
            f32x4 score[2][NT];
            for (int i = 0; i < 2; ++i)
                for (int t = 0; t < NT; ++t) score[i][t] = f32x4{0, 0, 0, 0};
            for (int s2 = 0; s2 < S::kSteps; ++s2)
                for (int i = 0; i < 2; ++i) {
                    const u32x4 k = S::k_operand(x.k[i], s2);
                    for (int t = 0; t < NT; ++t)
                        score[i][t] = product16<BF16>(k, kKeepQ ? q[kKeepQ ? t : 0][kKeepQ ? s2 : 0] : q_operand(t, s2), score[i][t]);
                }
            S::load_k(a, next_slot, h, lane, &x);        // also behind the last tile, of slot 0: loads on some paths only would be waited for on all
            float vs[8];
            for (int i = 0; i < 2; ++i) {
                if (E4M3) {
                    const f32x4 ks = *reinterpret_cast<const f32x4 *>(keys.k_scale[tile & 1] + 16 * i + 4 * g);
                    const f32x4 v = *reinterpret_cast<const f32x4 *>(keys.v_scale[tile & 1] + 16 * i + 4 * g);
                    for (int t = 0; t < NT; ++t) score[i][t] *= ks;
                    for (int e = 0; e < 4; ++e) vs[4 * i + e] = E4M3 ? v[e] * unit.inverse : v[e];
                } else {
                    for (int t = 0; t < NT; ++t) score[i][t] *= a.scale_log2;
                }
            }
            // Keys that some row does not see, or that are not there, are masked; their values may hold anything.
            const bool whole = base >= span.whole_lo && base + kTile <= span.whole_hi;
            bool odd = odd_scale;                        // a value that is not finite where it matters
            if (!whole || wave_any(slot[lane & 31] < 0)) {
                for (int i = 0; i < 2; ++i)
                    for (int e = 0; e < 4; ++e) {
                        const int at_key = 16 * i + 4 * g + e, key = base + at_key;
                        const bool there = slot[at_key] >= 0;
                        for (int t = 0; t < NT; ++t) {
                            const bool seen = there && key <= place[t] && (a.window == 0 || key > place[t] - a.window);
                            if (!seen) score[i][t][e] = kMinusInf;
                        }
                        for (int w = 0; w < S::kVWords; ++w) {
                            uint32_t &v = x.v[4 * i + e][w];
                            if (!there) v = 0;
                            const uint32_t bad = not_finite<BF16, E4M3>(v);
                            odd = odd || bad != 0;
                            v &= ~bad;
                        }
                    }
                odd = wave_any(odd);
            }
            uint32_t p[NT][4], rest[S::kTwice ? NT : 1][4];
            for (int t = 0; t < NT; ++t) {
                float best = score[0][t][0];
                for (int i = 0; i < 2; ++i)
                    for (int e = 0; e < 4; ++e) best = fmaxf(best, score[i][t][e]);
                // The maximum only moves when it is passed by far: probabilities up to 2^8 do no harm.
                if (wave_any(best > top[t] + kSlack)) {
                    best = fmaxf(best, lane_xor(best, 16));
                    best = fmaxf(best, lane_xor(best, 32));
                    const float now = fmaxf(top[t], best);
                    const float less = now == kMinusInf ? 1.0f : exp2_fast(top[t] - now);
                    top[t] = now;
                    sum[t] *= less;
                    for (int d = 0; d < S::kDims; ++d) acc[t][d] *= less;
                }
                const float from = top[t] == kMinusInf ? 0.0f : top[t] - kRaised<BF16, E4M3>;
                float e8[8];
                for (int e = 0; e < 8; ++e) {
                    e8[e] = exp2_fast(score[e / 4][t][e % 4] - from);
                    sum[t] += e8[e];
                    if (E4M3) e8[e] *= vs[e];
                }
                for (int e = 0; e < 4; ++e) {
                    p[t][e] = S::kPBf16 ? pack_bf16(e8[2 * e], e8[2 * e + 1]) : pack_f16(e8[2 * e], e8[2 * e + 1]);
                    // This value, and no other: rounded once more from a fused product, it differs near ties, and the rest with it.
                    if constexpr (S::kTwice) keep_here(p[t][e]);
                }
                if constexpr (S::kTwice)
                    for (int e = 0; e < 4; ++e)
                        rest[t][e] = S::kPBf16 ? pack_bf16(e8[2 * e] - bf16_lo(p[t][e]), e8[2 * e + 1] - bf16_hi(p[t][e]))
                                               : pack_f16(e8[2 * e] - f16_lo(p[t][e]), e8[2 * e + 1] - f16_hi(p[t][e]));
            }
            constexpr int kAtOnce = E4M3 ? 4 : 2;        // dims from one word
            for (int w = 0; w < S::kVWords; ++w) {
                u32x4 v[kAtOnce];
                S::v_operands(x, w, v);
                for (int e = 0; e < kAtOnce; ++e)
                    for (int t = 0; t < NT; ++t) {
                        f32x4 &x4 = acc[t][kAtOnce * w + e];
                        x4 = product16<S::kPBf16>(v[e], u32x4{p[t][0], p[t][1], p[t][2], p[t][3]}, x4);
                        if constexpr (S::kTwice) x4 = product16<S::kPBf16>(v[e], u32x4{rest[t][0], rest[t][1], rest[t][2], rest[t][3]}, x4);
                    }
            }
            if (odd) {                                   // rare: such values reach the rows that see them, and no others
                const int64_t seg = int64_t(D) * S::kElem;
                for (int at_key = 0; at_key < kTile; ++at_key) {
                    const int one = slot[at_key], key = base + at_key;
                    if (one < 0) continue;
                    const uint8_t *v = c.v_cache + one * (seg * c.heads) + h * seg;
                    const float by = E4M3 ? odd_scale_at(a, static_cast<int>(div_by(static_cast<uint32_t>(one), c.page_div)), h) : 1.0f;
                    for (int e = 0; e < 4; ++e)
                        for (int d = 0; d < S::kDims; ++d) {
                            const float f = element<BF16, E4M3>(v, (4 * g + e) * S::kDims + d) * by;
                            in_order();                  // one at a time: registers matter here, time does not
                            if (!wave_any(f - f != 0)) continue;
                            for (int t = 0; t < NT; ++t)
                                acc[t][d][e] += f - f != 0 && key <= place[t] && (a.window == 0 || key > place[t] - a.window) ? f : 0.0f;
                        }
                }
            }
            S::load_v(a, next_slot, h, lane, &x);
        };

        // A tile's pages are asked for two tiles ahead, and before the loads of the next tile, so that
        // waiting for them does not wait for those.
        put_slot(0, page_in(0));
        put_scales(0);
        wave_lds_fence();
        S::load_k(a, keys.slot[0], h, lane, &x);
        S::load_v(a, keys.slot[0], h, lane, &x);
        put_slot(1, page_in(1));
        wave_lds_fence();
        for (int i = 0; i < n; ++i) {
            const int page = page_in(i + 2);
            work(i);
            wave_lds_fence();
            put_scales(i + 1);
            put_slot(i + 2, page);
            wave_lds_fence();
        }

        const bool alone = at == seq_begin && stop == seq_end;
        int g4 = 4 * g, row0 = m;                        // addresses are computed here, not before the tiles, where registers are short
        keep_here(g4);
        keep_here(row0);
        for (int t = 0; t < NT; ++t) {
            sum[t] += lane_xor(sum[t], 16);
            sum[t] += lane_xor(sum[t], 32);
            const int row = 16 * t + row0;
            if (row >= rows) continue;
            if (alone) {
                const int token = static_cast<int>(div_by(static_cast<uint32_t>(row), a.group_div));
                const int qh = h * a.group + row - token * a.group;
                const float inv = sum[t] == 0 ? 0.0f : (E4M3 ? unit.unit : 1.0f) / sum[t];
                uint8_t *o = a.out + (s.row0 + token) * a.out_stride + int64_t(qh) * (2 * D);
                for (int e = 0; e < 4; ++e)
                    for (int d = 0; d < S::kDims; d += 2) {
                        const float x = acc[t][d][e] * inv, y = acc[t][d + 1][e] * inv;
                        *reinterpret_cast<uint32_t *>(o + 2 * ((g4 + e) * S::kDims + d)) = BF16 ? pack_bf16(x, y) : pack_f16(x, y);
                    }
                if (a.lse != nullptr && g == 0) a.lse[int64_t(s.row0 + token) * a.q_heads + qh] = lse_of(top[t] - kRaised<BF16, E4M3>, sum[t]);
            } else {
                // Which of the two contexts that a range can share with others: the one that began before it, or the one that goes on.
                float *o = a.partials + partial_at(a, worker, h, at != seq_begin ? 0 : 1, row, D);
                for (int e = 0; e < 4; ++e)
                    for (int d = 0; d < S::kDims; ++d) o[(g4 + e) * S::kDims + d] = E4M3 ? acc[t][d][e] * unit.unit : acc[t][d][e];
                if (g == 0) o[D] = top[t] - kRaised<BF16, E4M3>, o[D + 1] = sum[t];
            }
        }
        at = stop;
        seq_begin = seq_end;
        wave_lds_fence();
    }
}

// Join the partial results of a row and query head: a wave's work, or, where few rows have many partial results each,
// a workgroup's, each wave a run of them, then the first the waves'.
template <bool BF16, int D, int WAVES>
__global__ void __launch_bounds__(WAVES > 1 ? 64 * WAVES : kThreads) join_steps(const AttendArgs a) {
    constexpr int kDims = D / 64;
    __shared__ float shared[WAVES][D + 2];
    const CacheArgs &c = a.c;
    const int lane = static_cast<int>(threadIdx.x) & 63, wave = wave_first(static_cast<int>(threadIdx.x) >> 6);
    const int at = WAVES > 1 ? static_cast<int>(blockIdx.x) : static_cast<int>(blockIdx.x) * kWaves + wave;
    const int row = at / a.q_heads, qh = at - row * a.q_heads;
    if (row >= c.num_tokens) return;
    const int b = seq_with_row(c, row, lane);
    if (b < 0) return;
    const Seq s = seq_of(c, b);
    if (row < s.row0 || row >= s.row0 + s.rows) return;
    int64_t begin;
    const Ranges r = ranges_of(a, lane, b, &begin);
    const int tiles = span_of(a, s).tiles;
    if (tiles == 0) return;
    const int w0 = static_cast<int>(begin / r.per_worker), w1 = static_cast<int>((begin + tiles - 1) / r.per_worker);
    if (w0 == w1) return;
    const int h = qh / a.group, at_row = (row - s.row0) * a.group + qh - h * a.group;
    const int n = w1 - w0 + 1, share = (n + WAVES - 1) / WAVES;
    float top, sum, acc[kDims];
    auto sums = [&](int i) { return a.partials + partial_at(a, w0 + i, h, i == 0 ? 1 : 0, at_row, D); };
    const int from = WAVES > 1 ? wave * share : 0;
    join_partials<D>(from, from + share < n ? from + share : n, lane, sums, [&](int i) { return sums(i) + D; }, &top, &sum, acc);
    if constexpr (WAVES > 1) {
        if (lane == 0) shared[wave][D] = top, shared[wave][D + 1] = sum;
#pragma unroll
        for (int d = 0; d < kDims; ++d) shared[wave][d * 64 + lane] = acc[d];
        workgroup_barrier();
        if (wave != 0) return;
        join_partials<D>(0, (n + share - 1) / share, lane, [&](int i) { return shared[i]; }, [&](int i) { return shared[i] + D; }, &top, &sum, acc);
    }
    const float inv = sum == 0 ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int d = 0; d < kDims; ++d)
        reinterpret_cast<uint16_t *>(a.out + row * a.out_stride + int64_t(qh) * (2 * D))[d * 64 + lane] =
            static_cast<uint16_t>(BF16 ? pack_bf16(acc[d] * inv, 0) : pack_f16(acc[d] * inv, 0));
    if (a.lse != nullptr && lane == 0) a.lse[int64_t(row) * a.q_heads + qh] = lse_of(top, sum);
}

template <bool BF16, bool E4M3, int D>
hipError_t launch(const AttendArgs &a, const AttendPlan &plan, hipStream_t stream) {
    if (plan.columns == 1) hipLaunchKernelGGL((attend_steps<BF16, E4M3, D, 1>), dim3(plan.groups), dim3(kThreads), 0, stream, a);
    else if (plan.columns == 2) hipLaunchKernelGGL((attend_steps<BF16, E4M3, D, 2>), dim3(plan.groups), dim3(kThreads), 0, stream, a);
    else if constexpr (D <= 128) {
        if (plan.columns == 3) hipLaunchKernelGGL((attend_steps<BF16, E4M3, D, 3>), dim3(plan.groups), dim3(kThreads), 0, stream, a);
        else hipLaunchKernelGGL((attend_steps<BF16, E4M3, D, 4>), dim3(plan.groups), dim3(kThreads), 0, stream, a);
    }
    const int64_t rows = int64_t(a.c.num_tokens) * a.q_heads;
    if (plan.joined && rows <= kFewRows)
        hipLaunchKernelGGL((join_steps<BF16, D, 16>), dim3(static_cast<unsigned>(rows)), dim3(1024), 0, stream, a);
    else if (plan.joined)
        hipLaunchKernelGGL((join_steps<BF16, D, 1>), dim3(static_cast<unsigned>((rows + kWaves - 1) / kWaves)), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

template <bool BF16, bool E4M3>
hipError_t launch_dim(const AttendArgs &a, const AttendPlan &plan, hipStream_t stream) {
    if (a.c.head_dim == 64) return launch<BF16, E4M3, 64>(a, plan, stream);
    if (a.c.head_dim == 128) return launch<BF16, E4M3, 128>(a, plan, stream);
    return launch<BF16, E4M3, 256>(a, plan, stream);
}

}  // namespace

hipError_t launch_steps(const AttendArgs &a, const AttendPlan &plan, int32_t dtype, bool e4m3, hipStream_t stream) {
    if (dtype == KVIO_BF16) return e4m3 ? launch_dim<true, true>(a, plan, stream) : launch_dim<true, false>(a, plan, stream);
    return e4m3 ? launch_dim<false, true>(a, plan, stream) : launch_dim<false, false>(a, plan, stream);
}

AttendPlan plan_steps(bool e4m3, int32_t heads, int32_t q_heads, int32_t dim, const kvio_batch &b, int32_t max_query, int32_t max_ctx) {
    AttendPlan p = {};
    const int64_t rows = int64_t(max_query) * (q_heads / heads);
    p.few = true;
    p.columns = static_cast<int32_t>((rows + 15) / 16);
    p.heads_per_group = heads % 4 == 0 ? 4 : heads % 2 == 0 ? 2 : 1;
    const int64_t head_groups = heads / p.heads_per_group, splits = kWaves / p.heads_per_group;
    // As many workgroups as the GPU holds at once: 256 compute units, a wave on each SIMD for each of them.
    const int64_t most = std::max<int64_t>(256 * occupancy(e4m3, dim, p.columns) / head_groups, 1);
    // With 2 or 8 tiles at least: 4 contexts of 2000 tokens of 32 heads 19.1 and 24.2 us (21.2 with 4), 8 drafts of 8 contexts of
    // 3000 46.2 and 39.0 (43.4), 256 contexts of 200 44.7 and 50.9 (44.9).
    p.min_tiles = 4;
    const int64_t tiles = int64_t(b.num_seqs) * ((max_ctx + 2 * kTile - 1) / kTile);      // at most
    const int64_t workers = std::min(most * splits, (tiles + p.min_tiles - 1) / p.min_tiles);
    const int64_t blocks = (workers + splits - 1) / splits;
    p.workers = static_cast<int32_t>(blocks * splits);
    p.groups = static_cast<uint32_t>(blocks * head_groups);
    p.joined = tiles > p.min_tiles;
    p.slot_rows = static_cast<int32_t>(std::min<int64_t>(rows, 16 * p.columns));
    if (p.joined) p.bytes = uint64_t(p.workers) * uint64_t(heads) * 2 * uint64_t(p.slot_rows) * uint64_t(dim + 2) * 4;
    return p;
}

}  // namespace kvio
