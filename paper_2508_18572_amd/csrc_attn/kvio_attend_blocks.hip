// kvio_attend_blocks.hip -- attention of many new tokens to a sequence (prompts
// and the rest of partly cached ones), on the matrix units.
//
// A workgroup takes a block of 256 rows (128 with heads of 256 dims), query heads
// and tokens of one KV head, 64 (32) to a wave, and goes through its keys a tile at a time.  Rows are columns of
// both products,
//   scores^T (keys x rows) = K Q^T,  out^T (dims x rows) += V^T probabilities^T,
// so that the scores that a lane gets are the probabilities that it has to bring
// to the second product, and a row's maximum and sum concern two lanes.  Q and
// out^T stay in registers; K and V come from the pages through registers, where
// codes are widened to 16 bits, into LDS buffers shared by the four waves, a tile ahead.  V^T is read with the LDS' transposing loads.
//
// 4 D flops to a score against some six vector operations: both units have to be
// kept busy at once.  A wave's 512 registers hold the scores of two tiles, so
// that the products of the next tile's run beside the exponentials of this one's.
//
// Work is split over all blocks' keys, laid end to end, in equal ranges, one to a
// workgroup: ragged batches and causal triangles load the GPU evenly.  A block
// that lies in several ranges leaves partial results that a second kernel joins
// in order.
#include "kvio_attend.h"

#include <algorithm>
#include <type_traits>

// Registers that lambdas work on stay registers only where the calls are gone early.
#define KVIO_INLINE __attribute__((always_inline))

namespace kvio {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kJoinRows = 16;                            // rows that a workgroup joins

// The blocks of one sequence and the keys that each goes through.
struct Blocks {
    int32_t count, first, rows, tokens, window;          // `tokens` to a block
    __device__ __forceinline__ int end(int j) const {    // one past the last key that the block sees; maybe none are
        const int t = j + 1 < count ? (j + 1) * tokens : rows;
        return first + t;
    }
    // Blocks that see nothing go through one hidden key, and give zeros.
    __device__ __forceinline__ int hi(int j) const { return end(j) > 1 ? end(j) : 1; }
    __device__ __forceinline__ int lo(int j) const {
        const int64_t w = int64_t(first) + int64_t(j) * tokens - window + 1;
        return window > 0 && w > 0 ? static_cast<int>(w) : 0;
    }
    // Keys of all blocks before j, j < count: sums over i < j of hi(i) = max(1, first + (i + 1) tokens) and lo(i).
    __device__ __forceinline__ int64_t before(int j) const {
        const int64_t n = j, z = first < 1 ? std_min(n, (1 - first) / tokens) : 0;
        int64_t sum = z + (n - z) * first + tokens * ((n * (n + 1) - z * (z + 1)) / 2);
        if (window > 0) {
            const int64_t free = int64_t(window) - 1 - first;                  // lo(i) is 0 while i * tokens <= free
            const int64_t y = free < 0 ? 0 : std_min(n, int64_t(static_cast<int>(std_min(free, 0x7fffffff)) / tokens) + 1);
            sum -= (n - y) * (int64_t(first) - window + 1) + tokens * ((n * (n - 1) - y * (y - 1)) / 2);
        }
        return sum;
    }
    __device__ __forceinline__ int64_t keys() const { return count == 0 ? 0 : before(count - 1) + hi(count - 1) - lo(count - 1); }
    static __device__ __forceinline__ int64_t std_min(int64_t a, int64_t b) { return a < b ? a : b; }
};
__device__ __forceinline__ Blocks blocks_of(const AttendArgs &a, const Seq &s) {
    return {s.rows > 0 ? (s.rows - 1) / a.block_tokens + 1 : 0, s.first, s.rows, a.block_tokens, a.window};
}

// All keys, head after head, sequence after sequence, block after block.
struct Line {
    int64_t head, all, per_worker;           // keys of a KV head, of all, of a workgroup
};
__device__ __forceinline__ Line line_of(const AttendArgs &a, int lane) {
    int64_t n = 0;
    for (int i = lane; i < a.c.num_seqs; i += 64) n += blocks_of(a, seq_of(a.c, i)).keys();
    for (int by = 1; by < 64; by *= 2) n += lane_xor(n, by);
    Line l;
    l.head = wave_first(n);
    l.all = l.head * a.c.heads;
    l.per_worker = (l.all + a.workers - 1) / a.workers;
    if (l.per_worker < a.min_keys) l.per_worker = a.min_keys;
    return l;
}

// The block that holds a key of that line, and the key's place in it.
struct Where {
    int32_t h, b, j;
    int64_t begin;                           // where the block begins in the line
};
__device__ __forceinline__ Where where_is(const AttendArgs &a, const Line &l, int64_t at, int lane) {
    Where r;
    r.h = static_cast<int>(at / l.head);
    int64_t before = l.head * r.h;
    for (int i = 0;; i += 64) {
        const int64_t n = i + lane < a.c.num_seqs ? blocks_of(a, seq_of(a.c, i + lane)).keys() : 0;
        const int64_t upto = lanes_upto(n, lane);
        const uint64_t behind = wave_ballot(before + upto > at);
        if (behind != 0) {
            const int k = __builtin_ctzll(behind);
            r.b = i + k;
            before += wave_read(upto, k) - wave_read(n, k);
            break;
        }
        before += wave_read(upto, 63);
    }
    const Blocks blocks = blocks_of(a, seq_of(a.c, r.b));
    r.j = 0;
    for (int n = blocks.count; n > 1;) {     // of n blocks from r.j on, the last that begins no later
        const int step = (n + 63) / 64, j = r.j + lane * step;
        const uint64_t begun = wave_ballot(lane * step < n && before + blocks.before(j) <= at);
        const int k = 63 - __builtin_clzll(begun);
        r.j += k * step;
        n = n - k * step < step ? n - k * step : step;
    }
    r.begin = before + blocks.before(r.j);
    return r;
}

// Floats into the partial results of a workgroup: of each row its sums, behind all rows' the maximum and the sum of
// probabilities.  `which`: the block began before its range (0), or goes on after it (1).
__device__ __forceinline__ int64_t block_partial_at(const AttendArgs &a, int worker, int which, int dim) {
    return (int64_t(worker) * 2 + which) * a.slot_rows * (dim + 2);
}

template <bool BF16, bool E4M3, int D>
struct Shape {
    static constexpr int kElem = E4M3 ? 1 : 2, kSeg = D * kElem;
    static constexpr int kKeys = D <= 128 ? 64 : 32, kHalves = kKeys / 32;   // keys of a tile
    static constexpr int kWaveRows = block_rows(D) / kWaves, kColumns = kWaveRows / 32;   // rows to a wave, 32 to a column of products
    static constexpr int kSteps = D / 16, kDimBlocks = D / 32;
    static constexpr int kPieces = kSeg / 16, kRowsAtOnce = kThreads / kPieces, kPasses = kKeys / kRowsAtOnce;
    // 16 rows' pieces of 16 bytes lie in all banks; so do 32 bytes of 8 rows
    static constexpr int kKRow = 2 * D + 16, kVRow = 2 * D + 64;
    static constexpr bool kPBf16 = BF16 || E4M3;
    static constexpr int kKBuffers = 1 + kHalves;        // the second half's scores are computed after the next tile's K is due
    struct alignas(16) Lds {
        uint8_t k[kKBuffers][kKeys * kKRow], v[2][kKeys * kVRow];
        float k_scale[4][64], v_scale[4][64];            // of tiles, by their number & 3
        int32_t odd[4];                                  // the running number of a tile with values that are not finite
    };
};

template <bool BF16, bool E4M3, int D>
__global__ void __launch_bounds__(kThreads, 1) attend_blocks(const AttendArgs a) {
    using S = Shape<BF16, E4M3, D>;
    constexpr int kKeys = S::kKeys, kColumns = S::kColumns, kWaveRows = S::kWaveRows;
    __shared__ typename S::Lds lds;
    const CacheArgs &c = a.c;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = wave_first(tid >> 6);
    const int g = lane / 32, m = lane % 32;
    // Workgroups go to the 8 dies in turn; each die takes one stretch of the line, so that its cache serves few heads.
    const int worker = static_cast<int>(blockIdx.x % 8) * (a.workers / 8) + static_cast<int>(blockIdx.x / 8);

    const Line line = line_of(a, lane);
    int64_t pos = worker * line.per_worker;
    const int64_t stop = pos + line.per_worker < line.all ? pos + line.per_worker : line.all;
    if (pos >= stop) return;
    if (tid < 4) lds.odd[tid] = -1;
    int serial = 0;                                      // tiles so far
    Where at = where_is(a, line, pos, lane);
    while (pos < stop) {
        const int b = at.b, h = at.h;
        const Seq s = seq_of(c, b);
        const Blocks blocks = blocks_of(a, s);
        if (at.j >= blocks.count) {                      // on to the next sequence, and head
            at.j = 0;
            if (++at.b == c.num_seqs) at.b = 0, ++at.h;
            continue;
        }
        const int lo = blocks.lo(at.j), hi = blocks.hi(at.j), end = blocks.end(at.j);
        const int64_t next = at.begin + (hi - lo);
        const int tile0 = lo / kKeys, all_tiles = (hi + kKeys - 1) / kKeys - tile0;
        // A range's end is moved down to a tile's.
        const int from_tile = pos == at.begin ? 0 : static_cast<int>(lo + (pos - at.begin)) / kKeys - tile0;
        const int to_tile = stop >= next ? all_tiles : static_cast<int>(lo + (stop - at.begin)) / kKeys - tile0;
        const int block_row0 = at.j * a.block_tokens;    // in the sequence
        const int n = to_tile - from_tile;
        at.begin = pos = next;
        ++at.j;
        if (n <= 0) continue;
        const int base0 = (tile0 + from_tile) * kKeys;
        const int rows = (s.rows - block_row0 < a.block_tokens ? s.rows - block_row0 : a.block_tokens) * a.group;
        const int first = s.first + block_row0;          // place of the block's first token
        const int last = end - 1;                        // and of its last
        // Of the wave's rows.
        const int wave_row0 = wave * kWaveRows, wave_row1 = rows - 1 < wave_row0 + kWaveRows - 1 ? rows - 1 : wave_row0 + kWaveRows - 1;
        const bool idle = wave_row0 > wave_row1;
        const int wave_first_place = first + static_cast<int>(div_by(static_cast<uint32_t>(wave_row0), a.group_div));
        const int wave_last_place = first + static_cast<int>(div_by(static_cast<uint32_t>(idle ? 0 : wave_row1), a.group_div));

        int place[kColumns];                             // of the lane's columns; below any key for none
        u32x4 q[kColumns][S::kSteps];
#pragma unroll
        for (int t = 0; t < kColumns; ++t) {
            const int row = wave_row0 + 32 * t + m, token = static_cast<int>(div_by(static_cast<uint32_t>(row), a.group_div));
            place[t] = row < rows ? first + token : -1;
            const uint8_t *p = a.q + (s.row0 + block_row0 + token) * a.q_stride + int64_t(h * a.group + row - token * a.group) * (2 * D) + 16 * g;
#pragma unroll
            for (int i = 0; i < S::kSteps; ++i) q[t][i] = row < rows ? *reinterpret_cast<const u32x4 *>(p + 32 * i) : u32x4{0, 0, 0, 0};
        }
        f32x16 acc[kColumns][S::kDimBlocks];
        float top[kColumns], sum[kColumns];
#pragma unroll
        for (int t = 0; t < kColumns; ++t) {
#pragma unroll
            for (int d = 0; d < S::kDimBlocks; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[t][d][i] = 0;
            top[t] = kMinusInf;
            sum[t] = 0;
        }

        // ---- keys and values on their way into LDS ----------------------------------------
        const int lane_key = lane & (kKeys - 1);         // the key of a tile whose page the lane looks up
        auto page_in = [&](int tile) KVIO_INLINE {                   // -2 for a key that no row sees
            const int key = base0 + tile * kKeys + lane_key;
            if (tile >= n || key < lo || key >= end) return -2;
            return c.page_table[b * c.table_stride + static_cast<int>(div_by(static_cast<uint32_t>(key), c.page_div))];
        };
        float k_scale = 0, v_scale = 0;
        auto slot_from = [&](int tile, int page) KVIO_INLINE {       // -1 for a key that is not there; asks for its scales
            const int key = base0 + tile * kKeys + lane_key;
            const bool there = page >= 0 && page < c.num_pages;
            const int i = static_cast<int>(div_by(static_cast<uint32_t>(key), c.page_div));
            if (page != -2 && !there) record_bad_page(c, b, i);
            if (E4M3) {
                k_scale = there ? c.k_scale[page * c.scale_stride + h] * a.scale_log2 : 0.0f;
                v_scale = there ? c.v_scale[page * c.scale_stride + h] : 0.0f;
            }
            return there ? page * c.page_size + (key - i * c.page_size) : -1;
        };
        auto put_scales = [&](int tile) KVIO_INLINE {
            if (E4M3 && wave == 0) {
                lds.k_scale[tile & 3][lane] = k_scale;
                lds.v_scale[tile & 3][lane] = v_scale;
            }
        };
        const int piece = tid % S::kPieces, piece_row = tid / S::kPieces;
        const int64_t cache_row = int64_t(S::kSeg) * c.heads;
        auto load = [&](u32x4 *x, const uint8_t *cache, int slots) KVIO_INLINE {
            const uint8_t *p = cache + h * S::kSeg + 16 * piece;
#pragma unroll
            for (int i = 0; i < S::kPasses; ++i) {
                const int slot = lane_read(slots, piece_row + i * S::kRowsAtOnce);
                x[i] = *reinterpret_cast<const u32x4 *>(p + (slot < 0 ? 0 : slot) * cache_row);
            }
        };
        auto put = [&](uint8_t *to, int row_bytes, const u32x4 *x, auto of_v) KVIO_INLINE {
#pragma unroll
            for (int i = 0; i < S::kPasses; ++i) {
                uint8_t *p = to + (piece_row + i * S::kRowsAtOnce) * row_bytes + piece * (32 / S::kElem);
                if constexpr (E4M3) {
                    constexpr bool kBf16 = BF16 || decltype(of_v)::value;     // values meet probabilities
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        *reinterpret_cast<u32x4 *>(p + 16 * e) = u32x4{e4m3_16<kBf16, false>(x[i][2 * e]), e4m3_16<kBf16, true>(x[i][2 * e]),
                                                                       e4m3_16<kBf16, false>(x[i][2 * e + 1]), e4m3_16<kBf16, true>(x[i][2 * e + 1])};
                } else {
                    *reinterpret_cast<u32x4 *>(p) = x[i];
                }
            }
        };
        // Whether all rows of the block see all keys of a tile; `there`: the lanes with a slot.
        auto whole_for_all = [&](int tile, uint64_t there) KVIO_INLINE {
            const int base = base0 + tile * kKeys;
            return base + kKeys - 1 <= first && (a.window == 0 || base > last - a.window) && there == ~0ull;
        };
        u32x4 kx[S::kPasses], vx[S::kPasses];
        auto put_k = [&](int buffer) KVIO_INLINE { put(lds.k[buffer], S::kKRow, kx, std::false_type()); };
        // Hidden values may hold anything: those that are not finite become zeros, the tile is marked.
        auto put_v = [&](int tile, uint64_t there) KVIO_INLINE {
            if (!whole_for_all(tile, there)) {
                bool odd = false;
#pragma unroll
                for (int i = 0; i < S::kPasses; ++i) {
                    const bool is_there = (there >> (piece_row + i * S::kRowsAtOnce)) & 1;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t v = is_there ? vx[i][e] : 0;
                        const uint32_t bad = not_finite<BF16, E4M3>(v);
                        odd = odd || bad != 0;
                        vx[i][e] = v & ~bad;
                    }
                }
                if (odd) lds.odd[(serial + tile) & 3] = serial + tile;
            }
            put(lds.v[tile & 1], S::kVRow, vx, std::true_type());
        };

        // ---- products, 32 keys at a time: half i of a tile ---------------------------------
        f32x16 score[kColumns], ahead[kColumns];
        auto scores = [&](int buffer, int i, f32x16 (&x)[kColumns]) KVIO_INLINE {
            const uint8_t *k = lds.k[buffer] + (32 * i + m) * S::kKRow + 16 * g;
            const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < kColumns; ++t) x[t] = zero;
#pragma unroll
            for (int e = 0; e < S::kSteps; ++e) {
                const u32x4 op = *reinterpret_cast<const u32x4 *>(k + 32 * e);
#pragma unroll
                for (int t = 0; t < kColumns; ++t) x[t] = product32<BF16>(op, q[t][e], x[t]);
            }
        };
        // Scores by the keys' scales; hidden keys' at minus infinity.
        auto settle = [&](int tile, int i, uint64_t there, f32x16 (&x)[kColumns]) KVIO_INLINE {
            const int base = base0 + tile * kKeys + 32 * i;
            if constexpr (E4M3) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const f32x4 ks = *reinterpret_cast<const f32x4 *>(lds.k_scale[tile & 3] + 32 * i + 8 * r + 4 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int t = 0; t < kColumns; ++t) x[t][4 * r + e] *= ks[e];
                }
            }
            const bool whole = idle || (base + 31 <= wave_first_place && (a.window == 0 || base > wave_last_place - a.window) && there == ~0ull);
            if (!whole) {
                const uint32_t mine = static_cast<uint32_t>(there >> (32 * i + 4 * g));
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int at_key = 8 * (e / 4) + e % 4, key = base + at_key + 4 * g;
                    const bool is_there = (mine >> at_key) & 1;
#pragma unroll
                    for (int t = 0; t < kColumns; ++t)
                        if (!(is_there && key <= place[t] && (a.window == 0 || key > place[t] - a.window))) x[t][e] = kMinusInf;
                }
            }
        };
        // A new maximum where the old one is passed by far.  Scores are in powers of two once multiplied by `unit`.
        const float unit = E4M3 ? 1.0f : a.scale_log2;
        auto raise = [&](const f32x16 (&x)[kColumns]) KVIO_INLINE {
            float best[kColumns];
            bool any = false;
#pragma unroll
            for (int t = 0; t < kColumns; ++t) {
                best[t] = x[t][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) best[t] = fmaxf(best[t], x[t][e]);
                best[t] *= unit;
                any = any || best[t] > top[t] + kSlack;
            }
            if (wave_any(any)) {
#pragma unroll
                for (int t = 0; t < kColumns; ++t) {
                    const float other = lane_xor(best[t], 32);
                    const float now = fmaxf(top[t], fmaxf(best[t], other));
                    const float less = now == kMinusInf ? 1.0f : exp2_fast(top[t] - now);
                    top[t] = now;
                    sum[t] *= less;
#pragma unroll
                    for (int d = 0; d < S::kDimBlocks; ++d) acc[t][d] *= less;
                }
            }
        };
        u32x4 p[kColumns][2];
        auto probabilities = [&](int tile, int i, const f32x16 (&x)[kColumns]) KVIO_INLINE {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f32x4 vs = {1, 1, 1, 1};
                if (E4M3) vs = *reinterpret_cast<const f32x4 *>(lds.v_scale[tile & 3] + 32 * i + 8 * r + 4 * g);
#pragma unroll
                for (int t = 0; t < kColumns; ++t) {
                    const float from = top[t] == kMinusInf ? 0.0f : top[t];
                    float e4[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        e4[e] = exp2_fast(fmaf(x[t][4 * r + e], unit, -from));
                        sum[t] += e4[e];
                        if (E4M3) e4[e] *= vs[e];
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        p[t][r / 2][2 * (r % 2) + e] = S::kPBf16 ? pack_bf16(e4[2 * e], e4[2 * e + 1]) : pack_f16(e4[2 * e], e4[2 * e + 1]);
                }
            }
        };
        auto outs = [&](int tile, int i) KVIO_INLINE {
            const uint8_t *v = lds.v[tile & 1] + (32 * i + 4 * g + m % 16 / 4) * S::kVRow + 32 * (m / 16) + 8 * (m % 4);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int d = 0; d < S::kDimBlocks; ++d) {
                    const uint8_t *w = v + 16 * u * S::kVRow + 64 * d;
                    const u32x2 x = lds_turned(w), y = lds_turned(w + 8 * S::kVRow);
#pragma unroll
                    for (int t = 0; t < kColumns; ++t) acc[t][d] = product32<S::kPBf16>(u32x4{x.x, x.y, y.x, y.y}, p[t][u], acc[t][d]);
                }
        };
        // Rare: values that are not finite reach the rows that see them, and no others.
        auto add_odd = [&](int tile) KVIO_INLINE {
            const int base = base0 + tile * kKeys;
            for (int i = 0; i < kKeys; ++i) {
                const int key = base + i;
                if (key < lo || key >= end) continue;
                const int page = page_of(c, b, key);
                if (page < 0) continue;
                const int j = static_cast<int>(div_by(static_cast<uint32_t>(key), c.page_div));
                const uint8_t *v = c.v_cache + (int64_t(page) * c.page_size + (key - j * c.page_size)) * cache_row + h * S::kSeg;
#pragma unroll
                for (int d = 0; d < S::kDimBlocks; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float f = element<BF16, E4M3>(v, 32 * d + 8 * (e / 4) + 4 * g + e % 4);
                        in_order();
                        if (!wave_any(f - f != 0)) continue;
#pragma unroll
                        for (int t = 0; t < kColumns; ++t)
                            acc[t][d][e] += f - f != 0 && key <= place[t] && (a.window == 0 || key > place[t] - a.window) ? f : 0.0f;
                    }
            }
        };

        // ---- before the first tile ----------------------------------------------------------
        int slot2, slot3, page4;                         // of tiles j + 2, j + 3, j + 4 in iteration j
        uint64_t there0, there1, there2, there3;
        {
            const int page0 = page_in(0), page1 = page_in(1), page2 = page_in(2), page3 = page_in(3);
            page4 = page_in(4);
            workgroup_barrier();                         // the block before is done with LDS
            const int slot0 = slot_from(0, page0);
            load(kx, c.k_cache, slot0);
            load(vx, c.v_cache, slot0);
            put_scales(0);
            const int slot1 = slot_from(1, page1);
            put_k(0);
            load(kx, c.k_cache, slot1);
            put_scales(1);
            slot2 = slot_from(2, page2);
            put_scales(2);
            slot3 = slot_from(3, page3);
            there0 = wave_ballot(slot0 >= 0), there1 = wave_ballot(slot1 >= 0);
            there2 = wave_ballot(slot2 >= 0), there3 = wave_ballot(slot3 >= 0);
            put_v(0, there0);
            load(vx, c.v_cache, slot1);
            put_k(1);
            load(kx, c.k_cache, slot2);
            workgroup_barrier();
            scores(0, 0, score);
            settle(0, 0, there0, score);
            raise(score);
        }
        // ---- tile by tile; what is computed of tiles behind the last one, from no slots, is masked or not used ----
        int k0 = 0;                                      // where K of tile j lies
        for (int j = 0; j < n; ++j) {
            workgroup_barrier();                         // K of tile j + 1 and V of tile j are there; the buffers of those before free
            const int k1 = k0 + 1 == S::kKBuffers ? 0 : k0 + 1, k2 = k1 + 1 == S::kKBuffers ? 0 : k1 + 1;
            put_k(k2);
            put_v(j + 1, there1);
            put_scales(j + 3);
            const int slot4 = slot_from(j + 4, page4);
            page4 = page_in(j + 5);
            load(vx, c.v_cache, slot2);
            load(kx, c.k_cache, slot3);
            in_order();
#pragma unroll
            for (int i = 0; i < S::kHalves; ++i) {
                const bool next = i + 1 == S::kHalves;
                scores(next ? k1 : k0, next ? 0 : i + 1, ahead);
                probabilities(j, i, score);
                in_order();
                outs(j, i);
                settle(next ? j + 1 : j, next ? 0 : i + 1, next ? there1 : there0, ahead);
                if (next && lds.odd[(serial + j) & 3] == serial + j) add_odd(j);   // before the maximum moves
                raise(ahead);
#pragma unroll
                for (int t = 0; t < kColumns; ++t) score[t] = ahead[t];
                in_order();
            }
            slot2 = slot3, slot3 = slot4;
            k0 = k1;
            there0 = there1, there1 = there2, there2 = there3, there3 = wave_ballot(slot4 >= 0);
        }
        serial += n;

        const bool alone = n == all_tiles;
#pragma unroll
        for (int t = 0; t < kColumns; ++t) {
            sum[t] += lane_xor(sum[t], 32);
            const int row = wave_row0 + 32 * t + m;
            if (row >= rows) continue;
            if (alone) {
                const int token = static_cast<int>(div_by(static_cast<uint32_t>(row), a.group_div)), qh = h * a.group + row - token * a.group;
                const float inv = sum[t] == 0 ? 0.0f : 1.0f / sum[t];
                const int64_t array_row = s.row0 + block_row0 + token;
                uint8_t *o = a.out + array_row * a.out_stride + int64_t(qh) * (2 * D);
#pragma unroll
                for (int d = 0; d < S::kDimBlocks; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const f32x16 &x = acc[t][d];
                        const float x0 = x[4 * r] * inv, x1 = x[4 * r + 1] * inv, x2 = x[4 * r + 2] * inv, x3 = x[4 * r + 3] * inv;
                        *reinterpret_cast<u32x2 *>(o + 2 * (32 * d + 8 * r + 4 * g)) =
                            BF16 ? u32x2{pack_bf16(x0, x1), pack_bf16(x2, x3)} : u32x2{pack_f16(x0, x1), pack_f16(x2, x3)};
                    }
                if (a.lse != nullptr && g == 0) a.lse[array_row * a.q_heads + qh] = lse_of(top[t], sum[t]);
            } else {
                float *slot = a.partials + block_partial_at(a, worker, from_tile != 0 ? 0 : 1, D);
                float *o = slot + int64_t(row) * D;
#pragma unroll
                for (int d = 0; d < S::kDimBlocks; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        *reinterpret_cast<f32x4 *>(o + 32 * d + 8 * r + 4 * g) = f32x4{acc[t][d][4 * r], acc[t][d][4 * r + 1], acc[t][d][4 * r + 2], acc[t][d][4 * r + 3]};
                if (g == 0) *reinterpret_cast<f32x2 *>(slot + int64_t(a.slot_rows) * D + 2 * row) = f32x2{top[t], sum[t]};
            }
        }
    }
}

// Join the partial results of the block that the end of a workgroup's range cuts, by the first workgroup that cuts it.
template <bool BF16, int D>
__global__ void __launch_bounds__(kThreads) join_blocks(const AttendArgs a) {
    constexpr int kDims = D / 64, kKeys = Shape<BF16, false, D>::kKeys;
    const CacheArgs &c = a.c;
    const int lane = static_cast<int>(threadIdx.x) & 63, wave = wave_first(static_cast<int>(threadIdx.x) >> 6);
    const int parts = (a.slot_rows + kJoinRows - 1) / kJoinRows;
    const int worker = static_cast<int>(blockIdx.x) / parts, part = static_cast<int>(blockIdx.x) - worker * parts;
    const Line line = line_of(a, lane);
    const int64_t begin = worker * line.per_worker, cut = begin + line.per_worker;
    if (cut >= line.all) return;
    const Where at = where_is(a, line, cut, lane);
    const Seq s = seq_of(c, at.b);
    const Blocks blocks = blocks_of(a, s);
    const int lo = blocks.lo(at.j), hi = blocks.hi(at.j), block_row0 = at.j * a.block_tokens;
    const int64_t end = at.begin + (hi - lo);
    auto tile_of = [&](int64_t p) { return static_cast<int>(lo + (p - at.begin)) / kKeys - lo / kKeys; };
    if (tile_of(cut) == 0) return;                       // not cut after all
    if (begin > at.begin && tile_of(begin) != 0) return; // cut before
    const int others = static_cast<int>((end - 1 - cut) / line.per_worker) + 1;      // workgroups behind this one that have a share
    const int rows = (s.rows - block_row0 < a.block_tokens ? s.rows - block_row0 : a.block_tokens) * a.group;
    for (int row = part * kJoinRows + wave; row < (part + 1) * kJoinRows && row < rows; row += kWaves) {
        float top = kMinusInf, sum = 0, acc[kDims] = {};
        for (int i = 0; i <= others; ++i) {
            const float *slot = a.partials + block_partial_at(a, worker + i, i == 0 ? 1 : 0, D);
            const f32x2 ends = *reinterpret_cast<const f32x2 *>(slot + int64_t(a.slot_rows) * D + 2 * row);
            const float *o = slot + int64_t(row) * D;
            const float other = ends.x;
            const float now = other > top || other != other ? other : top;
            const float mine = top == kMinusInf || now == top ? 1.0f : exp2_fast(top - now);
            const float its = other == kMinusInf || now == other ? 1.0f : exp2_fast(other - now);
            sum = sum * mine + ends.y * its;
#pragma unroll
            for (int d = 0; d < kDims; ++d) acc[d] = acc[d] * mine + o[d * 64 + lane] * its;
            top = now;
        }
        const int token = static_cast<int>(div_by(static_cast<uint32_t>(row), a.group_div)), qh = at.h * a.group + row - token * a.group;
        const int64_t array_row = s.row0 + block_row0 + token;
        const float inv = sum == 0 ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int d = 0; d < kDims; ++d)
            reinterpret_cast<uint16_t *>(a.out + array_row * a.out_stride + int64_t(qh) * (2 * D))[d * 64 + lane] =
                static_cast<uint16_t>(BF16 ? pack_bf16(acc[d] * inv, 0) : pack_f16(acc[d] * inv, 0));
        if (a.lse != nullptr && lane == 0) a.lse[array_row * a.q_heads + qh] = lse_of(top, sum);
    }
}

template <bool BF16, bool E4M3, int D>
hipError_t launch(const AttendArgs &a, const AttendPlan &plan, hipStream_t stream) {
    hipLaunchKernelGGL((attend_blocks<BF16, E4M3, D>), dim3(plan.groups), dim3(kThreads), 0, stream, a);
    if (plan.joined)
        hipLaunchKernelGGL((join_blocks<BF16, D>), dim3(static_cast<unsigned>((a.workers - 1) * ((a.slot_rows + kJoinRows - 1) / kJoinRows))), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

template <bool BF16, bool E4M3>
hipError_t launch_dim(const AttendArgs &a, const AttendPlan &plan, hipStream_t stream) {
    if (a.c.head_dim == 64) return launch<BF16, E4M3, 64>(a, plan, stream);
    if (a.c.head_dim == 128) return launch<BF16, E4M3, 128>(a, plan, stream);
    return launch<BF16, E4M3, 256>(a, plan, stream);
}

}  // namespace

hipError_t launch_blocks(const AttendArgs &a, const AttendPlan &plan, int32_t dtype, bool e4m3, hipStream_t stream) {
    if (dtype == KVIO_BF16) return e4m3 ? launch_dim<true, true>(a, plan, stream) : launch_dim<true, false>(a, plan, stream);
    return e4m3 ? launch_dim<false, true>(a, plan, stream) : launch_dim<false, false>(a, plan, stream);
}

AttendPlan plan_blocks(int32_t heads, int32_t q_heads, int32_t dim, const kvio_batch &b, int32_t max_query, int32_t max_ctx) {
    AttendPlan p = {};
    const int32_t group = q_heads / heads;
    p.block_tokens = block_rows(dim) / group;
    p.min_keys = 512;                                    // writing and joining a partial result costs as much as some 300 keys
    const int64_t blocks = int64_t(heads) * (b.num_tokens / p.block_tokens + int64_t(b.num_seqs));   // at most
    const int64_t workers = std::min<int64_t>(256, (blocks * std::max(max_ctx, 1) + p.min_keys - 1) / p.min_keys);   // one to a compute unit
    p.groups = static_cast<uint32_t>((workers + 7) / 8 * 8);
    p.workers = static_cast<int32_t>(p.groups);
    p.joined = workers > 1;
    p.slot_rows = static_cast<int32_t>(std::min<int64_t>(p.block_tokens, max_query) * group + 1) & ~1;
    if (p.joined) p.bytes = uint64_t(p.workers) * 2 * uint64_t(p.slot_rows) * uint64_t(dim + 2) * 4;
    return p;
}

}  // namespace kvio
