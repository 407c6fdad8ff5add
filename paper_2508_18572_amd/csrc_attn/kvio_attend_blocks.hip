// kvio_attend_blocks.hip -- attention of many new tokens to a sequence (prompts
// and the rest of partly cached ones), on the matrix units.
//
// A workgroup takes a block of 256 rows (128 with heads of 256 dims), query heads
// and tokens of one KV head, 32 to a wave, and goes through its keys 64 at a time.
// Rows are columns of both products,
//   scores^T (keys x rows) = K Q^T,  out^T (dims x rows) += V^T probabilities^T,
// so that the scores that a lane gets are the probabilities that it has to bring
// to the second product, and a row's maximum and sum concern two lanes.  Q and
// out^T stay in registers; K and V come from the pages through registers, where
// codes are widened to 16 bits, into LDS buffers that all waves share, a tile
// ahead.  V^T is read with the LDS' transposing loads.
//
// 4 D flops to a score against some eight vector operations: both units have to be
// kept busy at once.  Eight waves, two to a SIMD with 256 registers each, fill each
// other's gaps, and a wave's registers hold the scores of two halves of a tile, so
// that the products of the next half's run beside the exponentials of this one's
// (8192 tokens of 32 heads, 128 dims: four waves of 64 rows 904 us, eight of 32
// 792 us).  Heads of 256 dims leave room for four waves, one to a SIMD.
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

constexpr int kJoinThreads = 256, kJoinWaves = kJoinThreads / 64;

// Beginning and ending a block takes about as long as so many keys.
constexpr int kBlockCost = 96;

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
    // Length of all blocks before j, j < count: kBlockCost and the keys of each, sums over i < j of hi(i) = max(1, first + (i + 1) tokens) and lo(i).
    __device__ __forceinline__ int64_t before(int j) const {
        const int64_t n = j, z = first < 1 ? std_min(n, (1 - first) / tokens) : 0;
        int64_t sum = z + (n - z) * first + tokens * ((n * (n + 1) - z * (z + 1)) / 2);
        if (window > 0) {
            const int64_t free = int64_t(window) - 1 - first;                  // lo(i) is 0 while i * tokens <= free
            const int64_t y = free < 0 ? 0 : std_min(n, int64_t(static_cast<int>(std_min(free, 0x7fffffff)) / tokens) + 1);
            sum -= (n - y) * (int64_t(first) - window + 1) + tokens * ((n * (n - 1) - y * (y - 1)) / 2);
        }
        return sum + n * kBlockCost;
    }
    __device__ __forceinline__ int64_t keys() const { return count == 0 ? 0 : before(count - 1) + length(count - 1); }
    __device__ __forceinline__ int length(int j) const { return kBlockCost + hi(j) - lo(j); }
    // The tile, counted from the block's first one, that a cut at `at` of its length begins with.
    __device__ __forceinline__ int tile_at(int j, int64_t at, int keys) const {
        const int key = lo(j) + (at > kBlockCost ? static_cast<int>(at) - kBlockCost : 0);
        return key / keys - lo(j) / keys;
    }
    static __device__ __forceinline__ int64_t std_min(int64_t a, int64_t b) { return a < b ? a : b; }
};
__device__ __forceinline__ Blocks blocks_of(const AttendArgs &a, const Seq &s) {
    return {s.rows > 0 ? (s.rows - 1) / a.block_tokens + 1 : 0, s.first, s.rows, a.block_tokens, a.window};
}

// All keys, head after head, sequence after sequence, block after block.
struct Line {
    int64_t head, all, per_worker;           // length of a KV head, of all, of a workgroup's range
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
    return int64_t(a.workers) * 4 + (int64_t(worker) * 2 + which) * a.slot_rows * (dim + 2);
}
// Before them, for each workgroup: the block that its range is the first to cut, and how many others have a share of it; 0: none.
struct alignas(16) Cut {
    int32_t h, b, j, others;
};

constexpr int waves_of(int dim) { return dim <= 128 ? 8 : 4; }

template <bool BF16, bool E4M3, int D>
struct Shape {
    static constexpr int kElem = E4M3 ? 1 : 2, kSeg = D * kElem;
    static constexpr int kKeys = 64;                     // of a tile
    static constexpr int kWaves = waves_of(D), kThreads = 64 * kWaves;
    static constexpr int kWaveRows = 32;                 // rows to a wave, columns of its products
    static_assert(kWaveRows * kWaves == block_rows(D));
    static constexpr int kSteps = D / 16, kDimBlocks = D / 32;
    static constexpr int kPieces = kSeg / 16, kRowsAtOnce = std::min(kKeys, kThreads / kPieces), kPasses = kKeys / kRowsAtOnce;
    // 16 rows' pieces of 16 bytes lie in all banks; so do 32 bytes of 8 rows
    static constexpr int kKRow = 2 * D + 16, kVRow = 2 * D + 64;
    // Probabilities' and values' type: fp16, in a ValueUnit, for e4m3 values.  One term: a second one, as single tokens and drafts
    // have, costs half a product more for each score (8192 tokens of 32 heads, 128 dims, in bf16: 669 -> 849 us and an error against
    // 64 bits of 0.0022 -> 0.0017 of the result's norm; windowed prompts of 256 dims in fp16: 156 -> 178 us, 0.00029 -> 0.00021).
    static constexpr bool kPBf16 = BF16 && !E4M3;
    // Operands in registers at a time; with fewer than a phase has, K of a tile is still read while the next but one is put.
    // As many as the registers last for: over e4m3 with 128 dims, four of K spill.  Three of V, not two: 676 against 679 us for
    // 8192 tokens of 32 heads, 128 dims, 504 against 509 us for two prompts of 3500 tokens, 16 heads of 256 dims over e4m3 (eight
    // instead of all); four change nothing.
    static constexpr int kKOps = D == 128 && E4M3 ? 2 : D <= 128 ? 4 : kSteps, kVOps = D <= 128 ? 3 : 2 * kDimBlocks, kKBuffers = kKOps < kSteps ? 3 : 2;
    struct alignas(16) Lds {
        uint8_t k[kKBuffers][kKeys * kKRow], v[2][kKeys * kVRow];
        float k_scale[4][64], v_scale[4][64];            // of tiles, by their number & 3
        int32_t odd[4];                                  // the running number of a tile with values that are not finite, or that has such scales
    };
};

template <bool BF16, bool E4M3, int D>
__global__ void __launch_bounds__(64 * waves_of(D), waves_of(D) / 4) attend_blocks(const AttendArgs a) {
    using S = Shape<BF16, E4M3, D>;
    constexpr int kKeys = S::kKeys, kWaveRows = S::kWaveRows;
    __shared__ typename S::Lds lds;
    const CacheArgs &c = a.c;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = wave_first(tid >> 6);
    const int g = lane / 32, m = lane % 32;
    // Workgroups go to the 8 dies in turn; each die takes one stretch of the line, so that its cache serves few heads.
    const int worker = static_cast<int>(blockIdx.x % 8) * (a.workers / 8) + static_cast<int>(blockIdx.x / 8);

    const Line line = line_of(a, lane);
    int64_t pos = worker * line.per_worker;
    const int64_t stop = pos + line.per_worker < line.all ? pos + line.per_worker : line.all;
    Cut cut = {0, 0, 0, 0};
    Cut *my_cut = reinterpret_cast<Cut *>(a.partials) + worker;
    if (pos >= stop) {
        if (a.joined && tid == 0) *my_cut = cut;
        return;
    }
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
        const int64_t next = at.begin + blocks.length(at.j);
        const int tile0 = lo / kKeys, all_tiles = (hi + kKeys - 1) / kKeys - tile0;
        // A range's end is moved down to a tile's.
        const int from_tile = blocks.tile_at(at.j, pos - at.begin, kKeys);
        const int to_tile = stop >= next ? all_tiles : blocks.tile_at(at.j, stop - at.begin, kKeys);
        const int block_row0 = at.j * a.block_tokens;    // in the sequence
        const int n = to_tile - from_tile;
        if (from_tile == 0 && to_tile < all_tiles && to_tile > 0)
            cut = Cut{h, b, at.j, static_cast<int>((next - 1 - stop) / line.per_worker) + 1};
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

        int g16 = 16 * g;
        keep_here(g16);
        // The lane's column is one row: its place, below any key for none.
        int place;
        u32x4 q[S::kSteps];
        {
            const int row = wave_row0 + m, token = static_cast<int>(div_by(static_cast<uint32_t>(row), a.group_div));
            place = row < rows ? first + token : -1;
            const uint8_t *p = a.q + (s.row0 + block_row0 + token) * a.q_stride + int64_t(h * a.group + row - token * a.group) * (2 * D) + g16;
#pragma unroll
            for (int i = 0; i < S::kSteps; ++i) q[i] = row < rows ? *reinterpret_cast<const u32x4 *>(p + 32 * i) : u32x4{0, 0, 0, 0};
        }
        f32x16 acc[S::kDimBlocks];
        float top = kMinusInf, sum = 0;
#pragma unroll
        for (int d = 0; d < S::kDimBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] = 0;

        // ---- keys and values on their way into LDS ----------------------------------------
        auto page_in = [&](int tile) KVIO_INLINE {       // of the lane's key; some page for one that no row sees
            const int key = base0 + tile * kKeys + lane;
            return c.page_table[b * c.table_stride + static_cast<int>(div_by(static_cast<uint32_t>(key < c.max_ctx ? key : c.max_ctx - 1), c.page_div))];
        };
        float k_scale = 0, v_scale = 0;
        f32x4 ks[2] = {}, vs[2] = {};                    // e4m3: scales of 4 g + 8 r .. + 3 of a half's keys, of r and r + 1; values' in value_unit
        ValueUnit value_unit;
        uint64_t there_now = 0;                          // the keys that are there
        int bad_page = -1;
        auto record_bad = [&]() KVIO_INLINE {
            if (wave_any(bad_page >= 0) && bad_page >= 0) record_bad_page(c, b, bad_page);
        };
        auto slot_from = [&](int tile, int page) KVIO_INLINE {   // 0 for a key that is not there; asks for its scales
            const int key = base0 + tile * kKeys + lane;
            const bool seen = tile < n && key >= lo && key < end;
            const bool there = seen && page >= 0 && page < c.num_pages;
            const int i = static_cast<int>(div_by(static_cast<uint32_t>(key), c.page_div));
            there_now = wave_ballot(there);
            bad_page = seen && !there ? i : -1;
            if (E4M3) {
                const int at_page = there ? page : 0;
                k_scale = c.k_scale[at_page * c.scale_stride + h] * a.scale_log2;
                v_scale = c.v_scale[at_page * c.scale_stride + h];
            }
            return there ? page * c.page_size + (key - i * c.page_size) : 0;
        };
        auto put_scales = [&](int tile, uint64_t there) KVIO_INLINE {
            if constexpr (!E4M3) return;
            const bool is_there = (there >> lane) & 1;   // what garbage holds does not count
            float vs_now = is_there ? v_scale : 0.0f;
            bool odd;
            const float less = value_unit.take(vs_now, odd);
            if (__builtin_expect(less != 1.0f, 0)) {                          // rare, and the same in all waves: what is in the old unit follows
#pragma unroll
                for (int d = 0; d < S::kDimBlocks; ++d) acc[d] *= less;
                vs[0] *= less, vs[1] *= less;
                workgroup_barrier();
                if (wave < 4) lds.v_scale[wave][lane] *= less;
                workgroup_barrier();
            }
            if (wave == 0) {
                lds.k_scale[tile & 3][lane] = is_there ? k_scale : 0.0f;
                lds.v_scale[tile & 3][lane] = vs_now * value_unit.inverse;
                if (odd) lds.odd[(serial + tile) & 3] = serial + tile;
            }
        };
        const int piece = tid % S::kPieces, piece_row = tid / S::kPieces % kKeys;
        const uint32_t cache_row = static_cast<uint32_t>(S::kSeg) * static_cast<uint32_t>(c.heads);
        auto row_slots = [&](uint32_t *slots, int slot) KVIO_INLINE {        // of the thread's rows
#pragma unroll
            for (int i = 0; i < S::kPasses; ++i) slots[i] = static_cast<uint32_t>(lane_read(slot, piece_row + i * S::kRowsAtOnce));
        };
        const uint8_t *k_from = c.k_cache + h * S::kSeg + 16 * piece, *v_from = c.v_cache + h * S::kSeg + 16 * piece;
        u32x4 kx[S::kPasses], vx[S::kPasses];
        auto load_one = [&](const uint8_t *from, uint32_t slot) KVIO_INLINE { return *reinterpret_cast<const u32x4 *>(from + uint64_t(slot) * cache_row); };
        auto load = [&](u32x4 *x, const uint8_t *from, const uint32_t *slots) KVIO_INLINE {
#pragma unroll
            for (int i = 0; i < S::kPasses; ++i) x[i] = load_one(from, slots[i]);
        };
        auto put_one = [&](uint8_t *to, int row_bytes, int i, u32x4 x, auto as_bf16) KVIO_INLINE {
            uint8_t *w = to + (piece_row + i * S::kRowsAtOnce) * row_bytes + piece * (32 / S::kElem);
            if constexpr (E4M3) {
                constexpr bool kBf16 = decltype(as_bf16)::value;
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    *reinterpret_cast<u32x4 *>(w + 16 * e) = u32x4{e4m3_16<kBf16, false>(x[2 * e]), e4m3_16<kBf16, true>(x[2 * e]),
                                                                   e4m3_16<kBf16, false>(x[2 * e + 1]), e4m3_16<kBf16, true>(x[2 * e + 1])};
            } else {
                *reinterpret_cast<u32x4 *>(w) = x;
            }
        };
        auto put_k = [&](int buffer, int i) KVIO_INLINE { put_one(lds.k[buffer], S::kKRow, i, kx[i], std::bool_constant<BF16>()); };
        auto put_v = [&](int tile, int i) KVIO_INLINE { put_one(lds.v[tile & 1], S::kVRow, i, vx[i], std::bool_constant<S::kPBf16>()); };
        // Whether all rows of the block see all keys of a tile.
        auto whole_for_all = [&](int tile, uint64_t there) KVIO_INLINE {
            const int base = base0 + tile * kKeys;
            return base + kKeys - 1 <= first && (a.window == 0 || base > last - a.window) && there == ~0ull;
        };
        // Hidden values may hold anything: those that are not finite become zeros, the tile is marked.
        auto clean_v = [&](int tile, uint64_t there) KVIO_INLINE {
            if (whole_for_all(tile, there)) return;
            if (there != ~0ull)
#pragma unroll
                for (int i = 0; i < S::kPasses; ++i)
                    if (((there >> (piece_row + i * S::kRowsAtOnce)) & 1) == 0) vx[i] = u32x4{0, 0, 0, 0};
            NotFinite<BF16, E4M3> any;
#pragma unroll
            for (int i = 0; i < S::kPasses; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) any.look(vx[i][e]);
            if (__builtin_expect(!wave_any(any.found()), 1)) return;
#pragma unroll
            for (int i = 0; i < S::kPasses; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) vx[i][e] &= ~not_finite<BF16, E4M3>(vx[i][e]);
            if (any.found()) lds.odd[(serial + tile) & 3] = serial + tile;
        };

        // ---- products, 32 keys at a time: half i of a tile ---------------------------------
        // Scores (of keys 8 (e / 4) + 4 g + e % 4) become probabilities, and take part in the maximum, in units of two.
        constexpr int kUnits = 8, kScoreProducts = S::kSteps, kOutProducts = 2 * S::kDimBlocks;
        f32x16 score, ahead;
        u32x4 k_op[S::kKOps], v_op[S::kVOps], p[2];
        auto fetch_k = [&](int buffer, int i, int e) KVIO_INLINE {
            k_op[e % S::kKOps] = *reinterpret_cast<const u32x4 *>(lds.k[buffer] + (32 * i + m) * S::kKRow + 16 * g + 32 * e);
        };
        auto fetch_v = [&](int tile, int i, int e) KVIO_INLINE {
            const uint8_t *w = lds.v[tile & 1] + (32 * i + 4 * g + m % 16 / 4) * S::kVRow + 32 * (m / 16) + 8 * (m % 4) +
                               e / S::kDimBlocks * 16 * S::kVRow + e % S::kDimBlocks * 64;
            const u32x2 x = lds_turned(w), y = lds_turned(w + 8 * S::kVRow);
            v_op[e % S::kVOps] = u32x4{x.x, x.y, y.x, y.y};
        };
        auto fetch_scales = [&](f32x4 *to, const float *scales, int i, int r) KVIO_INLINE {
            if constexpr (E4M3) to[r % 2] = *reinterpret_cast<const f32x4 *>(scales + 32 * i + 8 * r + 4 * g);
        };
        auto score_product = [&](int i, f32x16 &x) KVIO_INLINE {
            const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
            x = product32<BF16>(k_op[i % S::kKOps], q[i], i == 0 ? zero : x);
        };
        auto out_product = [&](int i) KVIO_INLINE {
            const int u = i / S::kDimBlocks, d = i % S::kDimBlocks;
            acc[d] = product32<S::kPBf16>(v_op[i % S::kVOps], p[u], acc[d]);
        };
        // Scores are in powers of two once multiplied by `unit`.
        const float unit = E4M3 ? 1.0f : a.scale_log2;
        float best, from = 0;                            // of a half; what is taken off a score: the maximum, or 0 where there is none
        auto largest = [&](int i, f32x16 &x) KVIO_INLINE {
            const int e = 2 * i;
            if (E4M3) x[e] *= ks[e / 4 % 2][e % 4], x[e + 1] *= ks[e / 4 % 2][e % 4 + 1];
            const float of_two = larger(x[e], x[e + 1]);
            best = e == 0 ? of_two : larger(best, of_two);
            if (e == 14) keep_here(best);
        };
        auto probability = [&](int i, const f32x16 &x) KVIO_INLINE {
            const int e = 2 * i;
            float y = exp2_fast(fmaf(x[e], unit, -from)), z = exp2_fast(fmaf(x[e + 1], unit, -from));
            sum += y + z;
            if (e == 14) keep_here(sum);
            if (E4M3) y *= vs[e / 4 % 2][e % 4], z *= vs[e / 4 % 2][e % 4 + 1];
            p[e / 8][e / 2 % 4] = S::kPBf16 ? pack_bf16(y, z) : pack_f16(y, z);
        };
        auto mask = [&](int tile, int i, uint64_t there, f32x16 &x) KVIO_INLINE { // hidden keys at minus infinity
            const int base = base0 + tile * kKeys + 32 * i;
            if (idle || (base + 31 <= wave_first_place && (a.window == 0 || base > wave_last_place - a.window) && there == ~0ull)) return;
            // Bit n of `seen`: the row sees key base + 4 g + n.
            const uint32_t mine = static_cast<uint32_t>(there >> (32 * i + 4 * g));
            const int up_to = place - (base + 4 * g);
            uint32_t seen = mine & low_bits(up_to);
            if (a.window > 0) seen &= ~low_bits(place < 0 ? -1 : up_to - a.window);
            best = kMinusInf;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                x[e] = where_bit(seen, 8 * (e / 4) + e % 4, x[e], kMinusInf);
                best = larger(best, x[e]);
            }
        };
        auto raise = [&]() KVIO_INLINE {                 // a new maximum where the old one is passed by far
            if (!wave_any(best * unit > top + kSlack)) return;
            const float mine = best * unit, now = fmaxf(top, fmaxf(mine, lane_xor(mine, 32)));
            const float less = now == kMinusInf ? 1.0f : exp2_fast(top - now);
            top = now;
            from = now == kMinusInf ? 0.0f : now - kRaised<BF16, E4M3>;
            sum *= less;
#pragma unroll
            for (int d = 0; d < S::kDimBlocks; ++d) acc[d] *= less;
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
                const float by = E4M3 ? odd_scale_at(a, page, h) : 1.0f;
#pragma unroll
                for (int d = 0; d < S::kDimBlocks; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float f = element<BF16, E4M3>(v, 32 * d + 8 * (e / 4) + 4 * g + e % 4) * by;
                        in_order();
                        if (!wave_any(f - f != 0)) continue;
                        acc[d][e] += f - f != 0 && key <= place && (a.window == 0 || key > place - a.window) ? f : 0.0f;
                    }
            }
        };

        // ---- before the first tile ----------------------------------------------------------
        // In iteration j: the slots of the thread's rows in tiles j + 2 and j + 3, the page of the lane's key in tile
        // j + 4, the keys that are there in tiles j to j + 3.
        uint32_t slots2[S::kPasses], slots3[S::kPasses];
        int page4;
        uint64_t there0, there1, there2, there3;
        {
            const int page0 = page_in(0), page1 = page_in(1), page2 = page_in(2), page3 = page_in(3);
            page4 = page_in(4);
            workgroup_barrier();                         // the block before is done with LDS
            const int slot0 = slot_from(0, page0);
            record_bad();
            there0 = there_now;
            put_scales(0, there0);
            row_slots(slots2, slot0);
            load(kx, k_from, slots2);
            load(vx, v_from, slots2);
            const int slot1 = slot_from(1, page1);
            record_bad();
            there1 = there_now;
            put_scales(1, there1);
            row_slots(slots3, slot1);
#pragma unroll
            for (int i = 0; i < S::kPasses; ++i) put_k(0, i);
            load(kx, k_from, slots3);
            const int slot2 = slot_from(2, page2);
            record_bad();
            there2 = there_now;
            put_scales(2, there2);
            row_slots(slots2, slot2);
            clean_v(0, there0);
#pragma unroll
            for (int i = 0; i < S::kPasses; ++i) put_v(0, i);
            load(vx, v_from, slots3);
            const int slot3 = slot_from(3, page3);
            record_bad();
            there3 = there_now;
            row_slots(slots3, slot3);
#pragma unroll
            for (int i = 0; i < S::kPasses; ++i) put_k(1, i);
            load(kx, k_from, slots2);
            workgroup_barrier();
#pragma unroll
            for (int e = 0; e < S::kKOps; ++e) fetch_k(0, 0, e);
#pragma unroll
            for (int i = 0; i < kScoreProducts; ++i) {
                score_product(i, score);
                if (i + S::kKOps < S::kSteps) fetch_k(0, 0, i + S::kKOps);
            }
#pragma unroll
            for (int e = 0; e < S::kKOps; ++e) fetch_k(0, 1, e);
            fetch_scales(vs, lds.v_scale[0], 0, 0);
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                if (i % 2 == 0) fetch_scales(ks, lds.k_scale[0], 0, i / 2);
                largest(i, score);
            }
            mask(0, 0, there0, score);
            raise();
        }
        // ---- tile by tile; what is computed of tiles behind the last one is masked or not used ----
        // Each half in two phases: the next half's scores beside this one's probabilities, then this one's part of out^T
        // beside the next half's maximum.  Operands are fetched, and tiles moved on, one phase or more before they are
        // used, a little beside each product: a matrix product takes as long as 8 other instructions, and the compiler,
        // left to itself, puts all of one kind first (8192 tokens of 32 heads, 128 dims: 912 us).  What is rare is said to be
        // (__builtin_expect): its code then lies behind the loop, not in it (windowed prompts of 256 dims 157 -> 147 us).
        int k0 = 0;                                      // where K of tile j lies
        for (int j = 0; j < n; ++j) {
            const int k1 = k0 + 1 == S::kKBuffers ? 0 : k0 + 1, k2 = k1 + 1 == S::kKBuffers ? 0 : k1 + 1;
            workgroup_barrier();                         // K of tile j + 1 and V of tile j are there; the buffers of those before free
            put_scales(j + 3, there3);
            const int page5 = page_in(j + 5);            // before the tiles' loads, so that waiting for it does not wait for them
            in_order();
            auto scores_phase = [&](int half, const f32x16 &now, f32x16 &next) KVIO_INLINE {
#pragma unroll
                for (int i = 0; i < kScoreProducts; ++i) {
                    score_product(i, next);
                    in_order();
                    if (i == kScoreProducts - 1) fetch_scales(ks, lds.k_scale[(j + half) & 3], 1 - half, 0);
                    if (half == 1 && i < S::kPasses) {
                        put_k(k2, i);
                        kx[i] = load_one(k_from, slots3[i]);
                    }
#pragma unroll
                    for (int e = i * S::kVOps / kScoreProducts; e < (i + 1) * S::kVOps / kScoreProducts; ++e) fetch_v(j, half, e);
                    if (i + S::kKOps < S::kSteps) fetch_k(half == 0 ? k0 : k1, 1 - half, i + S::kKOps);
#pragma unroll
                    for (int e = i * kUnits / kScoreProducts; e < (i + 1) * kUnits / kScoreProducts; ++e) {
                        if (e % 2 == 0 && e < 6) fetch_scales(vs, lds.v_scale[j & 3], half, e / 2 + 1);
                        probability(e, now);
                    }
                    in_order();
                }
            };
            auto out_phase = [&](int half, f32x16 &next) KVIO_INLINE {
#pragma unroll
                for (int i = 0; i < kOutProducts; ++i) {
                    out_product(i);
                    in_order();
                    if (i == kOutProducts - 1) fetch_scales(vs, lds.v_scale[(j + half) & 3], 1 - half, 0);
                    if (half == 1 && i < S::kPasses) {
                        put_v(j + 1, i);
                        vx[i] = load_one(v_from, slots2[i]);
                    }
#pragma unroll
                    for (int e = i * S::kKOps / kOutProducts; e < (i + 1) * S::kKOps / kOutProducts; ++e) fetch_k(k1, half, e);
                    if (i + S::kVOps < 2 * S::kDimBlocks) fetch_v(j, half, i + S::kVOps);
                    // not beside the first ones: the next scores are just being finished
                    constexpr int kLate = kOutProducts / 4;
                    if (i >= kLate)
#pragma unroll
                        for (int e = (i - kLate) * kUnits / (kOutProducts - kLate); e < (i + 1 - kLate) * kUnits / (kOutProducts - kLate); ++e) {
                            if (e % 2 == 0 && e < 6) fetch_scales(ks, lds.k_scale[(j + half) & 3], 1 - half, e / 2 + 1);
                            largest(e, next);
                        }
                    in_order();
                }
            };
            scores_phase(0, score, ahead);
            out_phase(0, ahead);
            mask(j, 1, there0, ahead);
            raise();
            in_order();
            clean_v(j + 1, there1);
            in_order();
            scores_phase(1, ahead, score);
            out_phase(1, score);
            if (__builtin_expect(lds.odd[(serial + j) & 3] == serial + j, 0)) add_odd(j);   // before the maximum moves
            mask(j + 1, 0, there1, score);
            raise();
            const int slot4 = slot_from(j + 4, page4);
            record_bad();
            page4 = page5;
#pragma unroll
            for (int i = 0; i < S::kPasses; ++i) slots2[i] = slots3[i];
            row_slots(slots3, slot4);
            k0 = k1;
            there0 = there1, there1 = there2, there2 = there3, there3 = there_now;
        }
        serial += n;

        const bool alone = n == all_tiles;
        sum += lane_xor(sum, 32);
        int g8 = 8 * g, last_m = m;                      // computed here, not kept from block to block where registers are short
        keep_here(g8);
        if constexpr (D > 64) keep_here(last_m);
        const int out_row = wave_row0 + last_m;
        if (out_row < rows && alone) {
            const int token = static_cast<int>(div_by(static_cast<uint32_t>(out_row), a.group_div)), qh = h * a.group + out_row - token * a.group;
            const float inv = sum == 0 ? 0.0f : (E4M3 ? value_unit.unit : 1.0f) / sum;
            const int64_t array_row = s.row0 + block_row0 + token;
            uint8_t *o = a.out + array_row * a.out_stride + int64_t(qh) * (2 * D);
#pragma unroll
            for (int d = 0; d < S::kDimBlocks; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const f32x16 &x = acc[d];
                    const float x0 = x[4 * r] * inv, x1 = x[4 * r + 1] * inv, x2 = x[4 * r + 2] * inv, x3 = x[4 * r + 3] * inv;
                    *reinterpret_cast<u32x2 *>(o + 64 * d + 16 * r + g8) =
                        BF16 ? u32x2{pack_bf16(x0, x1), pack_bf16(x2, x3)} : u32x2{pack_f16(x0, x1), pack_f16(x2, x3)};
                }
            if (a.lse != nullptr && g == 0) a.lse[array_row * a.q_heads + qh] = lse_of(top - kRaised<BF16, E4M3>, sum);
        } else if (out_row < rows) {
            float *slot = a.partials + block_partial_at(a, worker, from_tile != 0 ? 0 : 1, D);
            float *o = slot + int64_t(out_row) * D;
            const float by = E4M3 ? value_unit.unit : 1.0f;
#pragma unroll
            for (int d = 0; d < S::kDimBlocks; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    *reinterpret_cast<f32x4 *>(o + 32 * d + 8 * r + g8 / 2) = f32x4{acc[d][4 * r] * by, acc[d][4 * r + 1] * by, acc[d][4 * r + 2] * by, acc[d][4 * r + 3] * by};
            if (g == 0) *reinterpret_cast<f32x2 *>(slot + int64_t(a.slot_rows) * D + 2 * out_row) = f32x2{top - kRaised<BF16, E4M3>, sum};
        }
    }
    if (a.joined && tid == 0) *my_cut = cut;
}

// Join the partial results of the block that a workgroup was the first to cut, in order, a.join_rows rows to a workgroup.
template <bool BF16, int D>
__global__ void __launch_bounds__(kJoinThreads) join_blocks(const AttendArgs a) {
    constexpr int kDims = D / 64;
    const CacheArgs &c = a.c;
    const int lane = static_cast<int>(threadIdx.x) & 63, wave = wave_first(static_cast<int>(threadIdx.x) >> 6);
    const int parts = (a.slot_rows + a.join_rows - 1) / a.join_rows;
    const int worker = static_cast<int>(blockIdx.x) / parts, part = static_cast<int>(blockIdx.x) - worker * parts;
    const Cut cut = reinterpret_cast<const Cut *>(a.partials)[worker];
    if (cut.others == 0) return;
    const Seq s = seq_of(c, cut.b);
    const int block_row0 = cut.j * a.block_tokens, end = (part + 1) * a.join_rows;
    const int rows = (s.rows - block_row0 < a.block_tokens ? s.rows - block_row0 : a.block_tokens) * a.group;
    for (int row = part * a.join_rows + wave; row < end && row < rows; row += kJoinWaves) {
        float top, sum, acc[kDims];
        auto slot = [&](int i) { return a.partials + block_partial_at(a, worker + i, i == 0 ? 1 : 0, D); };
        join_partials<D>(0, cut.others + 1, lane, [&](int i) { return slot(i) + int64_t(row) * D; },
                         [&](int i) { return slot(i) + int64_t(a.slot_rows) * D + 2 * row; }, &top, &sum, acc);
        const int token = static_cast<int>(div_by(static_cast<uint32_t>(row), a.group_div)), qh = cut.h * a.group + row - token * a.group;
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
    hipLaunchKernelGGL((attend_blocks<BF16, E4M3, D>), dim3(plan.groups), dim3(64 * waves_of(D)), 0, stream, a);
    if (plan.joined)
        hipLaunchKernelGGL((join_blocks<BF16, D>), dim3(static_cast<unsigned>((a.workers - 1) * ((a.slot_rows + a.join_rows - 1) / a.join_rows))), dim3(kJoinThreads), 0, stream, a);
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
    // Writing and joining a partial result costs as much as some 300 keys.  With 256 or 1024: a prompt of 300 tokens of 32 heads
    // 32.0 and 61.4 us (40.6 with 512), 100 tokens behind 2000 38.2 and 49.9 (39.7); 100 behind 16384 64.4 and 64.7 (64.4).
    p.min_keys = 512;
    const int64_t blocks = int64_t(heads) * (b.num_tokens / p.block_tokens + int64_t(b.num_seqs));   // at most
    const int64_t workers = std::min<int64_t>(256, (blocks * (std::max(max_ctx, 1) + kBlockCost) + p.min_keys - 1) / p.min_keys);   // one to a compute unit
    p.groups = static_cast<uint32_t>((workers + 7) / 8 * 8);
    p.workers = static_cast<int32_t>(p.groups);
    p.joined = workers > 1;
    // Few blocks have many partial results each: 100 tokens behind 16384 of 32 heads take 64 us with 4 rows to a workgroup, 81
    // with 16; a prompt of 8192 tokens 705 and 700 us.
    p.join_rows = blocks <= 64 ? 4 : 16;
    p.slot_rows = static_cast<int32_t>(std::min<int64_t>(p.block_tokens, max_query) * group + 1) & ~1;
    if (p.joined) p.bytes = uint64_t(p.workers) * (sizeof(Cut) + 2 * uint64_t(p.slot_rows) * uint64_t(dim + 2) * 4);
    return p;
}

}  // namespace kvio
