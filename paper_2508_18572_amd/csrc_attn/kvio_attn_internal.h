// kvio_attn_internal.h -- what the checks of kvio_append and kvio_attend hand to
// their kernels, and what those share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvio_attn.h"
#include "kvio_internal.h"
#include "kvio_lane.h"

namespace kvio {

// A batch and the pool layer it works on, as kernels see them.
struct CacheArgs {
    const int32_t *page_table;
    const int32_t *ctx_len;
    const int32_t *q_start;        // null: one new token each
    unsigned long long *err;
    uint8_t *k_cache, *v_cache;    // the layer's K and V
    float *k_scale, *v_scale;      // e4m3
    int64_t scale_stride;
    int64_t table_stride;
    int32_t num_seqs, num_tokens, max_query, max_ctx;   // max_ctx = max_pages * P
    int32_t num_pages, page_size;
    Divider page_div;
    int32_t heads, head_dim;       // of the cache
};

struct AppendArgs {
    CacheArgs c;
    const uint8_t *k, *v, *q;
    uint8_t *q_out;
    int64_t k_stride, v_stride, q_stride, q_out_stride;   // bytes
    const float *inv_freq;
    const int32_t *positions;
    int32_t q_heads, rot_half, interleaved;
    int32_t page_items;            // e4m3: at most so many (sequence, page) pairs are written
};

struct AttendArgs {
    CacheArgs c;
    const uint8_t *q;
    uint8_t *out;
    float *lse;
    int64_t q_stride, out_stride;  // bytes
    int32_t q_heads, group;        // group = q_heads / heads
    Divider group_div;
    int32_t window;
    float scale_log2;              // softmax_scale * log2(e)
    // How the work is split (AttendPlan).
    float *partials;
    int32_t heads_per_group, workers, min_tiles, slot_rows;
    int32_t block_tokens, min_keys, join_rows;
    bool joined;
};

// How a call of given sizes is split; what it needs of workspace.
struct AttendPlan {
    bool few;                      // few rows to a sequence: kvio_attend_steps.hip, else kvio_attend_blocks.hip
    int32_t columns;               // blocks of 16 rows that a wave holds
    int32_t heads_per_group, workers, min_tiles, slot_rows;
    int32_t block_tokens, min_keys, join_rows;
    uint32_t groups;               // workgroups
    bool joined;                   // partial results may be left
    uint64_t bytes;
};
// Rows that a workgroup of kvio_attend_blocks.hip holds, 32 to a wave: out^T of these takes D / 2 of a lane's registers.
constexpr int block_rows(int dim) { return dim <= 128 ? 256 : 128; }
AttendPlan plan_steps(bool e4m3, int32_t heads, int32_t q_heads, int32_t dim, const kvio_batch &b, int32_t max_query, int32_t max_ctx);
AttendPlan plan_blocks(int32_t heads, int32_t q_heads, int32_t dim, const kvio_batch &b, int32_t max_query, int32_t max_ctx);

int64_t append_threads(const AppendArgs &a, bool e4m3);      // that launch_append starts; fewer than 2^32 can be
hipError_t launch_append(const AppendArgs &a, int32_t dtype, bool e4m3, hipStream_t stream);
hipError_t launch_steps(const AttendArgs &a, const AttendPlan &plan, int32_t dtype, bool e4m3, hipStream_t stream);
hipError_t launch_blocks(const AttendArgs &a, const AttendPlan &plan, int32_t dtype, bool e4m3, hipStream_t stream);

// ---- shared by the kernels -----------------------------------------------------------

__device__ __forceinline__ int clamp_int(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ uint32_t div_by(uint32_t n, Divider d) { return static_cast<uint32_t>((uint64_t(n) * d.mul) >> d.shift); }

// The rows of sequence b and the length of its context, cut to what the arrays hold.
struct Seq {
    int32_t row0, rows;            // rows [row0, row0 + rows) of the arrays of new tokens
    int32_t ctx;                   // tokens in the context, the new ones included
    int32_t first;                 // context place of row0, maybe negative
};
__device__ __forceinline__ Seq seq_of(const CacheArgs &c, int b) {
    Seq s;
    int end;
    if (c.q_start != nullptr) {
        s.row0 = clamp_int(c.q_start[b], 0, c.num_tokens);
        end = clamp_int(c.q_start[b + 1], s.row0, c.num_tokens);
    } else {
        s.row0 = b;
        end = b + 1;
    }
    s.ctx = clamp_int(c.ctx_len[b], 0, c.max_ctx);
    s.first = s.ctx - (end - s.row0);
    s.rows = end - s.row0 < c.max_query ? end - s.row0 : c.max_query;
    return s;
}

// The sequence that array row `row` belongs to, if any: the first that ends behind it; -1 behind the last.
__device__ __forceinline__ int seq_with_row(const CacheArgs &c, int row, int lane) {
    int b = row;
    if (c.q_start != nullptr) {
        b = 0;
        for (int i = 0; i < c.num_seqs; i += 64)
            b += __builtin_popcountll(wave_ballot(i + lane < c.num_seqs && c.q_start[i + lane + 1] <= row));
    }
    return b < c.num_seqs ? b : -1;
}

// 64-bit values between lanes, by halves.
__device__ __forceinline__ int64_t whole_of(int lo, int hi) { return static_cast<int64_t>((static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32) | static_cast<uint32_t>(lo)); }
__device__ __forceinline__ int64_t lane_xor(int64_t v, int mask) { return whole_of(lane_xor(static_cast<int>(v), mask), lane_xor(static_cast<int>(v >> 32), mask)); }
__device__ __forceinline__ int64_t wave_read(int64_t v, int lane) { return whole_of(wave_read(static_cast<int>(v), lane), wave_read(static_cast<int>(v >> 32), lane)); }
__device__ __forceinline__ int64_t wave_first(int64_t v) { return whole_of(wave_first(static_cast<int>(v)), wave_first(static_cast<int>(v >> 32))); }

// Sum of this and all lower lanes' values.
__device__ __forceinline__ int lanes_upto(int v, int lane) {
    for (int by = 1; by < 64; by *= 2) {
        const int other = lane_up(v, by);
        if (lane >= by) v += other;
    }
    return v;
}

__device__ __forceinline__ int64_t lanes_upto(int64_t v, int lane) {
    for (int by = 1; by < 64; by *= 2) {
        const int64_t other = whole_of(lane_up(static_cast<int>(v), by), lane_up(static_cast<int>(v >> 32), by));
        if (lane >= by) v += other;
    }
    return v;
}

// Record a page of sequence b outside the pool for kvio_check, unless one is recorded already.
__device__ __forceinline__ void record_bad_page(const CacheArgs &c, int b, int page) {
    atomicCAS(c.err, 0ull, (static_cast<unsigned long long>(b + 1) << kErrSpanShift) | static_cast<unsigned long long>(page));
}

// The pool page of context token t of sequence b (t within the table), -1 for one outside the pool.
__device__ __forceinline__ int page_of(const CacheArgs &c, int b, int t) {
    const int j = static_cast<int>(div_by(static_cast<uint32_t>(t), c.page_div));
    const int page = c.page_table[b * c.table_stride + j];
    if (page >= 0 && page < c.num_pages) return page;
    record_bad_page(c, b, j);
    return -1;
}

}  // namespace kvio
