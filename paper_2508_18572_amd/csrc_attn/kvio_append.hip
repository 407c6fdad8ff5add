// kvio_append.hip -- new tokens' keys and values into the pages of their
// sequences, keys and queries rotated by their positions on the way; the cache
// in 16 bits (append_rows) or in e4m3 with a scale for each page and head
// (append_pages).
//
// A head of D elements is D / 16 units of two pieces of 8 elements (16 bytes):
// the two sides of 8 pairs that are rotated together, or two neighbours.  Every
// element is read once and written once; nothing is computed that would bound this.
#include "kvio_attn_internal.h"

namespace kvio {
namespace {

constexpr int kThreads = 256;
constexpr int kPageThreads = 1024, kWaves = kPageThreads / 64;
constexpr int kAngles = 8192, kKept = 4;
constexpr int kMostPairs = 512;              // rotated pairs of a head; check in kvio_append
constexpr double kPerTurn = 0.15915494309189533577;   // 1 / (2 pi)

template <bool BF16> __device__ __forceinline__ float lo(uint32_t w) { return BF16 ? bf16_lo(w) : f16_lo(w); }
template <bool BF16> __device__ __forceinline__ float hi(uint32_t w) { return BF16 ? bf16_hi(w) : f16_hi(w); }
template <bool BF16> __device__ __forceinline__ uint32_t pack(float a, float b) { return BF16 ? pack_bf16(a, b) : pack_f16(a, b); }

// Sine and cosine of position * inv_freq.  The product is exact in 64 bits, and
// so many turns are taken off there: far positions lose nothing.
__device__ __forceinline__ f32x2 sin_cos(int position, float inv_freq) {
    const double turns = static_cast<double>(position) * static_cast<double>(inv_freq) * kPerTurn;
    return sin_cos_of(static_cast<float>(turns - rint(turns)));
}

struct Unit {
    u32x4 a, b;                              // 8 elements each
};

// Where unit j's pieces lie in a head and which of its pairs they hold.
struct Place {
    int a, b;                                // first element of each piece
    bool turned;
};
__device__ __forceinline__ Place place_of(int j, int half, bool interleaved) {
    if (interleaved || j >= half / 8) return {16 * j, 16 * j + 8, interleaved && j < half / 8};
    return {8 * j, half + 8 * j, true};
}

template <bool BF16>
__device__ __forceinline__ void turn(Unit &u, bool interleaved, const f32x2 *sc) {   // sc: of pairs 8 j .. 8 j + 7
    if (!interleaved) {
        for (int w = 0; w < 4; ++w) {
            const f32x2 s = sc[2 * w], t = sc[2 * w + 1];
            const float a0 = lo<BF16>(u.a[w]), a1 = hi<BF16>(u.a[w]), b0 = lo<BF16>(u.b[w]), b1 = hi<BF16>(u.b[w]);
            u.a[w] = pack<BF16>(a0 * s.y - b0 * s.x, a1 * t.y - b1 * t.x);
            u.b[w] = pack<BF16>(b0 * s.y + a0 * s.x, b1 * t.y + a1 * t.x);
        }
        return;
    }
    for (int w = 0; w < 8; ++w) {
        const uint32_t word = w < 4 ? u.a[w & 3] : u.b[w & 3];
        const float a = lo<BF16>(word), b = hi<BF16>(word);
        const uint32_t turned = pack<BF16>(a * sc[w].y - b * sc[w].x, b * sc[w].y + a * sc[w].x);
        if (w < 4) u.a[w & 3] = turned;
        else u.b[w & 3] = turned;
    }
}

__device__ __forceinline__ Unit load_unit(const uint8_t *head, const Place &p) {
    return {*reinterpret_cast<const u32x4 *>(head + 2 * p.a), *reinterpret_cast<const u32x4 *>(head + 2 * p.b)};
}
__device__ __forceinline__ void store_unit(uint8_t *head, const Place &p, const Unit &u) {
    *reinterpret_cast<u32x4 *>(head + 2 * p.a) = u.a;
    *reinterpret_cast<u32x4 *>(head + 2 * p.b) = u.b;
}

// One row by the kThreads threads that `tid` counts: its angles once for all heads (in `sc`), then the units of its heads:
// queries, and with CACHE keys and values too.  All threads of the workgroup come here.
template <bool BF16, bool CACHE>
__device__ __forceinline__ void append_row(const AppendArgs &a, int row, int tid, f32x2 *sc) {
    const CacheArgs &c = a.c;
    const int lane = tid & 63;
    Seq s = {0, 0, 0, 0};
    const int b = row < c.num_tokens ? seq_with_row(c, row, lane) : -1;
    if (b >= 0) s = seq_of(c, b);
    const int at = s.first + row - s.row0;
    const bool mine = b >= 0 && row >= s.row0 && row < s.row0 + s.rows && at >= 0;
    const int position = mine && a.positions != nullptr ? a.positions[row] : at;
    if (mine)
        for (int i = tid; i < a.rot_half; i += kThreads) sc[i] = sin_cos(position, a.inv_freq[i]);
    workgroup_barrier();
    if (!mine) return;

    int64_t slot = -1;
    if (CACHE) {
        const int page = page_of(c, b, at);
        if (page >= 0) slot = int64_t(page) * c.page_size + (at - static_cast<int>(div_by(static_cast<uint32_t>(at), c.page_div)) * c.page_size);
    }
    const int units = c.head_dim / 16, heads = a.q_heads + (CACHE ? 2 * c.heads : 0);
    const int64_t seg = int64_t(c.head_dim) * 2, cache_row = seg * c.heads;
    for (int i = tid; i < heads * units; i += kThreads) {
        const int h = i / units, j = i - h * units, kh = h - a.q_heads, vh = kh - c.heads;
        const bool is_v = vh >= 0;
        const Place p = place_of(j, is_v ? 0 : a.rot_half, a.interleaved);
        const uint8_t *from;
        uint8_t *to;
        if (kh < 0) {
            from = a.q + row * a.q_stride + h * seg;
            to = a.q_out + row * a.q_out_stride + h * seg;
        } else {
            if (slot < 0) continue;
            from = is_v ? a.v + row * a.v_stride + vh * seg : a.k + row * a.k_stride + kh * seg;
            to = is_v ? c.v_cache + slot * cache_row + vh * seg : c.k_cache + slot * cache_row + kh * seg;
        }
        Unit u = load_unit(from, p);
        if (p.turned) turn<BF16>(u, a.interleaved, sc + 8 * j);
        store_unit(to, p, u);
    }
}

// 16-bit caches: a workgroup a row.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) append_rows(const AppendArgs a) {
    __shared__ f32x2 sc[kMostPairs];
    append_row<BF16, true>(a, static_cast<int>(blockIdx.x), static_cast<int>(threadIdx.x), sc);
}

// The smallest power of two, 2^-100 at least, with `top` within 448 of it.
__device__ __forceinline__ float scale_for(float top) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, top);
    // 448 = 1.75 * 2^8: one more where the mantissa passes 0.75
    const int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
    return __builtin_bit_cast(float, static_cast<uint32_t>((e < -100 ? -100 : e) + 127) << 23);
}

// v * inv as an e4m3 value: within +-448, NaN kept.
__device__ __forceinline__ float within(float v) { return v != v ? v : fminf(fmaxf(v, -448.0f), 448.0f); }

constexpr float kLargest = 3.402823466e38f;

__device__ __forceinline__ float finite_abs(float v) { return fabsf(v) <= kLargest ? fabsf(v) : 0.0f; }

template <bool BF16>
__device__ __forceinline__ u32x2 codes_of(u32x4 x, float inv) {
    u32x2 r;
    for (int w = 0; w < 2; ++w)
        r[w] = pack_e4m3(within(lo<BF16>(x[2 * w]) * inv), within(hi<BF16>(x[2 * w]) * inv),
                         within(lo<BF16>(x[2 * w + 1]) * inv), within(hi<BF16>(x[2 * w + 1]) * inv));
    return r;
}

// A workgroup for one page that new tokens reach, and up to kWaves of its parts, K or V of one head, one to a wave: their
// largest element, the page's scale, its older rows again where that grew, the new rows.  The angles are computed once for
// all heads, as many tokens at a time as LDS holds; a wave keeps its first kKept passes' units in registers from the
// largest element to the codes.  (16K tokens of 8 heads, 128 dims, pages of 64: 54 us with angles for each head, twice.)
template <bool BF16>
__device__ __forceinline__ void append_page(const AppendArgs &a, int group, f32x2 *angles) {
    const CacheArgs &c = a.c;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = wave_first(tid >> 6);
    const int groups = (2 * c.heads + kWaves - 1) / kWaves;
    int item = group / groups;
    const int part = (group - item * groups) * kWaves + wave, h = part >> 1;
    const bool is_v = (part & 1) != 0;
    // The item-th page of all that sequences reach, in order.
    int b = -1, page_at = 0;
    for (int i = 0; i < c.num_seqs && b < 0; i += 64) {
        int pages = 0, first = 0;
        if (i + lane < c.num_seqs) {
            const Seq s = seq_of(c, i + lane);
            const int from = s.first > 0 ? s.first : 0, to = s.first + s.rows;    // tokens [from, to)
            if (to > from) {
                first = static_cast<int>(div_by(static_cast<uint32_t>(from), c.page_div));
                pages = static_cast<int>(div_by(static_cast<uint32_t>(to - 1), c.page_div)) - first + 1;
            }
        }
        const int upto = lanes_upto(pages, lane);
        const uint64_t behind = wave_ballot(upto > item);
        if (behind != 0) {
            const int at = __builtin_ctzll(behind);
            b = i + at;
            page_at = wave_read(first, at) + item - (wave_read(upto, at) - wave_read(pages, at));
        }
        item -= wave_read(upto, 63);
    }
    if (b < 0) return;
    const Seq s = seq_of(c, b);
    const int P = c.page_size, begin = page_at * P;
    const int from = s.first > begin ? s.first : begin, to = s.first + s.rows < begin + P ? s.first + s.rows : begin + P;
    const int page = page_of(c, b, begin);
    if (page < 0) return;

    const int units = c.head_dim / 16;
    int span = 1;                            // lanes of a row
    while (span < units) span *= 2;
    const int per_pass = 64 / span, j = lane & (span - 1), sub = lane / span;
    const bool mine = part < 2 * c.heads && j < units;
    const int64_t seg = c.head_dim, cache_row = seg * c.heads;
    uint8_t *cache = (is_v ? c.v_cache : c.k_cache) + (int64_t(page) * P) * cache_row + h * seg;
    const uint8_t *in = (is_v ? a.v : a.k) + h * seg * 2;
    const int64_t in_stride = is_v ? a.v_stride : a.k_stride;
    const Place p = place_of(j < units ? j : 0, is_v ? 0 : a.rot_half, a.interleaved);
    // Tokens whose angles LDS holds; without, so many that places and a step more stay below 2^31 (contexts end 4096 before it).
    const int at_once = a.rot_half == 0 ? 4096 : kAngles / a.rot_half;
    auto put_angles = [&](int t0) {          // of tokens t0 on
        workgroup_barrier();
        const int n = (to - t0 < at_once ? to - t0 : at_once) * a.rot_half;
        for (int i = tid; i < n; i += kPageThreads) {
            const int t = i / a.rot_half, row = s.row0 + (t0 + t - s.first);
            angles[i] = sin_cos(a.positions != nullptr ? a.positions[row] : t0 + t, a.inv_freq[i - t * a.rot_half]);
        }
        workgroup_barrier();
    };
    auto fetch = [&](int t, int t0) {        // the lane's unit of context token t, rotated, in the model's type
        Unit u = load_unit(in + (s.row0 + (t - s.first)) * in_stride, p);
        if (p.turned) turn<BF16>(u, a.interleaved, angles + (t - t0) * a.rot_half + 8 * j);
        return u;
    };
    float *at = (is_v ? c.v_scale : c.k_scale) + page * c.scale_stride + (part < 2 * c.heads ? h : 0);
    const float was = from != begin && part < 2 * c.heads ? *at : 0.0f;   // read by all lanes before one of them writes it
    float top = 0;
    Unit kept[kKept];
    auto look = [&](const Unit &u) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            top = fmaxf(top, fmaxf(finite_abs(lo<BF16>(u.a[w])), finite_abs(hi<BF16>(u.a[w]))));
            top = fmaxf(top, fmaxf(finite_abs(lo<BF16>(u.b[w])), finite_abs(hi<BF16>(u.b[w]))));
        }
    };
    for (int t0 = from; t0 < to; t0 += at_once) {
        if (a.rot_half > 0) put_angles(t0);
        const int t1 = to - t0 < at_once ? to : t0 + at_once;
        if (!mine) continue;
        int t = t0 + sub;
        if (t0 == from)
#pragma unroll
            for (int i = 0; i < kKept; ++i, t += per_pass)
                if (t < t1) look(kept[i] = fetch(t, t0));
        for (; t < t1; t += per_pass) look(fetch(t, t0));
    }
    for (int by = 1; by < 64; by *= 2) top = fmaxf(top, lane_xor(top, by));
    float scale = scale_for(top);
    if (from != begin) {
        // Not one that nothing can be divided by (a page of zeros from elsewhere may have 0).
        const float size = fabsf(was);
        if (size >= 0x1p-100f && size <= kLargest && top <= 448.0f * size) {
            scale = was;
        } else {
            const float by = was / scale;    // below one in size, or infinite or NaN
            for (int t = sub; t < from - begin; t += per_pass) {
                if (!mine) continue;
                u32x4 *row = reinterpret_cast<u32x4 *>(cache + t * cache_row + 16 * j);
                u32x4 x = *row;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x2 l = e4m3_f32<false>(x[w]), m = e4m3_f32<true>(x[w]);
                    x[w] = pack_e4m3(within(l.x * by), within(l.y * by), within(m.x * by), within(m.y * by));
                }
                *row = x;
            }
        }
    }
    if (lane == 0 && part < 2 * c.heads && scale != was) *at = scale;
    const float inv = 1.0f / scale;
    auto put = [&](int t, const Unit &u) {
        uint8_t *row = cache + (t - begin) * cache_row;
        *reinterpret_cast<u32x2 *>(row + p.a) = codes_of<BF16>(u.a, inv);
        *reinterpret_cast<u32x2 *>(row + p.b) = codes_of<BF16>(u.b, inv);
    };
    for (int t0 = from; t0 < to; t0 += at_once) {
        if (a.rot_half > 0 && to - from > at_once) put_angles(t0);
        const int t1 = to - t0 < at_once ? to : t0 + at_once;
        if (!mine) continue;
        int t = t0 + sub;
        if (t0 == from)
#pragma unroll
            for (int i = 0; i < kKept; ++i, t += per_pass)
                if (t < t1) put(t, kept[i]);
        for (; t < t1; t += per_pass) put(t, fetch(t, t0));
    }
}

// e4m3 caches: first the pages, then the queries' rows, kPageThreads / kThreads to a workgroup.
template <bool BF16>
__global__ void __launch_bounds__(kPageThreads) append_pages(const AppendArgs a) {
    __shared__ f32x2 angles[kAngles];
    const int groups = a.page_items * ((2 * a.c.heads + kWaves - 1) / kWaves), group = static_cast<int>(blockIdx.x) - groups;
    if (group < 0) {
        append_page<BF16>(a, static_cast<int>(blockIdx.x), angles);
    } else {
        const int tid = static_cast<int>(threadIdx.x), in_group = wave_first(tid / kThreads);
        append_row<BF16, false>(a, group * (kPageThreads / kThreads) + in_group, tid - in_group * kThreads, angles + in_group * kMostPairs);
    }
}

template <bool BF16>
hipError_t launch(const AppendArgs &a, bool e4m3, hipStream_t stream) {
    const dim3 groups(static_cast<unsigned>(append_threads(a, e4m3) / (e4m3 ? kPageThreads : kThreads)));
    if (e4m3) hipLaunchKernelGGL((append_pages<BF16>), groups, dim3(kPageThreads), 0, stream, a);
    else hipLaunchKernelGGL((append_rows<BF16>), groups, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

int64_t append_threads(const AppendArgs &a, bool e4m3) {
    const int64_t n = a.c.num_tokens;
    if (!e4m3) return n * kThreads;
    const int64_t rows = kPageThreads / kThreads;
    return (int64_t(a.page_items) * ((2 * a.c.heads + kWaves - 1) / kWaves) + (a.q_heads > 0 ? (n + rows - 1) / rows : 0)) * kPageThreads;
}

hipError_t launch_append(const AppendArgs &a, int32_t dtype, bool e4m3, hipStream_t stream) {
    return dtype == KVIO_BF16 ? launch<true>(a, e4m3, stream) : launch<false>(a, e4m3, stream);
}

}  // namespace kvio
