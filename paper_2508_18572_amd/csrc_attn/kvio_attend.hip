// kvio_attend.hip -- causal attention of new tokens over the pages of their
// contexts, the cache in 16 bits or in e4m3 with a scale for each page and head.
#include "kvio_attend.h"

namespace kvio {
namespace {

// One wave for one row and query head: 64 keys at a time, a key a lane for the
// scores, D / 64 dims a lane for the values.
template <bool BF16, bool E4M3, int D>
__global__ void __launch_bounds__(64) attend_rows(const AttendArgs a) {
    constexpr int kDims = D / 64;
    const CacheArgs &c = a.c;
    const int lane = static_cast<int>(threadIdx.x), row = static_cast<int>(blockIdx.x) / a.q_heads;
    const int qh = static_cast<int>(blockIdx.x) - row * a.q_heads, h = qh / a.group;
    const int b = seq_with_row(c, row, lane);
    if (b < 0) return;
    const Seq s = seq_of(c, b);
    if (row < s.row0 || row >= s.row0 + s.rows) return;
    const int last = s.first + row - s.row0;           // the row's own place
    const int first = a.window > 0 && last - a.window + 1 > 0 ? last - a.window + 1 : 0;
    const int64_t seg = int64_t(D) * (E4M3 ? 1 : 2), cache_row = seg * c.heads;
    const uint32_t *q = reinterpret_cast<const uint32_t *>(a.q + row * a.q_stride + int64_t(qh) * D * 2);
    float best = kMinusInf, sum = 0, acc[kDims] = {};
    for (int t0 = first; t0 <= last; t0 += 64) {
        const int t = t0 + lane;
        int64_t slot = -1;
        float score = kMinusInf, v_scale = 1;
        if (t <= last) {
            const int page = page_of(c, b, t);
            if (page >= 0) {
                slot = int64_t(page) * c.page_size + (t - static_cast<int>(div_by(static_cast<uint32_t>(t), c.page_div)) * c.page_size);
                const uint32_t *k = reinterpret_cast<const uint32_t *>(c.k_cache + slot * cache_row + h * seg);
                float dot = 0;
                for (int w = 0; w < D / 2; ++w) {
                    const uint32_t x = q[w];
                    float k0, k1;
                    if (E4M3) {
                        const f32x2 v = w & 1 ? e4m3_f32<true>(k[w / 2]) : e4m3_f32<false>(k[w / 2]);
                        k0 = v.x, k1 = v.y;
                    } else {
                        k0 = BF16 ? bf16_lo(k[w]) : f16_lo(k[w]), k1 = BF16 ? bf16_hi(k[w]) : f16_hi(k[w]);
                    }
                    dot += (BF16 ? bf16_lo(x) : f16_lo(x)) * k0 + (BF16 ? bf16_hi(x) : f16_hi(x)) * k1;
                }
                if (E4M3) {
                    dot *= c.k_scale[page * c.scale_stride + h];
                    v_scale = c.v_scale[page * c.scale_stride + h];
                }
                score = dot * a.scale_log2;
            }
        }
        float top = score;
        for (int by = 1; by < 64; by *= 2) top = fmaxf(top, lane_xor(top, by));
        if (top > best) {
            const float less = exp2_fast(best - top);
            sum *= less;
            for (int d = 0; d < kDims; ++d) acc[d] *= less;
            best = top;
        }
        const float p = slot >= 0 && best != kMinusInf ? exp2_fast(score - best) : 0.0f;
        float all = p;
        for (int by = 1; by < 64; by *= 2) all += lane_xor(all, by);
        sum += all;
        for (int i = 0; i < 64; ++i) {
            const float w = __builtin_bit_cast(float, lane_read(__builtin_bit_cast(int, p * v_scale), i));
            const int lo = lane_read(static_cast<int>(slot), i), hi = lane_read(static_cast<int>(slot >> 32), i);
            const int64_t at = (int64_t(hi) << 32) | static_cast<uint32_t>(lo);
            if (at < 0) continue;
            const uint8_t *v = c.v_cache + at * cache_row + h * seg;
            for (int d = 0; d < kDims; ++d) {
                const int e = d * 64 + lane;
                float x;
                if (E4M3) x = e4m3_f32<false>(v[e]).x;
                else {
                    const uint32_t u = reinterpret_cast<const uint16_t *>(v)[e];
                    x = BF16 ? bf16_lo(u) : f16_lo(u);
                }
                acc[d] += w * x;
            }
        }
    }
    for (int d = 0; d < kDims; ++d) {
        const float v = sum > 0 ? acc[d] / sum : sum != sum ? sum : 0.0f;
        reinterpret_cast<uint16_t *>(a.out + row * a.out_stride + int64_t(qh) * D * 2)[d * 64 + lane] =
            static_cast<uint16_t>(BF16 ? pack_bf16(v, 0) : pack_f16(v, 0));
    }
    if (a.lse != nullptr && lane == 0) a.lse[int64_t(row) * a.q_heads + qh] = (best + log2_fast(sum)) * 0.69314718055994530942f;
}

template <bool BF16, bool E4M3>
hipError_t launch(const AttendArgs &a, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(a.c.num_tokens) * static_cast<unsigned>(a.q_heads));
    if (a.c.head_dim == 64) hipLaunchKernelGGL((attend_rows<BF16, E4M3, 64>), grid, dim3(64), 0, stream, a);
    else if (a.c.head_dim == 128) hipLaunchKernelGGL((attend_rows<BF16, E4M3, 128>), grid, dim3(64), 0, stream, a);
    else hipLaunchKernelGGL((attend_rows<BF16, E4M3, 256>), grid, dim3(64), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(const AttendArgs &a, const AttendPlan &plan, int32_t dtype, bool e4m3, hipStream_t stream) {
    if (plan.few) return launch_steps(a, plan, dtype, e4m3, stream);
    if (dtype == KVIO_BF16) return e4m3 ? launch<true, true>(a, stream) : launch<true, false>(a, stream);
    return e4m3 ? launch<false, true>(a, stream) : launch<false, false>(a, stream);
}

}  // namespace kvio
