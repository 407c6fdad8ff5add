// kvio_lane.h -- the instructions that the cache kernels name, on the CPU (the
// kernels' own kvio_lane.h stands for gfx950).  A workgroup's waves take turns
// between barriers, the lanes of a wave between the operations that join them;
// lanes that wait at different ones, or waves of which some wait at a barrier
// that others never reach, are errors.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#define __shared__ static
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(k, grid, block, lds, stream, ...) \
    emu_attn_launch(grid, block, [=] { (k)(__VA_ARGS__); })

void emu_attn_launch(dim3 grid, dim3 block, const std::function<void()> &lane);
// Every lane brings `bytes` bytes; the address of all 64 lanes', 64 bytes apart.
const char *emu_attn_join(const void *mine, size_t bytes, const char *what);
void emu_attn_barrier();
int emu_attn_lane();

namespace kvio {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

inline float bf16_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
inline float bf16_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
inline uint32_t emu_bf16(float f) {
    const uint32_t u = __builtin_bit_cast(uint32_t, f);
    if (f != f) return (u >> 16) | 0x40u;
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}
inline uint32_t pack_bf16(float a, float b) { return emu_bf16(a) | (emu_bf16(b) << 16); }
inline float f16_lo(uint32_t w) { return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(w))); }
inline float f16_hi(uint32_t w) { return f16_lo(w >> 16); }
inline uint32_t emu_f16(float f) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(f)); }
inline uint32_t pack_f16(float a, float b) { return emu_f16(a) | (emu_f16(b) << 16); }

inline float emu_e4m3_value(uint32_t c) {
    const int e = (c >> 3) & 15, m = c & 7;
    if (e == 15 && m == 7) return __builtin_nanf("");
    const float v = e ? ldexpf(1.0f + m / 8.0f, e - 7) : ldexpf(m / 8.0f, -6);
    return c & 128 ? -v : v;
}
inline uint32_t emu_e4m3(float f) {
    if (f != f) return 0x7f;
    const uint32_t sign = signbit(f) ? 128 : 0;
    const float a = fabsf(f);
    int e;
    (void)frexpf(a, &e);
    e = a == 0 || e - 1 < -6 ? -6 : e - 1;
    const float steps = nearbyintf(ldexpf(a, 3 - e));            // of 2^(e - 3), to nearest even
    const float v = ldexpf(steps, e - 3);
    if (v > 448) return sign | 0x7f;
    for (uint32_t c = 0; c < 0x7f; ++c)
        if (emu_e4m3_value(c) == v) return sign | c;
    return sign | 0x7f;
}
inline uint32_t pack_e4m3(float a, float b, float c, float d) {
    return emu_e4m3(a) | (emu_e4m3(b) << 8) | (emu_e4m3(c) << 16) | (emu_e4m3(d) << 24);
}
template <bool HIGH>
f32x2 e4m3_f32(uint32_t w) {
    const uint32_t h = HIGH ? w >> 16 : w;
    return f32x2{emu_e4m3_value(h & 255), emu_e4m3_value((h >> 8) & 255)};
}

template <bool BF16, bool HIGH>
uint32_t e4m3_16(uint32_t w) {
    const f32x2 v = e4m3_f32<HIGH>(w);
    return BF16 ? pack_bf16(v.x, v.y) : pack_f16(v.x, v.y);
}
inline uint32_t larger_halves(uint32_t a, uint32_t b) {
    const uint32_t l = (a & 0xffffu) > (b & 0xffffu) ? a & 0xffffu : b & 0xffffu, h = a >> 16 > b >> 16 ? a >> 16 : b >> 16;
    return l | (h << 16);
}
inline uint32_t bytes_of(uint32_t a, uint32_t b, uint32_t sel) {
    const uint64_t all = (uint64_t(a) << 32) | b;
    uint32_t r = 0;
    for (int i = 0; i < 4; ++i) r |= static_cast<uint32_t>((all >> (8 * ((sel >> (8 * i)) & 7))) & 255) << (8 * i);
    return r;
}
template <bool BF16>
float emu_16(const uint32_t *words, int i) {
    const uint32_t w = words[i / 2];
    return i & 1 ? (BF16 ? bf16_hi(w) : f16_hi(w)) : (BF16 ? bf16_lo(w) : f16_lo(w));
}
// The lane's 8 elements of each operand go to the others as floats.
template <bool BF16>
const char *emu_operands(u32x4 a, u32x4 b, const char *what) {
    uint32_t words[8];
    float both[16];
    memcpy(words, &a, 16);
    memcpy(words + 4, &b, 16);
    for (int i = 0; i < 16; ++i) both[i] = emu_16<BF16>(words, i);
    return emu_attn_join(both, sizeof both, what);
}
inline const float *emu_of(const char *all, int lane) { return reinterpret_cast<const float *>(all + lane * 64); }
template <bool BF16>
f32x4 product16(u32x4 a, u32x4 b, f32x4 c) {
    const char *all = emu_operands<BF16>(a, b, "product16");
    const int l = emu_attn_lane();
    for (int g = 0; g < 4; ++g) {
        const float *y = emu_of(all, 16 * g + l % 16) + 8;
        for (int r = 0; r < 4; ++r) {
            const float *x = emu_of(all, 16 * g + 4 * (l / 16) + r);
            for (int i = 0; i < 8; ++i) c[r] += x[i] * y[i];
        }
    }
    return c;
}
template <bool BF16>
f32x16 product32(u32x4 a, u32x4 b, f32x16 c) {
    const char *all = emu_operands<BF16>(a, b, "product32");
    const int l = emu_attn_lane();
    for (int g = 0; g < 2; ++g) {
        const float *y = emu_of(all, 32 * g + l % 32) + 8;
        for (int r = 0; r < 16; ++r) {
            const float *x = emu_of(all, 32 * g + 8 * (r / 4) + 4 * (l / 32) + r % 4);
            float sum = 0;
            for (int i = 0; i < 8; ++i) sum += x[i] * y[i];
            c[r] += sum;
        }
    }
    return c;
}
// Each group of 16 lanes: lane 4 r + i names elements 4 i .. 4 i + 3 of row r, and gets element 4 r + i of all four.
inline u32x2 lds_turned(const uint8_t *p) {
    uint16_t mine[4], got[4];
    memcpy(mine, p, 8);
    const char *all = emu_attn_join(mine, sizeof mine, "lds_turned");
    const int l = emu_attn_lane(), i = l % 16;
    for (int r = 0; r < 4; ++r) memcpy(&got[r], all + (l - i + 4 * r + i / 4) * 64 + 2 * (i % 4), 2);
    u32x2 v;
    memcpy(&v, got, 8);
    return v;
}

template <class T>
T emu_from(T v, int lane, const char *what) {
    const char *all = emu_attn_join(&v, sizeof v, what);
    T r;
    memcpy(&r, all + (lane & 63) * 64, sizeof r);
    return r;
}
inline float lane_xor(float v, int mask) { return emu_from(v, emu_attn_lane() ^ mask, "lane_xor"); }
inline int lane_read(int v, int lane) { return emu_from(v, lane, "lane_read"); }
inline int wave_read(int v, int lane) { return emu_from(v, lane, "wave_read"); }
int wave_first(int v);
uint64_t wave_ballot(bool v);
inline bool wave_any(bool v) { return wave_ballot(v) != 0; }
inline int lane_xor(int v, int mask) { return emu_from(v, emu_attn_lane() ^ mask, "lane_xor"); }
inline int lane_up(int v, int by) { return emu_from(v, emu_attn_lane() < by ? emu_attn_lane() : emu_attn_lane() - by, "lane_up"); }
inline float exp2_fast(float v) { return exp2f(v); }
inline float larger(float a, float b) { return a != a ? a : b != b ? b : a > b ? a : b; }
inline float log2_fast(float v) { return log2f(v); }
inline f32x2 sin_cos_of(float revolutions) {
    const double t = 6.283185307179586476925 * revolutions;
    return f32x2{static_cast<float>(sin(t)), static_cast<float>(cos(t))};
}
inline void in_order() {}
template <class T>
void keep_here(T &) {}
inline void wave_lds_fence() { wave_ballot(true); }
inline void workgroup_barrier() { emu_attn_barrier(); }

}  // namespace kvio
