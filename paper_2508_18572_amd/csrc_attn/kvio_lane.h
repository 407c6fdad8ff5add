// kvio_lane.h -- what the cache kernels take from the gfx950 instruction set, by
// one name each, so that the CPU tests can put plain code in its place.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kvio {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// ---- 16-bit elements, two to a word, low half first ----------------------------------
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2 v = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float f16_lo(uint32_t w) { return static_cast<float>(__builtin_bit_cast(f16x2, w).x); }
__device__ __forceinline__ float f16_hi(uint32_t w) { return static_cast<float>(__builtin_bit_cast(f16x2, w).y); }
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const f16x2 v = {static_cast<_Float16>(a), static_cast<_Float16>(b)};
    return __builtin_bit_cast(uint32_t, v);
}

// ---- e4m3 ----------------------------------------------------------------------------
// Four codes of values within [-448, 448] or NaN, to nearest even.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}
template <bool HIGH>
__device__ __forceinline__ f32x2 e4m3_f32(uint32_t w) { return __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), HIGH); }

// The two codes in the low (HIGH: high) half of w, in the 16-bit type of Q; exact.
template <bool BF16, bool HIGH>
__device__ __forceinline__ uint32_t e4m3_16(uint32_t w) {
    if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HIGH));
}

// The larger of each half, as whole numbers.
__device__ __forceinline__ uint32_t larger_halves(uint32_t a, uint32_t b) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// Byte i of the result is byte (sel >> 8 i) & 7 of the eight in b (0 to 3) and a (4 to 7).
__device__ __forceinline__ uint32_t bytes_of(uint32_t a, uint32_t b, uint32_t sel) { return __builtin_amdgcn_perm(a, b, sel); }

// ---- matrix products -----------------------------------------------------------------
// c + A B, 16-bit elements, fp32 sums.
// 16x16 from 32: lane l brings row l % 16 of A and column l % 16 of B, their elements
// 8 (l / 16) .. + 7 along the sum; it gets column l % 16, rows 4 (l / 16) .. + 3.
template <bool BF16>
__device__ __forceinline__ f32x4 product16(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// 32x32 from 16: row and column l % 32, elements 8 (l / 32) .. + 7; it gets column l % 32,
// rows 8 (i / 4) + 4 (l / 32) + i % 4 for i = 0 .. 15.
template <bool BF16>
__device__ __forceinline__ f32x16 product32(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Four 16-bit elements a lane from LDS, turned: each group of 16 lanes names 4 rows of 16 elements, lane i the elements
// 4 (i % 4) .. + 3 of row i / 4, and lane i gets element i of the rows, in their order.
__device__ __forceinline__ u32x2 lds_turned(const uint8_t *p) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p)));
}

// ---- between lanes -------------------------------------------------------------------
__device__ __forceinline__ float lane_xor(float v, int mask) { return __shfl_xor(v, mask); }
__device__ __forceinline__ int lane_read(int v, int lane) { return __shfl(v, lane); }       // `lane` may differ by lane
__device__ __forceinline__ int wave_read(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }   // the same for all
__device__ __forceinline__ int wave_first(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint64_t wave_ballot(bool v) { return __ballot(v); }
__device__ __forceinline__ bool wave_any(bool v) { return __any(v); }
__device__ __forceinline__ int lane_xor(int v, int mask) { return __shfl_xor(v, mask); }
__device__ __forceinline__ int lane_up(int v, int by) { return __shfl_up(v, by); }
__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float log2_fast(float v) { return __builtin_amdgcn_logf(v); }
// The larger one; NaN if either is (one instruction, where fmaxf first has to quiet signalling ones).
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// Sine and cosine of so many revolutions, up to half of one either way.
__device__ __forceinline__ f32x2 sin_cos_of(float revolutions) {
    float s, c;
    sincospif(2 * revolutions, &s, &c);
    return f32x2{s, c};
}
// The compiler moves nothing past this.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }
// v is computed here, not later where it is first used.
template <class T>
__device__ __forceinline__ void keep_here(T &v) { asm volatile("" : "+v"(v)); }
// What lanes of a wave wrote to LDS before is there for its others after.
__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ void workgroup_barrier() { __syncthreads(); }

}  // namespace kvio
