// Pieces shared by the kernels over the paged cache: 8-bit codes, rounding to the model's type, looking up
// pages and the sequence that a row of a ragged call belongs to.
#pragma once
#include "attention_common.h"

namespace leoam {

// 8-bit pages: e4m3 codes (4 exponent bits, 3 fraction bits, largest 448, no infinity), a lane moves 8 of them
struct E4M3 { static constexpr int kBytes = 1; };

typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;

// four codes of a register to floats (exact)
__device__ __forceinline__ void unpack_e4m3(uint32_t w, float* x) {
    const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}

// Four floats of at most 448 (the conversion gives NaN beyond) to four codes, round half to even; NaN stays NaN.
__device__ __forceinline__ uint32_t pack_e4m3(const float* x) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
}
// x within +-most, NaN stays NaN
__device__ __forceinline__ float clamp_nan(float x, float most) { return x > most ? most : x < -most ? -most : x; }

// floats rounded once to the model's type (half to even): the 16 bytes a lane holds of a row
template <typename T> __device__ __forceinline__ uint4 round_pack(const float* x);
template <> __device__ __forceinline__ uint4 round_pack<F32>(const float* x) { return pack<F32>(x); }
template <> __device__ __forceinline__ uint4 round_pack<F16>(const float* x) { return pack<F16>(x); }
template <> __device__ __forceinline__ uint4 round_pack<BF16>(const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bf16x2_t p;
        p.x = (__bf16)x[2 * i];
        p.y = (__bf16)x[2 * i + 1];
        w[i] = __builtin_bit_cast(uint32_t, p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Number of entries i in 1..n of an ascending list with value(i) <= x, found by the whole wave 64 entries at a
// time: the sequence that owns element x when value(i) is where sequence i begins.
template <typename F> __device__ __forceinline__ int wave_count_below(int n, int x, F&& value) {
    int found = 0;
    for (int i0 = 1; i0 <= n; i0 += LEOAM_WAVE) {
        const int i = i0 + lane_id();
        const uint64_t hit = __ballot(i <= n && value(min(i, n)) <= x);
        found += __popcll(hit);
        if (hit != ~0ull) break;
    }
    return found;
}

// a value that is the same in every lane, held once for the wave
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// eight codes to the operand type, times a power of two (exact)
template <typename T> __device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b, float scale);
template <> __device__ __forceinline__ uint4 widen8<BF16>(uint32_t a, uint32_t b, float s) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true)));
}
template <> __device__ __forceinline__ uint4 widen8<F16>(uint32_t a, uint32_t b, float s) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, s, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, s, true)));
}

// two floats rounded to the 16-bit type, and back
__device__ __forceinline__ uint32_t pair_of(BF16, float a, float b) {
    bf16x2_t p;
    p.x = (__bf16)a;
    p.y = (__bf16)b;
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ uint32_t pair_of(F16, float a, float b) {
    f16x2_t p;
    p.x = (_Float16)a;
    p.y = (_Float16)b;
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ void pair_back(BF16, uint32_t w, float& a, float& b) {
    a = bits_to_float(w << 16);
    b = bits_to_float(w & 0xffff0000u);
}
__device__ __forceinline__ void pair_back(F16, uint32_t w, float& a, float& b) {
    const f16x2_t p = __builtin_bit_cast(f16x2_t, w);
    a = (float)p.x;
    b = (float)p.y;
}

// ln(2^m l).  Where the reference m was taken `bias` below the largest logit both are brought back first: the logarithm of
// a sum near 2^bias would cost the result bits.
__device__ __forceinline__ float log_sum_exp(float m, float l, int bias) {
    return l == 0.f ? -INFINITY : ((m + (float)bias) + log2f(ldexpf(l, -bias))) * kLn2;
}

}  // namespace leoam
