// The 4-bit form of matrices and caches: blocks of 32 values share a power of two 2^e and each value is one of
// +-{0, 1/2, 1, 3/2, 2, 3, 4, 6} * 2^e (E2M1 codes, sign in bit 3; e stored as the byte e + 127).  e is the smallest exponent with
// max|v| <= 6 * 2^e, within [-126, 125]; a value goes to the nearest of the grid, ties to the even code.  Multiplying by a power of
// two is exact, so the codes do not depend on the order or the width of the arithmetic, and what they stand for is exact in bf16
// and fp32.  A block that holds a NaN gets the byte 255 and reads as NaN throughout.
// The chip's own converters do the rounding and the way back, two values an instruction: they take the scale as a float and look
// at its exponent field only (255 reads as NaN), so that a byte of a word is put there by one shift.
#pragma once
#include "spts_internal.h"

namespace spts {

constexpr int FP4_BLOCK = 32;

// the scale byte of a block from the largest of its values' bit patterns without sign (of fp32)
__device__ inline uint32_t fp4_scale_byte(uint32_t amax_bits) {
    if (amax_bits > 0x7f800000u) return 255u;
    const int e = (int)((amax_bits + 0x3fffffu) >> 23) - 2;   // 6 = 1.5 * 2^2: one more where the significand is above 1.5
    return (uint32_t)(e < 1 ? 1 : e > 252 ? 252 : e);
}
// byte i of w as a scale for the converters (bits beside the exponent field are those of the neighbours)
template <int I> __device__ inline float fp4_scale_of(uint32_t w) { return __uint_as_float(I == 0 ? w << 23 : I == 1 ? w << 15 : I == 2 ? w << 7 : w >> 1); }

// eight fp32 values -> eight codes, value i in bits 4i .. 4i + 3
__device__ inline uint32_t fp4_encode8(const float* v, float scale) {
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], scale, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], scale, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], scale, 3);
    return q;
}
typedef float fp4_f32x2 __attribute__((ext_vector_type(2)));
// codes 2 I and 2 I + 1 of w as fp32 / as two bf16
template <int I> __device__ inline fp4_f32x2 fp4_pair(uint32_t w, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, I); }
template <int I> __device__ inline uint32_t fp4_pair_bf16(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, I));
}
// eight codes as fp32
__device__ inline void fp4_decode8(uint32_t w, float scale, float* v) {
    fp4_f32x2 p;
    p = fp4_pair<0>(w, scale); v[0] = p[0]; v[1] = p[1];
    p = fp4_pair<1>(w, scale); v[2] = p[0]; v[3] = p[1];
    p = fp4_pair<2>(w, scale); v[4] = p[0]; v[5] = p[1];
    p = fp4_pair<3>(w, scale); v[6] = p[0]; v[7] = p[1];
}
// eight codes as eight bf16
__device__ inline u32x4 fp4_decode8_bf16(uint32_t w, float scale) {
    return u32x4{fp4_pair_bf16<0>(w, scale), fp4_pair_bf16<1>(w, scale), fp4_pair_bf16<2>(w, scale), fp4_pair_bf16<3>(w, scale)};
}

// eight consecutive values of T that are read once
template <typename T> __device__ inline void load8(const T* p, float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    } else {
        const u32x4 a = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)), b = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(a[i]); v[4 + i] = __uint_as_float(b[i]); }
    }
}

// ------------------------------------------------------------------ matrix cores
typedef __bf16 mfma_bf16x8 __attribute__((ext_vector_type(8)));
typedef float mfma_f32x4 __attribute__((ext_vector_type(4)));

__device__ inline mfma_f32x4 mfma16(u32x4 a, u32x4 b, mfma_f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(mfma_bf16x8, a), __builtin_bit_cast(mfma_bf16x8, b), c, 0, 0, 0);
}

// eight fp32 values as N bf16 vectors whose sum they are (to 8 N bits, three are exact): every part but the last is the upper half of what is left, so that no
// finite value becomes infinite on the way.  INF: an infinity is its first part alone (the others would be NaN).
template <int N, bool INF = false>
__device__ inline void bf16_parts(const float* v, u32x4 (&out)[N]) {
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = v[j];
#pragma unroll
    for (int p = 0; p < N; ++p)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (p + 1 == N) { out[p][j] = cvt_pk_bf16(r[2 * j], r[2 * j + 1]); continue; }
            out[p][j] = __builtin_amdgcn_perm(__float_as_uint(r[2 * j + 1]), __float_as_uint(r[2 * j]), 0x07060302);
#pragma unroll
            for (int h = 2 * j; h < 2 * j + 2; ++h) {
                const float rest = r[h] - __uint_as_float(__float_as_uint(r[h]) & 0xffff0000u);
                r[h] = INF && p == 0 && fabsf(r[h]) == INFINITY ? 0.f : rest;
            }
        }
}

// the same for eight values in two registers of four: all 24 bits, infinities as they are
__device__ inline void bf16_parts3(u32x4 lo, u32x4 hi, u32x4 (&out)[3]) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[j] = __uint_as_float(lo[j]); v[4 + j] = __uint_as_float(hi[j]); }
    bf16_parts<3, true>(v, out);
}

}  // namespace spts
