// Matrices in 4 bits and their products with one to sixteen vectors.
#include "spts_fp4.h"

namespace spts {

// One thread per piece and slab: four blocks of one row, 128 values apart.
template <typename T>
__global__ void __launch_bounds__(256) q4_pack_kernel(const T* __restrict__ W, int64_t rows, int64_t K, int64_t slabs, int64_t pieces,
                                                      u32x4* __restrict__ codes, uint32_t* __restrict__ scales) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const int lane = (int)(i & 63);
    const int64_t slab = (i >> 6) % slabs, strip = (i >> 6) / slabs, row = strip * 16 + (lane & 15);
    uint32_t sc = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int64_t k0 = slab * Q4_SLAB + t * 128 + (lane >> 4) * 32;
        float v[32];
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            v[j] = row < rows && k0 + j < K ? to_f32(W[row * K + k0 + j]) : 0.f;
            const uint32_t m = __float_as_uint(v[j]) & 0x7fffffffu;
            top = m > top ? m : top;
        }
        const uint32_t byte = fp4_scale_byte(top);
        u32x4 c;
#pragma unroll
        for (int g = 0; g < 4; ++g) c[g] = fp4_encode8(v + 8 * g, __uint_as_float(byte << 23));
        codes[((i >> 6) * 4 + t) * 64 + lane] = c;
        sc |= byte << (8 * t);
    }
    scales[i] = sc;
}

hipError_t launch_q4_pack(const void* W, int64_t rows, int64_t K, void* codes, void* scales, bool bf16, hipStream_t s) {
    const int64_t pieces = (rows + 15) / 16 * q4_slabs(K) * 64;
    const dim3 g((unsigned)((pieces + 255) / 256)), b(256);
    if (bf16) q4_pack_kernel<bf16_t><<<g, b, 0, s>>>((const bf16_t*)W, rows, K, q4_slabs(K), pieces, (u32x4*)codes, (uint32_t*)scales);
    else q4_pack_kernel<float><<<g, b, 0, s>>>((const float*)W, rows, K, q4_slabs(K), pieces, (u32x4*)codes, (uint32_t*)scales);
    return hipGetLastError();
}

// One wavefront per strip and vector: a lane sums the products of its pieces, and the four lanes of a row meet at the end.
template <typename T, int MODE>
__global__ void __launch_bounds__(64) q4_matvec_kernel(Q4Args a) {
    const int lane = threadIdx.x, b = blockIdx.y;
    const int64_t slabs = (a.K + Q4_SLAB - 1) / Q4_SLAB;
    int64_t strip = blockIdx.x;
    int which = 0;
    if (MODE != Q4_SILU)
        while (which < 2 && strip >= (a.rows[which] + 15) / 16) strip -= (a.rows[which++] + 15) / 16;
    const T* x = (const T*)a.x + (int64_t)b * a.K;
    float acc[2] = {0.f, 0.f};
    for (int m = 0; m < (MODE == Q4_SILU ? 2 : 1); ++m) {
        const u32x4* codes = (const u32x4*)a.codes[which + m] + strip * slabs * 256;
        const uint32_t* scales = (const uint32_t*)a.scales[which + m] + strip * slabs * 64;
        for (int64_t slab = 0; slab < slabs; ++slab) {
            const uint32_t sc = scales[slab * 64 + lane];
            for (int t = 0; t < 4; ++t) {
                const u32x4 c = codes[(slab * 4 + t) * 64 + lane];
                const float scale = __uint_as_float(((sc >> (8 * t)) & 255u) << 23);
                const int64_t k0 = slab * Q4_SLAB + t * 128 + (lane >> 4) * 32;
                for (int g = 0; g < 4; ++g) {
                    float v[8];
                    fp4_decode8(c[g], scale, v);
                    for (int j = 0; j < 8; ++j)
                        if (k0 + 8 * g + j < a.K) acc[m] = fmaf(v[j], to_f32(x[k0 + 8 * g + j]), acc[m]);
                }
            }
        }
        acc[m] += __shfl_xor(acc[m], 16);
        acc[m] += __shfl_xor(acc[m], 32);
    }
    const int64_t row = strip * 16 + lane;
    if (lane >= 16 || row >= a.rows[which]) return;
    const int64_t at = (int64_t)b * a.rows[which] + row;
    if (MODE == Q4_F32) ((float*)a.y[which])[at] = acc[0];
    else {
        T* y = (T*)a.y[which] + at;
        *y = from_f32<T>(MODE == Q4_SILU ? acc[0] / (1.0f + __expf(-acc[0])) * acc[1] : MODE == Q4_RESID ? to_f32(*y) + acc[0] : acc[0]);
    }
}

template <typename T>
static hipError_t launch_q4_matvec_t(const Q4Args& a, hipStream_t s) {
    int64_t strips = 0;
    for (int i = 0; i < (a.mode == Q4_SILU ? 1 : 3); ++i) strips += (a.rows[i] + 15) / 16;
    if (strips == 0) return hipSuccess;
    const dim3 g((unsigned)strips, (unsigned)a.nb), b(64);
    switch (a.mode) {
        case Q4_STORE: q4_matvec_kernel<T, Q4_STORE><<<g, b, 0, s>>>(a); break;
        case Q4_F32: q4_matvec_kernel<T, Q4_F32><<<g, b, 0, s>>>(a); break;
        case Q4_RESID: q4_matvec_kernel<T, Q4_RESID><<<g, b, 0, s>>>(a); break;
        case Q4_SILU: q4_matvec_kernel<T, Q4_SILU><<<g, b, 0, s>>>(a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

hipError_t launch_q4_matvec(const Q4Args& a, bool bf16, hipStream_t s) {
    if (a.nb < 1 || a.nb > DECODE_MAX_BATCH) return hipErrorInvalidValue;
    return bf16 ? launch_q4_matvec_t<bf16_t>(a, s) : launch_q4_matvec_t<float>(a, s);
}

}  // namespace spts
