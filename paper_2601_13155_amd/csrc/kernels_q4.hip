// Matrices in 4 bits and their products with one to sixteen vectors.
#include "spts_fp4.h"
#include "spts_lanes.h"

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

// y = x W^T on the matrix cores for up to 16 vectors: a row of W is an operand row (lane l16), a vector a column, and lane group kg takes 32 of a tile's 128 k:
// one stored block, so that a 16-byte load brings four operands of one scale each, already where the matrix core wants them, and the decoder's
// bf16 pairs are the operand.  Vectors are read from the caches (lanes without a vector feed zeros); an fp32 vector is taken as three bf16 parts, which is all
// of its 24 bits.  The NW wavefronts of a workgroup share the slabs of NS strips in turn and meet in LDS; the order of a row's sum depends on K alone.
template <typename T, int MODE, int NS, int NW>
__global__ void __launch_bounds__(NW * 64) q4_matvec_kernel(Q4Args a) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NP = F32 ? 3 : 1;
    __shared__ __attribute__((aligned(16))) float sred[NW][NS][16][20];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, kg = lane >> 4;
    const int slabs = (int)((a.K + Q4_SLAB - 1) / Q4_SLAB), K = (int)a.K;
    int64_t blk = blockIdx.x;
    int which = 0;
    if (MODE != Q4_SILU)
        while (which < 2 && blk >= (a.rows[which] + 16 * NS - 1) / (16 * NS)) blk -= (a.rows[which++] + 16 * NS - 1) / (16 * NS);
    const u32x4* codes[NS];
    const uint32_t* scales[NS];
    const int64_t last = (a.rows[which] + 15) / 16 - 1;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int64_t strip = MODE == Q4_SILU ? blk : blk * NS + s < last ? blk * NS + s : last;
        const int m = MODE == Q4_SILU ? s : which;
        codes[s] = (const u32x4*)a.codes[m] + strip * slabs * 256;
        scales[s] = (const uint32_t*)a.scales[m] + strip * slabs * 64;
    }
    const bool vec = l16 < a.nb;
    const T* const x = (const T*)a.x + (int64_t)(vec ? l16 : 0) * K + kg * 32;
    mfma_f32x4 acc[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) acc[s] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 cn[NS][4];
    uint32_t sn[NS];
    auto load = [&](int slab) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
#pragma unroll
            for (int t = 0; t < 4; ++t) cn[s][t] = __builtin_nontemporal_load(codes[s] + (slab * 4 + t) * 64 + lane);
            sn[s] = __builtin_nontemporal_load(scales[s] + slab * 64 + lane);
        }
    };
    if (wave < slabs) load(wave);
    for (int slab = wave; slab < slabs; slab += NW) {
        u32x4 c[NS][4];
        uint32_t sc[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
#pragma unroll
            for (int t = 0; t < 4; ++t) c[s][t] = cn[s][t];
            sc[s] = sn[s];
        }
        const int k0 = slab * Q4_SLAB;
        auto multiply = [&](int t, int i, const u32x4 (&xf)[NP]) {
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const float scale = __uint_as_float(t == 0 ? sc[s] << 23 : t == 1 ? sc[s] << 15 : t == 2 ? sc[s] << 7 : sc[s] >> 1);
                const u32x4 w = fp4_decode8_bf16(c[s][t][i], scale);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) acc[s] = mfma16(w, xf[p], acc[s]);
            }
        };
        if constexpr (F32) {
            if (slab + NW < slabs) load(slab + NW);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = t * 128 + 8 * i;
                    const bool in = vec && k0 + kg * 32 + k < K;
                    const f32x4* p = reinterpret_cast<const f32x4*>(x + k0 + k);
                    const f32x4 lo = in ? p[0] : f32x4{0.f, 0.f, 0.f, 0.f}, hi = in ? p[1] : f32x4{0.f, 0.f, 0.f, 0.f};
                    const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                    u32x4 xf[NP];
                    bf16_parts<NP>(v, xf);
                    multiply(t, i, xf);
                }
        } else {
            u32x4 xv[4][4];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = t * 128 + 8 * i;
                    xv[t][i] = vec && k0 + kg * 32 + k < K ? *reinterpret_cast<const u32x4*>(x + k0 + k) : u32x4{0, 0, 0, 0};
                }
            if (slab + NW < slabs) load(slab + NW);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u32x4 xf[NP] = {xv[t][i]};
                    multiply(t, i, xf);
                }
        }
    }
    // lane (vector l16, row group kg) holds rows 4 kg .. 4 kg + 3 of its strips
#pragma unroll
    for (int s = 0; s < NS; ++s) *reinterpret_cast<mfma_f32x4*>(&sred[wave][s][l16][4 * kg]) = acc[s];
    __syncthreads();
    constexpr int OUT = MODE == Q4_SILU ? 1 : NS;
    for (int t = tid; t < OUT * 256; t += NW * 64) {
        const int r = t & 15, s = (t >> 4) % OUT, b = t / (16 * OUT);
        const int64_t row = (MODE == Q4_SILU ? blk : blk * NS + s) * 16 + r;
        if (b >= a.nb || row >= a.rows[which]) continue;
        float v = 0.f, u = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            v += sred[w][s][b][r];
            if (MODE == Q4_SILU) u += sred[w][NS - 1][b][r];
        }
        const int64_t at = (int64_t)b * a.rows[which] + row;
        if (MODE == Q4_F32) ((float*)a.y[which])[at] = v;
        else {
            T* y = (T*)a.y[which] + at;
            *y = from_f32<T>(MODE == Q4_SILU ? v / (1.0f + __expf(-v)) * u : MODE == Q4_RESID ? to_f32(*y) + v : v);
        }
    }
}

template <typename T>
static hipError_t launch_q4_matvec_t(const Q4Args& a, hipStream_t s) {
    constexpr int NW = 8;
    auto blocks = [&](int ns) {
        int64_t n = 0;
        for (int i = 0; i < 3; ++i) n += (a.rows[i] + 16 * ns - 1) / (16 * ns);
        return n;
    };
    const dim3 b(NW * 64);
    if (a.mode == Q4_SILU) {
        if (a.rows[0] > 0) q4_matvec_kernel<T, Q4_SILU, 2, NW><<<dim3((unsigned)((a.rows[0] + 15) / 16)), b, 0, s>>>(a);
        return hipGetLastError();
    }
    if (blocks(1) == 0) return hipSuccess;
    const dim3 g((unsigned)blocks(1));
    switch (a.mode) {
        case Q4_STORE: q4_matvec_kernel<T, Q4_STORE, 1, NW><<<g, b, 0, s>>>(a); break;
        case Q4_F32: q4_matvec_kernel<T, Q4_F32, 1, NW><<<g, b, 0, s>>>(a); break;
        case Q4_RESID: q4_matvec_kernel<T, Q4_RESID, 1, NW><<<g, b, 0, s>>>(a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

hipError_t launch_q4_matvec(const Q4Args& a, bool bf16, hipStream_t s) {
    if (a.nb < 1 || a.nb > DECODE_MAX_BATCH) return hipErrorInvalidValue;
    return bf16 ? launch_q4_matvec_t<bf16_t>(a, s) : launch_q4_matvec_t<float>(a, s);
}

}  // namespace spts
