// Matrices in 4 bits and their products with one to sixteen vectors.
#include "spts_fp4.h"
#include "spts_lanes.h"

namespace spts {

// One thread per piece and slab: eight values of sixteen blocks of one row; the other values of a block are 16, 32 and 48 lanes away.
template <typename T>
__global__ void __launch_bounds__(256) q4_pack_kernel(const T* __restrict__ W, int64_t rows, int64_t K, int64_t slabs, int64_t pieces,
                                                      u32x4* __restrict__ codes, uint32_t* __restrict__ scales) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;                      // (whole wavefronts)
    const int lane = (int)(i & 63), kg = lane >> 4;
    const int64_t slab = (i >> 6) % slabs, strip = (i >> 6) / slabs, row = strip * 16 + (lane & 15);
    u32x4 sc{0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        u32x4 c;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t k = slab * Q4_SLAB + t * 128 + j * 32 + kg * 8;
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (row < rows && k < K) load8(W + row * K + k, v);   // K % 8 == 0
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t m = __float_as_uint(v[e]) & 0x7fffffffu;
                top = m > top ? m : top;
            }
            uint32_t o = (uint32_t)__shfl_xor((int)top, 16);
            top = o > top ? o : top;
            o = (uint32_t)__shfl_xor((int)top, 32);
            top = o > top ? o : top;
            const uint32_t byte = fp4_scale_byte(top);
            c[j] = fp4_encode8(v, __uint_as_float(byte << 23));
            sc[t] |= byte << (8 * j);
        }
        codes[((i >> 6) * 4 + t) * 64 + lane] = c;
    }
    scales[i] = kg == 0 ? sc[0] : kg == 1 ? sc[1] : kg == 2 ? sc[2] : sc[3];   // (all four lanes of a row have all four)
}

hipError_t launch_q4_pack(const void* W, int64_t rows, int64_t K, void* codes, void* scales, bool bf16, hipStream_t s) {
    const int64_t pieces = (rows + 15) / 16 * q4_slabs(K) * 64;
    const dim3 g((unsigned)((pieces + 255) / 256)), b(256);
    if (bf16) q4_pack_kernel<bf16_t><<<g, b, 0, s>>>((const bf16_t*)W, rows, K, q4_slabs(K), pieces, (u32x4*)codes, (uint32_t*)scales);
    else q4_pack_kernel<float><<<g, b, 0, s>>>((const float*)W, rows, K, q4_slabs(K), pieces, (u32x4*)codes, (uint32_t*)scales);
    return hipGetLastError();
}

// y = x W^T on the matrix cores for up to 16 vectors: a row of W is an operand row (lane l16), a vector a column; a dword of codes is an operand's eight values of a
// lane, and the decoder's bf16 pairs are the operand.  Vectors are read from the caches, 64 bytes of each per load; an fp32 vector is taken as three bf16
// parts, which is all of its 24 bits.  The NW wavefronts of a workgroup share the slabs of NS strips in turn, each with the codes and scales of its next slab on
// their way while it works on one, and meet in LDS.  The order of a row's sum depends on K and NW alone, not on the vectors.  (Vectors asked for a slab ahead too take
// 200 registers a lane, which halves the wavefronts on a CU: 28672 x 4096, one vector, 16.0 -> 22.6 us.)
// (few arguments: quick launches)
template <int NM> struct Q4Mats { const u32x4* codes[NM]; const uint32_t* scales[NM]; void* y[NM]; int32_t rows[NM]; const void* x; int32_t K, nb; const void* gamma; float eps; };

// One vector x [K] normalised on its way in: every workgroup takes its sum of squares and leaves the normalised vector, rounded as rmsnorm_kernel does it, in LDS
// (zeros up to whole slabs), where the products read it.  The first codes are already on their way; a norm of its own would be a launch of 3 us.
template <int NW>
__device__ inline void norm_to_lds(const bf16_t* __restrict__ x, const bf16_t* __restrict__ gamma, float eps, int K, int slabs, u32x4* xl, float* red) {
    const int tid = threadIdx.x, chunks = K / 8;
    float ss = 0.f;
    for (int c = tid; c < chunks; c += NW * 64) {
        const u32x4 w = reinterpret_cast<const u32x4*>(x)[c];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = __uint_as_float(w[i] << 16), b = __uint_as_float(w[i] & 0xffff0000u);
            ss += a * a; ss += b * b;
        }
    }
    ss = wave_sum(ss);
    if ((tid & 63) == 0) red[tid >> 6] = ss;
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) ss += red[w];
    const float inv = 1.0f / sqrtf(ss / (float)K + eps);
    for (int c = tid; c < slabs * (Q4_SLAB / 8); c += NW * 64) {
        u32x4 o{0, 0, 0, 0};
        if (c < chunks) {
            const u32x4 w = reinterpret_cast<const u32x4*>(x)[c], g = reinterpret_cast<const u32x4*>(gamma)[c];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                o[i] = cvt_pk_bf16(__uint_as_float(w[i] << 16) * inv * __uint_as_float(g[i] << 16),
                                   __uint_as_float(w[i] & 0xffff0000u) * inv * __uint_as_float(g[i] & 0xffff0000u));
        }
        xl[c] = o;
    }
    __syncthreads();
}
constexpr int Q4_NORM_K = 16384;   // longest: 32 KB of LDS

template <typename T, int MODE, int NM, int NS, int NW, bool NORM>
__global__ void __launch_bounds__(NW * 64) q4_matvec_kernel(Q4Mats<NM> a) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NP = F32 ? 3 : 1, OWN = MODE == Q4_SILU ? NS / 2 : NS;   // strips of one matrix (SiLU: half are gate rows, half the same up rows)
    __shared__ __attribute__((aligned(16))) float sred[NW][NS][16][20];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, kg = lane >> 4;
    const int slabs = (a.K + Q4_SLAB - 1) / Q4_SLAB, K = a.K;
    int blk = blockIdx.x;
    int which = 0;
    if (MODE != Q4_SILU) {
#pragma unroll
        for (int i = 0; i + 1 < NM; ++i) {
            const int n = (a.rows[i] + 16 * NS - 1) / (16 * NS);
            if (which == i && blk >= n) { blk -= n; which = i + 1; }
        }
    }
    const u32x4* codes[NS];
    const uint32_t* scales[NS];
    const int last = (a.rows[which] + 15) / 16 - 1;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int at = blk * OWN + s % OWN, m = MODE == Q4_SILU ? s / OWN : which;
        const int64_t strip = at < last ? at : last;
        codes[s] = a.codes[m] + strip * slabs * 256;
        scales[s] = a.scales[m] + strip * slabs * 64;
    }
    const bool vec = l16 < a.nb;
    const T* const x = (const T*)a.x + (int64_t)(vec ? l16 : 0) * K + kg * 8;
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
    extern __shared__ u32x4 xl[];
    if constexpr (NORM) norm_to_lds<NW>((const bf16_t*)a.x, (const bf16_t*)a.gamma, a.eps, K, slabs, xl, &sred[0][0][0][0]);
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
        u32x4 xv[F32 ? 1 : 4][4];
        if constexpr (!F32) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if constexpr (NORM) xv[t][i] = vec ? xl[(k0 + t * 128 + i * 32) / 8 + kg] : u32x4{0, 0, 0, 0};
                    else xv[t][i] = vec && k0 + t * 128 + i * 32 + kg * 8 < K ? *reinterpret_cast<const u32x4*>(x + k0 + t * 128 + i * 32) : u32x4{0, 0, 0, 0};
        }
        if (slab + NW < slabs) load(slab + NW);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            uint32_t w4[NS];   // the tile's four scales of the lane's row, which lane 16 t + l16 has loaded
#pragma unroll
            for (int s = 0; s < NS; ++s) w4[s] = (uint32_t)__builtin_amdgcn_ds_bpermute((16 * t + l16) * 4, (int)sc[s]);
            f32x4 xw[F32 ? 4 : 1][2];
            if constexpr (F32) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = k0 + t * 128 + i * 32;
                    const bool in = vec && k + kg * 8 < K;
#pragma unroll
                    for (int h = 0; h < 2; ++h) xw[i][h] = in ? reinterpret_cast<const f32x4*>(x + k)[h] : f32x4{0.f, 0.f, 0.f, 0.f};
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u32x4 xf[NP];
                if constexpr (F32) {
                    const float v[8] = {xw[i][0][0], xw[i][0][1], xw[i][0][2], xw[i][0][3], xw[i][1][0], xw[i][1][1], xw[i][1][2], xw[i][1][3]};
                    bf16_parts<NP>(v, xf);
                } else xf[0] = xv[t][i];
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const u32x4 w = fp4_decode8_bf16(c[s][t][i], i == 0 ? fp4_scale_of<0>(w4[s]) : i == 1 ? fp4_scale_of<1>(w4[s]) : i == 2 ? fp4_scale_of<2>(w4[s]) : fp4_scale_of<3>(w4[s]));
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p) acc[s] = mfma16(w, xf[p], acc[s]);
                }
            }
        }
    }
    // lane (vector l16, row group kg) holds rows 4 kg .. 4 kg + 3 of its strips.  (NORM: everyone has read the norm's sums, which stood here, before the second barrier)
#pragma unroll
    for (int s = 0; s < NS; ++s) *reinterpret_cast<mfma_f32x4*>(&sred[wave][s][l16][4 * kg]) = acc[s];
    __syncthreads();
    for (int t = tid; t < OWN * 256; t += NW * 64) {
        const int r = t & 15, s = (t >> 4) % OWN, b = t / (16 * OWN);
        const int64_t row = ((int64_t)blk * OWN + s) * 16 + r;
        if (b >= a.nb || row >= a.rows[which]) continue;
        float v = 0.f, u = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            v += sred[w][s][b][r];
            if (MODE == Q4_SILU) u += sred[w][NS - OWN + s][b][r];
        }
        const int64_t at = (int64_t)b * a.rows[which] + row;
        if (MODE == Q4_F32) ((float*)a.y[which])[at] = v;
        else {
            T* y = (T*)a.y[which] + at;
            *y = from_f32<T>(MODE == Q4_SILU ? v / (1.0f + __expf(-v)) * u : MODE == Q4_RESID ? to_f32(*y) + v : v);
        }
    }
}

template <typename T, int MODE, int NM, int NS, int NW>
static hipError_t launch_q4_matvec_n(const Q4Args& a, hipStream_t s) {
    constexpr int OWN = MODE == Q4_SILU ? NS / 2 : NS;   // strips of one matrix
    Q4Mats<NM> m{};
    int64_t blocks = 0;
    for (int i = 0; i < NM; ++i) {
        m.codes[i] = (const u32x4*)a.codes[i]; m.scales[i] = (const uint32_t*)a.scales[i]; m.y[i] = a.y[i]; m.rows[i] = (int32_t)a.rows[i];
        if (MODE != Q4_SILU || i == 0) blocks += (a.rows[i] + 16 * OWN - 1) / (16 * OWN);
    }
    m.x = a.x; m.K = (int32_t)a.K; m.nb = a.nb;
    if (blocks == 0) return hipSuccess;
    if constexpr (sizeof(T) == 2 && (MODE == Q4_F32 || MODE == Q4_SILU) && NM > 1 && NS <= 2) {   // (a single vector never takes four strips)
        if (a.gamma) {
            m.gamma = a.gamma; m.eps = a.eps;
            const int lds = (m.K + Q4_SLAB - 1) / Q4_SLAB * Q4_SLAB * 2;
            q4_matvec_kernel<T, MODE, NM, NS, NW, true><<<dim3((unsigned)blocks), dim3(NW * 64), lds, s>>>(m);
            return hipGetLastError();
        }
    }
    q4_matvec_kernel<T, MODE, NM, NS, NW, false><<<dim3((unsigned)blocks), dim3(NW * 64), 0, s>>>(m);
    return hipGetLastError();
}

template <typename T, int NS, int NW>
static hipError_t launch_q4_matvec_m(const Q4Args& a, hipStream_t s) {
    switch (a.mode) {
        case Q4_STORE: return launch_q4_matvec_n<T, Q4_STORE, 1, NS, NW>(a, s);
        case Q4_F32: return a.rows[1] || a.rows[2] ? launch_q4_matvec_n<T, Q4_F32, 3, NS, NW>(a, s) : launch_q4_matvec_n<T, Q4_F32, 1, NS, NW>(a, s);
        case Q4_RESID: return launch_q4_matvec_n<T, Q4_RESID, 1, NS, NW>(a, s);
        case Q4_SILU: return launch_q4_matvec_n<T, Q4_SILU, 2, (NS < 2 ? 2 : NS), NW>(a, s);
        default: return hipErrorInvalidValue;
    }
}

// How many strips a workgroup takes.  A launch costs 4 us before the codes stream at 6 TB/s, so few strips are spread over the chip, one or two
// workgroups of eight wavefronts to a CU; of many, fewer and longer workgroups lose less on their ends, and several strips share what is read of the vectors,
// which many vectors feel most.  bf16, us for 1 / 2 / 4 strips with 8, 8 / 4 wavefronts: 4096 x 4096, one vector 4.3 / 5.0 / 7.5, sixteen 6.7 / 7.4 / 9.9; 6144 rows 5.9 / 5.3 / 7.8
// and 10.8 / 7.6 / 10.1; 8192 x 8192, sixteen 19.4 / 13.9 / 16.5; 12288 x 4096 8.8 / 9.2 / 8.6 (two strips, 4 wavefronts 8.5) and 14.7 / 14.1 / 10.9 (13.2);
// 28672 x 4096 16.3 / 17.9 / 15.0 (14.7) and 30.6 / 27.8 / 18.7 (22.7); 128256 x 4096 58.6 / 66.2 / 46.5 (48.0) and 128 / 106 / 60.0 (79).
// The number of wavefronts, and with it the order of a sum, goes by the matrices alone.
template <typename T>
static hipError_t launch_q4_matvec_t(const Q4Args& a, hipStream_t s) {
    int64_t strips = 0;
    for (int i = 0; i < 3; ++i) strips += (a.rows[i] + 15) / 16;
    if (a.mode == Q4_SILU) strips = 2 * ((a.rows[0] + 15) / 16);
    if (strips <= 256) return launch_q4_matvec_m<T, 1, 8>(a, s);
    if (strips <= 512) return launch_q4_matvec_m<T, 2, 8>(a, s);
    return a.nb <= 2 ? launch_q4_matvec_m<T, 2, 4>(a, s) : launch_q4_matvec_m<T, 4, 4>(a, s);
}

// a: Q4_STORE and Q4_RESID take one matrix, Q4_SILU two, Q4_F32 up to three
bool q4_norm_inside(int64_t K, int nb, bool bf16) { return bf16 && nb == 1 && K <= Q4_NORM_K; }

hipError_t launch_q4_matvec(const Q4Args& a, bool bf16, hipStream_t s) {
    if (a.nb < 1 || a.nb > DECODE_MAX_BATCH) return hipErrorInvalidValue;
    if (a.gamma && (!q4_norm_inside(a.K, a.nb, bf16) || (a.mode != Q4_SILU && !(a.mode == Q4_F32 && (a.rows[1] || a.rows[2]))))) return hipErrorInvalidValue;
    return bf16 ? launch_q4_matvec_t<bf16_t>(a, s) : launch_q4_matvec_t<float>(a, s);
}

}  // namespace spts
