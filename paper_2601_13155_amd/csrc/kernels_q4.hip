// Matrices in 4 bits and their products with one to sixteen vectors.
#include "spts_fp4.h"
#include "spts_lanes.h"

namespace spts {

// One thread per piece and slab: eight values of sixteen blocks of one row; the other values of a block are 16, 32 and 48 lanes away.  Done once for a matrix: 28672 x 4096 in bf16
// 87.9 us, 3.4 TB/s read and written (a copy's rate would be 60.0; a wavefront's load is 16 rows of 64 bytes), 4096 x 4096 15.8 (8.6).
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

// A kernel's view of its matrices (few arguments make quick launches)
template <int NM> struct Q4Mats { const u32x4* codes[NM]; const uint32_t* scales[NM]; void* y[NM]; int32_t rows[NM]; const void* x; int32_t K, nb; const void* gamma; float eps; };

// Up to four vectors normalised on their way in.  Every workgroup reads them and gamma into LDS (norm_load, a KB of a vector an instruction; ahead of the ring's
// loads, which a load behind them would have to wait for), takes the sums of squares and leaves the normalised vectors, rounded as rmsnorm_kernel does it,
// in their place (zeros up to whole slabs).  Piece c (16 bytes) of vector b lies at slot c ^ 4 b, which spreads the vectors of an operand over the banks.
// A wavefront reads only what it has loaded itself until the sums meet.
// Where that is done: up to four vectors, in 40 KB of LDS with gamma, beside which two workgroups' rings fit a CU.  us of a decode layer over 1000 pairs, inside / with two
// launches: hidden size 4096, 1 / 2 / 4 vectors 40.3 / 42.7 / 46.1 and 46.9 / 49.4 / 50.3; 2048 28.9 / 31.1 / 34.1 and 33.6 / 35.6 / 36.8; beyond, 8192, two vectors in 48 KB
// 105.1 and 103.2, four in 80 KB 117.0 and 103.9; 4096, eight vectors inside Q/K/V alone 54.8 and 53.4.
constexpr int Q4_NORM_NB = 4;
constexpr int Q4_NORM_SLABS = 40;
template <int NW>
__device__ inline void norm_load(const bf16_t* x, const bf16_t* gamma, int K, int slabs, int nb, uint32_t at) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int b = 0; b <= nb; ++b)
        for (int s = wave; s < slabs; s += NW) {
            const int piece = s * 64 + (b < nb ? lane ^ (4 * b) : lane);
            dma16s(piece * 8 < K ? (uint32_t)piece * 16 : 0u, b < nb ? x + (int64_t)b * K : gamma, at + (uint32_t)(b * slabs + s) * 1024);
        }
}
// NV: vectors taken together, so that their latencies overlap (those behind the last repeat the first and are not stored)
template <int NW, int NV>
__device__ inline void norm_in_lds(u32x4* xl, float* red, float eps, int K, int slabs, int nb) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u32x4* const gl = xl + nb * slabs * 64;
    float ss[NV];
#pragma unroll
    for (int b = 0; b < NV; ++b) ss[b] = 0.f;
    for (int s = wave; s < slabs; s += NW) {
#pragma unroll
        for (int b = 0; b < NV; ++b) {
            const int at = b < nb ? b : 0, slot = s * 64 + lane;
            u32x4 w = xl[at * slabs * 64 + slot];
            w = (slot ^ (4 * at)) * 8 < K ? w : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xffff0000u);
                ss[b] += lo * lo; ss[b] += hi * hi;
            }
        }
    }
#pragma unroll
    for (int b = 0; b < NV; ++b) {
        ss[b] = group_sum<16>(ss[b]);
        ss[b] += __shfl_xor(ss[b], 16);
        ss[b] += __shfl_xor(ss[b], 32);
    }
#pragma unroll
    for (int b = 0; b < NV; ++b)
        if (lane == 0) red[b * NW + wave] = ss[b];
    __syncthreads();
    float inv[NV];
#pragma unroll
    for (int b = 0; b < NV; ++b) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += red[b * NW + w];
        inv[b] = 1.0f / sqrtf(sum / (float)K + eps);
    }
    for (int s = wave; s < slabs; s += NW) {
        const int slot = s * 64 + lane;
        u32x4 o[NV];
#pragma unroll
        for (int b = 0; b < NV; ++b) {
            const int at = b < nb ? b : 0, piece = slot ^ (4 * at);
            const u32x4 w = xl[at * slabs * 64 + slot], g = gl[piece];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                o[b][i] = cvt_pk_bf16(__uint_as_float(w[i] << 16) * inv[b] * __uint_as_float(g[i] << 16),
                                      __uint_as_float(w[i] & 0xffff0000u) * inv[b] * __uint_as_float(g[i] & 0xffff0000u));
            o[b] = piece * 8 < K ? o[b] : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int b = 0; b < NV; ++b)
            if (b < nb) xl[b * slabs * 64 + slot] = o[b];
    }
    __syncthreads();
}

// which strips a workgroup has: NS consecutive ones of one matrix (SiLU: half are gate rows, half the same up rows); behind the last one, that again
template <int NS> struct Q4Strips { const u32x4* codes[NS]; const uint32_t* scales[NS]; int blk, which; };
template <int MODE, int NM, int NS>
__device__ inline Q4Strips<NS> q4_strips(const Q4Mats<NM>& a, int slabs) {
    constexpr int OWN = MODE == Q4_SILU ? NS / 2 : NS;
    Q4Strips<NS> r;
    r.blk = blockIdx.x;
    r.which = 0;
    if (MODE != Q4_SILU) {
#pragma unroll
        for (int i = 0; i + 1 < NM; ++i) {
            const int n = (a.rows[i] + 16 * NS - 1) / (16 * NS);
            if (r.which == i && r.blk >= n) { r.blk -= n; r.which = i + 1; }
        }
    }
    const int last = (a.rows[r.which] + 15) / 16 - 1;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int at = r.blk * OWN + s % OWN, m = MODE == Q4_SILU ? s / OWN : r.which;
        const int64_t strip = at < last ? at : last;
        r.codes[s] = a.codes[m] + strip * slabs * 256;
        r.scales[s] = a.scales[m] + strip * slabs * 64;
    }
    return r;
}

// The wavefronts' partial tiles meet in LDS and leave.  Lane (vector l16, row group kg) holds rows 4 kg .. 4 kg + 3 of its strips.  Sums of three parts of the
// vectors are columns (4 part + vector, four vectors a tile) or tiles of their own, added in one order either way.
template <typename T, int MODE, int NM, int NS, int NW, int TILES, int PARTS, bool APART>
__device__ inline void q4_finish(const Q4Mats<NM>& a, const Q4Strips<NS>& st, const mfma_f32x4 (&acc)[TILES][NS], float (*sred)[TILES][NS][16][20]) {
    constexpr int OWN = MODE == Q4_SILU ? NS / 2 : NS;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int p = 0; p < TILES; ++p)
#pragma unroll
        for (int s = 0; s < NS; ++s) *reinterpret_cast<mfma_f32x4*>(&sred[wave][p][s][lane & 15][4 * (lane >> 4)]) = acc[p][s];
    __syncthreads();
    for (int t = tid; t < OWN * 256; t += NW * 64) {
        const int r = t & 15, s = (t >> 4) % OWN, b = t / (16 * OWN);
        const int64_t row = ((int64_t)st.blk * OWN + s) * 16 + r;
        if (b >= a.nb || row >= a.rows[st.which]) continue;
        float v = 0.f, u = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w)
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p) {
                const int tile = APART ? b / 4 : p, col = APART ? 4 * p + b % 4 : b;
                v += sred[w][tile][s][col][r];
                if (MODE == Q4_SILU) u += sred[w][tile][NS - OWN + s][col][r];
            }
        const int64_t at = (int64_t)b * a.rows[st.which] + row;
        if (MODE == Q4_F32) ((float*)a.y[st.which])[at] = v;
        else {
            T* y = (T*)a.y[st.which] + at;
            *y = from_f32<T>(MODE == Q4_SILU ? v / (1.0f + __expf(-v)) * u : MODE == Q4_RESID ? to_f32(*y) + v : v);
        }
    }
}

// y = x W^T on the matrix cores for up to 16 vectors: a row of W is an operand row (lane l16), a vector a column; a dword of codes is an operand's eight values of a
// lane, and the decoder's bf16 pairs are the operand.  The NW wavefronts of a workgroup share the tiles of NS strips in turn and meet in LDS, so the order of a
// row's sum depends on K and NW alone, not on the vectors.  (A slab at a time instead of a tile: 28672 x 4096 12.8 instead of 12.1 us, 3584 x 18944 8.9 instead of 8.1.)
// fp32 vectors are taken as three bf16 parts, which is all of their 24 bits.  Up to eight vectors are taken apart by all lanes together, eight values of four vectors
// a lane, and the parts are columns of their own (4 part + vector), so that a matrix instruction does for all three; more are taken apart as operands are read.  (One kernel
// that split operands of any number and read them from the caches: 28672 x 4096, 1 / 4 / 8 / 16 vectors 24.6 / 25.0 / 26.3 / 28.8 us; this way
// 13.8 / 13.9 / 18.2 / 26.2.  Taking them apart is what bounds them: 7.5 instructions a value.)
// Read by lanes, an operand of 16 vectors is 16 half cache lines, of which a CU takes in 22 bytes a clock: a product of 4096 x 14336 took 0.55 us more with
// every vector, on however many CUs.  So codes, scales and vectors go to LDS with loads that are laid out for memory, whole lines of 4 vectors an instruction, into a
// ring of DEPTH tiles (128 k) of each wavefront; a wavefront reads only what it has loaded itself, after its own vmcnt wait, so there is no barrier in the loop.
// Piece c (16 bytes) of vector r lies at slot c ^ r of its row, which spreads the 16 rows of an operand over the banks.  4096 x 14336, 2 / 4 / 8 / 16 vectors 9.7 / 10.9 /
// 12.8 / 17.5 -> 7.1 / 7.9 / 9.3 / 11.9 us; of sixteen a CU still takes in no more than 30 bytes a clock, with three tiles in flight or with workgroups
// that begin at different tiles as well (14.8 / 14.9 / 14.8 us for 3584 x 18944).  4 XI: vectors there is room for; 0: up to four that are normalised on their way in.
constexpr int Q4_APART = 12 * 256;
template <typename T, int NS, int XI> constexpr int q4_stage_bytes() { return NS * 1024 + 256 + XI * 512 * (int)sizeof(T); }
template <typename T, int MODE, int NM, int NS, int NW, int XI, int DEPTH>
__global__ void __launch_bounds__(NW * 64) q4_matvec_kernel(Q4Mats<NM> a) {
    constexpr bool NORM = XI == 0, F32 = sizeof(T) == 4, APART = F32 && XI <= 2;
    constexpr uint32_t STAGE = q4_stage_bytes<T, NS, XI>();
    constexpr int RV = F32 ? 2 : 4, XN = 4 * XI / RV;   // vectors of a load, loads of all
    constexpr int NI = NS + 1 + XN;                // loads of a stage: codes of each strip, scales of all, vectors
    static_assert(NS <= 4 && DEPTH * NI <= 63, "vmcnt field");
    constexpr int TILES = APART ? XI : F32 ? 3 : 1;
    static_assert((size_t)DEPTH * STAGE >= sizeof(float) * TILES * NS * 16 * 20, "the partial tiles reuse the ring");
    extern __shared__ __attribute__((aligned(16))) char ring[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, kg = lane >> 4;
    const int K = a.K, slabs = (K + Q4_SLAB - 1) / Q4_SLAB, ntiles = (K + 127) / 128;
    const Q4Strips<NS> st = q4_strips<MODE, NM, NS>(a, slabs);
    const int N = wave < ntiles ? (ntiles - wave + NW - 1) / NW : 0;   // tiles wave, wave + NW, ...
    const int lrow = lane * RV / 64;               // vector of a load that the lane has a part of
    int row[XN + NORM];
#pragma unroll
    for (int j = 0; j < XN; ++j) row[j] = RV * j + lrow < a.nb ? RV * j + lrow : a.nb - 1;   // (behind the last vector any: its column is not stored)
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring + (uint32_t)wave * (DEPTH * STAGE);
    const uint32_t* sp = st.scales[0];             // lane (kg, l16): scales of strip kg % NS, row l16
#pragma unroll
    for (int s = 1; s < NS; ++s) sp = kg % NS == s ? st.scales[s] : sp;
    sp += l16;
    auto issue = [&](int n) {
        const int tile = wave + NW * n, k0 = tile * 128;
        const uint32_t slot = base + (uint32_t)(n % DEPTH) * STAGE;
#pragma unroll
        for (int s = 0; s < NS; ++s) dma16s_nt((uint32_t)lane * 16, (const char*)st.codes[s] + (int64_t)tile * 1024, slot + s * 1024);
        dma4_nt(sp + (int64_t)tile * 16, slot + NS * 1024);
#pragma unroll
        for (int j = 0; j < XN; ++j) {
            // the lane's 16 bytes go to row RV j + lrow, bf16: slot l16, fp32: half lane % 2 of slot l16
            const int at = F32 ? lane % 32 / 2 : l16;
            int piece = at ^ (RV * j + lrow);
            piece = k0 + piece * 8 < K ? piece : 0;
            dma16s(((uint32_t)row[j] * (uint32_t)K + (uint32_t)piece * 8) * (uint32_t)sizeof(T) + (F32 ? lane % 2 * 16 : 0), (const char*)a.x + (int64_t)k0 * (int)sizeof(T),
                   slot + NS * 1024 + 256 + j * 1024);
        }
    };
    mfma_f32x4 acc[TILES][NS];
#pragma unroll
    for (int p = 0; p < TILES; ++p)
#pragma unroll
        for (int s = 0; s < NS; ++s) acc[p][s] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
    int vx = 0;
    // behind the rings: the vectors to normalise, gamma, the sums
    u32x4* xl = reinterpret_cast<u32x4*>(ring + NW * DEPTH * STAGE);
    char* const apart = ring + NW * DEPTH * STAGE + wave * Q4_APART;   // or a tile's parts, of each wavefront
    if constexpr (NORM) norm_load<NW>((const bf16_t*)a.x, (const bf16_t*)a.gamma, K, slabs, a.nb, base + (uint32_t)(NW - wave) * (DEPTH * STAGE));
    for (int n = 0; n < (N < DEPTH ? N : DEPTH); ++n) issue(n);
    if constexpr (NORM) {
        if (N >= DEPTH) SPTS_WAIT_VMCNT(DEPTH * NI); else SPTS_WAIT_VMCNT(0);
        asm volatile("" ::: "memory");
        float* const red = reinterpret_cast<float*>(xl + (a.nb + 1) * slabs * 64);
        if (a.nb == 1) norm_in_lds<NW, 1>(xl, red, a.eps, K, slabs, 1);
        else if (a.nb == 2) norm_in_lds<NW, 2>(xl, red, a.eps, K, slabs, 2);
        else norm_in_lds<NW, Q4_NORM_NB>(xl, red, a.eps, K, slabs, a.nb);
        const int v = (l16 & 3) < a.nb ? l16 & 3 : a.nb - 1;
        xl += v * slabs * 64 + kg;
        vx = v;
    }
    for (int n = 0; n < N; ++n) {
        if (n + DEPTH <= N) SPTS_WAIT_VMCNT((DEPTH - 1) * NI); else SPTS_WAIT_VMCNT(0);
        asm volatile("" ::: "memory");
        const char* const slot = ring + (size_t)wave * (DEPTH * STAGE) + (size_t)(n % DEPTH) * STAGE;
        u32x4 c[NS], xv[APART ? XI : 1][4], raw[F32 ? (APART ? 2 * XI : 8) : 1];
        uint32_t sc[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            c[s] = *reinterpret_cast<const u32x4*>(slot + s * 1024 + lane * 16);
            sc[s] = *reinterpret_cast<const uint32_t*>(slot + NS * 1024 + s * 64 + l16 * 4);
        }
        const int xr = l16 & (4 * XI - 1);         // (with room for 4 or 8 vectors the columns behind repeat them)
        const int k0 = (wave + NW * n) * 128;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (NORM) xv[0][i] = xl[k0 / 8 + 4 * (i ^ vx)];
            else if constexpr (!F32) xv[0][i] = *reinterpret_cast<const u32x4*>(slot + NS * 1024 + 256 + xr * 256 + (((4 * i + kg) ^ xr) * 16));
            else if constexpr (!APART) {
#pragma unroll
                for (int h = 0; h < 2; ++h) raw[2 * i + h] = *reinterpret_cast<const u32x4*>(slot + NS * 1024 + 256 + xr * 512 + (((4 * i + kg) ^ xr) * 32) + h * 16);
            }
        }
        if constexpr (APART) {                     // piece l16 of vectors 4 j + kg
#pragma unroll
            for (int j = 0; j < 2 * XI; ++j) {
                const int r = j / 2 * 4 + kg;
                raw[j] = *reinterpret_cast<const u32x4*>(slot + NS * 1024 + 256 + r * 512 + ((l16 ^ r) * 32) + j % 2 * 16);
            }
        }
        // the slot is filled again only after its operands have arrived in registers
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (n + DEPTH < N) issue(n + DEPTH);
        if (!NORM && k0 + 128 > K) {
            const u32x4 none{0, 0, 0, 0};
            if constexpr (APART) {
#pragma unroll
                for (int j = 0; j < 2 * XI; ++j) raw[j] = k0 + l16 * 8 < K ? raw[j] : none;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool in = k0 + i * 32 + kg * 8 < K;
                    if constexpr (!F32) xv[0][i] = in ? xv[0][i] : none;
                    else { raw[2 * i] = in ? raw[2 * i] : none; raw[2 * i + 1] = in ? raw[2 * i + 1] : none; }
                }
            }
        }
        if constexpr (APART) {
            const int col = l16 < 12 ? l16 : l16 - 4;
#pragma unroll
            for (int j = 0; j < XI; ++j) {
                u32x4 xf[3];
                bf16_parts3(raw[2 * j], raw[2 * j + 1], xf);
#pragma unroll
                for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4*>(apart + (4 * p + kg) * 256 + ((l16 ^ (4 * p + kg)) * 16)) = xf[p];
#pragma unroll
                for (int i = 0; i < 4; ++i) xv[j][i] = *reinterpret_cast<const u32x4*>(apart + col * 256 + (((4 * i + kg) ^ col) * 16));
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32x4 xf[3];
            if constexpr (F32 && !APART) bf16_parts3(raw[2 * i], raw[2 * i + 1], xf);
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const u32x4 w = fp4_decode8_bf16(c[s][i], i == 0 ? fp4_scale_of<0>(sc[s]) : i == 1 ? fp4_scale_of<1>(sc[s]) : i == 2 ? fp4_scale_of<2>(sc[s]) : fp4_scale_of<3>(sc[s]));
#pragma unroll
                for (int p = 0; p < TILES; ++p) acc[p][s] = mfma16(w, F32 && !APART ? xf[p] : xv[APART ? p : 0][i], acc[p][s]);
            }
        }
    }
    __syncthreads();   // every ring has drained: its last tile waited for vmcnt 0
    q4_finish<T, MODE, NM, NS, NW, TILES, F32 ? 3 : 1, APART>(a, st, acc, reinterpret_cast<float (*)[TILES][NS][16][20]>(ring));
}

// (Depth of the ring: four tiles where they are small, 4096 x 14336, one vector, 2 / 3 / 4 tiles 8.5 / 7.6 / 7.1 us; otherwise two, which leaves room for more workgroups:
// 12288 x 4096, one vector 2 / 3 tiles 7.3 / 7.8, 128256 x 4096, sixteen 53.0 / 66.4; one strip of eight fp32 vectors, 4096 x 14336, 18.8 / 19.3.)
template <typename T, int MODE, int NM, int NS, int NW, int XI>
static hipError_t launch_q4_matvec_x(const Q4Mats<NM>& m, unsigned blocks, hipStream_t s) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int DEPTH = NS == 1 && XI < (F32 ? 2 : 4) ? 4 : 2, SUMS = Q4_NORM_NB * NW * (int)sizeof(float);
    constexpr int RING = NW * DEPTH * q4_stage_bytes<T, NS, XI>() + (F32 && XI <= 2 ? NW * Q4_APART : 0), MOST = RING + (XI ? 0 : Q4_NORM_SLABS * 1024 + SUMS);
    static_assert(MOST <= 160 * 1024, "LDS of a CU");
    const int lds = XI ? RING : RING + (m.nb + 1) * (int)q4_slabs(m.K) * 1024 + SUMS;
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(&q4_matvec_kernel<T, MODE, NM, NS, NW, XI, DEPTH>), MOST);
    if (e != hipSuccess) return e;
    q4_matvec_kernel<T, MODE, NM, NS, NW, XI, DEPTH><<<dim3(blocks), dim3(NW * 64), lds, s>>>(m);
    return hipGetLastError();
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
    const unsigned g = (unsigned)blocks;
    if constexpr (NM > 1 && sizeof(T) == 2) {
        if (a.gamma) {
            m.gamma = a.gamma; m.eps = a.eps;
            return launch_q4_matvec_x<T, MODE, NM, NS, NW, 0>(m, g, s);
        }
    }
    return a.nb <= 4   ? launch_q4_matvec_x<T, MODE, NM, NS, NW, 1>(m, g, s)
           : a.nb <= 8 ? launch_q4_matvec_x<T, MODE, NM, NS, NW, 2>(m, g, s)
                       : launch_q4_matvec_x<T, MODE, NM, NS, NW, 4>(m, g, s);
}

template <typename T, int NS, int NW>
static hipError_t launch_q4_matvec_m(const Q4Args& a, hipStream_t s) {
    switch (a.mode) {
        case Q4_STORE: return launch_q4_matvec_n<T, Q4_STORE, 1, NS, NW>(a, s);
        case Q4_F32: return a.rows[1] || a.rows[2] ? launch_q4_matvec_n<T, Q4_F32, 3, NS, NW>(a, s) : launch_q4_matvec_n<T, Q4_F32, 1, NS, NW>(a, s);
        case Q4_RESID: return launch_q4_matvec_n<T, Q4_RESID, 1, NS, NW>(a, s);
        case Q4_SILU: return launch_q4_matvec_n<T, Q4_SILU, 2, (NS < 2 ? 2 : NS), (NS < 2 && sizeof(T) == 4 ? NW / 2 : NW)>(a, s);
        default: return hipErrorInvalidValue;
    }
}

// How many strips a workgroup takes.  A launch costs about 4 us before the codes stream at 6 TB/s, so few strips are spread over the chip, one or two workgroups
// of eight wavefronts to a CU; of many, fewer and longer workgroups lose less on their ends, and several strips share what is read of the vectors.  bf16, us for
// 1 / 2 strips with 8 / 4 strips with 4 wavefronts (2 with 4, 4 with 8): 4096 x 14336, one vector 7.2 / 9.0 / 15.8 (12.8, 13.8), sixteen 12.0 / 14.4 / 19.2; 6144 x
// 4096 5.1 / 4.6 / 6.4 and 8.1 / 5.9 / 7.5; 8192 x 8192 9.6 / 7.6 / 10.7 and 13.9 / 9.8 / 12.5; 12288 x 4096 7.4 / 6.7 / 6.9 (6.5, 6.8) and 12.1 / 10.2 / 7.9 (9.3, 8.2);
// 28672 x 4096 14.6 / 12.6 / 12.3 (12.4, 13.5) and 26.6 / 19.4 / 14.0 (16.1, 15.4); 128256 x 4096 56.1 / 42.2 / 43.2 (42.4, 49.9) and 117 / 76.2 / 49.5 (59.9, 59.4).
// fp32, 28672 x 4096, 1 strip with 8 / 2 with 4 / 4 with 4 wavefronts: 29.1 / 15.9 / 13.7 and 55.9 / 39.5 / 26.4.  It goes by the matrices alone, and with it the order of a sum.
template <typename T>
static hipError_t launch_q4_matvec_t(const Q4Args& a, hipStream_t s) {
    int64_t strips = 0;
    for (int i = 0; i < 3; ++i) strips += (a.rows[i] + 15) / 16;
    if (a.mode == Q4_SILU) strips = 2 * ((a.rows[0] + 15) / 16);
    if (strips <= 256) return launch_q4_matvec_m<T, 1, 8>(a, s);
    if (strips <= 512) return launch_q4_matvec_m<T, 2, (sizeof(T) == 4 ? 4 : 8)>(a, s);   // (eight rings of 16 fp32 vectors do not fit a CU)
    return launch_q4_matvec_m<T, 4, 4>(a, s);
}

// a: Q4_STORE and Q4_RESID take one matrix, Q4_SILU two, Q4_F32 up to three
bool q4_norm_inside(int64_t K, int nb, bool bf16) { return bf16 && nb <= Q4_NORM_NB && (nb + 1) * q4_slabs(K) <= Q4_NORM_SLABS; }

hipError_t launch_q4_matvec(const Q4Args& a, bool bf16, hipStream_t s) {
    if (a.nb < 1 || a.nb > DECODE_MAX_BATCH) return hipErrorInvalidValue;
    if (a.gamma && (!q4_norm_inside(a.K, a.nb, bf16) || (a.mode != Q4_SILU && !(a.mode == Q4_F32 && (a.rows[1] || a.rows[2]))))) return hipErrorInvalidValue;
    return bf16 ? launch_q4_matvec_t<bf16_t>(a, s) : launch_q4_matvec_t<float>(a, s);
}

}  // namespace spts
