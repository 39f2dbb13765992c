// Caches in 4 bits: appending pairs, reading them back, and the attention of one query per sequence over them.
#include "spts_fp4.h"

namespace spts {

namespace {
// byte offsets of a key's code row / of the d / 32 bytes of values that piece n of a key holds / of the scale bytes
__device__ inline int64_t key_at(int g, int64_t cap, int64_t key, int d) { return ((int64_t)g * cap + key) * (d / 2); }
__device__ inline int64_t key_scale_at(int g, int64_t cap, int64_t key, int blk, int d) { return ((int64_t)g * cap + key) * (d / 32) + blk; }
__device__ inline int64_t value_at(int g, int64_t cap, int64_t key, int n, int d) { return ((((int64_t)g * cap + key) >> 3) * 16 + n) * (d / 4) + (key & 7) * (d / 32); }
__device__ inline int64_t value_scale_at(int g, int64_t cap, int64_t key, int blk, int d) { return ((((int64_t)g * cap + key) >> 3) * (d / 32) + blk) * 8 + (key & 7); }

// the cache that row `row` of a call belongs to, and the row's place in it
__device__ inline int cache_of(const Kv4Batch& kb, int64_t row, int64_t* at) {
    int b = 0;
    while (b + 1 < kb.n && row >= kb.off[b + 1]) ++b;
    *at = kb.count[b] + (row - kb.off[b]);
    return b;
}
}  // namespace

// One thread per row, head and block of 32, keys (blockIdx.y = 0) or values.
template <typename T>
__global__ void __launch_bounds__(256) kv4_append_kernel(const T* __restrict__ k, const T* __restrict__ v, const int32_t* __restrict__ pos, Kv4Batch kb, int Hkv, int d) {
    const int blocks = Hkv * (d / 32);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / blocks;
    if (row >= kb.off[kb.n]) return;
    const int g = (int)(i % blocks) / (d / 32), blk = (int)(i % blocks) % (d / 32);
    int64_t key;
    const int b = cache_of(kb, row, &key);
    const T* src = (blockIdx.y ? v : k) + (row * Hkv + g) * d + blk * 32;
    float f[32];
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        f[j] = to_f32(src[j]);
        const uint32_t m = __float_as_uint(f[j]) & 0x7fffffffu;
        top = m > top ? m : top;
    }
    const uint32_t byte = fp4_scale_byte(top);
    u32x4 c;
#pragma unroll
    for (int q = 0; q < 4; ++q) c[q] = fp4_encode8(f + 8 * q, __uint_as_float(byte << 23));
    if (blockIdx.y == 0) {
        *reinterpret_cast<u32x4*>((char*)kb.k[b] + key_at(g, kb.cap[b], key, d) + blk * 16) = c;
        ((uint8_t*)kb.ks[b])[key_scale_at(g, kb.cap[b], key, blk, d)] = (uint8_t)byte;
        if (i % blocks == 0) kb.pos[b][key] = pos[row];
    } else {
        const int per = d / 32;   // bytes of a piece
        for (int j = 0; j < 16; ++j) ((uint8_t*)kb.v[b])[value_at(g, kb.cap[b], key, (blk * 16 + j) / per, d) + j % per] = (uint8_t)(c[j / 4] >> (8 * (j % 4)));
        ((uint8_t*)kb.vs[b])[value_scale_at(g, kb.cap[b], key, blk, d)] = (uint8_t)byte;
    }
}

hipError_t launch_kv4_append(const void* k, const void* v, const int32_t* pos, const Kv4Batch& kb, int Hkv, int d, bool bf16, hipStream_t s) {
    const int64_t items = kb.off[kb.n] * Hkv * (d / 32);
    if (items == 0) return hipSuccess;
    const dim3 g((unsigned)((items + 255) / 256), 2), b(256);
    if (bf16) kv4_append_kernel<bf16_t><<<g, b, 0, s>>>((const bf16_t*)k, (const bf16_t*)v, pos, kb, Hkv, d);
    else kv4_append_kernel<float><<<g, b, 0, s>>>((const float*)k, (const float*)v, pos, kb, Hkv, d);
    return hipGetLastError();
}

template <typename T>
__global__ void __launch_bounds__(256) kv4_read_kernel(Kv4Batch kb, T* __restrict__ k, T* __restrict__ v, int Hkv, int d) {
    const int blocks = Hkv * (d / 32);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / blocks;
    if (row >= kb.off[kb.n]) return;
    const int g = (int)(i % blocks) / (d / 32), blk = (int)(i % blocks) % (d / 32);
    int64_t key;
    const int b = cache_of(kb, row, &key);
    T* dst = (blockIdx.y ? v : k) + (row * Hkv + g) * d + blk * 32;
    u32x4 c{0, 0, 0, 0};
    uint32_t byte;
    if (blockIdx.y == 0) {
        c = *reinterpret_cast<const u32x4*>((const char*)kb.k[b] + key_at(g, kb.cap[b], key, d) + blk * 16);
        byte = ((const uint8_t*)kb.ks[b])[key_scale_at(g, kb.cap[b], key, blk, d)];
    } else {
        const int per = d / 32;
        for (int j = 0; j < 16; ++j) c[j / 4] |= (uint32_t)((const uint8_t*)kb.v[b])[value_at(g, kb.cap[b], key, (blk * 16 + j) / per, d) + j % per] << (8 * (j % 4));
        byte = ((const uint8_t*)kb.vs[b])[value_scale_at(g, kb.cap[b], key, blk, d)];
    }
    for (int q = 0; q < 4; ++q) {
        float f[8];
        fp4_decode8(c[q], __uint_as_float(byte << 23), f);
        for (int j = 0; j < 8; ++j) dst[8 * q + j] = from_f32<T>(f[j]);
    }
}

hipError_t launch_kv4_read(const Kv4Batch& kb, void* k, void* v, int Hkv, int d, bool bf16, hipStream_t s) {
    const int64_t items = kb.off[kb.n] * Hkv * (d / 32);
    if (items == 0) return hipSuccess;
    const dim3 g((unsigned)((items + 255) / 256), 2), b(256);
    if (bf16) kv4_read_kernel<bf16_t><<<g, b, 0, s>>>(kb, (bf16_t*)k, (bf16_t*)v, Hkv, d);
    else kv4_read_kernel<float><<<g, b, 0, s>>>(kb, (float*)k, (float*)v, Hkv, d);
    return hipGetLastError();
}

// One workgroup per query head and sequence, 256 keys at a time with the running maximum and sum: a thread takes a key's score, then a thread takes
// a dimension of the weighted values.
template <typename T>
__global__ void __launch_bounds__(256) kv4_attn_kernel(const T* __restrict__ q, Kv4Batch kb, int H, int Hkv, int d, float scale_log2e, T* __restrict__ out) {
    __shared__ float sp[256], sq[128], red[4];
    const int h = blockIdx.x, b = blockIdx.y, g = h / (H / Hkv), tid = threadIdx.x;
    const int64_t n = kb.count[b], cap = kb.cap[b];
    if (tid < d) sq[tid] = to_f32(q[((int64_t)b * H + h) * d + tid]);
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int64_t k0 = 0; k0 < n; k0 += 256) {
        __syncthreads();
        float s = -INFINITY;
        if (k0 + tid < n) {
            s = 0.f;
            for (int c = 0; c < d / 8; ++c) {
                float f[8];
                const uint32_t w = *reinterpret_cast<const uint32_t*>((const char*)kb.k[b] + key_at(g, cap, k0 + tid, d) + c * 4);
                fp4_decode8(w, __uint_as_float((uint32_t)((const uint8_t*)kb.ks[b])[key_scale_at(g, cap, k0 + tid, c / 4, d)] << 23), f);
                for (int j = 0; j < 8; ++j) s = fmaf(f[j], sq[c * 8 + j], s);
            }
            s *= scale_log2e;
        }
        float mx = s;
        for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
        if ((tid & 63) == 0) red[tid >> 6] = mx;
        __syncthreads();
        const float mn = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        const float alpha = exp2f(m - mn);
        m = mn;
        sp[tid] = exp2f(s - mn);
        __syncthreads();
        l *= alpha;
        o *= alpha;
        const int64_t left = n - k0 < 256 ? n - k0 : 256;
        for (int j = 0; j < left; ++j) {
            l += sp[j];
            if (tid < d) {
                const int per = d / 16;   // values of a piece
                const uint8_t byte = ((const uint8_t*)kb.v[b])[value_at(g, cap, k0 + j, tid / per, d) + tid % per / 2];
                const fp4_f32x2 f = fp4_pair<0>(byte, __uint_as_float((uint32_t)((const uint8_t*)kb.vs[b])[value_scale_at(g, cap, k0 + j, tid / 32, d)] << 23));
                o = fmaf(sp[j], f[tid & 1], o);
            }
        }
    }
    if (tid < d) out[((int64_t)b * H + h) * d + tid] = from_f32<T>(n > 0 ? o / l : 0.f);
}

hipError_t launch_kv4_attn(const void* q, const Kv4Batch& kb, int H, int Hkv, int d, float* part, size_t part_floats, void* out, bool bf16, hipStream_t s) {
    (void)part; (void)part_floats;
    const float c = 1.4426950408889634f / sqrtf((float)d);
    const dim3 g((unsigned)H, (unsigned)kb.n), b(256);
    if (bf16) kv4_attn_kernel<bf16_t><<<g, b, 0, s>>>((const bf16_t*)q, kb, H, Hkv, d, c, (bf16_t*)out);
    else kv4_attn_kernel<float><<<g, b, 0, s>>>((const float*)q, kb, H, Hkv, d, c, (float*)out);
    return hipGetLastError();
}

}  // namespace spts
