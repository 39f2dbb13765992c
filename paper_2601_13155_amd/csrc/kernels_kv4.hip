// Caches in 4 bits: appending pairs, reading them back, and the attention of one query per sequence over them.
#include "spts_fp4.h"

#include <algorithm>
#include <type_traits>

namespace spts {

namespace {
// byte offsets of a key's code row / of the d / 32 bytes of values that piece n of a key holds / of the scale bytes
__device__ inline int64_t key_at(int g, int64_t cap, int64_t key, int d) { return ((int64_t)g * cap + key) * (d / 2); }
__device__ inline int64_t key_scale_at(int g, int64_t cap, int64_t key, int blk, int d) { return ((int64_t)g * cap + key) * (d / 32) + blk; }
__device__ inline int64_t value_at(int g, int64_t cap, int64_t key, int n, int d) { return ((((int64_t)g * cap + key) >> 3) * 16 + n) * (d / 4) + (key & 7) * (d / 32); }
__device__ inline int64_t value_scale_at(int g, int64_t cap, int64_t key, int blk, int d) { return ((((int64_t)g * cap + key) >> 3) * (d / 32) + blk) * 8 + (key & 7); }

// A kernel's view of up to NB caches: one, or sixteen (the launches' arguments are then 752 bytes for the attention, 860 for reading, 868 for appending, 952 for the rotation with the
// append; 84 to 120 for one).  What it costs is finding the sequence and its pointers, not the arguments' bytes (an empty kernel takes 2.4 us with 24 bytes and with 1288): one sequence
// by the descriptor of one / of sixteen, 517 keys 6.3 / 7.0 us, 13107 keys (two launches) 9.6 / 10.7, a pair appended and read back 9.0 / 10.3.
template <int NB> struct Kv4Rows {
    char *k[NB], *v[NB];
    uint8_t *ks[NB], *vs[NB];
    int32_t* pos[NB];
    int32_t cap[NB], at[NB], end[NB];   // capacity, cache row of the sequence's first row, its end among the call's rows
    int32_t row0, rows;                 // rows of this launch
};
template <int NB> struct Kv4Caches {
    const char *k[NB], *v[NB];
    const uint8_t *ks[NB], *vs[NB];
    int32_t cap[NB], n[NB];
    int32_t end[NB];                    // splits of sequence b: those before end[b] that are none of b - 1's; behind the last sequence its end
    uint32_t per;                       // keys of a split, a multiple of 32 (a little above 2^31 where one share takes the longest cache)
};

// the sequence that item i is in, and the first item of that sequence
template <int NB> __device__ inline int sequence_of(const int32_t (&end)[NB], int i, int* first) {
    int b = 0;
    *first = 0;
#pragma unroll
    for (int j = 0; j + 1 < NB; ++j)
        if (i >= end[j]) { b = j + 1; *first = end[j]; }
    return b;
}
}  // namespace

// Eight dimensions of one row and head per thread, of the key and of the value: 16 bytes of bf16 in, a dword of codes out.  A workgroup takes 2048 / D
// consecutive rows of one head (blockIdx.y), so that rows arrive in whole pieces of 2 D bytes and the codes of a head leave in one stretch; the four lanes of a block
// find its largest value by two exchanges.
// codes of eight values and their block's scale byte; the block is the quad of lanes
__device__ inline uint32_t encode_quad(const float (&v)[8], uint32_t* byte) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t m = __float_as_uint(v[j]) & 0x7fffffffu;
        top = m > top ? m : top;
    }
    uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true);   // quad_perm [1, 0, 3, 2]
    top = o > top ? o : top;
    o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true);            // quad_perm [2, 3, 0, 1]
    top = o > top ? o : top;
    *byte = fp4_scale_byte(top);
    return fp4_encode8(v, __uint_as_float(*byte << 23));
}

template <typename T, int D, int NB>
__global__ void __launch_bounds__(256) kv4_append_kernel(const T* __restrict__ k, const T* __restrict__ v, const int32_t* __restrict__ pos, Kv4Rows<NB> kb, int Hkv) {
    constexpr int CH = D / 8, PB = D / 32;   // threads of a row, bytes of a piece of values
    const int g = blockIdx.y, c = threadIdx.x % CH;
    const int64_t row = kb.row0 + (int64_t)blockIdx.x * (256 / CH) + threadIdx.x / CH;
    if (row >= kb.rows) return;         // (whole quads)
    const T* const ks = k + (row * Hkv + g) * D + 8 * c;
    const T* const vs = v + (row * Hkv + g) * D + 8 * c;
    float kf[8], vf[8];
    load8(ks, kf);
    load8(vs, vf);
    int first;
    const int b = sequence_of(kb.end, (int)row, &first);
    const int64_t cap = kb.cap[b], key = kb.at[b] + (row - first);
    uint32_t kbyte, vbyte;
    const uint32_t kc = encode_quad(kf, &kbyte), vc = encode_quad(vf, &vbyte);
    *reinterpret_cast<uint32_t*>(kb.k[b] + key_at(g, cap, key, D) + 4 * c) = kc;
    char* const vp = kb.v[b] + value_at(g, cap, key, c * 4 / PB, D);   // pieces of one key are 8 PB bytes apart
    if constexpr (PB == 4) *reinterpret_cast<uint32_t*>(vp) = vc;
    else if constexpr (PB == 2) {
        *reinterpret_cast<uint16_t*>(vp) = (uint16_t)vc;
        *reinterpret_cast<uint16_t*>(vp + 16) = (uint16_t)(vc >> 16);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) vp[8 * j] = (char)(vc >> (8 * j));
    }
    if (c % 4 == 0) {
        kb.ks[b][key_scale_at(g, cap, key, c / 4, D)] = (uint8_t)kbyte;
        kb.vs[b][value_scale_at(g, cap, key, c / 4, D)] = (uint8_t)vbyte;
    }
    if (g == 0 && c == 0) kb.pos[b][key] = pos[row];
}

template <typename T> __device__ inline void store8(T* p, const float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        const u32x4 w{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])};
        __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p));
    } else {
        const u32x4 a{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])},
            b{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
        __builtin_nontemporal_store(a, reinterpret_cast<u32x4*>(p));
        __builtin_nontemporal_store(b, reinterpret_cast<u32x4*>(p) + 1);
    }
}

// The way back, same threads.
template <typename T, int D, int NB>
__global__ void __launch_bounds__(256) kv4_read_kernel(Kv4Rows<NB> kb, T* __restrict__ k, T* __restrict__ v, int Hkv) {
    constexpr int CH = D / 8, PB = D / 32;
    const int g = blockIdx.y, c = threadIdx.x % CH;
    const int64_t row = kb.row0 + (int64_t)blockIdx.x * (256 / CH) + threadIdx.x / CH;
    if (row >= kb.rows) return;
    int first;
    const int b = sequence_of(kb.end, (int)row, &first);
    const int64_t cap = kb.cap[b], key = kb.at[b] + (row - first);
    const uint32_t kc = *reinterpret_cast<const uint32_t*>(kb.k[b] + key_at(g, cap, key, D) + 4 * c);
    const char* const vp = kb.v[b] + value_at(g, cap, key, c * 4 / PB, D);
    uint32_t vc;
    if constexpr (PB == 4) vc = *reinterpret_cast<const uint32_t*>(vp);
    else if constexpr (PB == 2) vc = (uint32_t)*reinterpret_cast<const uint16_t*>(vp) | (uint32_t)*reinterpret_cast<const uint16_t*>(vp + 16) << 16;
    else vc = (uint32_t)(uint8_t)vp[0] | (uint32_t)(uint8_t)vp[8] << 8 | (uint32_t)(uint8_t)vp[16] << 16 | (uint32_t)(uint8_t)vp[24] << 24;
    const uint32_t kbyte = kb.ks[b][key_scale_at(g, cap, key, c / 4, D)], vbyte = kb.vs[b][value_scale_at(g, cap, key, c / 4, D)];
    float f[8];
    fp4_decode8(kc, __uint_as_float(kbyte << 23), f);
    store8(k + (row * Hkv + g) * D + 8 * c, f);
    fp4_decode8(vc, __uint_as_float(vbyte << 23), f);
    store8(v + (row * Hkv + g) * D + 8 * c, f);
}

constexpr int64_t KV4_LAUNCH_ROWS = 1 << 24;   // a launch has fewer than 2^32 threads along a dimension; a row of a head has at most 16

template <int NB> static Kv4Rows<NB> rows_of(const Kv4Batch& kb) {
    Kv4Rows<NB> r{};
    for (int b = 0; b < NB; ++b) {
        const int i = b < kb.n ? b : kb.n - 1;
        r.k[b] = (char*)kb.k[i]; r.v[b] = (char*)kb.v[i]; r.ks[b] = (uint8_t*)kb.ks[i]; r.vs[b] = (uint8_t*)kb.vs[i]; r.pos[b] = kb.pos[i];
        r.cap[b] = (int32_t)kb.cap[i]; r.at[b] = (int32_t)kb.count[i]; r.end[b] = (int32_t)kb.off[i + 1];
    }
    r.rows = (int32_t)kb.off[kb.n];
    return r;
}

template <typename T, int D, int NB>
static hipError_t launch_kv4_rows_n(const T* k, const T* v, const int32_t* pos, T* k_out, T* v_out, const Kv4Batch& kb, int Hkv, hipStream_t s) {
    Kv4Rows<NB> r = rows_of<NB>(kb);
    const int64_t rows = r.rows;
    for (int64_t r0 = 0; r0 < rows; r0 += KV4_LAUNCH_ROWS) {
        const int64_t n = rows - r0 < KV4_LAUNCH_ROWS ? rows - r0 : KV4_LAUNCH_ROWS;
        r.row0 = (int32_t)r0; r.rows = (int32_t)(r0 + n);
        const dim3 g((unsigned)((n + 2048 / D - 1) / (2048 / D)), (unsigned)Hkv), t(256);
        if (k) kv4_append_kernel<T, D, NB><<<g, t, 0, s>>>(k, v, pos, r, Hkv);
        else kv4_read_kernel<T, D, NB><<<g, t, 0, s>>>(r, k_out, v_out, Hkv);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int D>
static hipError_t launch_kv4_rows(const T* k, const T* v, const int32_t* pos, T* k_out, T* v_out, const Kv4Batch& kb, int Hkv, hipStream_t s) {
    if (kb.off[kb.n] == 0) return hipSuccess;
    return kb.n == 1 ? launch_kv4_rows_n<T, D, 1>(k, v, pos, k_out, v_out, kb, Hkv, s)
                     : launch_kv4_rows_n<T, D, DECODE_MAX_BATCH>(k, v, pos, k_out, v_out, kb, Hkv, s);
}

template <typename T>
static hipError_t launch_kv4_rows_t(const void* k, const void* v, const int32_t* pos, void* k_out, void* v_out, const Kv4Batch& kb, int Hkv, int d, hipStream_t s) {
    switch (d) {
        case 128: return launch_kv4_rows<T, 128>((const T*)k, (const T*)v, pos, (T*)k_out, (T*)v_out, kb, Hkv, s);
        case 64: return launch_kv4_rows<T, 64>((const T*)k, (const T*)v, pos, (T*)k_out, (T*)v_out, kb, Hkv, s);
        case 32: return launch_kv4_rows<T, 32>((const T*)k, (const T*)v, pos, (T*)k_out, (T*)v_out, kb, Hkv, s);
        default: return hipErrorInvalidValue;
    }
}

hipError_t launch_kv4_append(const void* k, const void* v, const int32_t* pos, const Kv4Batch& kb, int Hkv, int d, bool bf16, hipStream_t s) {
    return bf16 ? launch_kv4_rows_t<bf16_t>(k, v, pos, nullptr, nullptr, kb, Hkv, d, s) : launch_kv4_rows_t<float>(k, v, pos, nullptr, nullptr, kb, Hkv, d, s);
}

hipError_t launch_kv4_read(const Kv4Batch& kb, void* k, void* v, int Hkv, int d, bool bf16, hipStream_t s) {
    return bf16 ? launch_kv4_rows_t<bf16_t>(nullptr, nullptr, nullptr, k, v, kb, Hkv, d, s) : launch_kv4_rows_t<float>(nullptr, nullptr, nullptr, k, v, kb, Hkv, d, s);
}

// The pairs of one new token per sequence, from the projections' fp32 sums q32 [n, H, D], k32 / v32 [n, Hkv, D]: queries and keys are rotated, everything is rounded to T
// once, keys and values then go into the caches (blockIdx.y = sequence).  A thread has the dimensions j and j + D / 2 of a head, 32 lanes a block of each half (both halves
// one block for D = 32); neighbours share a byte.  The angle is formed in fp64, as everywhere here.
template <int NB> struct Kv4Tokens { Kv4Rows<NB> rows; int32_t pos[NB]; double neg2_over_d_log2base; };
template <typename T, int D, int NB>
__global__ void __launch_bounds__(256) kv4_rope_append_kernel(const float* __restrict__ q32, const float* __restrict__ k32, const float* __restrict__ v32, T* __restrict__ q,
                                                              int H, int Hkv, Kv4Tokens<NB> tk) {
    constexpr int HALF = D / 2, PB = D / 32;
    const int b = NB > 1 ? (int)blockIdx.y : 0, i = blockIdx.x * 256 + threadIdx.x, j = i % HALF;
    int head = i / HALF;
    if (i == 0) tk.rows.pos[b][tk.rows.at[b]] = tk.pos[b];
    if (head >= H + 2 * Hkv) return;                  // (whole heads: the lanes of a block leave together)
    const bool is_q = head < H, is_v = head >= H + Hkv;
    head -= is_q ? 0 : is_v ? H + Hkv : H;
    const float* src = (is_q ? q32 + (int64_t)b * H * D : (is_v ? v32 : k32) + (int64_t)b * Hkv * D) + (int64_t)head * D + j;
    float x0 = src[0], x1 = src[HALF];
    if (!is_v) {
        double sn, cs;
        sincos((double)tk.pos[b] * exp2((double)j * tk.neg2_over_d_log2base), &sn, &cs);
        const float c = (float)cs, s = (float)sn, r0 = x0 * c - x1 * s;
        x1 = x1 * c + x0 * s;
        x0 = r0;
    }
    const T t0 = from_f32<T>(x0), t1 = from_f32<T>(x1);
    if (is_q) {
        T* to = q + ((int64_t)b * H + head) * D + j;
        to[0] = t0;
        to[HALF] = t1;
    }
    x0 = to_f32(t0); x1 = to_f32(t1);
    uint32_t top0 = __float_as_uint(x0) & 0x7fffffffu, top1 = __float_as_uint(x1) & 0x7fffffffu;
    if (D == 32) top0 = top1 = top0 > top1 ? top0 : top1;
#pragma unroll
    for (int off = 1; off < (D == 32 ? 16 : 32); off <<= 1) {
        const uint32_t o0 = (uint32_t)__shfl_xor((int)top0, off), o1 = (uint32_t)__shfl_xor((int)top1, off);
        top0 = o0 > top0 ? o0 : top0;
        top1 = o1 > top1 ? o1 : top1;
    }
    const float n0 = __shfl_xor(x0, 1), n1 = __shfl_xor(x1, 1);
    if (is_q || (j & 1)) return;
    const uint32_t byte0 = fp4_scale_byte(top0), byte1 = fp4_scale_byte(top1);
    const uint32_t c0 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x0, n0, __uint_as_float(byte0 << 23), 0);
    const uint32_t c1 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x1, n1, __uint_as_float(byte1 << 23), 0);
    const int64_t cap = tk.rows.cap[b], key = tk.rows.at[b];
    const int p0 = j / 2, p1 = (j + HALF) / 2;        // bytes of the row
    if (!is_v) {
        char* const to = tk.rows.k[b] + key_at(head, cap, key, D);
        to[p0] = (char)c0;
        to[p1] = (char)c1;
    } else {
        tk.rows.v[b][value_at(head, cap, key, p0 / PB, D) + p0 % PB] = (char)c0;
        tk.rows.v[b][value_at(head, cap, key, p1 / PB, D) + p1 % PB] = (char)c1;
    }
    if (j % 32 == 0) {
        uint8_t* const to = is_v ? tk.rows.vs[b] : tk.rows.ks[b];
        const int b0 = j / 32, b1 = (j + HALF) / 32;
        to[is_v ? value_scale_at(head, cap, key, b0, D) : key_scale_at(head, cap, key, b0, D)] = (uint8_t)byte0;
        if (D > 32) to[is_v ? value_scale_at(head, cap, key, b1, D) : key_scale_at(head, cap, key, b1, D)] = (uint8_t)byte1;
    }
}

template <typename T, int D, int NB>
static hipError_t launch_kv4_rope_append_n(const float* q32, const float* k32, const float* v32, void* q, int H, int Hkv, float base, const Kv4Batch& kb, const int32_t* pos,
                                           hipStream_t s) {
    Kv4Tokens<NB> tk{rows_of<NB>(kb), {}, -2.0 / (double)D * log2((double)base)};
    for (int b = 0; b < kb.n; ++b) tk.pos[b] = pos[b];
    kv4_rope_append_kernel<T, D, NB><<<dim3((unsigned)(((H + 2 * Hkv) * (D / 2) + 255) / 256), (unsigned)kb.n), dim3(256), 0, s>>>(q32, k32, v32, (T*)q, H, Hkv, tk);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_kv4_rope_append_t(const float* q32, const float* k32, const float* v32, void* q, int H, int Hkv, int d, float base, const Kv4Batch& kb,
                                           const int32_t* pos, hipStream_t s) {
#define SPTS_KV4_ROPE(D_)                                                                                                                          \
    return kb.n == 1 ? launch_kv4_rope_append_n<T, D_, 1>(q32, k32, v32, q, H, Hkv, base, kb, pos, s)                                              \
                     : launch_kv4_rope_append_n<T, D_, DECODE_MAX_BATCH>(q32, k32, v32, q, H, Hkv, base, kb, pos, s);
    switch (d) {
        case 128: SPTS_KV4_ROPE(128)
        case 64: SPTS_KV4_ROPE(64)
        case 32: SPTS_KV4_ROPE(32)
        default: return hipErrorInvalidValue;
    }
#undef SPTS_KV4_ROPE
}

hipError_t launch_kv4_rope_append(const float* q32, const float* k32, const float* v32, void* q, int H, int Hkv, int d, float base, const Kv4Batch& kb, const int32_t* pos,
                                  bool bf16, hipStream_t s) {
    return bf16 ? launch_kv4_rope_append_t<bf16_t>(q32, k32, v32, q, H, Hkv, d, base, kb, pos, s) : launch_kv4_rope_append_t<float>(q32, k32, v32, q, H, Hkv, d, base, kb, pos, s);
}

// ------------------------------------------------------------------------------------------------- attention
// W dwords from p
template <int W> __device__ inline void load_words(const char* p, uint32_t (&w)[W]) {
    if constexpr (W == 8) {
        const u32x4 a = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)), b = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) { w[i] = a[i]; w[4 + i] = b[i]; }
    } else if constexpr (W == 4) {
        const u32x4 a = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = a[i];
    } else if constexpr (W == 2) {
        const u32x2 a = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
        w[0] = a[0]; w[1] = a[1];
    } else {
        w[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
    }
}

// pair I (two dimensions) of key J in a lane's piece of values: D / 32 bytes a key, eight keys
template <int D, int J, int I> __device__ inline uint32_t value_pair(const uint32_t* w, float scale) {
    constexpr int byte = J * (D / 32) + I;
    return fp4_pair_bf16<byte % 4>(w[byte / 4], scale);
}

constexpr float KV4_LOWEST = -3.402823466e38f;

// what one lane needs of 32 keys
template <int D> struct Kv4Step {
    uint32_t k[2][D / 32], v[D / 16], vs[2];
    uint32_t ks[2];
};

// One workgroup of NW wavefronts per split of a sequence's keys and key/value head (4; 8 or 16 where one has a whole short cache); a wavefront takes 32 keys at a time with its own running maximum
// and sum, all query heads of the head at once on the matrix cores:
//   S^T = K Q^T: a key is an operand row (lane l16 = key, lane group kg = a quarter of the dimensions, one stored block), a query head a column.
//     Of the two products of 16 keys, operand row m of product t is key 8 (m / 4) + 4 t + m % 4: lane group kg then holds the scores of the keys 8 kg .. 8 kg + 7.
//   O^T = V^T P^T: these eight scores are already the second operand's eight values of the lane, no exchange needed; the first needs eight keys of one dimension in
//     a lane, which is how the values are stored (piece n of eight keys: D / 16 dimensions): decoding gives pairs of dimensions, two byte permutes pairs of keys.
//   In both results a column, i.e. lane % 16, is a query head, so the running maximum, the sum and the rescaling are the lane's own.
// The maximum moves only when a score is 2^8 times above it (the sums stand that easily), so most steps have no rescaling.  It begins at the lowest finite number, below
// every finite score, so that scores that are -inf in fp32 weigh nothing even where a wavefront has met no other yet.
// The weights of a bf16 output go into the matrix instructions as two bf16 parts (off by 2^-15 of a weight at most; one part, off by 2^-8, is as much again as the output's own rounding),
// those of an fp32 output as three, all of their 24 bits.  With up to eight query heads the two parts are columns of one instruction (PAIRED: column c is head c % 8, the
// upper eight columns have the second part; the scores are computed in both), added where the wavefronts meet, otherwise an instruction each.
template <typename T, int D, int NW, int NB, bool PAIRED>
__global__ void __launch_bounds__(NW * 64, NW == 4 ? 2 : 1) kv4_attn_kernel(const T* q, Kv4Caches<NB> kb, int H, int Hkv, float scale_log2e, float* __restrict__ part,
                                                                          T* out) {   // (may be q: a workgroup has read its heads' queries before it writes them)
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NP = F32 ? 3 : 1;                       // bf16 parts of a query
    constexpr int WP = F32 ? 3 : PAIRED ? 1 : 2;          // instructions for the parts of a weight
    static_assert(!(F32 && PAIRED), "three parts");
    constexpr int KW = D / 32, VM = D / 16, LD = D + 4;
    extern __shared__ __attribute__((aligned(16))) float lds[];   // [NW][group][LD] weighted values, then [NW][16][2] maximum and sum
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, kg = lane >> 4;
    const int g = blockIdx.y, grp = H / Hkv, head = PAIRED ? l16 & 7 : l16;   // the head of the lane's column
    float* const sml = lds + NW * grp * LD;
    int first;
    const int b = sequence_of(kb.end, (int)blockIdx.x, &first);
    const int ns = kb.end[b] - first, split = (int)blockIdx.x - first;
    const int64_t n = kb.n[b], cap = kb.cap[b], m0 = (int64_t)split * kb.per, m1 = m0 + kb.per < n ? m0 + kb.per : n;

    // the queries, columns beyond the group zero
    u32x4 qf[NP][KW];
    {
        const T* qh = q + ((int64_t)b * H + g * grp + (head < grp ? head : 0)) * D + kg * (D / 4);
#pragma unroll
        for (int i = 0; i < KW; ++i) {
            if constexpr (F32) {
                float v[8];
                u32x4 parts[NP];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = head < grp ? qh[8 * i + j] : 0.f;
                bf16_parts<NP>(v, parts);
#pragma unroll
                for (int p = 0; p < NP; ++p) qf[p][i] = parts[p];
            } else {
                qf[0][i] = head < grp ? *reinterpret_cast<const u32x4*>(qh + 8 * i) : u32x4{0, 0, 0, 0};
            }
        }
    }
    // a head's rows; a lane's offsets within 32 keys
    const char* const kh = kb.k[b] + (int64_t)g * cap * (D / 2);
    const char* const vh = kb.v[b] + (int64_t)g * cap * (D / 2);
    const uint8_t* const ksh = kb.ks[b] + (int64_t)g * cap * (D / 32);
    const uint8_t* const vsh = kb.vs[b] + (int64_t)g * cap * (D / 32);
    const int kblk = kg * (D / 4) / 32, vblk = l16 * (D / 16) / 32;
    int krow[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) krow[t] = 8 * (l16 >> 2) + 4 * t + (l16 & 3);

    // keys from key0 on (a multiple of 32, below m1); rows at and beyond n are not read
    auto load = [&](int64_t key0, Kv4Step<D>& s) {
        const int left = (int)(n - key0 < 32 ? n - key0 : 32);
        const char* kp = kh + key0 * (D / 2);
        const uint8_t* ksp = ksh + key0 * (D / 32);
        const char* vp = vh + key0 * (D / 2);
        const uint8_t* vsp = vsh + key0 * (D / 32);
        int row[2] = {krow[0], krow[1]}, grp8 = kg;
        if (left < 32) {
#pragma unroll
            for (int t = 0; t < 2; ++t) row[t] = row[t] < left ? row[t] : left - 1;
            grp8 = grp8 < (left + 7) / 8 ? grp8 : (left - 1) / 8;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            load_words<KW>(kp + (uint32_t)(row[t] * (D / 2) + kg * (D / 8)), s.k[t]);
            s.ks[t] = ksp[(uint32_t)(row[t] * (D / 32) + kblk)];
        }
        load_words<D / 16>(vp + (uint32_t)((grp8 * 16 + l16) * (D / 4)), s.v);
        load_words<2>((const char*)vsp + (uint32_t)((grp8 * (D / 32) + vblk) * 8), s.vs);
    };

    const float less = PAIRED && l16 >= 8 ? -1.f : 0.f;
    float m = KV4_LOWEST, l = 0.f;
    mfma_f32x4 acc[VM];
#pragma unroll
    for (int i = 0; i < VM; ++i) acc[i] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
    Kv4Step<D> next;
    int64_t key0 = m0 + wave * 32;
    if (key0 < m1) load(key0, next);
    for (; key0 < m1; key0 += NW * 32) {
        Kv4Step<D> cur = next;
        if (key0 + NW * 32 < m1) load(key0 + NW * 32, next);
        const int left = (int)(n - key0 < 32 ? n - key0 : 32);
        mfma_f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
            const float sc = __uint_as_float(cur.ks[t] << 23);
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                const u32x4 kf = fp4_decode8_bf16(cur.k[t][i], sc);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) s[t] = mfma16(kf, qf[p][i], s[t]);
            }
        }
        if (left < 32) {
            // the last keys: weights of rows that are not there are 0, and so are their values (the bytes may be anything)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (kg * 8 + j >= left) {
                    s[j / 4][j % 4] = -INFINITY;
                    const uint32_t clear = 0xffu << (8 * (j % 4));
                    cur.vs[j / 4] = (cur.vs[j / 4] & ~clear) | (0x7f7f7f7fu & clear);
                    if constexpr (D == 128) cur.v[j] = 0;
                    else if constexpr (D == 64) cur.v[j / 2] &= j % 2 ? 0xffffu : 0xffff0000u;
                    else cur.v[j / 4] &= ~clear;
                }
            }
        }
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))) * scale_log2e;
        if (__ballot(mx > m + 8.0f) != 0) {
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float mn = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int i = 0; i < VM; ++i) acc[i] *= alpha;
        }
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j / 4][j % 4], scale_log2e, -m));
        l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        u32x4 pf[WP];
        if constexpr (PAIRED) {
            // the lower columns have the rounded weight, the upper columns what that leaves
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t h = cvt_pk_bf16(p[2 * j], p[2 * j + 1]);
                pf[0][j] = cvt_pk_bf16(__builtin_fmaf(__uint_as_float(h << 16), less, p[2 * j]), __builtin_fmaf(__uint_as_float(h & 0xffff0000u), less, p[2 * j + 1]));
            }
        } else {
            bf16_parts<WP>(p, pf);
        }
        float vsc[8];
        vsc[0] = fp4_scale_of<0>(cur.vs[0]); vsc[1] = fp4_scale_of<1>(cur.vs[0]); vsc[2] = fp4_scale_of<2>(cur.vs[0]); vsc[3] = fp4_scale_of<3>(cur.vs[0]);
        vsc[4] = fp4_scale_of<0>(cur.vs[1]); vsc[5] = fp4_scale_of<1>(cur.vs[1]); vsc[6] = fp4_scale_of<2>(cur.vs[1]); vsc[7] = fp4_scale_of<3>(cur.vs[1]);
        auto weigh = [&](auto at) {   // dimensions 2 I and 2 I + 1 of the lane's piece
            constexpr int I = decltype(at)::value;
            const uint32_t d[8] = {value_pair<D, 0, I>(cur.v, vsc[0]), value_pair<D, 1, I>(cur.v, vsc[1]), value_pair<D, 2, I>(cur.v, vsc[2]), value_pair<D, 3, I>(cur.v, vsc[3]),
                                   value_pair<D, 4, I>(cur.v, vsc[4]), value_pair<D, 5, I>(cur.v, vsc[5]), value_pair<D, 6, I>(cur.v, vsc[6]), value_pair<D, 7, I>(cur.v, vsc[7])};
            u32x4 lo, hi;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lo[j] = __builtin_amdgcn_perm(d[2 * j + 1], d[2 * j], 0x05040100);
                hi[j] = __builtin_amdgcn_perm(d[2 * j + 1], d[2 * j], 0x07060302);
            }
#pragma unroll
            for (int p2 = WP - 1; p2 >= 0; --p2) {
                acc[2 * I] = mfma16(lo, pf[p2], acc[2 * I]);
                acc[2 * I + 1] = mfma16(hi, pf[p2], acc[2 * I + 1]);
            }
        };
        weigh(std::integral_constant<int, 0>{});
        if constexpr (D >= 64) weigh(std::integral_constant<int, 1>{});
        if constexpr (D >= 128) { weigh(std::integral_constant<int, 2>{}); weigh(std::integral_constant<int, 3>{}); }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if constexpr (PAIRED) {
#pragma unroll
        for (int i = 0; i < VM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][r] += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(acc[i][r]), 0x128, 0xF, 0xF, true));   // row_ror 8
    }
    // the wavefronts meet.  acc[i][r]: head l16, dimension (4 kg + r) D / 16 + i
    if (l16 < grp) {
        float* const to = lds + (wave * grp + l16) * LD + 4 * kg * VM;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < VM; ++i) to[r * VM + i] = acc[i][r];
        if (kg == 0) { sml[(wave * 16 + l16) * 2] = m; sml[(wave * 16 + l16) * 2 + 1] = l; }
    }
    __syncthreads();
    for (int t = tid; t < grp * D; t += NW * 64) {
        const int hg = t / D, e = t % D;
        float mn = KV4_LOWEST;
#pragma unroll
        for (int w = 0; w < NW; ++w) mn = fmaxf(mn, sml[(w * 16 + hg) * 2]);
        float ls = 0.f, o = 0.f;
#pragma unroll 4
        for (int w = 0; w < NW; ++w) {
            const float a = __builtin_amdgcn_exp2f(sml[(w * 16 + hg) * 2] - mn);
            ls += sml[(w * 16 + hg) * 2 + 1] * a;
            o += lds[(w * grp + hg) * LD + e] * a;
        }
        if (ns == 1) {
            out[((int64_t)b * H + g * grp + hg) * D + e] = from_f32<T>(n == 0 ? 0.f : o / ls);
        } else {
            float* dst = part + (((int64_t)blockIdx.x * Hkv + g) * grp + hg) * (D + 2);
            if (e == 0) { dst[0] = mn; dst[1] = ls; }
            dst[2 + e] = o;
        }
    }
}

// The splits of one query head meet: blockIdx.x = head, blockIdx.y = sequence, blockIdx.z = W of its dimensions; 512 / W groups of threads walk the splits.
constexpr int KV4_MAX_SPLITS = 256;
template <int NB> struct Kv4Ends { int32_t end[NB]; };
template <typename T, int D, int NB>
__global__ void __launch_bounds__(512) kv4_merge_kernel(const float* __restrict__ part, Kv4Ends<NB> sp, int H, int Hkv, T* __restrict__ out) {
    constexpr int W = 32, GROUPS = 512 / W, AHEAD = 4;
    __shared__ float sa[KV4_MAX_SPLITS], red[2][8], so[512];
    const int h = blockIdx.x, b = blockIdx.y, grp = H / Hkv, g = h / grp, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, e = blockIdx.z * W + tid % W;
    const int first = NB > 1 && b > 0 ? sp.end[NB > 1 ? b - 1 : 0] : 0, ns = sp.end[NB > 1 ? b : 0] - first;
    if (ns == 1) return;
    const float* base = part + (((int64_t)first * Hkv + g) * grp + h % grp) * (D + 2);
    const int64_t stride = (int64_t)H * (D + 2);
    const float m = tid < ns ? base[tid * stride] : -INFINITY, l = tid < ns ? base[tid * stride + 1] : 0.f;
    float early[AHEAD];   // the first values, asked for before their weights are known
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) early[i] = tid / W + i * GROUPS < ns ? base[(tid / W + i * GROUPS) * stride + 2 + e] : 0.f;
    float mx = m;
    for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
    if (lane == 0) red[0][wave] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    const float a = __builtin_amdgcn_exp2f(m - mx);
    if (tid < KV4_MAX_SPLITS) sa[tid] = a;
    float ls = l * a;
    for (int off = 32; off > 0; off >>= 1) ls += __shfl_xor(ls, off);
    if (lane == 0) red[1][wave] = ls;
    __syncthreads();
    const float L = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    float o = 0.f;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (tid / W + i * GROUPS < ns) o += early[i] * sa[tid / W + i * GROUPS];
#pragma unroll 4
    for (int s = tid / W + AHEAD * GROUPS; s < ns; s += GROUPS) o += base[s * stride + 2 + e] * sa[s];
    so[tid] = o;
    __syncthreads();
    if (tid >= W) return;
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) t += so[k * W + tid];
    out[((int64_t)b * H + h) * D + e] = from_f32<T>(t / L);
}

// Of up to KV4_FEW splits: a thread has a dimension and takes all of them at once, one round trip without a barrier.
constexpr int KV4_FEW = 16;
template <typename T, int D, int NB>
__global__ void __launch_bounds__(D) kv4_merge_few_kernel(const float* __restrict__ part, Kv4Ends<NB> sp, int H, int Hkv, T* __restrict__ out) {
    const int h = blockIdx.x, b = blockIdx.y, grp = H / Hkv, g = h / grp, e = threadIdx.x;
    const int first = NB > 1 && b > 0 ? sp.end[NB > 1 ? b - 1 : 0] : 0, ns = sp.end[NB > 1 ? b : 0] - first;
    if (ns == 1) return;
    const float* base = part + (((int64_t)first * Hkv + g) * grp + h % grp) * (D + 2);
    const int64_t stride = (int64_t)H * (D + 2);
    float m[KV4_FEW], l[KV4_FEW], o[KV4_FEW], mx = -INFINITY;
#pragma unroll
    for (int s = 0; s < KV4_FEW; ++s) {
        const float* const at = base + (s < ns ? s : 0) * stride;
        m[s] = s < ns ? at[0] : -INFINITY;
        l[s] = at[1];
        o[s] = at[2 + e];
    }
#pragma unroll
    for (int s = 0; s < KV4_FEW; ++s) mx = fmaxf(mx, m[s]);
    float L = 0.f, t = 0.f;
#pragma unroll
    for (int s = 0; s < KV4_FEW; ++s) {
        const float a = __builtin_amdgcn_exp2f(m[s] - mx);
        L += s < ns ? l[s] * a : 0.f;
        t += s < ns ? o[s] * a : 0.f;
    }
    out[((int64_t)b * H + h) * D + e] = from_f32<T>(t / L);
}

template <typename T, int D, int NW, int NB, bool PAIRED>
static hipError_t launch_kv4_attn_p(const T* q, const Kv4Batch& kb, int64_t per, int H, int Hkv, float* part, T* out, hipStream_t s) {
    Kv4Caches<NB> c{};
    Kv4Ends<NB> ends{};
    for (int b = 0; b < NB; ++b) {
        const int i = b < kb.n ? b : kb.n - 1;
        c.k[b] = (const char*)kb.k[i]; c.v[b] = (const char*)kb.v[i]; c.ks[b] = (const uint8_t*)kb.ks[i]; c.vs[b] = (const uint8_t*)kb.vs[i];
        c.cap[b] = (int32_t)kb.cap[i]; c.n[b] = (int32_t)kb.count[i];
        ends.end[b] = c.end[b] = (b > 0 ? c.end[b - 1] : 0) + (b < kb.n ? (int32_t)(kb.count[b] > per ? (kb.count[b] + per - 1) / per : 1) : 0);
    }
    c.per = (uint32_t)per;
    const int splits = c.end[NB - 1], lds = (NW * (H / Hkv) * (D + 4) + NW * 32) * (int)sizeof(float);
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(&kv4_attn_kernel<T, D, NW, NB, PAIRED>), (NW * KV4_MAX_GROUP * (D + 4) + NW * 32) * (int)sizeof(float));
    if (e != hipSuccess) return e;
    kv4_attn_kernel<T, D, NW, NB, PAIRED><<<dim3((unsigned)splits, (unsigned)Hkv), dim3(NW * 64), lds, s>>>(q, c, H, Hkv, 1.4426950408889634f / sqrtf((float)D), part, out);
    if (splits > kb.n) {
        // us by four workgroups a head / in one round trip: 16 sequences of up to 3000 / 13107 keys of 28 heads, 12 shares, 13.5 / 21.0 and 10.9 / 18.4; one sequence of 2000 keys, 16
        // shares, 7.5 and 7.5; many shares, 5000 / 13107 / 131072 keys of 32 heads, 40 or 64 shares, by four workgroups a head 8.3 / 9.5 / 27.9, by one a head 1.0 / 1.7 / 0.9 more
        int most = 1;
        for (int b = 0; b < kb.n; ++b) most = std::max(most, ends.end[b] - (b > 0 ? ends.end[b - 1] : 0));
        if (most > KV4_FEW) kv4_merge_kernel<T, D, NB><<<dim3((unsigned)H, (unsigned)kb.n, D / 32), dim3(512), 0, s>>>(part, ends, H, Hkv, out);
        else kv4_merge_few_kernel<T, D, NB><<<dim3((unsigned)H, (unsigned)kb.n), dim3(D), 0, s>>>(part, ends, H, Hkv, out);
    }
    return hipGetLastError();
}

// Pairing saves every step half of the value product's instructions and costs an addition of all sums at the end, so short caches (a step or two a wavefront) go without.
// us with one part of a weight / two, an instruction each / two, paired: 517 keys of 32 / 8 heads 6.0 / 6.2 / 6.5, 13107 keys 9.2 / 9.45 / 9.45, 131072 keys 27.4 / 27.9 / 27.6,
// 16 sequences of 1048 .. 13107 keys of 28 / 4 heads 17.6 / 18.5 / 18.1 (three parts, an instruction each: 6.6, 9.7, 30.4, 20.0).
template <typename T, int D, int NW, int NB>
static hipError_t launch_kv4_attn_n(const T* q, const Kv4Batch& kb, int64_t per, int H, int Hkv, float* part, T* out, hipStream_t s) {
    if constexpr (sizeof(T) == 2) {
        if (NW == 4 && H / Hkv <= 8) return launch_kv4_attn_p<T, D, NW, NB, true>(q, kb, per, H, Hkv, part, out, s);
    }
    return launch_kv4_attn_p<T, D, NW, NB, false>(q, kb, per, H, Hkv, part, out, s);
}

constexpr int KV4_WORKGROUPS = 512;   // two per CU
template <typename T, int D>
static hipError_t launch_kv4_attn_t(const T* q, const Kv4Batch& kb, int H, int Hkv, float* part, size_t part_floats, T* out, hipStream_t s) {
    constexpr int WIDE = sizeof(T) == 4 && D == 128 ? 8 : 16;   // wavefronts that a CU's registers hold
    constexpr int SHORT = WIDE * 64;
    int64_t total = 0, longest = 1;
    for (int b = 0; b < kb.n; ++b) { total += kb.count[b]; longest = kb.count[b] > longest ? kb.count[b] : longest; }
    // short caches whole, by one wide workgroup each: no second launch
    if (longest <= SHORT) {
        return kb.n == 1 ? launch_kv4_attn_n<T, D, WIDE, 1>(q, kb, SHORT, H, Hkv, part, out, s)
                         : launch_kv4_attn_n<T, D, WIDE, DECODE_MAX_BATCH>(q, kb, SHORT, H, Hkv, part, out, s);
    }
    // Shares of equal length over all sequences, none below 128 keys, the shortest with which no CU gets a third workgroup: 131072 keys of 8 heads in 64 / 60 /
    // 70 / 128 shares 27.9 / 28.9 / 35.0 / 29.7 us; 16 sequences of 1048 .. 13107 keys, 4 heads, room for 480 / 512 / 560 / 1024 workgroups 18.3 / 18.4 / 21.4 / 22.8 us.  Sequences and heads that are many on their own
    // have room for four shares a sequence nevertheless, else the longest one's workgroups stay behind: the same sequences, 32 heads, 1 / 2 / 4 / 8 shares a sequence on average 118.5 /
    // 96.7 / 87.9 / 85.9 us; 16 of 120 .. 1500 keys in fp32, 32 heads of 64, 15.1 / 15.4 / 15.9 / 19.2.
    const int64_t most = std::max<int64_t>(KV4_WORKGROUPS, 4 * (int64_t)kb.n * Hkv);
    int64_t per = (total * Hkv + most - 1) / most;
    per = per < 128 ? 128 : per > (1 << 30) ? (1 << 30) : (per + 31) / 32 * 32;
    const int64_t room = (int64_t)(part_floats / ((size_t)H * (D + 2)));
    for (;; per += (per / 64 + 31) / 32 * 32) {
        int64_t splits = 0;
        for (int b = 0; b < kb.n; ++b) splits += kb.count[b] > per ? (kb.count[b] + per - 1) / per : 1;
        if (longest <= per * KV4_MAX_SPLITS && (splits == kb.n || (splits <= room && splits * Hkv <= most))) break;
    }
    return kb.n == 1 ? launch_kv4_attn_n<T, D, 4, 1>(q, kb, per, H, Hkv, part, out, s)
                     : launch_kv4_attn_n<T, D, 4, DECODE_MAX_BATCH>(q, kb, per, H, Hkv, part, out, s);
}

hipError_t launch_kv4_attn(const void* q, const Kv4Batch& kb, int H, int Hkv, int d, float* part, size_t part_floats, void* out, bool bf16, hipStream_t s) {
#define SPTS_KV4_ATTN(D_)                                                                                                                   \
    return bf16 ? launch_kv4_attn_t<bf16_t, D_>((const bf16_t*)q, kb, H, Hkv, part, part_floats, (bf16_t*)out, s)                           \
                : launch_kv4_attn_t<float, D_>((const float*)q, kb, H, Hkv, part, part_floats, (float*)out, s);
    switch (d) {
        case 128: SPTS_KV4_ATTN(128)
        case 64: SPTS_KV4_ATTN(64)
        case 32: SPTS_KV4_ATTN(32)
        default: return hipErrorInvalidValue;
    }
#undef SPTS_KV4_ATTN
}

}  // namespace spts
