// Attention of a chunk of new tokens of each sequence over its cache in pages, and the attention that every cached row got.
//
//   out[i, h] = sum_{j <= c + i} p_ij v_j,  p_ij = softmax_j(q[i, h] . k_j / sqrt(d)),  c = rows cached before the chunk
//   weight[j] = decay * weight[j] + sum_{i, h} p_ij
//
// The queries of a key/value head are columns: column n of sequence b is query n / G, head n % G of the G heads that read it, so that any group and any chunk
// fill blocks of 32 columns and a key that is loaded serves them all.
#include "spts_lanes.h"

#include <algorithm>

namespace spts {

namespace {
typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LOWEST = -3.402823466e38f;   // a running maximum starts here: below every finite score, and a score of -inf then weighs 2^-inf = 0

// A kernel's view of up to NB sequences
template <int NB> struct PagedSeqs {
    const int32_t* table[NB];
    float* weight[NB];
    int32_t count[NB], first[NB], nq[NB];   // rows, the call's first query row, queries
    int32_t end[NB];                        // work items of the sequences up to here
    int32_t at[NB];                         // first row of sequence b in arrays over all sequences' rows (weights) / first partial result (attention)
};
struct Pool { const char* k; const char* v; uint32_t pages; int32_t shift; };

template <int NB> __device__ inline int seq_of(const int32_t (&end)[NB], int i, int* first) {
    int b = 0;
    *first = 0;
#pragma unroll
    for (int j = 0; j + 1 < NB; ++j)
        if (i >= end[j]) { b = j + 1; *first = end[j]; }
    return b;
}
// element offset of the first row of a page's half of 16 rows that holds `row` (a multiple of 16)
__device__ inline int64_t page_at(const Pool& pool, const int32_t* table, int64_t row, int g, int Hkv, int D) {
    uint32_t id = (uint32_t)table[row >> pool.shift];
    id = id < pool.pages ? id : 0;
    return (((int64_t)id * Hkv + g) << pool.shift) * D + (row & ((1 << pool.shift) - 1)) * D;
}

__device__ inline f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
__device__ inline f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}
// N consecutive elements as fp32 (16-byte aligned)
template <int N> __device__ inline void load_row(const float* p, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i + e] = w[e];
    }
}
template <int N> __device__ inline void load_row(const bf16_t* p, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(p + i);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i + e] = chunk_elem(w, e, bf16_t{});
    }
}
}  // namespace

// On the fp32 matrix instruction 32x32x2.  S^T = K Q^T: operand rows are keys, columns queries; of the two halves of a wavefront one multiplies the first, one the second half of the
// dimensions, so a lane's operand is half a row.  O^T += V^T P^T: result element r of lane (l, half) is key 8 (r / 4) + 4 half + r % 4 of column l, which is the second operand of the
// r-th product of V^T as it stands.  The four wavefronts of a workgroup take blocks of 32 keys in turn and meet in LDS.
// A block that some column does not see entirely has its scores set to -inf there, and values that are not finite kept out of the product (0 times them would be NaN): two more products
// count those that a column does see and put the infinity or NaN where it belongs.
constexpr int AW = 4;
template <typename T, int D, int NB>
__global__ void __launch_bounds__(AW * 64) kvp_attn_kernel(const T* q, Pool pool, PagedSeqs<NB> sq, int H, int Hkv, int64_t per, float c, float* __restrict__ part,
                                                           float2* __restrict__ stats, T* out) {
    constexpr int DB = D / 32, LD = D + 4;
    __shared__ float so[AW][32][LD];
    __shared__ float sm[AW][32], sl[AW][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh = lane >> 5;
    const int g = (int)(blockIdx.x % Hkv), G = H / Hkv;
    int first;
    const int b = seq_of(sq.end, (int)(blockIdx.x / Hkv), &first);
    const int item = (int)(blockIdx.x / Hkv) - first;
    const int n = sq.count[b], nq = sq.nq[b], cols = nq * G, blocks = (cols + 31) / 32;
    const int splits = (int)((n + per - 1) / per), split = item % splits, blk = blocks - 1 - item / splits;
    const int32_t* const table = sq.table[b];
    const int col = blk * 32 + l32, cc = col < cols ? col : cols - 1, last = blk * 32 + 31 < cols ? blk * 32 + 31 : cols - 1;
    const int seen = n - nq + cc / G + 1;                                   // keys that the lane's column sees
    const int seen_all = n - nq + blk * 32 / G + 1, seen_any = n - nq + last / G + 1;
    const int64_t k0 = split * per, k1 = k0 + per < seen_any ? k0 + per : seen_any;

    float qf[D / 2];
    load_row(q + ((int64_t)(sq.first[b] + cc / G) * H + g * G + cc % G) * D + lh * (D / 2), qf);
    f32x16 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = zero16();
    float m = LOWEST, l = 0.f;
    for (int64_t key0 = k0 + wave * 32; key0 < k1; key0 += AW * 32) {
        const int left = (int)(n - key0 < 32 ? n - key0 : 32);
        const int64_t p0 = page_at(pool, table, key0, g, Hkv, D), p1 = left > 16 ? page_at(pool, table, key0 + 16, g, Hkv, D) - 16 * D : p0;
        const int row = l32 < left ? l32 : left - 1;
        f32x16 s = zero16();
        {
            float kf[D / 2];
            load_row((const T*)pool.k + (row < 16 ? p0 : p1) + row * D + lh * (D / 2), kf);
#pragma unroll
            for (int i = 0; i < D / 2; ++i) s = mfma_f32(kf[i], qf[i], s);
        }
        const bool masked = key0 + 32 > seen_all;
        float mx = LOWEST;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int64_t key = key0 + 8 * (r >> 2) + 4 * lh + (r & 3);
            s[r] = masked && key >= seen ? -INFINITY : s[r] * c;
            mx = fmaxf(mx, s[r]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mn = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r] - m);
            l += s[r];
        }
#pragma unroll
        for (int i = 0; i < DB; ++i) {
            float vf[16];
            bool odd = false;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int at = 8 * (r >> 2) + 4 * lh + (r & 3), vr = at < left ? at : left - 1;
                vf[r] = to_f32(((const T*)pool.v)[(vr < 16 ? p0 : p1) + vr * D + 32 * i + l32]);
                odd |= !(fabsf(vf[r]) < INFINITY);
            }
            if (masked && __ballot(odd) != 0) {
                f32x16 up = zero16(), down = zero16();
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float sees = key0 + 8 * (r >> 2) + 4 * lh + (r & 3) < seen ? 1.f : 0.f;
                    const float v = vf[r];
                    up = mfma_f32(v == INFINITY || v != v ? 1.f : 0.f, sees, up);
                    down = mfma_f32(v == -INFINITY || v != v ? 1.f : 0.f, sees, down);
                    vf[r] = fabsf(v) < INFINITY ? v : 0.f;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] += (up[r] > 0.f ? INFINITY : 0.f) - (down[r] > 0.f ? INFINITY : 0.f);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i] = mfma_f32(vf[r], s[r], o[i]);
        }
    }
    l += __shfl_xor(l, 32);
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) so[wave][l32][32 * i + 8 * (r >> 2) + 4 * lh + (r & 3)] = o[i][r];
    if (lh == 0) { sm[wave][l32] = m; sl[wave][l32] = l; }
    __syncthreads();
    // D / 4 threads a column
    for (int i = tid; i < 32 * (D / 4); i += AW * 64) {
        const int cl = i / (D / 4), e = i % (D / 4) * 4, cn = blk * 32 + cl;
        if (cn >= cols) continue;
        float M = LOWEST, L = 0.f;
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < AW; ++w) M = fmaxf(M, sm[w][cl]);
#pragma unroll
        for (int w = 0; w < AW; ++w) {
            const float a = __builtin_amdgcn_exp2f(sm[w][cl] - M);
            L += sl[w][cl] * a;
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] += so[w][cl][e + j] * a;
        }
        if (splits > 1) {
            float* const to = part + ((int64_t)sq.at[b] + ((int64_t)split * Hkv + g) * cols + cn) * (D + 2);
            if (e == 0) { to[0] = M; to[1] = L; }
#pragma unroll
            for (int j = 0; j < 4; ++j) to[2 + e + j] = t[j];
        } else {
            const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;
            const int64_t head = (int64_t)(sq.first[b] + cn / G) * H + g * G + cn % G;
#pragma unroll
            for (int j = 0; j < 4; ++j) out[head * D + e + j] = from_f32<T>(t[j] * inv);
            if (stats && e == 0) stats[head] = make_float2(M, inv);
        }
    }
}

// The shares of a head's keys, one workgroup of D threads per query and head
template <typename T, int NB>
__global__ void kvp_merge_kernel(const float* __restrict__ part, PagedSeqs<NB> sq, int H, int Hkv, int64_t per, float2* __restrict__ stats, T* __restrict__ out) {
    const int h = blockIdx.x % H, G = H / Hkv, D = blockDim.x, e = threadIdx.x;
    const int64_t row = blockIdx.x / H;
    int b = 0;
#pragma unroll
    for (int j = 1; j < NB; ++j)
        if (sq.nq[j] > 0 && row >= sq.first[j]) b = j;
    const int splits = (int)((sq.count[b] + per - 1) / per), cols = sq.nq[b] * G;
    if (splits <= 1) return;
    const int cn = (int)(row - sq.first[b]) * G + h % G;
    const float* const base = part + ((int64_t)sq.at[b] + (int64_t)(h / G) * cols + cn) * (D + 2);
    const int64_t stride = (int64_t)Hkv * cols * (D + 2);
    float M = LOWEST, L = 0.f, t = 0.f;
    for (int s = 0; s < splits; ++s) M = fmaxf(M, base[s * stride]);
    for (int s = 0; s < splits; ++s) {
        const float a = __builtin_amdgcn_exp2f(base[s * stride] - M);
        L += base[s * stride + 1] * a;
        t += base[s * stride + 2 + e] * a;
    }
    const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;
    out[(row * H + h) * D + e] = from_f32<T>(t * inv);
    if (stats && e == 0) stats[row * H + h] = make_float2(M, inv);
}

// Column sums of the probabilities: a wavefront holds the keys of 32 rows and goes over the blocks of columns of its part of all heads, the scores anew (storing them would be
// more bytes than the products cost, but for a few columns); stats has each column's maximum and 1 / sum.
template <typename T, int D, int NB>
__global__ void __launch_bounds__(AW * 64) kvp_weights_kernel(const T* __restrict__ q, Pool pool, PagedSeqs<NB> sq, int H, int Hkv, int parts, int64_t rows, float c,
                                                              const float2* __restrict__ stats, float* __restrict__ wpart, float decay) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh = lane >> 5, G = H / Hkv;
    const int p = (int)(blockIdx.x % parts);
    int first;
    const int b = seq_of(sq.end, (int)(blockIdx.x / parts), &first);
    const int n = sq.count[b], nq = sq.nq[b], cols = nq * G, blocks = (cols + 31) / 32;
    const int64_t key0 = ((int64_t)(blockIdx.x / parts) - first) * (AW * 32) + wave * 32;
    if (key0 >= n) return;
    const int left = (int)(n - key0 < 32 ? n - key0 : 32), row = l32 < left ? l32 : left - 1;
    const int64_t total = (int64_t)blocks * Hkv;
    const int64_t i0 = total * p / parts, i1 = total * (p + 1) / parts;
    float acc[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    float kf[D / 2];
    int have = -1;
    for (int64_t i = i0; i < i1; ++i) {
        const int g = (int)(i / blocks), blk = (int)(i % blocks);
        const int col = blk * 32 + l32, cc = col < cols ? col : cols - 1, last = blk * 32 + 31 < cols ? blk * 32 + 31 : cols - 1;
        if (key0 >= n - nq + last / G + 1) continue;
        if (g != have) {
            have = g;
            load_row((const T*)pool.k + page_at(pool, sq.table[b], key0 + (row & 16), g, Hkv, D) + (row & 15) * D + lh * (D / 2), kf);
        }
        const int64_t head = (int64_t)(sq.first[b] + cc / G) * H + g * G + cc % G;
        float qf[D / 2];
        load_row(q + head * D + lh * (D / 2), qf);
        const float2 st = stats[head];
        const int seen = col < cols ? n - nq + cc / G + 1 : 0;
        f32x16 s = zero16();
#pragma unroll
        for (int j = 0; j < D / 2; ++j) s = mfma_f32(kf[j], qf[j], s);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int64_t key = key0 + 8 * (r >> 2) + 4 * lh + (r & 3);
            const float e = __builtin_amdgcn_exp2f(s[r] * c - st.x) * st.y;
            acc[r] += key < seen ? e : 0.f;
        }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const float w = group_sum<32>(acc[r]);
        const int64_t key = key0 + 8 * (r >> 2) + 4 * lh + (r & 3);
        if (l32 != 0 || key >= n) continue;
        if (parts > 1) wpart[p * rows + sq.at[b] + key] = w;
        else sq.weight[b][key] = decay == 0.f ? w : decay * sq.weight[b][key] + w;
    }
}

template <int NB>
__global__ void __launch_bounds__(256) kvp_add_weights_kernel(const float* __restrict__ wpart, PagedSeqs<NB> sq, int parts, int64_t rows, float decay) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows) return;
    int b = 0;
#pragma unroll
    for (int j = 1; j < NB; ++j)
        if (sq.nq[j] > 0 && i >= sq.at[j]) b = j;
    float w = 0.f;
    for (int p = 0; p < parts; ++p) w += wpart[p * rows + i];
    float* const at = sq.weight[b] + (i - sq.at[b]);
    *at = decay == 0.f ? w : decay * *at + w;
}

size_t kvp_attn_min_floats(int64_t rows, int H) { return ((size_t)rows * H * 2 + 63) / 64 * 64; }   // the statistics of every column

constexpr int64_t ATT_WORKGROUPS = 1024;
template <typename T, int D, int NB>
static hipError_t launch_kvp_attn_t(const T* q, const PagedPool& pool, const PagedBatch& pb, int H, int Hkv, float* part, size_t part_floats, T* out, bool add, float decay,
                                    hipStream_t s) {
    const int G = H / Hkv;
    const int64_t rows = pb.off[pb.n];
    const float c = LOG2E / sqrtf((float)D);
    const Pool pl{(const char*)pool.k, (const char*)pool.v, (uint32_t)pool.pages, pool.shift};
    float2* const stats = add ? (float2*)part : nullptr;
    const size_t used = add ? kvp_attn_min_floats(rows, H) : 0;
    float* const rest = part + used;
    const size_t room = part_floats - used;
    int64_t total = 0, blocks = 0;   // keys times blocks of columns
    for (int b = 0; b < pb.n; ++b) {
        const int64_t nb = ((pb.off[b + 1] - pb.off[b]) * G + 31) / 32;
        total += nb * pb.count[b];
        blocks += nb;
    }
    // keys of a share: the chip's workgroups where blocks of columns and heads are few
    int64_t per = (total * Hkv + ATT_WORKGROUPS - 1) / ATT_WORKGROUPS;
    per = per < 256 ? 256 : (per + 127) / 128 * 128;
    auto splits_of = [&](int b) { return (pb.count[b] + per - 1) / per; };
    for (;; per *= 2) {
        int64_t floats = 0, split = 0;
        for (int b = 0; b < pb.n; ++b)
            if (splits_of(b) > 1) { floats += splits_of(b) * (pb.off[b + 1] - pb.off[b]) * H * (D + 2); split += pb.off[b + 1] - pb.off[b]; }
        if (split == 0 || ((size_t)floats <= room && floats <= 0x7fffffff)) break;
    }
    PagedSeqs<NB> sq{};
    int64_t items = 0, parts_at = 0, most = 1;
    for (int b = 0; b < NB; ++b) {
        if (b < pb.n) {
            const int64_t nq = pb.off[b + 1] - pb.off[b], sp = splits_of(b);
            sq.table[b] = pb.table[b]; sq.weight[b] = pb.weight[b];
            sq.count[b] = (int32_t)pb.count[b]; sq.first[b] = (int32_t)pb.off[b]; sq.nq[b] = (int32_t)nq; sq.at[b] = (int32_t)parts_at;
            items += (nq * G + 31) / 32 * sp;
            if (nq > 0 && sp > 1) { parts_at += sp * nq * H; most = std::max(most, sp); }
        }
        sq.end[b] = (int32_t)items;
    }
    if (items * Hkv > 0x7fffffff) return hipErrorInvalidValue;
    kvp_attn_kernel<T, D, NB><<<dim3((unsigned)(items * Hkv)), dim3(AW * 64), 0, s>>>(q, pl, sq, H, Hkv, per, c, rest, stats, out);
    if (most > 1) kvp_merge_kernel<T, NB><<<dim3((unsigned)(rows * H)), dim3(D), 0, s>>>(rest, sq, H, Hkv, per, stats, out);
    if (add) {
        int64_t tiles = 0, keys = 0;
        for (int b = 0; b < NB; ++b) {
            if (b < pb.n && sq.nq[b] > 0) {
                sq.at[b] = (int32_t)keys;
                keys += pb.count[b];
                tiles += (pb.count[b] + AW * 32 - 1) / (AW * 32);
            }
            sq.end[b] = (int32_t)tiles;
        }
        int64_t parts = std::max<int64_t>(1, std::min<int64_t>({ATT_WORKGROUPS / std::max<int64_t>(1, tiles), blocks * Hkv, (int64_t)(room / (size_t)keys)}));
        if (tiles * parts > 0x7fffffff) return hipErrorInvalidValue;
        kvp_weights_kernel<T, D, NB><<<dim3((unsigned)(tiles * parts)), dim3(AW * 64), 0, s>>>(q, pl, sq, H, Hkv, (int)parts, keys, c, stats, rest, decay);
        if (parts > 1) kvp_add_weights_kernel<NB><<<dim3((unsigned)((keys + 255) / 256)), dim3(256), 0, s>>>(rest, sq, (int)parts, keys, decay);
    }
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_kvp_attn_d(const T* q, const PagedPool& pool, const PagedBatch& pb, int H, int Hkv, int d, float* part, size_t part_floats, T* out, bool add, float decay,
                                    hipStream_t s) {
#define SPTS_KVP_ATTN(D_)                                                                                                                   \
    return pb.n == 1 ? launch_kvp_attn_t<T, D_, 1>(q, pool, pb, H, Hkv, part, part_floats, out, add, decay, s)                              \
                     : launch_kvp_attn_t<T, D_, DECODE_MAX_BATCH>(q, pool, pb, H, Hkv, part, part_floats, out, add, decay, s);
    switch (d) {
        case 128: SPTS_KVP_ATTN(128)
        case 64: SPTS_KVP_ATTN(64)
        case 32: SPTS_KVP_ATTN(32)
        default: return hipErrorInvalidValue;
    }
#undef SPTS_KVP_ATTN
}

hipError_t launch_kvp_attn(const void* q, const PagedPool& pool, const PagedBatch& pb, int H, int Hkv, int d, float* part, size_t part_floats, void* out, bool add, float decay,
                           bool bf16, hipStream_t s) {
    if (pb.n < 1 || pb.n > DECODE_MAX_BATCH || pb.off[pb.n] < 1) return hipErrorInvalidValue;
    return bf16 ? launch_kvp_attn_d<bf16_t>((const bf16_t*)q, pool, pb, H, Hkv, d, part, part_floats, (bf16_t*)out, add, decay, s)
                : launch_kvp_attn_d<float>((const float*)q, pool, pb, H, Hkv, d, part, part_floats, (float*)out, add, decay, s);
}

}  // namespace spts
