// Attention of a chunk of new tokens of each sequence over its cache in pages, and the attention that every cached row got.
//
//   out[i, h] = sum_{j <= c + i} p_ij v_j,  p_ij = softmax_j(q[i, h] . k_j / sqrt(d)),  c = rows cached before the chunk
//   weight[j] = decay * weight[j] + sum_{i, h} p_ij
//
// The queries of a key/value head are columns: column n of sequence b is query n / G, head n % G of the G heads that read it, so that any group and any chunk
// fill blocks of 32 columns and a key that is loaded serves them all.
#include "spts_paged.h"

#include <algorithm>

namespace spts {

namespace {
typedef paged_f32x16 f32x16;
__device__ inline f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
// N of 2 N elements, every other four (16-byte aligned)
template <int N> __device__ inline void load_quads(const float* p, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(p + 2 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i + e] = w[e];
    }
}
__device__ inline void store4(float* p, f32x4 v, float f) { *reinterpret_cast<f32x4*>(p) = f32x4{v[0] * f, v[1] * f, v[2] * f, v[3] * f}; }
__device__ inline void store4(bf16_t* p, f32x4 v, float f) { *reinterpret_cast<u32x2*>(p) = u32x2{cvt_pk_bf16(v[0] * f, v[1] * f), cvt_pk_bf16(v[2] * f, v[3] * f)}; }
}  // namespace

// On the fp32 matrix instruction 32x32x2.  S^T = K Q^T: operand rows are keys, columns queries; the two halves of a wavefront multiply every other four of the dimensions, so a lane's
// operand is half a row and a load takes 32 bytes of each key (halves that are 64 dimensions apart touch twice the lines a load, more than the first cache holds until the rest of them is
// wanted: 128 tokens after 3872 rows of 8 heads of 4, d = 128, 126 us for 115, their accounts 57 for 45).  O^T += V^T P^T: result element r of lane (l, half) is key
// 8 (r / 4) + 4 half + r % 4 of column l, which is the second operand of the r-th product of V^T as it stands.  The four wavefronts of a workgroup take blocks of 32 keys in turn and meet in
// LDS; a lane asks for the next piece of a key, and the next 32 dimensions of the values, before it multiplies these: those 128 tokens 99 us with the
// rows in the last cache and 117 behind a kernel that wrote 1 GB, 84 and 71 TFLOP/s of the 154 that a large fp32 product reaches here.
// A block that some column does not see entirely has its scores set to -inf there, and values that are not finite kept out of the product (0 times them would be NaN): two more products
// count those that a column does see and put the infinity or NaN where it belongs.
constexpr int AW = 4;
template <int D, int NB>
__global__ void __launch_bounds__(AW * 64, 2) kvp_attn_kernel(const float* q, PoolView pool, PagedSeqs<NB> sq, int H, int Hkv, float c, Shares sh, float2* __restrict__ stats,
                                                              float* out) {   // (out may be q: a workgroup has read its columns before it writes them)
    constexpr int DB = D / 32, LD = D + 4;
    __shared__ float so[AW][32][LD];
    __shared__ float sm[AW][32], sl[AW][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh = lane >> 5;
    const int g = (int)(blockIdx.x % Hkv), G = H / Hkv;
    int first;
    const int b = seq_of(sq.end, (int)(blockIdx.x / Hkv), &first);
    const int item = (int)(blockIdx.x / Hkv) - first;
    const int n = sq.count[b], nq = sq.nq[b], cols = nq * G, blocks = (cols + 31) / 32;
    const int splits = sq.splits[b], split = item % splits, blk = blocks - 1 - item / splits;
    const int32_t* const table = sq.table[b];
    const int col = blk * 32 + l32, cc = col < cols ? col : cols - 1, last = blk * 32 + 31 < cols ? blk * 32 + 31 : cols - 1;
    const int seen = n - nq + cc / G + 1;                                   // keys that the lane's column sees
    const int seen_all = n - nq + blk * 32 / G + 1, seen_any = n - nq + last / G + 1;
    const int64_t k0 = (int64_t)split * sq.per[b], k1 = k0 + sq.per[b] < seen_any ? k0 + sq.per[b] : seen_any;

    float qf[D / 2];
    load_quads(q + ((int64_t)(sq.first[b] + cc / G) * H + g * G + cc % G) * D + 4 * lh, qf);
    f32x16 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = zero16();
    float m = PAGED_LOWEST, l = 0.f;
    constexpr int CH = D == 128 ? 8 : 16, NCH = D / 2 / CH;          // a lane's half row of a key in pieces, the next one on its way
    struct Rows { const float *k, *v; int64_t upper; };             // the lane's key; element 4 lh of dimension l32 of the block's values, and what lies between its halves of 16 rows
    auto rows_of = [&](int64_t key0) {
        const int left = (int)(n - key0 < 32 ? n - key0 : 32), row = l32 < left ? l32 : left - 1;
        const int64_t p0 = page_at(pool, table, key0, g, Hkv, D), p1 = left > 16 ? page_at(pool, table, key0 + 16, g, Hkv, D) : p0 + 16 * D;
        return Rows{(const float*)pool.k + (row < 16 ? p0 + row * D : p1 + (row - 16) * D) + 4 * lh, (const float*)pool.v + p0 + 4 * lh * D + l32, p1 - p0 - 16 * D};
    };
    auto load_key = [&](const Rows& at, int ch, float (&v)[CH]) __attribute__((always_inline)) { load_quads(at.k + 2 * ch * CH, v); };
    auto load_values = [&](const Rows& at, int i, int left, float (&v)[16]) __attribute__((always_inline)) {
        if (left == 32) {
#pragma unroll
            for (int r = 0; r < 16; ++r) v[r] = at.v[(r < 8 ? 0 : at.upper) + (8 * (r >> 2) + (r & 3)) * D + 32 * i];
        } else {   // rows behind the last one are the last one again
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int want = 8 * (r >> 2) + 4 * lh + (r & 3), row = want < left ? want : left - 1;
                v[r] = at.v[(row < 16 ? 0 : at.upper) + (row - 4 * lh) * D + 32 * i];
            }
        }
    };
    int64_t key0 = k0 + wave * 32;
    Rows here{};
    float kb[2][CH], vb[2][16];
    if (key0 < k1) {
        here = rows_of(key0);
        load_key(here, 0, kb[0]);
    }
    for (; key0 < k1; key0 += AW * 32) {
        const int left = (int)(n - key0 < 32 ? n - key0 : 32);
        f32x16 s = zero16();
#pragma unroll
        for (int ch = 0; ch < NCH; ++ch) {
            if (ch + 1 < NCH) load_key(here, ch + 1, kb[(ch + 1) & 1]);
            else load_values(here, 0, left, vb[0]);
#pragma unroll
            for (int i = 0; i < CH; ++i) s = mfma_f32(kb[ch & 1][i], qf[ch * CH + i], s);
        }
        const bool masked = key0 + 32 > seen_all;
        float mx = PAGED_LOWEST;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = masked && (int)(seen - key0) - 4 * lh <= 8 * (r >> 2) + (r & 3) ? -INFINITY : s[r] * c;
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
        Rows next = here;
        if (key0 + AW * 32 < k1) next = rows_of(key0 + AW * 32);
#pragma unroll
        for (int i = 0; i < DB; ++i) {
            if (i + 1 < DB) load_values(here, i + 1, left, vb[(i + 1) & 1]);
            else load_key(next, 0, kb[0]);
            float (&vf)[16] = vb[i & 1];
            if (masked) {
                bool odd = false;
#pragma unroll
                for (int r = 0; r < 16; ++r) odd |= !(fabsf(vf[r]) < INFINITY);
                if (__ballot(odd) != 0) {
                    f32x16 up = zero16(), down = zero16();
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float sees = (int)(seen - key0) - 4 * lh > 8 * (r >> 2) + (r & 3) ? 1.f : 0.f;
                        const float v = vf[r];
                        up = mfma_f32(v == INFINITY || v != v ? 1.f : 0.f, sees, up);
                        down = mfma_f32(v == -INFINITY || v != v ? 1.f : 0.f, sees, down);
                        vf[r] = fabsf(v) < INFINITY ? v : 0.f;
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[i][r] += (up[r] > 0.f ? INFINITY : 0.f) - (down[r] > 0.f ? INFINITY : 0.f);
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i] = mfma_f32(vf[r], s[r], o[i]);
        }
        here = next;
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
        float M = PAGED_LOWEST, L = 0.f;
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
            const int64_t to = (int64_t)sq.at[b] + ((int64_t)split * Hkv + g) * cols + cn;
            if (e == 0) sh.ml[to] = make_float2(M, L);
            *reinterpret_cast<f32x4*>(sh.o + to * D + e) = t;
        } else {
            const float inv = inverse_sum(L);
            const int64_t head = (int64_t)(sq.first[b] + cn / G) * H + g * G + cn % G;
#pragma unroll
            for (int j = 0; j < 4; ++j) out[head * D + e + j] = t[j] * inv;
            if (stats && e == 0) stats[head] = make_float2(M, inv);
        }
    }
}

// The shares of a column's keys, up to MOST: D / 4 threads a column, which ask for everything at once
constexpr int MERGE_T = 256;
template <typename T, int D, int NB, int MOST>
__global__ void __launch_bounds__(MERGE_T) kvp_merge_few_kernel(Shares sh, PagedSeqs<NB> sq, uint32_t total, int H, int Hkv, float2* __restrict__ stats, T* __restrict__ out) {
    constexpr uint32_t TG = D / 4;
    const uint32_t item = blockIdx.x * (MERGE_T / TG) + threadIdx.x / TG;   // query and head among those of sequences in shares
    if (item >= total) return;
    const int e = (int)(threadIdx.x % TG) * 4, row = (int)(item / (uint32_t)H), h = (int)item - row * H, G = H / Hkv, g = h / G;
    int first;
    const int b = seq_of(sq.end, row, &first);
    const int qi = row - first, splits = sq.splits[b], cols = sq.nq[b] * G;
    const int64_t base = (int64_t)sq.at[b] + g * cols + qi * G + (h - g * G), step = (int64_t)Hkv * cols;
    float2 ml[MOST];
    f32x4 o[MOST];
#pragma unroll
    for (int s = 0; s < MOST; ++s) {   // (all at once; those that are not there weigh nothing)
        const int64_t at = base + (s < splits ? s : 0) * step;
        ml[s] = sh.ml[at];
        o[s] = *reinterpret_cast<const f32x4*>(sh.o + at * D + e);
    }
    float M = PAGED_LOWEST, L = 0.f;
#pragma unroll
    for (int s = 0; s < MOST; ++s) M = fmaxf(M, s < splits ? ml[s].x : PAGED_LOWEST);
    f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < MOST; ++s) {
        const float a = __builtin_amdgcn_exp2f(ml[s].x - M);
        L += s < splits ? ml[s].y * a : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] += s < splits ? o[s][j] * a : 0.f;
    }
    const float inv = inverse_sum(L);
    const int64_t head = (int64_t)(sq.first[b] + qi) * H + h;
    store4(out + head * D + e, t, inv);
    if (stats && e == 0) stats[head] = make_float2(M, inv);
}

// ... and many: a workgroup a column.  Every wavefront finds the column's maximum and sum (a lane a share), then groups of D / 4 threads take shares in turn.
template <typename T, int D, int NB>
__global__ void __launch_bounds__(MERGE_T) kvp_merge_kernel(Shares sh, PagedSeqs<NB> sq, int H, int Hkv, float2* __restrict__ stats, T* __restrict__ out) {
    constexpr int TG = D / 4, GROUPS = MERGE_T / TG;
    __shared__ float so[GROUPS][D];
    const int h = blockIdx.x % H, G = H / Hkv, tid = threadIdx.x, lane = tid & 63, grp = tid / TG, e = tid % TG * 4;
    int first;
    const int b = seq_of(sq.end, (int)(blockIdx.x / H), &first);   // (of sequences in shares)
    const int qi = (int)(blockIdx.x / H) - first, splits = sq.splits[b], cols = sq.nq[b] * G;
    const int64_t base = (int64_t)sq.at[b] + (int64_t)(h / G) * cols + qi * G + h % G, step = (int64_t)Hkv * cols;
    float M = PAGED_LOWEST, L = 0.f;
    for (int s = lane; s < splits; s += 64) M = fmaxf(M, sh.ml[base + s * step].x);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
    for (int s = lane; s < splits; s += 64) {
        const float2 w = sh.ml[base + s * step];
        L += w.y * __builtin_amdgcn_exp2f(w.x - M);
    }
    L = wave_sum(L);
    f32x4 t = {0.f, 0.f, 0.f, 0.f};
    for (int s = grp; s < splits; s += GROUPS) {
        const float a = __builtin_amdgcn_exp2f(sh.ml[base + s * step].x - M);
        const f32x4 o = *reinterpret_cast<const f32x4*>(sh.o + (base + s * step) * D + e);
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] += o[j] * a;
    }
    *reinterpret_cast<f32x4*>(&so[grp][e]) = t;
    __syncthreads();
    const float inv = inverse_sum(L);
    const int64_t head = (int64_t)(sq.first[b] + qi) * H + h;
    if (tid < D) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) v += so[i][tid];
        out[head * D + tid] = from_f32<T>(v * inv);
    }
    if (stats && tid == 0) stats[head] = make_float2(M, inv);
}

// Column sums of the probabilities in fp32: a wavefront holds 32 keys and goes over the blocks of columns of its part of all heads, the scores anew; stats has each column's maximum
// and 1 / sum.
template <int D, int NB>
__global__ void __launch_bounds__(AW * 64) kvp_weights_kernel(const float* __restrict__ q, PoolView pool, PagedSeqs<NB> sq, int H, int Hkv, float c, const float2* __restrict__ stats,
                                                              float* __restrict__ sums, float decay) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh = lane >> 5, G = H / Hkv;
    int first;
    const int b = seq_of(sq.end, (int)blockIdx.x, &first);
    const int parts = sq.parts[b], p = ((int)blockIdx.x - first) % parts;
    const int n = sq.count[b], nq = sq.nq[b], cols = nq * G, blocks = (cols + 31) / 32;   // (nq > 0: others have no tiles)
    const int64_t key0 = (int64_t)(((int)blockIdx.x - first) / parts) * (AW * 32) + wave * 32;
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
            load_quads((const float*)pool.k + page_at(pool, sq.table[b], key0 + (row & 16), g, Hkv, D) + (row & 15) * D + 4 * lh, kf);
        }
        const int64_t head = (int64_t)(sq.first[b] + cc / G) * H + g * G + cc % G;
        float qf[D / 2];
        load_quads(q + head * D + 4 * lh, qf);
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
        if (parts > 1) sums[(int64_t)sq.at[b] + (int64_t)p * n + key] = w;
        else sq.weight[b][key] = decay == 0.f ? w : decay * sq.weight[b][key] + w;
    }
}

// Accounts from kept scores (few columns): a thread has a place of the scores' rows and goes over all heads' columns
template <int NB>
__global__ void __launch_bounds__(256) kvp_scores_weights_kernel(const float* __restrict__ scores, PagedSeqs<NB> sq, int H, int Hkv, const float2* __restrict__ stats, float decay) {
    int first;
    const int b = seq_of(sq.end, (int)blockIdx.x, &first);
    const int n = sq.count[b], G = H / Hkv, cols = sq.nq[b] * G;
    const int64_t at = (int64_t)((int)blockIdx.x - first) * 256 + threadIdx.x, stride = score_blocks(n) * 32;
    const int64_t key = (at & ~31) + 8 * (at >> 2 & 3) + 4 * (at >> 4 & 1) + (at & 3);   // as the scores were stored
    if (key >= n) return;
    const float* row = scores + (int64_t)sq.scores[b] * 32 + at;
    float w = 0.f;
    const float2* const st0 = stats + (int64_t)sq.first[b] * H;
    int64_t st = 0;                      // the column's place among the statistics, [query][head]
    int j = 0, cn = 0, g = 0;            // head of the group, column of the head, head
#pragma unroll 8
    for (int r = 0; r < cols * Hkv; ++r) {
        const float2 z = st0[st];
        const float x = *row, e = __builtin_amdgcn_exp2f(x - z.x) * z.y;
        w += x == -INFINITY ? 0.f : e;   // (unseen by the column, whose sum may be NaN)
        row += stride;
        ++st;
        if (++j == G) { j = 0; st += H - G; }
        if (++cn == cols) { cn = 0; ++g; st = g * G; }
    }
    sq.weight[b][key] = decay == 0.f ? w : decay * sq.weight[b][key] + w;
}

// The parts' sums of a key, in their order
template <int NB>
__global__ void __launch_bounds__(256) kvp_add_weights_kernel(const float* __restrict__ sums, PagedSeqs<NB> sq, float decay) {
    int first;
    const int b = seq_of(sq.end, (int)blockIdx.x, &first);
    const int key = ((int)blockIdx.x - first) * 256 + threadIdx.x, n = sq.count[b], parts = sq.parts[b];
    if (key >= n) return;
    float w = 0.f;
#pragma unroll 16
    for (int p = 0; p < parts; ++p) w += sums[(int64_t)sq.at[b] + (int64_t)p * n + key];
    sq.weight[b][key] = decay == 0.f ? w : decay * sq.weight[b][key] + w;
}

size_t kvp_attn_min_floats(int64_t rows, int H) { return ((size_t)rows * H * 2 + 63) / 64 * 64; }   // the statistics of every column

static int64_t columns(const PagedBatch& pb, int b, int G) { return (pb.off[b + 1] - pb.off[b]) * G; }

// per[b], splits[b] of the sequences that `mine` picks: shares of about equal length (none below `least` keys), so many that blocks of `cols_wg` columns, heads and shares make
// about `wgs` workgroups.  Returns the workgroups; *longest: keys of the longest share.
template <int NB, typename F>
static int64_t share_keys(PagedSeqs<NB>& sq, const PagedBatch& pb, int Hkv, int G, int64_t cols_wg, int64_t wgs, int64_t least, F mine, int64_t* longest = nullptr) {
    int64_t total = 0, n_wgs = 0, most = 0;    // keys times blocks of columns
    for (int b = 0; b < pb.n; ++b)
        if (mine(b)) total += (columns(pb, b, G) + cols_wg - 1) / cols_wg * pb.count[b];
    int64_t per = (total * Hkv + wgs - 1) / wgs;
    per = per < least ? least : (per + 127) / 128 * 128;
    for (int b = 0; b < pb.n; ++b)
        if (mine(b)) {
            const int64_t n = (pb.count[b] + per - 1) / per, even = ((pb.count[b] + n - 1) / n + 127) / 128 * 128;
            sq.per[b] = (int32_t)std::min<int64_t>(even, 1 << 30);
            sq.splits[b] = (int32_t)((pb.count[b] + sq.per[b] - 1) / sq.per[b]);
            n_wgs += (columns(pb, b, G) + cols_wg - 1) / cols_wg * Hkv * sq.splits[b];
            most = std::max<int64_t>(most, std::min<int64_t>(sq.per[b], pb.count[b]));
        }
    if (longest) *longest = most;
    return n_wgs;
}

// Workgroups of many columns, one a CU: a share costs about 12 us and 1.6 us for 64 keys of 128 dimensions (1.35 with a quarter of the chip at work, 1.87 with all of it), shares are
// merged at about 4 us and 4 TB/s.  The number of them for which that sum is least (us for all keys in one share / this choice: 64 tokens after 4096, 8 heads of 4, 36.6 / 24; 256 after
// 4096 110 / 39; 1024 tokens alone 33 / 33, in two shares 28 and a merge of 8).
template <int NB, typename F>
static int64_t pick_workgroups(PagedSeqs<NB>& sq, const PagedBatch& pb, int H, int Hkv, int D, int64_t cols_wg, int64_t least, F mine) {
    const double tile = D == 128 ? 1.6 : D == 64 ? 1.0 : 0.6;
    double best = 0.0;
    int64_t choice = 1;
    for (const int64_t wgs : {1, 32, 64, 96, 128, 192, 256, 384, 512, 768, 1024}) {
        int64_t longest;
        const int64_t n = share_keys(sq, pb, Hkv, H / Hkv, cols_wg, wgs, least, mine, &longest);
        const double unit = 12.0 + tile * ((longest + 63) / 64);
        double all = 0.0, bytes = 0.0;
        for (int b = 0; b < pb.n; ++b) {
            if (!mine(b)) continue;
            all += (double)((columns(pb, b, H / Hkv) + cols_wg - 1) / cols_wg * Hkv * sq.splits[b]) * (12.0 + tile * (sq.per[b] < pb.count[b] ? sq.per[b] : pb.count[b]) / 64);
            if (sq.splits[b] > 1) bytes += (double)sq.splits[b] * (pb.off[b + 1] - pb.off[b]) * H * D * 8;
        }
        const double rounds = (double)((n + 255) / 256) * unit, spread = n <= 256 ? unit : std::min(rounds, all / 256 + 0.5 * unit);
        const double t = spread + (bytes > 0 ? 4.0 + bytes / 4e6 : 0.0);
        if (choice == 1 && best == 0.0) { best = t; continue; }
        if (t < best) { best = t; choice = wgs; }
    }
    return choice;
}

constexpr int64_t MAX_GROUPS = (1 << 24) - 1;   // of 256 threads: a launch has fewer than 2^32
constexpr int64_t F32_WORKGROUPS = 512;
template <typename T, int D, int NB>
static hipError_t launch_kvp_attn_t(const T* q, const PagedPool& pool, const PagedBatch& pb, int H, int Hkv, float* part, size_t part_floats, T* out, bool add, float decay,
                                    hipStream_t s) {
    constexpr bool BF16 = sizeof(T) == 2;
    const int G = H / Hkv;
    const int64_t rows = pb.off[pb.n];
    const float c = PAGED_LOG2E / sqrtf((float)D);
    const PoolView pl{(const char*)pool.k, (const char*)pool.v, (uint32_t)pool.pages, pool.shift};
    float2* const stats = add ? (float2*)part : nullptr;
    const size_t used = add ? kvp_attn_min_floats(rows, H) : 0;
    float* const rest = part + used;
    const size_t room = part_floats - used;
    PagedSeqs<NB> sq{};
    for (int b = 0; b < pb.n; ++b) {
        sq.table[b] = pb.table[b]; sq.weight[b] = pb.weight[b];
        sq.count[b] = (int32_t)pb.count[b]; sq.first[b] = (int32_t)pb.off[b]; sq.nq[b] = (int32_t)(pb.off[b + 1] - pb.off[b]);
        sq.per[b] = 1 << 30; sq.splits[b] = sq.nq[b] > 0 ? 1 : 0; sq.scores[b] = -1;
    }
    auto few = [&](int b) { return sq.nq[b] > 0 && columns(pb, b, G) <= KVP_FEW_COLS; };
    auto many = [&](int b) { return sq.nq[b] > 0 && columns(pb, b, G) > KVP_FEW_COLS; };
    auto any = [&](int b) { return sq.nq[b] > 0; };
    constexpr int64_t COLS = kvp_many_waves(D) * 32;
    int64_t want = F32_WORKGROUPS, want_few = 256, least_few = 256, least = 256;
    if constexpr (BF16) {
        want = pick_workgroups(sq, pb, H, Hkv, D, COLS, 256, many);
        // Few columns: a workgroup a CU where the shares come out alike (the longest times the CUs within 1.25 of all keys), with accounts such that their scores wait in LDS; otherwise, of several
        // sequences, 384, two of which fit a CU, to even them out.  Us at 384 / so, behind reads of other data: 16 sequences of 1048 .. 13106 rows, 4 heads of 7, 59 / 53, with accounts 74 / 62;
        // five of 1600 .. 20000, 8 heads, 55 / 48 and 64 / 54; two of up to 60000, 4 heads, 43 / 36 and 52 / 43; 16 of 640 .. 8000, 8 heads, where the least number of shares is uneven, 64 at
        // 384, 85 at 224.  Short caches in one share, without a merge: 301 rows 7.7 for 9.1, 16 of up to 501 10.4 for 11.8; two shares of 517 rows 9.2, one 9.9.
        int n = 0;
        int64_t longest = 0, total = 0, cols = 0;
        for (int b = 0; b < pb.n; ++b)
            if (few(b)) { ++n; longest = std::max(longest, pb.count[b]); total += pb.count[b] * Hkv; cols = std::max(cols, columns(pb, b, G)); }
        if (n > 1) want_few = 384;
        if (longest <= 512) least_few = 512;
        for (int64_t w = CUS; n > 0 && w >= CUS * 5 / 8; w -= 8) {
            int64_t share;
            if (share_keys(sq, pb, Hkv, G, KVP_FEW_COLS, w, least_few, few, &share) > CUS) continue;
            if ((!add || kvp_few_keeps(D, (int)cols, share)) && 4 * share * CUS <= 5 * total) want_few = w;
            break;
        }
    } else {
        // Two workgroups a CU (us at 256 / 512 / 1024: 128 tokens after 4000 rows, 8 heads of 4, d = 128, 125 / 121 / 136, one token after 60000 163 / 152 / 155, four of 300 after 3000
        // 33 / 29 / 32), and a block of keys for every wavefront where that leaves most of the chip idle (one token after 500 rows of two heads 8.3, with two blocks each 11.7; three
        // sequences of up to 333 after 1500 17.3 / 15.4)
        int64_t n = 0;
        for (int b = 0; b < pb.n; ++b) n += (columns(pb, b, G) + 31) / 32 * Hkv;
        if (n < 32) least = 128;
    }
    int64_t shares = 0;
    for (int64_t scale = 1;; scale *= 2) {   // (fewer and longer shares where they would not fit the scratch)
        if constexpr (BF16) {
            share_keys(sq, pb, Hkv, G, KVP_FEW_COLS, std::max<int64_t>(1, want_few / scale), least_few * scale, few);
            share_keys(sq, pb, Hkv, G, COLS, std::max<int64_t>(1, want / scale), 256 * scale, many);
        } else {
            share_keys(sq, pb, Hkv, G, 32, std::max<int64_t>(1, want / scale), least * scale, any);
        }
        shares = 0;
        for (int b = 0; b < pb.n; ++b)
            if (sq.splits[b] > 1) { sq.at[b] = (int32_t)std::min<int64_t>(shares, 0x7fffffff); shares += (int64_t)sq.splits[b] * sq.nq[b] * H; }
        if (shares == 0 || (shares <= 0x7fffffff && (size_t)shares * (D + 2) + 64 <= room)) break;
    }
    const Shares sh{(float2*)rest, rest + (2 * shares + 63) / 64 * 64};
    size_t taken = shares > 0 ? (2 * shares + 63) / 64 * 64 + (size_t)shares * D : 0;
    // scores of few columns are kept for the accounts where there is room
    float* const scores = rest + taken;
    if (BF16 && add) {
        int64_t at = 0;
        for (int b = 0; b < pb.n; ++b) {
            const int64_t need = score_blocks(pb.count[b]) * columns(pb, b, G) * Hkv;
            if (!few(b) || (size_t)(at + need) * 32 > room - taken || at + need > 0x7fffffff) continue;
            sq.scores[b] = (int32_t)at;
            at += need;
        }
    }
    // work items of the sequences that `mine` picks, in blocks of w columns
    auto items_of = [&](auto mine, int64_t w) {
        int64_t n = 0;
        for (int b = 0; b < NB; ++b) {
            if (b < pb.n && mine(b)) n += (columns(pb, b, G) + w - 1) / w * sq.splits[b];
            sq.end[b] = (int32_t)std::min<int64_t>(n, 0x7fffffff);
        }
        return n;
    };
    hipError_t e = hipSuccess;
    if constexpr (BF16) {
        const int64_t nm = items_of(many, COLS);
        if (nm * Hkv > MAX_GROUPS / 2) return hipErrorInvalidValue;
        if (nm > 0) e = launch_kvp_attn_many<NB>(q, pl, sq, (int)nm, H, Hkv, D, sh, stats, out, s);
        if (e != hipSuccess) return e;
        for (const bool keep : {true, false}) {   // those whose scores are kept, and those for which there was no room, or no wish
            const int64_t nf = items_of([&](int b) { return few(b) && (sq.scores[b] >= 0) == keep; }, KVP_FEW_COLS);
            if (nf > 0 && e == hipSuccess) e = launch_kvp_attn_few<NB>(q, pl, sq, (int)nf, H, Hkv, D, sh, stats, keep ? scores : nullptr, out, s);
        }
    } else {
        const int64_t n = items_of(any, 32);
        if (n * Hkv > MAX_GROUPS) return hipErrorInvalidValue;
        kvp_attn_kernel<D, NB><<<dim3((unsigned)(n * Hkv)), dim3(AW * 64), 0, s>>>(q, pl, sq, H, Hkv, c, sh, stats, out);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    if (shares > 0) {
        int64_t n = 0;
        for (int b = 0; b < NB; ++b) {
            if (b < pb.n && sq.splits[b] > 1) n += sq.nq[b];
            sq.end[b] = (int32_t)n;
        }
        if (n * H > MAX_GROUPS) return hipErrorInvalidValue;
        int most = 1;
        for (int b = 0; b < pb.n; ++b) most = std::max(most, sq.splits[b]);
        const dim3 grid((unsigned)((n * H + MERGE_T / (D / 4) - 1) / (MERGE_T / (D / 4))));
        if (most <= 2) kvp_merge_few_kernel<T, D, NB, 2><<<grid, dim3(MERGE_T), 0, s>>>(sh, sq, (uint32_t)(n * H), H, Hkv, stats, out);
        else if (most <= 4) kvp_merge_few_kernel<T, D, NB, 4><<<grid, dim3(MERGE_T), 0, s>>>(sh, sq, (uint32_t)(n * H), H, Hkv, stats, out);
        else if (most <= 8) kvp_merge_few_kernel<T, D, NB, 8><<<grid, dim3(MERGE_T), 0, s>>>(sh, sq, (uint32_t)(n * H), H, Hkv, stats, out);
        else if (most <= 16) kvp_merge_few_kernel<T, D, NB, 16><<<grid, dim3(MERGE_T), 0, s>>>(sh, sq, (uint32_t)(n * H), H, Hkv, stats, out);
        else kvp_merge_kernel<T, D, NB><<<dim3((unsigned)(n * H)), dim3(MERGE_T), 0, s>>>(sh, sq, H, Hkv, stats, out);
    }
    if (add) {
        auto kept = [&](int b) { return sq.scores[b] >= 0; };
        auto anew = [&](int b) { return sq.nq[b] > 0 && sq.scores[b] < 0; };
        // workgroups of `keys` rows of the sequences that `mine` picks, each `parts` times
        auto tiles_of = [&](auto mine, int64_t keys, bool in_parts) {
            int64_t t = 0;
            for (int b = 0; b < NB; ++b) {
                if (b < pb.n && mine(b)) t += (pb.count[b] + keys - 1) / keys * (in_parts ? sq.parts[b] : 1);
                sq.end[b] = (int32_t)std::min<int64_t>(t, 0x7fffffff);
            }
            return t;
        };
        const int64_t ns = tiles_of(kept, 256, false);
        if (ns > 0) kvp_scores_weights_kernel<NB><<<dim3((unsigned)ns), dim3(256), 0, s>>>(scores, sq, H, Hkv, stats, decay);
        // parts of the heads and blocks of columns of each sequence, so that all workgroups have about the same number of blocks (the shares' and scores' room is free again, but for what
        // the kept scores' kernel still reads: it is ahead in the stream)
        constexpr int64_t KEYS = BF16 ? KVP_WEIGHT_KEYS : AW * 32;
        int64_t work = 0;
        for (int b = 0; b < pb.n; ++b)
            if (anew(b)) work += (pb.count[b] + KEYS - 1) / KEYS * ((columns(pb, b, G) + 31) / 32) * Hkv;
        // Three workgroups for each of the 512 that are at work at a time, but no fewer than 10 blocks each as long as all 512 have one (us with 1024 workgroups / so, all kernels of the call: 300
        // tokens after 3700 rows, 8 heads of 4, 83 / 75; six of 300 after 3700, 4 heads of 7, 216 / 208; six of 600 after 8400 871 / 824; 20 after 7980 47 / 45; 64 after 1936 42 / 42)
        bool joined = false;
        for (int64_t target = std::max(std::max<int64_t>(1, work / 1536), std::min<int64_t>((work + 511) / 512, 10)); work > 0; target *= 2) {
            int64_t at = 0;
            joined = false;
            for (int b = 0; b < pb.n; ++b) {
                if (!anew(b)) continue;
                const int64_t all = (columns(pb, b, G) + 31) / 32 * Hkv;
                sq.parts[b] = (int32_t)std::max<int64_t>(1, std::min<int64_t>(256, all / target));
                sq.at[b] = (int32_t)std::min<int64_t>(at, 0x7fffffff);
                if (sq.parts[b] > 1) { at += sq.parts[b] * pb.count[b]; joined = true; }
            }
            if (!joined || ((size_t)at <= room && at <= 0x7fffffff)) break;
        }
        const int64_t nt = tiles_of(anew, KEYS, true);
        if (nt > MAX_GROUPS) return hipErrorInvalidValue;
        if (nt > 0) {
            if constexpr (BF16) {
                e = launch_kvp_weights_many<NB>(q, pl, sq, (int)nt, H, Hkv, D, stats, rest, decay, s);
                if (e != hipSuccess) return e;
            } else {
                kvp_weights_kernel<D, NB><<<dim3((unsigned)nt), dim3(AW * 64), 0, s>>>(q, pl, sq, H, Hkv, c, stats, rest, decay);
            }
        }
        if (joined) {
            const int64_t na = tiles_of([&](int b) { return anew(b) && sq.parts[b] > 1; }, 256, false);
            kvp_add_weights_kernel<NB><<<dim3((unsigned)na), dim3(256), 0, s>>>(rest, sq, decay);
        }
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
    if (pb.n < 1 || pb.n > DECODE_MAX_BATCH || pb.off[pb.n] < 1 || pb.off[pb.n] * H > 0x7fffffff) return hipErrorInvalidValue;
    return bf16 ? launch_kvp_attn_d<bf16_t>((const bf16_t*)q, pool, pb, H, Hkv, d, part, part_floats, (bf16_t*)out, add, decay, s)
                : launch_kvp_attn_d<float>((const float*)q, pool, pb, H, Hkv, d, part, part_floats, (float*)out, add, decay, s);
}

}  // namespace spts
