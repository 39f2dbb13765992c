// What the attention kernels over caches in pages share: a kernel's view of the sequences, where rows lie, how scores and values that are not finite are kept out.
#pragma once
#include "spts_lanes.h"

namespace spts {
typedef float paged_f32x16 __attribute__((ext_vector_type(16)));
constexpr float PAGED_LOG2E = 1.4426950408889634f;
constexpr float PAGED_LOWEST = -3.402823466e38f;   // a running maximum starts here: below every finite score, and a score of -inf then weighs 2^-inf = 0

// A kernel's view of up to NB sequences
template <int NB> struct PagedSeqs {
    const int32_t* table[NB];
    float* weight[NB];
    int32_t count[NB], first[NB], nq[NB];   // rows, the call's first query row, queries
    int32_t per[NB], splits[NB];            // keys of a share (a multiple of 128), shares
    int32_t end[NB];                        // work items of the sequences up to here
    int32_t at[NB];                         // first share of sequence b (attention) / first of its partial sums (accounts)
    int32_t scores[NB];                     // where the scores of sequence b begin, in blocks of 32 (-1: not kept)
    int32_t parts[NB];                      // accounts: parts of its heads and columns
};
struct PoolView { const char* k; const char* v; uint32_t pages; int32_t shift; };
// Shares of a column's keys, each with its maximum and sum (ml) and its unnormalised output (o [D]); column n of head g in share s is at at[b] + (s * Hkv + g) * columns + n
struct Shares { float2* ml; float* o; };
// x / G: the upper half of x times ceil(2^32 / G) is that, or one more
struct DivG { uint32_t m; int32_t G; };
__device__ inline uint32_t div_g(uint32_t x, DivG g) {
    if (g.G == 1) return x;
    const uint32_t y = __umulhi(x, g.m);
    return y - (y * (uint32_t)g.G > x ? 1u : 0u);
}

template <int NB> __device__ inline int seq_of(const int32_t (&end)[NB], int i, int* first) {
    int b = 0;
    *first = 0;
#pragma unroll
    for (int j = 0; j + 1 < NB; ++j)
        if (i >= end[j]) { b = j + 1; *first = end[j]; }
    return b;
}
// Blocks of 32 scores from a column's row to the next one's: no power of two, which would put the same keys of all columns into one memory channel (131004 rows, 128 columns, stored
// while the cache is read: 127 us, this way 121)
__host__ __device__ inline int64_t score_blocks(int64_t n) {
    const int64_t blocks = (n + 31) / 32;
    return blocks < 512 ? blocks : (blocks + 63) / 64 * 64 + 9;
}
// the pool's page of a row; the table does not change while kernels read it
__device__ inline uint32_t page_id(const PoolView& pool, const int32_t* table, int64_t row) {
    typedef const __attribute__((address_space(4))) int32_t* constant_i32;
    const uint32_t id = (uint32_t)((constant_i32)(uintptr_t)table)[row >> pool.shift];
    return id < pool.pages ? id : 0;
}
// element offset of a row (a multiple of 16) of kv head g on a page
__device__ inline int64_t row_at(const PoolView& pool, uint32_t id, int64_t row, int g, int Hkv, int D) {
    return (((int64_t)id * Hkv + g) << pool.shift) * D + (row & ((1 << pool.shift) - 1)) * D;
}
__device__ inline int64_t page_at(const PoolView& pool, const int32_t* table, int64_t row, int g, int Hkv, int D) {
    return row_at(pool, page_id(pool, table, row), row, g, Hkv, D);
}

__device__ inline paged_f32x16 zero16() {
    paged_f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}
// 1 / sum of a column's probabilities: 0 where all scores are -inf
__device__ inline float inverse_sum(float L) { return L > 0.f ? 1.f / L : L == 0.f ? 0.f : L; }

// kernels_paged_mfma.hip: bf16 on the bf16 matrix instructions.  `few`: sequences whose columns fit 16, `many`: the others (items of either may be none)
template <int NB> hipError_t launch_kvp_attn_few(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, int d, const Shares& sh, float2* stats,
                                                 float* scores, bf16_t* out, hipStream_t s);
template <int NB> hipError_t launch_kvp_attn_many(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, int d, const Shares& sh,
                                                  float2* stats, bf16_t* out, hipStream_t s);
// accounts of the sequences that have parts, over tiles of KVP_WEIGHT_KEYS keys; sums: partial sums of sequences in more than one part
template <int NB> hipError_t launch_kvp_weights_many(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, int d, const float2* stats, float* sums,
                                                     float decay, hipStream_t s);
constexpr int KVP_FEW_COLS = 16, KVP_WEIGHT_KEYS = 256;
// Few columns: wavefronts of a workgroup, its LDS (two stages of 32 values each, then outputs, maxima and sums where they meet), and the scores of a share that are kept behind it: rows of
// `longest` keys, whose 16 words more spread the columns over the banks.  They are kept where the call has no more workgroups than CUs.
constexpr int KVP_FEW_WAVES = 4, KVP_LDS = 160 * 1024, CUS = 256;
constexpr int kvp_few_lds(int d) { return KVP_FEW_WAVES * (2 * 32 * 2 * d > 16 * (d + 6) * 4 ? 2 * 32 * 2 * d : 16 * (d + 6) * 4); }
constexpr int64_t kvp_kept_row(int64_t longest) { return (longest + 31) / 32 * 32 + 16; }
constexpr bool kvp_few_keeps(int d, int cols, int64_t longest) { return cols * kvp_kept_row(longest) * 4 <= KVP_LDS - kvp_few_lds(d); }
constexpr int kvp_many_waves(int d) { return d == 32 ? 4 : 8; }   // of a workgroup, 32 columns each (a tile of 64 keys of 32 dimensions is four loads)
}  // namespace spts
