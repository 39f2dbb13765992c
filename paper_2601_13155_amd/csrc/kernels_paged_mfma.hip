// Attention of new tokens over caches in pages, bf16 on the matrix cores (what is computed stands at the head of kernels_paged_attn.hip).
//
// Values lie by rows, a row being a key, and O^T = V^T P^T wants eight keys of one dimension in a lane: the transposing LDS read (ds_read_b64_tr_b16: of four rows of sixteen
// columns that sixteen lanes address, each lane gets a column) gives them four at a time, so a cache needs no transposed copy and a row is written once.
#include "spts_paged.h"

#include <algorithm>
#include <type_traits>

namespace spts {

namespace {
typedef paged_f32x16 f32x16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// eight keys of the lane's dimension: two transposing reads of four rows
__device__ inline bf16x8 read_values(uint32_t at, uint32_t second) {
    union { s16x4 h[2]; bf16x8 v; } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)at);
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at + second));
    return u.v;
}
// whether one of eight bf16 values is an infinity or NaN
__device__ inline bool any_odd(bf16x8 v) {
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) odd |= (w[j] & 0x7f80u) == 0x7f80u || (w[j] & 0x7f800000u) == 0x7f800000u;
    return odd;
}
// The first of two bf16 parts of a probability: the largest number of that type below it (0 for 0), so that the second is above 0 too and an infinite value times either is that infinity
__device__ inline uint32_t first_part(float p) { return __builtin_elementwise_sub_sat(__float_as_uint(p), 1u) & 0xffff0000u; }
// v without its infinities and NaN; up / down: 1 where v is +inf / -inf, both where it is NaN
__device__ inline bf16x8 split_odd(bf16x8 v, bf16x8* up, bf16x8* down) {
    u32x4 w = __builtin_bit_cast(u32x4, v), u, d;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t keep = 0, uu = 0, dd = 0;
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
            const uint32_t x = w[j] >> h & 0xffffu, one = 0x3f80u << h;
            const bool odd = (x & 0x7f80u) == 0x7f80u, nan = odd && (x & 0x7fu);
            keep |= odd ? 0u : x << h;
            uu |= nan || (odd && !(x & 0x8000u)) ? one : 0u;
            dd |= nan || (odd && (x & 0x8000u)) ? one : 0u;
        }
        w[j] = keep; u[j] = uu; d[j] = dd;
    }
    *up = __builtin_bit_cast(bf16x8, u);
    *down = __builtin_bit_cast(bf16x8, d);
    return __builtin_bit_cast(bf16x8, w);
}

// A tile of rows of D values in LDS, in chunks of 16 bytes.  A wavefront reads 32 (16) keys at one chunk, and 4 rows at two neighbouring chunks at a time; both are spread over
// the banks by exchanging a row's chunks, pairs of them for the values.
template <int D> struct Tile {
    static constexpr int ROW = 2 * D, CPR = D / 8, RPB = 256 / ROW;   // bytes and chunks of a row, rows of 256 bytes
    static constexpr int ROWS_PER_LOAD = 1024 / ROW;
    __device__ static inline int kswz(int row) { return (row / RPB) % CPR; }
    __device__ static inline int vswz(int row) { return (row / RPB) % (CPR / 2) * 2; }
    __device__ static inline int k_at(int row, int c) { return row * ROW + ((c ^ kswz(row)) << 4); }
    __device__ static inline int v_at(int row, int c) { return row * ROW + ((c ^ vswz(row)) << 4); }
};
}  // namespace

// ------------------------------------------------------------------ many columns
// A workgroup of NW wavefronts has NW * 32 columns of a key/value head and takes its keys in tiles of 64, which travel from the pool to LDS directly (a ring of five
// stages; a load moves 1 KB of rows of one page).  A wavefront's pipeline is by blocks of 32 keys: while the scores S^T = K Q^T of block b + 1 and the outputs of block b - 1 are on the matrix core
// (32x32x16: columns of the result are the lane's column), the lane takes the exponentials of block b.  Each step is one matrix instruction, one operand read ahead and
// a share of the exponentials.  The reference that the exponents are relative to is the first block's maximum and moves only when a lane's sum of 16 probabilities exceeds SUM_MAX (an exponent of
// more than 8 or so, an overflow included).
// Probabilities are rounded to bf16 for the second product, half a step (2^-8) of each at most and at random: as much as the output's own rounding where nothing cancels.  Their sums are
// of the unrounded ones, which the accounts of attention are relative to.
constexpr int BKV = 64, NST = 5;
constexpr float TAU = 8.0f, SUM_MAX = 4096.0f;

// ONCE: the sequences' columns fit a workgroup, so that nobody else reads their rows and the caches need not keep them (64 tokens after 30000 rows 59 us either way, behind a kernel that
// wrote 1 GB 70 / 60).
template <int D, int NW, int NB, bool ONCE>
__global__ void __launch_bounds__(NW * 64, NW == 8 ? 2 : 1) kvp_many_kernel(const bf16_t* q, PoolView pool, PagedSeqs<NB> sq, int H, int Hkv, float c, Shares sh,
                                                                          float2* __restrict__ stats, bf16_t* out) {   // (out may be q: a workgroup has read its columns)
    using L = Tile<D>;
    constexpr int KS = D / 16, DB = D / 32, NSTEP = KS + 2 * DB, FD = NSTEP > 4 ? 3 : 2;
    constexpr int TILE = BKV * L::ROW, STAGE = 2 * TILE;
    constexpr int LOADS = BKV / NW / L::ROWS_PER_LOAD, PER = 2 * LOADS;
    static_assert(LOADS >= 1, "whole loads");
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh = lane >> 5;
    const int g = (int)(blockIdx.x % Hkv), G = H / Hkv;
    int first;
    const int b = seq_of(sq.end, (int)(blockIdx.x / Hkv), &first);
    const int item = (int)(blockIdx.x / Hkv) - first, n = sq.count[b], nq = sq.nq[b], cols = nq * G, blocks = (cols + NW * 32 - 1) / (NW * 32);
    const int splits = sq.splits[b], split = item % splits, blk = blocks - 1 - item / splits;
    const int32_t* const table = sq.table[b];
    const int c0 = blk * (NW * 32), c0w = c0 + wave * 32;
    const int k0 = split * sq.per[b], kend = (int64_t)k0 + sq.per[b] < n ? k0 + sq.per[b] : n;   // this share's keys
    auto seen_by = [&](int col) {                                                             // keys of the share before which a column sees
        const int s = n - nq + (col < cols ? col : cols - 1) / G + 1;
        return s < kend ? s : kend;
    };
    const int col = c0w + l32 < cols ? c0w + l32 : cols - 1;
    const int seen = seen_by(col);
    const int n_tiles = (seen_by(c0 + NW * 32 - 1) - k0 + BKV - 1) / BKV;        // of the workgroup (none or less: no column sees a key of the share)
    const int live = c0w < cols ? seen_by(c0w + 31) - k0 : 0;
    const int nbw = live > 0 ? (live + 31) / 32 : 0;                             // blocks that the wavefront works on
    const int whole = seen_by(c0w) - k0;                                         // keys that all of its columns see
    const int nbf = live > 0 && whole > 0 ? whole / 32 : 0;                      // blocks that all of its columns see entirely

    const int64_t qrow = ((int64_t)(sq.first[b] + col / G) * H + g * G + col % G) * D;
    bf16x8 qf[KS];   // lane (l32, lh): q[column l32][16 ks + 8 lh ..]
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(q + qrow + 16 * ks + 8 * lh);

    // ---- tile loads: wavefront w moves rows [64 / NW * w, ..), a lane the chunk that belongs at its place in LDS
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int lrow = lane / L::CPR, lchunk = lane % L::CPR;
    uint32_t koff[LOADS], voff[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int row = wave * (BKV / NW) + i * L::ROWS_PER_LOAD + lrow;
        koff[i] = (uint32_t)(lrow * L::ROW + ((lchunk ^ L::kswz(row)) << 4));
        voff[i] = (uint32_t)(lrow * L::ROW + ((lchunk ^ L::vswz(row)) << 4));
    }
    // Pages of the next tiles: lane i has entry window + i of the table
    const int last_page = (n - 1) >> pool.shift;
    int window = k0 >> pool.shift;
    auto entries = [&]() {
        const int at = window + lane < last_page ? window + lane : last_page;
        const uint32_t id = (uint32_t)table[at];
        return (int)(id < pool.pages ? id : 0);
    };
    int ids = entries();
    auto dma = [&](int t, uint32_t tile) {
        const int key0 = k0 + t * BKV + wave * (BKV / NW);
        const uint32_t to = tile + (uint32_t)(wave * (BKV / NW) * L::ROW);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int row = key0 + i * L::ROWS_PER_LOAD;
            if (row + L::ROWS_PER_LOAD <= n) {
                const int page = row >> pool.shift;
                if (page - window > 63) { window = page; ids = entries(); }
                const uint32_t id = (uint32_t)__builtin_amdgcn_readlane(ids, page - window);
                const int64_t at = row_at(pool, id, row, g, Hkv, D) * 2;
                if constexpr (ONCE) {
                    dma16s_nt(koff[i], pool.k + at, to + i * 1024);
                    dma16s_nt(voff[i], pool.v + at, to + TILE + i * 1024);
                } else {
                    dma16s(koff[i], pool.k + at, to + i * 1024);
                    dma16s(voff[i], pool.v + at, to + TILE + i * 1024);
                }
            } else {   // rows behind the last one are the last one again
                const int r = row + lrow < n ? row + lrow : n - 1;
                uint32_t kin = koff[i] - (uint32_t)(lrow * L::ROW), vin = voff[i] - (uint32_t)(lrow * L::ROW);
                asm volatile("" : "+v"(kin), "+v"(vin));   // (keeps the addresses of this rare way out of the loop's registers)
                const int64_t at = (page_at(pool, table, r & ~15, g, Hkv, D) + (r & 15) * D) * 2;
                dma16(pool.k + at + kin, to + i * 1024);
                dma16(pool.v + at + vin, to + TILE + i * 1024);
            }
        }
    };

    f32x16 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = zero16();
    float l_run = 0.f, ref = 0.f;         // sum of the probabilities, the reference of the exponents
    f32x16 sa = zero16(), sb = zero16();   // scores of two consecutive blocks (one being produced, one in the softmax)
    bf16x8 pa[2], pb[2];                   // their probabilities (one being produced, one multiplied)
    // a lane's places: of key row l32 in a block, chunk 2 ks + lh; of value rows 4 lh + (lane % 16) / 4 (and 8 on) of 16, dimensions 16 (lane / 16 % 2) + 4 (lane % 4) of 32
    // (exchanged chunks: ks and i only flip bits of the place inside the row)
    const uint32_t kplace = (uint32_t)L::k_at(l32, lh);
    const int vr = 4 * lh + ((lane & 15) >> 2), vc = (lane >> 4 & 1) * 2 + ((lane & 3) >> 1);
    const uint32_t vplace = (uint32_t)(L::v_at(vr, vc) + (lane & 1) * 8 + TILE);
    constexpr uint32_t EIGHT = 8 * L::ROW;
    static_assert(8 % (L::RPB * (L::CPR / 2)) == 0, "eight rows on, the chunks are exchanged alike");
    static_assert(32 % (L::RPB * L::CPR) == 0, "32 rows on, the chunks are exchanged alike");
    auto key_frag = [&](uint32_t at, int kb, int ks) {   // at: the tile's place + kplace
        return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)((at ^ (uint32_t)(ks << 5)) + (uint32_t)(kb * 32 * L::ROW));
    };
    auto value_frag = [&](uint32_t at, int kb, int hf, int i) {   // at: the tile's place + vplace
        return read_values((at ^ (uint32_t)(i << 6)) + (uint32_t)((kb * 32 + hf * 16) * L::ROW), EIGHT);
    };
    // the reference goes to a maximum that is TAU above it, to the first block's in any case (-inf alone: to the lowest number, and any later score moves it)
    auto move_reference = [&](bool first_block, float mx) __attribute__((always_inline)) {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        const float to = first_block || mx > ref + TAU ? mx : ref;
        const float alpha = first_block ? 1.f : __builtin_amdgcn_exp2f(ref - to);
        ref = to;
        l_run *= alpha;
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
    };

    // Slot bb of the pipeline: scores of block bb + 1 into SN, outputs of block bb - 1 from PP, exponentials of block bb (scores SC) into PC.  The slot behind the last whole block only
    // multiplies that block's probabilities: its other parts run on stale data and leave no trace.
    auto slot = [&](int bb, uint32_t key_tile, uint32_t value_tile, auto half, f32x16& SC, f32x16& SN, bf16x8 (&PC)[2], bf16x8 (&PP)[2]) __attribute__((always_inline)) {
        if (bb > nbf || nbf == 0) return;
        constexpr int KB = decltype(half)::value;   // which half of its tile both blocks are
        const uint32_t ka = key_tile + kplace, va = value_tile + vplace;
        auto frag = [&](int i) { return i < KS ? key_frag(ka, KB, i % KS) : value_frag(va, KB, (i - KS) / DB & 1, (i - KS) % DB); };
        bf16x8 fr[FD + 1];
#pragma unroll
        for (int i = 0; i < FD; ++i) fr[i] = frag(i);
        float p[16], sum = 0.f;
        u32x4 pk[2];
        auto pair = [&](int i) {
            pk[i >> 2][i & 3] = cvt_pk_bf16(p[2 * i], p[2 * i + 1]);
            sum += p[2 * i] + p[2 * i + 1];
        };
        constexpr int EPS = 16 / NSTEP;   // exponentials of a step
#pragma unroll
        for (int i = 0; i < NSTEP; ++i) {
            if (i + FD < NSTEP) fr[(i + FD) % (FD + 1)] = frag(i + FD);
            if (i < KS) SN = mfma32(fr[i % (FD + 1)], qf[i % KS], i == 0 ? zero16() : SN);
            else o[(i - KS) % DB] = mfma32(fr[i % (FD + 1)], PP[(i - KS) / DB & 1], o[(i - KS) % DB]);
#pragma unroll
            for (int e = i * EPS; e < (i + 1) * EPS; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(SC[e], c, -ref));
            if (EPS == 1) { if (i & 1) pair(i >> 1); }
            else
#pragma unroll
                for (int e = i * EPS / 2; e < (i + 1) * EPS / 2; ++e) pair(e);
            __builtin_amdgcn_sched_barrier(0);
        }
        // a use of the probabilities here: without it the exponentials sink past the branch below, away from the matrix instructions that they overlap
        asm volatile("" ::"v"(pk[0]), "v"(pk[1]), "v"(sum));
        if (bb == 0) {   // (what it multiplied are no probabilities)
#pragma unroll
            for (int i = 0; i < DB; ++i) o[i] = zero16();
        }
        const bool is_live = bb < nbf;
        if (__ballot(is_live && (bb == 0 || !(sum <= SUM_MAX))) != 0) {
            asm volatile("");   // keeps this a branch
            float mx = PAGED_LOWEST;
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, SC[r] * c);
            move_reference(bb == 0, mx);
            sum = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(SC[r], c, -ref));
#pragma unroll
            for (int i = 0; i < 8; ++i) pair(i);
        }
        PC[0] = __builtin_bit_cast(bf16x8, pk[0]);
        PC[1] = __builtin_bit_cast(bf16x8, pk[1]);
        l_run += is_live ? sum : 0.f;
    };

    // A block that some column does not see entirely, on its own: scores of unseen keys are -inf, and values that are not finite are kept out of the product (0 times them would be NaN);
    // two more products count those that a column does see and put the infinity or NaN where it belongs.
    auto edge = [&](int bb) __attribute__((always_inline)) {
        const uint32_t st = lds0 + (uint32_t)((bb >> 1) % NST * STAGE) + (uint32_t)((bb & 1) * 32 * L::ROW);
        const int key0 = k0 + bb * 32;
        f32x16 S;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) S = mfma32(key_frag(st + kplace, 0, ks), qf[ks], ks == 0 ? zero16() : S);
        float mx = PAGED_LOWEST;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            S[r] = key0 + 8 * (r >> 2) + 4 * lh + (r & 3) < seen ? S[r] * c : -INFINITY;
            mx = fmaxf(mx, S[r]);
        }
        move_reference(bb == 0, mx);
        u32x4 pk[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p0 = __builtin_amdgcn_exp2f(S[2 * i] - ref), p1 = __builtin_amdgcn_exp2f(S[2 * i + 1] - ref);
            pk[i >> 2][i & 3] = cvt_pk_bf16(p0, p1);
            l_run += p0 + p1;
        }
#pragma unroll 1
        for (int hf = 0; hf < 2; ++hf) {
            const bf16x8 P = __builtin_bit_cast(bf16x8, hf ? pk[1] : pk[0]);
            u32x4 sees;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const int key = key0 + hf * 16 + 8 * (j >> 2) + 4 * lh + (j & 3);
                sees[j >> 1] = (key < seen ? 0x3f80u : 0u) | (key + 1 < seen ? 0x3f800000u : 0u);
            }
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                bf16x8 v = value_frag(st + vplace, 0, hf, i);
                if (__ballot(any_odd(v)) != 0) {
                    bf16x8 up, down;
                    v = split_odd(v, &up, &down);
                    const f32x16 u = mfma32(up, __builtin_bit_cast(bf16x8, sees), zero16()), w = mfma32(down, __builtin_bit_cast(bf16x8, sees), zero16());
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[i][r] += (u[r] > 0.f ? INFINITY : 0.f) - (w[r] > 0.f ? INFINITY : 0.f);
                }
                o[i] = mfma32(v, P, o[i]);
            }
        }
    };

    // ---- tiles 0..2 in flight, tile 0 landed, scores of block 0
    if (n_tiles > 0) dma(0, lds0);
    if (n_tiles > 1) dma(1, lds0 + STAGE);
    if (n_tiles > 2) dma(2, lds0 + 2 * STAGE);
    // All of it lands here: the compiler does not see these loads, and a wait of its own for one of its loads would drain the ring later
    SPTS_WAIT_VMCNT(0);
    __syncthreads();
    if (nbf > 0) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sa = mfma32(key_frag(lds0 + kplace, 0, ks), qf[ks], ks == 0 ? zero16() : sa);
    }
    uint32_t before = lds0, here = lds0, ahead = lds0 + STAGE, into = lds0 + 3 * STAGE;   // places of tiles t - 1, t, t + 1 and t + 3
    auto next_stage = [&](uint32_t at) { return at == lds0 + (NST - 1) * STAGE ? lds0 : at + STAGE; };
    for (int t = 0; t < n_tiles; ++t) {
        // tile t + 1 is published; the place of tile t + 3 had tile t - 2, which nobody reads behind this barrier (values of tile t - 1 are still multiplied)
        if (t + 1 < n_tiles) {
            if (t + 2 < n_tiles) { SPTS_WAIT_VMCNT(PER); } else { SPTS_WAIT_VMCNT(0); }
        }
        __syncthreads();
        if (t + 3 < n_tiles) dma(t + 3, into);
        slot(2 * t, here, before, std::integral_constant<int, 1>{}, sa, sb, pa, pb);
        slot(2 * t + 1, ahead, here, std::integral_constant<int, 0>{}, sb, sa, pb, pa);
        before = here; here = ahead;
        ahead = next_stage(ahead); into = next_stage(into);
    }
    if (n_tiles > 0) slot(2 * n_tiles, here, before, std::integral_constant<int, 1>{}, sa, sb, pa, pb);
    // The blocks at the columns' ends: the queries of NW * 32 columns end within 256 keys of each other, and with the block before them those lie in the last five tiles, all in LDS still
#pragma unroll 1
    for (int bb = nbf; bb < nbw; ++bb) edge(bb);

    // ---- results.  A lane has four consecutive dimensions of its column at a time; they leave as whole rows through LDS (the ring is free behind the barrier)
    const float sum = l_run + __shfl_xor(l_run, 32);
    const float M = nbw > 0 ? ref : PAGED_LOWEST;
    if (splits > 1) {
        const int cn = c0w + l32;
        const int64_t to = (int64_t)sq.at[b] + ((int64_t)split * Hkv + g) * cols + cn;
        if (cn < cols) {
            if (lh == 0) sh.ml[to] = make_float2(M, sum);
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    *reinterpret_cast<f32x4*>(sh.o + to * D + 32 * i + 8 * r + 4 * lh) = f32x4{o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
        }
        return;
    }
    const float inv = inverse_sum(sum);
    __syncthreads();
    char* const stg = smem + wave * (32 * L::ROW);
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const u32x2 w = {cvt_pk_bf16(o[i][4 * r] * inv, o[i][4 * r + 1] * inv), cvt_pk_bf16(o[i][4 * r + 2] * inv, o[i][4 * r + 3] * inv)};
            *reinterpret_cast<u32x2*>(stg + l32 * L::ROW + (((4 * i + r) ^ (l32 % L::CPR)) << 4) + lh * 8) = w;
        }
    if (stats && lh == 0 && c0w + l32 < cols) stats[qrow / D] = make_float2(M, inv);
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 32 / L::ROWS_PER_LOAD; ++p) {
        const int r = p * L::ROWS_PER_LOAD + lrow, cn = c0w + r;
        if (cn < cols) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(stg + r * L::ROW + ((lchunk ^ (r % L::CPR)) << 4));
            *reinterpret_cast<u32x4*>(out + ((int64_t)(sq.first[b] + cn / G) * H + g * G + cn % G) * D + lchunk * 8) = v;
        }
    }
}

// ------------------------------------------------------------------ few columns
// Up to 16 columns (single tokens, mostly): bound by the cache's bytes.  The wavefronts of a workgroup take blocks of 32 keys in turn, each on its own, without barriers: keys come into
// registers, values into its two stages of LDS, a block ahead.  16x16x32: S^T = K Q^T with key 8 (m / 4) + 4 t + m % 4 as operand row m of the t-th product, so that lane group kg
// has the scores of keys 8 kg .. 8 kg + 7, which is the operand of O^T = V^T P^T as it stands.  Probabilities go in as two bf16 parts, both above 0 (off by 2^-16 of each at most), which
// costs nothing here.  The maximum moves only when a score is 2^8 above it.
// Scores for the accounts wait in LDS for the end where a share's fit there and a workgroup has a CU to itself: stores among the reads cost more than their bytes (131071 rows 110 us by these
// for 92, five of 1600 .. 20000 64 / 54; without accounts 87).
// Rows are read once, by loads that do not leave them in the caches, where they would push out what other kernels wrote (us by plain loads / so, when scores went to memory as they came:
// one token after 131071 rows with accounts 117 / 110, behind a kernel that wrote 1 GB 174 / 118; 16 of up to 13106 in 384 workgroups 53 / 51, behind such a kernel 152 / 92.  Where it costs:
// all of 16 caches of 4000 rows in the last cache from the call before 50 / 58, 16 sequences of 13106 rows on the same pages 58 / 63).
template <int D, int NW, int NB, bool SCORES>
__global__ void __launch_bounds__(NW * 64, 2) kvp_few_kernel(const bf16_t* q, PoolView pool, PagedSeqs<NB> sq, int H, int Hkv, float c, Shares sh, float2* __restrict__ stats,
                                                                 float* __restrict__ scores, int kept, bf16_t* out) {
    using L = Tile<D>;
    constexpr int KI = D / 32, VM = D / 16, BLOCK = 32 * L::ROW, LOADS = BLOCK / 1024, LD = D + 4;
    extern __shared__ __attribute__((aligned(1024))) char smem[];   // [NW][2][BLOCK] values; then [NW][16][LD] outputs and [NW][16][2] maxima and sums.  Behind these [cols][kept] scores
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, kg = lane >> 4;
    const int g = (int)(blockIdx.x % Hkv), G = H / Hkv;
    int first;
    const int b = seq_of(sq.end, (int)(blockIdx.x / Hkv), &first);
    const int split = (int)(blockIdx.x / Hkv) - first, n = sq.count[b], nq = sq.nq[b], cols = nq * G, splits = sq.splits[b];
    const int32_t* const table = sq.table[b];
    const int k0 = split * sq.per[b], k1 = (int64_t)k0 + sq.per[b] < n ? k0 + sq.per[b] : n;
    const int col = l16 < cols ? l16 : cols - 1, seen = n - nq + col / G + 1, all_see = n - nq + 1;
    const int64_t qrow = ((int64_t)(sq.first[b] + col / G) * H + g * G + col % G) * D;
    bf16x8 qf[KI];
#pragma unroll
    for (int i = 0; i < KI; ++i) qf[i] = *reinterpret_cast<const bf16x8*>(q + qrow + 32 * i + 8 * kg);

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + (uint32_t)(wave * 2 * BLOCK);
    const int lrow = lane / L::CPR, lchunk = lane % L::CPR;
    const int krow = 8 * (l16 >> 2) + (l16 & 3);   // key of operand row l16, first product
    struct Ids { uint32_t a, b; };
    auto ids_of = [&](int key0) {   // pages of the block's halves
        const int ka = key0 < n ? key0 : (n - 1) & ~15, kb = key0 + 16 < n ? key0 + 16 : ka;
        return Ids{page_id(pool, table, ka), page_id(pool, table, kb)};
    };
    bf16x8 kf[2][KI];
    auto load = [&](int key0, Ids id, int stage) __attribute__((always_inline)) {
        const int64_t pa = row_at(pool, id.a, key0, g, Hkv, D), pb = key0 + 16 < n ? row_at(pool, id.b, key0 + 16, g, Hkv, D) - 16 * D : pa;
        const int left = n - key0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int lr = i * L::ROWS_PER_LOAD + lrow, r = lr < left ? lr : left - 1;
            dma16_nt(pool.v + ((i * L::ROWS_PER_LOAD < 16 || r < 16 ? pa : pb) + r * D) * 2 + ((lchunk ^ L::vswz(lr)) << 4), lds0 + (uint32_t)(stage * BLOCK + i * 1024));
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int lr = krow + 4 * t, r = lr < left ? lr : left - 1;
            const bf16_t* const kr = (const bf16_t*)pool.k + (r < 16 ? pa : pb) + r * D + 8 * kg;
#pragma unroll
            for (int i = 0; i < KI; ++i) kf[t][i] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(kr + 32 * i));
        }
    };
    // the lane's place among value rows 8 kg + (lane % 16) / 4 (and 4 on), dimensions 4 (lane % 4) of 16
    const int vr = 8 * kg + (l16 >> 2), vc = (l16 & 3) >> 1;
    float* const to_scores = SCORES ? scores + ((int64_t)sq.scores[b] + (g * cols + col) * score_blocks(n)) * 32 + 4 * kg : nullptr;
    f32x4 o[VM];
#pragma unroll
    for (int i = 0; i < VM; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = PAGED_LOWEST, l = 0.f;
    int key0 = k0 + wave * 32, stage = 0;
    Ids next{};
    if (key0 < k1) {
        load(key0, ids_of(key0), 0);
        next = ids_of(key0 + NW * 32);
    }
    for (; key0 < k1; key0 += NW * 32, stage ^= 1) {
        // The values have landed where all but two operations have: behind them went at least two loads of keys (which the compiler waits for itself), and two stores of scores that
        // need not have.
        SPTS_WAIT_VMCNT(2);
        asm volatile("" ::: "memory");   // (the values' reads stay behind the wait)
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KI; ++i) s[t] = mfma16(kf[t][i], qf[i], s[t]);
        }
        if (key0 + NW * 32 < k1) {
            load(key0 + NW * 32, next, stage ^ 1);
            next = ids_of(key0 + 2 * NW * 32);
        }
        const bool masked = key0 + 32 > all_see;
        float mx = PAGED_LOWEST;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float x = s[j >> 2][j & 3] * c;
            if (masked) x = key0 + 8 * kg + j < seen ? x : -INFINITY;
            s[j >> 2][j & 3] = x;
            mx = fmaxf(mx, x);
        }
        if constexpr (SCORES) {   // behind the next block's loads, so that the wait for those is none for these; rows of whole blocks of 32 keys, in the order that stores whole
            // pieces of 64 bytes: place 16 t + 4 kg + r has key 8 kg + 4 t + r (lanes without a column store the last column's again)
            if (kept > 0) {
                float* const to = reinterpret_cast<float*>(smem + kvp_few_lds(D)) + l16 * kept + (key0 - k0) + 4 * kg;
                if (l16 < cols) {
                    *reinterpret_cast<f32x4*>(to) = s[0];
                    *reinterpret_cast<f32x4*>(to + 16) = s[1];
                }
            } else {
                *reinterpret_cast<f32x4*>(to_scores + key0) = s[0];
                *reinterpret_cast<f32x4*>(to_scores + key0 + 16) = s[1];
            }
        }
        if (__ballot(mx > m + TAU) != 0) {
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float to = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= alpha;
#pragma unroll
            for (int i = 0; i < VM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] *= alpha;
        }
        u32x4 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const float p0 = __builtin_amdgcn_exp2f(s[j >> 2][j & 3] - m), p1 = __builtin_amdgcn_exp2f(s[j >> 2][(j & 3) + 1] - m);
            l += p0 + p1;
            const uint32_t h0 = first_part(p0), h1 = first_part(p1);
            hi[j >> 1] = __builtin_amdgcn_perm(h1, h0, 0x07060302u);
            lo[j >> 1] = cvt_pk_bf16(p0 - __uint_as_float(h0), p1 - __uint_as_float(h1));
        }
        const bf16x8 ph = __builtin_bit_cast(bf16x8, hi), pl = __builtin_bit_cast(bf16x8, lo);
        const uint32_t at = lds0 + (uint32_t)(stage * BLOCK);
#pragma unroll
        for (int i = 0; i < VM; ++i) {
            union { s16x4 h[2]; bf16x8 v; } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at + (uint32_t)(L::v_at(vr, 2 * i + vc) + (l16 & 1) * 8)));
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at + (uint32_t)(L::v_at(vr + 4, 2 * i + vc) + (l16 & 1) * 8)));
            bf16x8 v = u.v;
            if (masked && __ballot(any_odd(v)) != 0) {
                bf16x8 up, down;
                v = split_odd(v, &up, &down);
                u32x4 sees;
#pragma unroll
                for (int j = 0; j < 8; j += 2) sees[j >> 1] = (key0 + 8 * kg + j < seen ? 0x3f80u : 0u) | (key0 + 8 * kg + j + 1 < seen ? 0x3f800000u : 0u);
                const f32x4 z = {0.f, 0.f, 0.f, 0.f};
                const f32x4 pu = mfma16(up, __builtin_bit_cast(bf16x8, sees), z), pd = mfma16(down, __builtin_bit_cast(bf16x8, sees), z);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] += (pu[r] > 0.f ? INFINITY : 0.f) - (pd[r] > 0.f ? INFINITY : 0.f);
            }
            o[i] = mfma16(v, pl, o[i]);
            o[i] = mfma16(v, ph, o[i]);
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    // ---- the wavefronts meet
    __syncthreads();
    float* const so = reinterpret_cast<float*>(smem);
    float* const sml = so + NW * 16 * LD;
#pragma unroll
    for (int i = 0; i < VM; ++i) *reinterpret_cast<f32x4*>(so + (wave * 16 + l16) * LD + 16 * i + 4 * kg) = o[i];
    if (kg == 0) { sml[(wave * 16 + l16) * 2] = m; sml[(wave * 16 + l16) * 2 + 1] = l; }
    __syncthreads();
    if constexpr (SCORES) {
        if (kept > 0) {
            const float* const from = reinterpret_cast<const float*>(smem + kvp_few_lds(D));
            const int len = k1 > k0 ? (k1 - k0 + 31) / 32 * 32 : 0;
            for (int cn = 0; cn < cols; ++cn) {
                float* const to = scores + ((int64_t)sq.scores[b] + (g * cols + cn) * score_blocks(n)) * 32 + k0;
                for (int i = 4 * tid; i < len; i += 4 * NW * 64) *reinterpret_cast<f32x4*>(to + i) = *reinterpret_cast<const f32x4*>(from + cn * kept + i);
            }
        }
    }
    for (int i = tid; i < cols * (D / 4); i += NW * 64) {
        const int cn = i / (D / 4), e = i % (D / 4) * 4;
        float M = PAGED_LOWEST, sum = 0.f;
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, sml[(w * 16 + cn) * 2]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float a = __builtin_amdgcn_exp2f(sml[(w * 16 + cn) * 2] - M);
            const f32x4 ow = *reinterpret_cast<const f32x4*>(so + (w * 16 + cn) * LD + e);
            sum += sml[(w * 16 + cn) * 2 + 1] * a;
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] += ow[j] * a;
        }
        if (splits > 1) {
            const int64_t to = (int64_t)sq.at[b] + ((int64_t)split * Hkv + g) * cols + cn;
            if (e == 0) sh.ml[to] = make_float2(M, sum);
            *reinterpret_cast<f32x4*>(sh.o + to * D + e) = t;
        } else {
            const float inv = inverse_sum(sum);
            const int64_t head = (int64_t)(sq.first[b] + cn / G) * H + g * G + cn % G;
            const u32x2 w = {cvt_pk_bf16(t[0] * inv, t[1] * inv), cvt_pk_bf16(t[2] * inv, t[3] * inv)};
            *reinterpret_cast<u32x2*>(out + head * D + e) = w;
            if (stats && e == 0) stats[head] = make_float2(M, inv);
        }
    }
}

// ------------------------------------------------------------------ accounts of many columns
// Column sums of the probabilities, the scores anew: storing them would be more bytes than the products cost.  A workgroup has 256 keys, a wavefront 64 of them in registers, and
// goes over the blocks of 32 columns of its part of (head, block); the queries of a block and the columns' maxima and 1 / sums come into LDS by direct loads, three blocks ahead in a ring
// of four.  While the scores of the next block are on the matrix core, the lane takes the exponentials of this one's; a step is one operand read ahead, two matrix instructions
// and four exponentials (operands read where they are used instead: 792 us for 2048 tokens after 30720 rows, so 682).
constexpr int WW = 4, WST = 4;
template <int D, int NB>
__global__ void __launch_bounds__(WW * 64, 2) kvp_weights_mfma_kernel(const bf16_t* __restrict__ q, PoolView pool, PagedSeqs<NB> sq, int H, int Hkv, DivG dg, float c,
                                                                      const float2* __restrict__ stats, float* __restrict__ sums, float decay) {
    using L = Tile<D>;
    constexpr int KS = D / 16, BLOCK = 32 * L::ROW, LOADS = BLOCK / 1024, STAGE = BLOCK + 256;
    __shared__ __attribute__((aligned(1024))) char ring[WST * BLOCK];
    __shared__ __attribute__((aligned(256))) float2 col_stats[WST][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh = lane >> 5, G = dg.G;
    int first;
    const int b = seq_of(sq.end, (int)blockIdx.x, &first);
    const int parts = sq.parts[b], item = (int)blockIdx.x - first, part = item % parts;
    const int n = sq.count[b], nq = sq.nq[b], cols = nq * G, blocks = (cols + 31) / 32;
    const int tile0 = item / parts * (WW * 64), key0 = tile0 + wave * 64;
    // blocks that see nothing of the tile come first: a column sees row n - nq + col / G at last
    const int skip = tile0 > n - nq ? (int)((int64_t)(tile0 - (n - nq)) * G / 32) : 0;
    const int each = blocks - skip;
    const int64_t total = (int64_t)each * Hkv;
    const int64_t i0 = total * part / parts, i1 = total * (part + 1) / parts;
    const int steps = (int)(i1 - i0);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring;
    const uint32_t st0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float2*)&col_stats[0][0];
    const int lrow = lane / L::CPR, lchunk = lane % L::CPR;
    // head and block of the next block to load
    int lg = (int)(i0 / each), lblk = skip + (int)(i0 % each);
    constexpr int EACH = (LOADS + WW - 1) / WW + 1;   // loads of every wavefront a block: its share of the queries and, each the same, the statistics
    auto issue = [&](int i) __attribute__((always_inline)) {
        const int st = i % WST;
        auto head_of = [&](int cn) {
            cn = cn < cols ? cn : cols - 1;
            const uint32_t qi = div_g((uint32_t)cn, dg);
            return (uint32_t)((sq.first[b] + (int)qi) * H + lg * G + (cn - (int)qi * G));   // (queries times heads stay below 2^31: checked on the host)
        };
#pragma unroll
        for (int j = 0; j < EACH - 1; ++j) {
            const int ld = (j * WW + wave) % LOADS, row = ld * L::ROWS_PER_LOAD + lrow;
            dma16(q + (int64_t)head_of(lblk * 32 + row) * D + ((lchunk ^ L::kswz(row)) << 3), lds0 + (uint32_t)(st * BLOCK + ld * 1024));
        }
        dma4_nt((const float*)(stats + head_of(lblk * 32 + (lane >> 1))) + (lane & 1), st0 + (uint32_t)(st * 256));
        if (++lblk == blocks) { lblk = skip; ++lg; }
    };

    f32x16 acc[2] = {zero16(), zero16()};
    bf16x8 kf[2][KS];
    const uint32_t kplace = (uint32_t)L::k_at(l32, lh);
    int64_t krow[2];    // element offsets of the lane's two keys on head 0's page
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = key0 + 32 * h + l32 < n ? key0 + 32 * h + l32 : n - 1;
            krow[h] = page_at(pool, sq.table[b], r & ~15, 0, Hkv, D) + (r & 15) * D + 8 * lh;
        }
    }
    const int64_t head_step = (int64_t)D << pool.shift;
    auto load_keys = [&](int g) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kf[h][ks] = *reinterpret_cast<const bf16x8*>((const bf16_t*)pool.k + krow[h] + g * head_step + 16 * ks);
    };
    auto frag = [&](uint32_t at, int ks) { return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)(at ^ (uint32_t)(ks << 5)); };
    // scores of the block at `at` into N, while the exponentials of the block before it, C, are added to the accounts
    constexpr int FD = KS > 2 ? 3 : 1, EPS = 16 / KS;
    auto step = [&](uint32_t at, f32x16 (&N)[2], f32x16 (&C)[2], float2 st) __attribute__((always_inline)) {
        bf16x8 fr[FD + 1];
#pragma unroll
        for (int ks = 0; ks < FD; ++ks) fr[ks] = frag(at, ks);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (ks + FD < KS) fr[(ks + FD) % (FD + 1)] = frag(at, ks + FD);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                N[h] = mfma32(kf[h][ks], fr[ks % (FD + 1)], ks == 0 ? zero16() : N[h]);
#pragma unroll
                for (int e = ks * EPS; e < (ks + 1) * EPS; ++e) acc[h][e] = fmaf(__builtin_amdgcn_exp2f(fmaf(C[h][e], c, -st.x)), st.y, acc[h][e]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (steps > 0) {
        for (int i = 0; i < 3 && i < steps; ++i) issue(i);
        int g = (int)(i0 / each), blk = skip + (int)(i0 % each);
        load_keys(g);
        SPTS_WAIT_VMCNT(0);
        __syncthreads();
        f32x16 sa[2], sb[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) sa[h] = mfma32(kf[h][ks], frag(lds0 + kplace, ks), ks == 0 ? zero16() : sa[h]);
        auto block = [&](int i, f32x16 (&N)[2], f32x16 (&C)[2]) __attribute__((always_inline)) {
            if (i >= steps) return;
            // block i + 1 has landed for everyone, and block i - 1's place is free
            if (i > 0) {
                if (i + 2 < steps) { SPTS_WAIT_VMCNT(EACH); } else { SPTS_WAIT_VMCNT(0); }
                __syncthreads();
            }
            if (i + 3 < steps) issue(i + 3);
            float2 st = col_stats[i % WST][l32];
            const int col = blk * 32 + l32;
            const int seen = (col < cols ? n - nq + (int)div_g((uint32_t)col, dg) + 1 : 0) - key0 - 4 * lh;   // of the lane's keys, from its first one
            const bool masked = blk * 32 + 32 > cols || n - nq + (int)div_g((uint32_t)(blk * 32), dg) + 1 < key0 + 64;
            if (++blk == blocks) { blk = skip; if (++g < Hkv && i + 1 < steps) load_keys(g); }
            const uint32_t at = lds0 + (uint32_t)((i + 1) % WST * BLOCK) + kplace;
            if (masked) {   // unseen keys weigh nothing, not even of a column whose sum is NaN
                const bool odd = !(st.y < INFINITY);
                st.y = odd ? 1.f : st.y;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 16; ++e) C[h][e] = 32 * h + 8 * (e >> 2) + (e & 3) < seen ? (odd ? NAN : C[h][e]) : -INFINITY;
            }
            step(at, N, C, st);
        };
        for (int i = 0; i < steps; i += 2) {
            block(i, sb, sa);
            block(i + 1, sa, sb);
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float w = group_sum<32>(acc[h][r]);
            const int key = key0 + 32 * h + 8 * (r >> 2) + 4 * lh + (r & 3);
            if (l32 != 0 || key >= n) continue;
            if (parts > 1) sums[(int64_t)sq.at[b] + (int64_t)part * n + key] = w;
            else sq.weight[b][key] = decay == 0.f ? w : decay * sq.weight[b][key] + w;
        }
}

// ------------------------------------------------------------------ launches
template <int D, int NB, bool ONCE>
static hipError_t launch_many_once(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, const Shares& sh, float2* stats, bf16_t* out, hipStream_t s) {
    constexpr int LDS = NST * 2 * BKV * Tile<D>::ROW, NW = kvp_many_waves(D);
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(&kvp_many_kernel<D, NW, NB, ONCE>), LDS);
    if (e != hipSuccess) return e;
    kvp_many_kernel<D, NW, NB, ONCE><<<dim3((unsigned)(items * Hkv)), dim3(NW * 64), LDS, s>>>(q, pool, sq, H, Hkv, PAGED_LOG2E / sqrtf((float)D), sh, stats, out);
    return hipGetLastError();
}

template <int D, int NB>
static hipError_t launch_many(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, const Shares& sh, float2* stats, bf16_t* out, hipStream_t s) {
    bool once = true;
    for (int b = 0; b < NB; ++b) once = once && (int64_t)sq.nq[b] * (H / Hkv) <= kvp_many_waves(D) * 32;
    return once ? launch_many_once<D, NB, true>(q, pool, sq, items, H, Hkv, sh, stats, out, s) : launch_many_once<D, NB, false>(q, pool, sq, items, H, Hkv, sh, stats, out, s);
}

template <int NB>
hipError_t launch_kvp_attn_many(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, int d, const Shares& sh, float2* stats, bf16_t* out,
                                hipStream_t s) {
    return d == 128 ? launch_many<128, NB>(q, pool, sq, items, H, Hkv, sh, stats, out, s)
         : d == 64 ? launch_many<64, NB>(q, pool, sq, items, H, Hkv, sh, stats, out, s) : launch_many<32, NB>(q, pool, sq, items, H, Hkv, sh, stats, out, s);
}
template hipError_t launch_kvp_attn_many<1>(const bf16_t*, const PoolView&, const PagedSeqs<1>&, int, int, int, int, const Shares&, float2*, bf16_t*, hipStream_t);
template hipError_t launch_kvp_attn_many<DECODE_MAX_BATCH>(const bf16_t*, const PoolView&, const PagedSeqs<DECODE_MAX_BATCH>&, int, int, int, int, const Shares&, float2*, bf16_t*,
                                                           hipStream_t);

template <int D, int NB, bool SCORES>
static hipError_t launch_few_s(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, const Shares& sh, float2* stats, float* scores, bf16_t* out,
                             hipStream_t s) {
    constexpr int NW = KVP_FEW_WAVES, LDS = kvp_few_lds(D);
    static_assert(LDS % 16 == 0, "scores lie behind it");
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(&kvp_few_kernel<D, NW, NB, SCORES>), SCORES ? KVP_LDS : LDS);
    if (e != hipSuccess) return e;
    int kept = 0, bytes = 0;
    if (SCORES && (int64_t)items * Hkv <= CUS) {
        int cols = 0;
        int64_t longest = 0;
        for (int b = 0; b < NB; ++b) {
            if (sq.scores[b] < 0) continue;
            cols = std::max(cols, sq.nq[b] * (H / Hkv));
            longest = std::max<int64_t>(longest, std::min(sq.per[b], sq.count[b]));
        }
        if (kvp_few_keeps(D, cols, longest)) {
            kept = (int)kvp_kept_row(longest);
            bytes = cols * kept * 4;
        }
    }
    kvp_few_kernel<D, NW, NB, SCORES><<<dim3((unsigned)(items * Hkv)), dim3(NW * 64), LDS + bytes, s>>>(q, pool, sq, H, Hkv, PAGED_LOG2E / sqrtf((float)D), sh, stats, scores, kept, out);
    return hipGetLastError();
}

template <int D, int NB>
static hipError_t launch_few(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, const Shares& sh, float2* stats, float* scores, bf16_t* out,
                             hipStream_t s) {
    return scores ? launch_few_s<D, NB, true>(q, pool, sq, items, H, Hkv, sh, stats, scores, out, s) : launch_few_s<D, NB, false>(q, pool, sq, items, H, Hkv, sh, stats, scores, out, s);
}

template <int NB>
hipError_t launch_kvp_attn_few(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, int d, const Shares& sh, float2* stats, float* scores, bf16_t* out,
                               hipStream_t s) {
    if ((int64_t)items * Hkv > 0x7fffffff) return hipErrorInvalidValue;
    return d == 128 ? launch_few<128, NB>(q, pool, sq, items, H, Hkv, sh, stats, scores, out, s)
         : d == 64 ? launch_few<64, NB>(q, pool, sq, items, H, Hkv, sh, stats, scores, out, s)
                    : launch_few<32, NB>(q, pool, sq, items, H, Hkv, sh, stats, scores, out, s);
}
template hipError_t launch_kvp_attn_few<1>(const bf16_t*, const PoolView&, const PagedSeqs<1>&, int, int, int, int, const Shares&, float2*, float*, bf16_t*, hipStream_t);
template hipError_t launch_kvp_attn_few<DECODE_MAX_BATCH>(const bf16_t*, const PoolView&, const PagedSeqs<DECODE_MAX_BATCH>&, int, int, int, int, const Shares&, float2*, float*, bf16_t*,
                                                          hipStream_t);

template <int D, int NB>
static hipError_t launch_weights(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, const float2* stats, float* sums, float decay, hipStream_t s) {
    const int G = H / Hkv;
    const DivG dg{(uint32_t)((((uint64_t)1 << 32) + G - 1) / G), G};
    kvp_weights_mfma_kernel<D, NB><<<dim3((unsigned)items), dim3(WW * 64), 0, s>>>(q, pool, sq, H, Hkv, dg, PAGED_LOG2E / sqrtf((float)D), stats, sums, decay);
    return hipGetLastError();
}

template <int NB>
hipError_t launch_kvp_weights_many(const bf16_t* q, const PoolView& pool, const PagedSeqs<NB>& sq, int items, int H, int Hkv, int d, const float2* stats, float* sums, float decay,
                                   hipStream_t s) {
    return d == 128 ? launch_weights<128, NB>(q, pool, sq, items, H, Hkv, stats, sums, decay, s)
         : d == 64 ? launch_weights<64, NB>(q, pool, sq, items, H, Hkv, stats, sums, decay, s) : launch_weights<32, NB>(q, pool, sq, items, H, Hkv, stats, sums, decay, s);
}
template hipError_t launch_kvp_weights_many<1>(const bf16_t*, const PoolView&, const PagedSeqs<1>&, int, int, int, int, const float2*, float*, float, hipStream_t);
template hipError_t launch_kvp_weights_many<DECODE_MAX_BATCH>(const bf16_t*, const PoolView&, const PagedSeqs<DECODE_MAX_BATCH>&, int, int, int, int, const float2*, float*, float,
                                                              hipStream_t);

}  // namespace spts
