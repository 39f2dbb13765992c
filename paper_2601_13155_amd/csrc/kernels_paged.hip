// Caches in pages: appending rows, and cutting a cache down to the rows with the most accumulated attention.
#include "spts_lanes.h"

#include <algorithm>

namespace spts {

namespace {
template <int NB> struct AppendSeqs {
    const int32_t* table[NB];
    int32_t* pos[NB];
    float* weight[NB];
    int32_t at[NB], end[NB];   // cache row of the sequence's first row, its end among the call's rows
};
template <int NB> struct EvictSeqs {
    const int32_t* table[NB];
    int32_t* pos[NB];
    float* weight[NB];
    int32_t count[NB], keep[NB], below[NB], above[NB];  // positions below / above which rows go before others; count = 0: nothing leaves
    int32_t list[NB];                                   // where the sequence's list of moves begins
    int32_t old[NB];                                    // where its part of `old` begins
};
struct Move { int32_t src, dst; };
}  // namespace

// A thread copies 16 bytes of a key and of a value; the rows of a head lie next to each other in a page.
template <int NB>
__global__ void __launch_bounds__(256) kvp_append_kernel(const u32x4* __restrict__ k, const u32x4* __restrict__ v, const int32_t* __restrict__ pos, u32x4* __restrict__ pk,
                                                         u32x4* __restrict__ pv, uint32_t pages, int shift, AppendSeqs<NB> sq, int64_t total, int Hkv, int chunks) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const int per = Hkv * chunks, e = (int)(i % per), g = e / chunks, ch = e % chunks;
    const int32_t row = (int32_t)(i / per);
    int b = 0, first = 0;
#pragma unroll
    for (int j = 0; j + 1 < NB; ++j)
        if (row >= sq.end[j]) { b = j + 1; first = sq.end[j]; }
    const int32_t at = sq.at[b] + (row - first);
    const u32x4 kw = k[i], vw = v[i];
    const uint32_t id = (uint32_t)sq.table[b][at >> shift];
    if (id < pages) {
        const int64_t to = ((((int64_t)id * Hkv + g) << shift) + (at & ((1 << shift) - 1))) * chunks + ch;
        pk[to] = kw;
        pv[to] = vw;
    }
    if (e == 0) {
        sq.pos[b][at] = pos[row];
        if (sq.weight[b]) sq.weight[b][at] = 0.f;
    }
}

template <int NB>
static hipError_t launch_kvp_append_n(const void* k, const void* v, const int32_t* pos, const PagedPool& pool, const PagedBatch& pb, int Hkv, int chunks, hipStream_t s) {
    AppendSeqs<NB> sq{};
    for (int b = 0; b < NB; ++b) {
        const int i = b < pb.n ? b : pb.n - 1;
        sq.table[b] = pb.table[i]; sq.pos[b] = pb.pos[i]; sq.weight[b] = pb.weight[i];
        sq.at[b] = (int32_t)pb.count[i]; sq.end[b] = (int32_t)pb.off[i + 1];
    }
    const int64_t total = pb.off[pb.n] * Hkv * chunks, groups = (total + 255) / 256;
    if (groups > 0x7fffffff) return hipErrorInvalidValue;
    kvp_append_kernel<NB><<<dim3((unsigned)groups), dim3(256), 0, s>>>((const u32x4*)k, (const u32x4*)v, pos, (u32x4*)pool.k, (u32x4*)pool.v, (uint32_t)pool.pages, pool.shift, sq,
                                                                       total, Hkv, chunks);
    return hipGetLastError();
}

hipError_t launch_kvp_append(const void* k, const void* v, const int32_t* pos, const PagedPool& pool, const PagedBatch& pb, int Hkv, int d, bool bf16, hipStream_t s) {
    if (pb.n < 1 || pb.n > DECODE_MAX_BATCH) return hipErrorInvalidValue;
    const int chunks = d * (bf16 ? 2 : 4) / 16;
    return pb.n == 1 ? launch_kvp_append_n<1>(k, v, pos, pool, pb, Hkv, chunks, s) : launch_kvp_append_n<DECODE_MAX_BATCH>(k, v, pos, pool, pb, Hkv, chunks, s);
}

// ------------------------------------------------------------------ eviction
// The order of the rows as unsigned numbers: rows that go before others have the upper bit, which no weight needs.  A NaN is above every number.
__device__ inline uint32_t evict_key(float w, int32_t pos, int32_t below, int32_t above) {
    const uint32_t u = w < 0.f ? 0u : __float_as_uint(w) & 0x7fffffffu;
    return u | (pos < below || pos > above ? 0x80000000u : 0u);
}

constexpr int ET = 1024, EWV = ET / 64, EBITS = 11, EBINS = 1 << EBITS;

// One workgroup per sequence.  Three radix passes of 11, 11 and 10 bits find the smallest key that stays and how many of its equals do; a wavefront has a stretch of rows, so that
// counts of wavefronts give every row its rank without a barrier in between.  The rows that move, and the places they go to, are listed for kvp_move_kernel; positions, weights and `old`
// are written here (sources lie from `keep` on, places below it).
template <int NB>
__global__ void __launch_bounds__(ET) kvp_select_kernel(EvictSeqs<NB> sq, Move* __restrict__ moves, int32_t* __restrict__ n_moves, int32_t* __restrict__ old) {
    __shared__ uint32_t hist[EBINS];
    __shared__ uint32_t swave[EWV], sgone[EWV], pick[2];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = sq.count[b], k = sq.keep[b];
    int32_t* const o = old ? old + sq.old[b] : nullptr;
    if (n <= k) {   // everything stays (n = 0: the host's word for it)
        if (o) for (int i = tid; i < k; i += ET) o[i] = i;
        if (tid == 0) n_moves[b] = 0;
        return;
    }
    const int32_t* const pos = sq.pos[b];
    const float* const weight = sq.weight[b];
    const int32_t below = sq.below[b], above = sq.above[b];
    const int stretch = (n + EWV * 64 - 1) / (EWV * 64) * 64, w0 = wave * stretch, w1 = w0 + stretch < n ? w0 + stretch : n;
    uint32_t prefix = 0, want = (uint32_t)k;   // of the keys that agree with the prefix so far the `want` largest stay
    for (int pass = 0; pass < 3; ++pass) {
        const int sh = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t bins = pass == 2 ? EBINS / 2 : EBINS;
        for (int i = tid; i < EBINS; i += ET) hist[i] = 0;
        __syncthreads();
        const uint32_t known = pass == 0 ? 0u : ~0u << (pass == 1 ? 21 : 10);
        for (int i = w0 + lane; i < w1; i += 64) {
            const uint32_t key = evict_key(weight[i], pos[i], below, above);
            if ((key & known) == prefix) atomicAdd(&hist[(key >> sh) & (bins - 1)], 1u);
        }
        __syncthreads();
        // counts of the bins from the highest down: thread t has bins 2 (ET - 1 - t) + 1 and 2 (ET - 1 - t)
        const int hi = 2 * (ET - 1 - tid) + 1;
        const uint32_t c1 = hist[hi], c0 = hist[hi - 1];
        uint32_t sum = c0 + c1;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t t = __shfl_up(sum, off);
            sum += lane >= off ? t : 0;
        }
        if (lane == 63) swave[wave] = sum;
        __syncthreads();
        for (int w = 0; w < wave; ++w) sum += swave[w];
        const uint32_t before = sum - c0 - c1;   // keys in higher bins
        if (before < want && want <= before + c1) { pick[0] = (uint32_t)hi; pick[1] = want - before; }
        else if (before + c1 < want && want <= sum) { pick[0] = (uint32_t)hi - 1; pick[1] = want - before - c1; }
        __syncthreads();
        prefix |= pick[0] << sh;
        want = pick[1];
        __syncthreads();
    }
    // `want` of the keys equal to prefix stay, the lowest rows of them
    uint32_t ties = 0;
    for (int i = w0 + lane; i - lane < w1; i += 64) {
        const bool t = i < w1 && evict_key(weight[i], pos[i], below, above) == prefix;
        ties += (uint32_t)__popcll(__ballot(t));
    }
    if (lane == 0) swave[wave] = ties;
    __syncthreads();
    uint32_t tie0 = 0;
    for (int w = 0; w < wave; ++w) tie0 += swave[w];
    __syncthreads();
    const uint64_t lower = lane ? ~0ull >> (64 - lane) : 0ull;
    // rank 0 of a stretch's free places and movers, then the lists
    uint32_t free0 = 0, move0 = 0;
    for (int sweep = 0; sweep < 2; ++sweep) {
        uint32_t tie = tie0, nfree = free0, nmove = move0;
        for (int i = w0 + lane; i - lane < w1; i += 64) {
            const uint32_t key = i < w1 ? evict_key(weight[i], pos[i], below, above) : 0u;
            const bool t = i < w1 && key == prefix;
            const uint64_t tb = __ballot(t);
            const bool stays = i < w1 && (key > prefix || (t && tie + (uint32_t)__popcll(tb & lower) < want));
            tie += (uint32_t)__popcll(tb);
            const uint64_t fb = __ballot(i < k && i < w1 && !stays), mb = __ballot(i >= k && stays);
            if (sweep == 1) {
                Move* const list = moves + sq.list[b];
                if (fb >> lane & 1) list[nfree + (uint32_t)__popcll(fb & lower)].dst = i;
                if (mb >> lane & 1) list[nmove + (uint32_t)__popcll(mb & lower)].src = i;
                if (o && i < k && stays) o[i] = i;
            }
            nfree += (uint32_t)__popcll(fb);
            nmove += (uint32_t)__popcll(mb);
        }
        if (sweep == 0) {
            if (lane == 0) { swave[wave] = nfree; sgone[wave] = nmove; }
            __syncthreads();
            for (int w = 0; w < wave; ++w) { free0 += swave[w]; move0 += sgone[w]; }
        }
    }
    __threadfence_block();
    __syncthreads();
    uint32_t all = 0;
    for (int w = 0; w < EWV; ++w) all += sgone[w];
    if (tid == 0) n_moves[b] = (int32_t)all;
    for (uint32_t i = tid; i < all; i += ET) {
        const Move mv = moves[sq.list[b] + i];
        if (o) o[mv.dst] = mv.src;
        sq.pos[b][mv.dst] = pos[mv.src];
        sq.weight[b][mv.dst] = weight[mv.src];
    }
}

// One workgroup per row that may move: its keys and values of all heads, 16 bytes a thread
template <int NB>
__global__ void __launch_bounds__(256) kvp_move_kernel(u32x4* __restrict__ pk, u32x4* __restrict__ pv, uint32_t pages, int shift, EvictSeqs<NB> sq, const Move* __restrict__ moves,
                                                       const int32_t* __restrict__ n_moves, int Hkv, int chunks) {
    const int b = blockIdx.y;
    if ((int)blockIdx.x >= n_moves[b]) return;
    const Move mv = moves[sq.list[b] + blockIdx.x];
    const int mask = (1 << shift) - 1;
    uint32_t from = (uint32_t)sq.table[b][mv.src >> shift];
    const uint32_t to = (uint32_t)sq.table[b][mv.dst >> shift];
    from = from < pages ? from : 0;
    if (to >= pages) return;
    for (int e = threadIdx.x; e < Hkv * chunks; e += 256) {
        const int g = e / chunks, ch = e % chunks;
        const int64_t f = ((((int64_t)from * Hkv + g) << shift) + (mv.src & mask)) * chunks + ch;
        const int64_t t = ((((int64_t)to * Hkv + g) << shift) + (mv.dst & mask)) * chunks + ch;
        const u32x4 kw = pk[f], vw = pv[f];
        pk[t] = kw;
        pv[t] = vw;
    }
}

static int64_t most_moves(const PagedBatch& pb, const PagedEvict& ev, int b) {
    return pb.count[b] > ev.keep[b] ? std::min(ev.keep[b], pb.count[b] - ev.keep[b]) : 0;
}

size_t kvp_evict_scratch(const PagedBatch& pb, const PagedEvict& ev) {
    size_t n = 0;
    for (int b = 0; b < pb.n; ++b) n += (size_t)most_moves(pb, ev, b);
    return n * sizeof(Move) + DECODE_MAX_BATCH * sizeof(int32_t);
}

template <int NB>
static hipError_t launch_kvp_evict_n(const PagedPool& pool, const PagedBatch& pb, const PagedEvict& ev, int32_t* old, int Hkv, int chunks, void* scratch, hipStream_t s) {
    EvictSeqs<NB> sq{};
    int64_t at = 0, kept = 0, most = 0;
    for (int b = 0; b < pb.n; ++b) {
        const bool leaves = pb.count[b] > ev.keep[b] && ev.keep[b] > 0;
        sq.table[b] = pb.table[b]; sq.pos[b] = pb.pos[b]; sq.weight[b] = pb.weight[b];
        sq.count[b] = leaves ? (int32_t)pb.count[b] : 0;
        sq.keep[b] = (int32_t)std::min(ev.keep[b], pb.count[b]);
        sq.below[b] = ev.below[b]; sq.above[b] = ev.above[b];
        sq.list[b] = (int32_t)at; sq.old[b] = (int32_t)kept;
        at += most_moves(pb, ev, b);
        kept += sq.keep[b];
        most = std::max(most, most_moves(pb, ev, b));
    }
    int32_t* const n_moves = (int32_t*)scratch;
    Move* const moves = (Move*)(n_moves + DECODE_MAX_BATCH);
    kvp_select_kernel<NB><<<dim3((unsigned)pb.n), dim3(ET), 0, s>>>(sq, moves, n_moves, old);
    if (most > 0) kvp_move_kernel<NB><<<dim3((unsigned)most, (unsigned)pb.n), dim3(256), 0, s>>>((u32x4*)pool.k, (u32x4*)pool.v, (uint32_t)pool.pages, pool.shift, sq, moves, n_moves,
                                                                                               Hkv, chunks);
    return hipGetLastError();
}

hipError_t launch_kvp_evict(const PagedPool& pool, const PagedBatch& pb, const PagedEvict& ev, int32_t* old, int Hkv, int d, bool bf16, void* scratch, hipStream_t s) {
    if (pb.n < 1 || pb.n > DECODE_MAX_BATCH) return hipErrorInvalidValue;
    const int chunks = d * (bf16 ? 2 : 4) / 16;
    return pb.n == 1 ? launch_kvp_evict_n<1>(pool, pb, ev, old, Hkv, chunks, scratch, s) : launch_kvp_evict_n<DECODE_MAX_BATCH>(pool, pb, ev, old, Hkv, chunks, scratch, s);
}

}  // namespace spts
