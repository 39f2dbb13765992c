// Caches in pages: appending rows, and cutting a cache down to the rows with the most accumulated attention.
#include "spts_lanes.h"

#include <algorithm>
#include <type_traits>

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
constexpr int64_t MAX_GROUPS = (1 << 24) - 1;   // of 256 threads: a launch has fewer than 2^32
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
    if (groups > MAX_GROUPS) return hipErrorInvalidValue;
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

// One workgroup per sequence.  Three radix passes of 11, 11 and 10 bits find the smallest key that stays and how many of its equals do; then the rows that move and the places
// they go to are listed for kvp_move_kernel.  A wavefront has a stretch of rows, K4 quads of neighbouring ones a lane, their keys in registers: ballots give
// ranks inside it, and counts of wavefronts the rest.
constexpr int K4 = 4;   // quads of rows a lane
template <int NB>
__global__ void __launch_bounds__(ET) kvp_select_kernel(EvictSeqs<NB> sq, Move* __restrict__ moves, int32_t* __restrict__ n_moves, int32_t* __restrict__ old) {
    __shared__ uint32_t hist[EBINS];
    __shared__ uint32_t swave[EWV], smove[EWV], pick[2];
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
    const int stretch = ((n + EWV - 1) / EWV + 255) / 256 * 256, w0 = wave * stretch, w1 = w0 + stretch < n ? w0 + stretch : n;
    const int last4 = (n - 1) & ~3;   // (whole quads: capacities are multiples of a page)
    uint32_t key[K4][4];   // rows behind the last one have 0: they are the last of their equals, of which enough come before them
#pragma unroll
    for (int j = 0; j < K4; ++j) {
        const int i = w0 + 256 * j + 4 * lane, at = i < last4 ? i : last4;
        const f32x4 w = *reinterpret_cast<const f32x4*>(weight + at);
        const u32x4 p = *reinterpret_cast<const u32x4*>(pos + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) key[j][e] = i + e < n ? evict_key(w[e], (int32_t)p[e], below, above) : 0u;
    }
    uint32_t prefix = 0, want = (uint32_t)k;   // of the keys that agree with the prefix so far the `want` largest stay
    for (int pass = 0; pass < 3; ++pass) {
        const int sh = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t bins = pass == 2 ? EBINS / 2 : EBINS;
        for (int i = tid; i < EBINS; i += ET) hist[i] = 0;
        __syncthreads();
        const uint32_t known = pass == 0 ? 0u : ~0u << (pass == 1 ? 21 : 10);
#pragma unroll
        for (int j = 0; j < K4; ++j) {
            if (w0 + 256 * j >= w1) break;
            // (one count of 256 where rows are all alike, zeros for instance)
            const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane((int)key[j][0]);
            const bool alike = key[j][0] == first && key[j][1] == first && key[j][2] == first && key[j][3] == first;
            if (__ballot(alike) == ~0ull) {
                if (lane == 0 && (first & known) == prefix) atomicAdd(&hist[(first >> sh) & (bins - 1)], 256u);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if ((key[j][e] & known) == prefix) atomicAdd(&hist[(key[j][e] >> sh) & (bins - 1)], 1u);
            }
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
    // of the rows with the key `prefix` the first `want` stay
    uint32_t ties = 0;
#pragma unroll
    for (int j = 0; j < K4; ++j) {
        if (w0 + 256 * j >= w1) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) ties += (uint32_t)__popcll(__ballot(key[j][e] == prefix));
    }
    if (lane == 0) swave[wave] = ties;
    __syncthreads();
    uint32_t tie0 = 0, all_ties = 0;
    for (int w = 0; w < EWV; ++w) {
        tie0 += w < wave ? swave[w] : 0;
        all_ties += swave[w];
    }
    __syncthreads();
    auto below_lane = [&](uint64_t m) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u)); };
    // f(first row of the lane's quad, which of the four are free places / move, ranks of the first of each in the wavefront, which stay) for all quads; counts in nfree, nmove.
    // choose: only some of the rows with the key `prefix` stay
    uint32_t nfree = 0, nmove = 0;
    auto quads = [&](auto choose, auto f) __attribute__((always_inline)) {
        uint32_t tie = tie0;
        nfree = nmove = 0;
#pragma unroll
        for (int j = 0; j < K4; ++j) {
            const int q0 = w0 + 256 * j, i0 = q0 + 4 * lane;
            if (q0 >= w1) break;
            bool stays[4], is_free[4], moves_[4];
            uint32_t seen = tie;
            if constexpr (decltype(choose)::value) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint64_t m = __ballot(key[j][e] == prefix);
                    seen += below_lane(m);
                    tie += (uint32_t)__popcll(m);
                }
            }
            uint32_t frank = nfree, mrank = nmove;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                stays[e] = key[j][e] >= prefix && i0 + e < n;
                if constexpr (decltype(choose)::value) {
                    const bool t = key[j][e] == prefix;
                    stays[e] = stays[e] && (!t || seen < want);
                    seen += t ? 1u : 0u;
                }
                is_free[e] = i0 + e < k && !stays[e];
                moves_[e] = i0 + e >= k && stays[e];
                const uint64_t fm = __ballot(is_free[e]), mm = __ballot(moves_[e]);
                frank += below_lane(fm);
                mrank += below_lane(mm);
                nfree += (uint32_t)__popcll(fm);
                nmove += (uint32_t)__popcll(mm);
            }
            f(i0, is_free, moves_, stays, frank, mrank);
        }
    };
    auto both = [&](auto f) __attribute__((always_inline)) {
        if (all_ties > want) quads(std::true_type{}, f);
        else quads(std::false_type{}, f);
    };
    both([](int, bool (&)[4], bool (&)[4], bool (&)[4], uint32_t, uint32_t) {});
    if (lane == 0) { swave[wave] = nfree; smove[wave] = nmove; }
    __syncthreads();
    uint32_t free0 = 0, move0 = 0, total = 0;
    for (int w = 0; w < EWV; ++w) {
        free0 += w < wave ? swave[w] : 0;
        move0 += w < wave ? smove[w] : 0;
        total += smove[w];
    }
    if (tid == 0) n_moves[b] = (int32_t)total;
    Move* const list = moves + sq.list[b];
    both([&](int i0, bool (&is_free)[4], bool (&moves_)[4], bool (&stays)[4], uint32_t frank, uint32_t mrank) {
        frank += free0;
        mrank += move0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (is_free[e]) list[frank++].dst = i0 + e;
            if (moves_[e]) list[mrank++].src = i0 + e;
            if (o && stays[e] && i0 + e < k) o[i0 + e] = i0 + e;
        }
    });
}

// ---- the same over the chip, for long sequences: a chunk of rows per workgroup, none on both sides of `keep`.  Launch p (0 .. 2) counts the p-th digit of the chunk's keys, after it has found
// the digit before from all chunks' counts; the last launch knows from the third digit's counts and from `above` (keys of a chunk beyond the upper 22 bits) how many rows stay in every
// chunk before its own, and lists the free places and movers of its own.  65536 rows, 16384 to stay: 4 + 7 + 7 + 11 us.
constexpr int CHUNK = 4096, MAX_CHUNKS = 132;
struct ChipState { uint32_t prefix, want; };
struct ChipScratch {
    uint32_t* hist;      // [pass][sequence][chunk][EBINS]
    uint32_t* above;     // [sequence][chunk]
    ChipState* state;    // [pass][sequence]
    int chunks;          // room for that many of each sequence
    int64_t rows;        // of a chunk
};
struct Chunks { int low, all; };
__device__ inline Chunks chunks_of(int n, int k, int64_t rows) { return Chunks{(int)((k + rows - 1) / rows), (int)((k + rows - 1) / rows + (n - k + rows - 1) / rows)}; }

template <int NB, int PASS>
__global__ void __launch_bounds__(ET) kvp_select_chip_kernel(EvictSeqs<NB> sq, ChipScratch cs, int seqs, Move* __restrict__ moves, int32_t* __restrict__ n_moves, int32_t* __restrict__ old) {
    __shared__ uint32_t hist[PASS < 3 ? EBINS : 1];
    __shared__ uint32_t swave[EWV], smove[EWV], pick[2], stie[MAX_CHUNKS], sabove[MAX_CHUNKS];
    const int b = blockIdx.y, c = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = sq.count[b], k = sq.keep[b];
    int32_t* const o = old ? old + sq.old[b] : nullptr;
    if (n <= k) {
        if (PASS == 3 && c == 0) {
            if (o) for (int i = tid; i < k; i += ET) o[i] = i;
            if (tid == 0) n_moves[b] = 0;
        }
        return;
    }
    const Chunks ch = chunks_of(n, k, cs.rows);
    if (c >= ch.all) return;
    auto hist_of = [&](int pass, int chunk) { return cs.hist + (((int64_t)pass * seqs + b) * cs.chunks + chunk) * EBINS; };
    // rows [lo, hi) of the chunk
    const int64_t first = c < ch.low ? c * cs.rows : k + (c - ch.low) * cs.rows, end = c < ch.low ? k : n;
    const int lo = (int)first, hi = (int)(first + cs.rows < end ? first + cs.rows : end);
    const int stretch = (int)(cs.rows / EWV), w0 = lo + wave * stretch, w1 = w0 + stretch < hi ? w0 + stretch : hi;
    const int32_t below = sq.below[b], above = sq.above[b];
    const int32_t* const pos = sq.pos[b];
    const float* const weight = sq.weight[b];
    // f(first row, whether the lane's is one, its key) for the wavefront's rows, 64 at a time; four keys a lane are asked for together, and at the beginning where that is all of them
    constexpr int KS = 4;
    uint32_t keys[KS];
    auto load = [&](int s0) __attribute__((always_inline)) {
        float w[KS];
        int32_t p[KS];
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const int i = s0 + 64 * j + lane, at = i < hi ? i : hi - 1;
            w[j] = weight[at];
            p[j] = pos[at];
        }
#pragma unroll
        for (int j = 0; j < KS; ++j) keys[j] = evict_key(w[j], p[j], below, above);
    };
    const bool once = stretch <= 64 * KS;
    if (once) load(w0);
    auto each_row = [&](auto f) __attribute__((always_inline)) {
        for (int s0 = w0; s0 < w1; s0 += 64 * KS) {
            if (!once) load(s0);
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                if (s0 + 64 * j >= w1) break;
                f(s0 + 64 * j, s0 + 64 * j + lane < w1, keys[j]);
            }
        }
    };

    uint32_t prefix = 0, want = (uint32_t)k;
    if (PASS > 0) {
        if (PASS > 1) {
            const ChipState z = cs.state[(PASS - 1) * seqs + b];
            prefix = z.prefix;
            want = z.want;
        }
        constexpr int sh = PASS == 1 ? 21 : PASS == 2 ? 10 : 0;
        const int hb = 2 * (ET - 1 - tid) + 1;   // bins from the highest down, two a thread
        uint32_t c1 = 0, c0 = 0;
#pragma unroll 8
        for (int i = 0; i < ch.all; ++i) {
            const u32x2 v = *reinterpret_cast<const u32x2*>(hist_of(PASS - 1, i) + hb - 1);
            c0 += v[0];
            c1 += v[1];
        }
        uint32_t sum = c0 + c1;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t t = __shfl_up(sum, off);
            sum += lane >= off ? t : 0;
        }
        if (lane == 63) swave[wave] = sum;
        __syncthreads();
        for (int w = 0; w < wave; ++w) sum += swave[w];
        const uint32_t before = sum - c0 - c1;
        if (before < want && want <= before + c1) { pick[0] = (uint32_t)hb; pick[1] = want - before; }
        else if (before + c1 < want && want <= sum) { pick[0] = (uint32_t)hb - 1; pick[1] = want - before - c1; }
        __syncthreads();
        prefix |= pick[0] << sh;
        want = pick[1];
        if (PASS < 3 && c == 0 && tid == 0) cs.state[PASS * seqs + b] = ChipState{prefix, want};
    }
    if constexpr (PASS < 3) {
        constexpr int sh = PASS == 0 ? 21 : PASS == 1 ? 10 : 0;
        constexpr uint32_t bins = PASS == 2 ? EBINS / 2 : EBINS, known = PASS == 0 ? 0u : PASS == 1 ? ~0u << 21 : ~0u << 10;
        for (int i = tid; i < EBINS; i += ET) hist[i] = 0;
        __syncthreads();
        uint32_t more = 0;
        each_row([&](int, bool there, uint32_t key) {
            const uint32_t first_key = (uint32_t)__builtin_amdgcn_readfirstlane((int)key);
            const bool in = there && (key & known) == prefix;
            if (__ballot(there && key == first_key) == ~0ull) {   // (one count of 64 where rows are all alike)
                if (in && lane == 0) atomicAdd(&hist[(key >> sh) & (bins - 1)], 64u);
            } else if (in) {
                atomicAdd(&hist[(key >> sh) & (bins - 1)], 1u);
            }
            if (PASS == 2) more += (uint32_t)__popcll(__ballot(there && (key & known) > prefix));
        });
        if (PASS == 2 && lane == 0) smove[wave] = more;
        __syncthreads();
        uint32_t* const to = hist_of(PASS, c);
        for (int i = tid; i < EBINS; i += ET) to[i] = hist[i];
        if (PASS == 2 && tid == 0) {
            uint32_t all = 0;
            for (int w = 0; w < EWV; ++w) all += smove[w];
            cs.above[(int64_t)b * cs.chunks + c] = all;
        }
    } else {
        // of every chunk the keys above prefix and those equal to it
        for (int i = wave; i < ch.all; i += EWV) {
            const uint32_t* const h = hist_of(2, i);
            uint32_t more = 0;
#pragma unroll
            for (int j = 0; j < EBINS / 2 / 64; ++j) {
                const uint32_t bin = (uint32_t)(lane + 64 * j);
                const uint32_t v = h[bin];
                more += bin > pick[0] ? v : 0u;
            }
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) more += (uint32_t)__shfl_xor((int)more, off);
            if (lane == 0) { sabove[i] = more + cs.above[(int64_t)b * cs.chunks + i]; stie[i] = h[pick[0]]; }
        }
        __syncthreads();
        // equals before this chunk; free places (or movers) before it; movers in all: a lane a chunk, every wavefront for itself
        uint32_t tie = 0, base = 0, total = 0, ties_before = 0;
        for (int j0 = 0; j0 < ch.all; j0 += 64) {
            const int i = j0 + lane;
            const bool there = i < ch.all;
            const uint32_t t = there ? stie[i] : 0u;
            uint32_t upto = t;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const uint32_t v = __shfl_up(upto, off);
                upto += lane >= off ? v : 0;
            }
            const uint32_t mine = ties_before + upto - t, room = mine < want ? want - mine : 0u, stay = there ? sabove[i] + (t < room ? t : room) : 0u;
            const int64_t left = k - i * cs.rows;
            const uint32_t r = (uint32_t)(left < cs.rows ? left : cs.rows);   // (rows of a chunk below `keep`)
            if (i == c) tie = mine;
            base += there && i < c && (i < ch.low) == (c < ch.low) ? (i < ch.low ? r - stay : stay) : 0u;
            total += there && i >= ch.low ? stay : 0u;
            ties_before += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            tie += (uint32_t)__shfl_xor((int)tie, off);   // (one lane has it)
            base += (uint32_t)__shfl_xor((int)base, off);
            total += (uint32_t)__shfl_xor((int)total, off);
        }
        if (c == 0 && tid == 0) n_moves[b] = (int32_t)total;
        // the chunk's rows, a wavefront's stretch each
        uint32_t ties = 0;
        each_row([&](int, bool there, uint32_t key) { ties += (uint32_t)__popcll(__ballot(there && key == prefix)); });
        if (lane == 0) swave[wave] = ties;
        __syncthreads();
        for (int w = 0; w < wave; ++w) tie += swave[w];
        const uint64_t lower = lane ? ~0ull >> (64 - lane) : 0ull;
        Move* const list = moves + sq.list[b];
        uint32_t rank = 0;
        for (int sweep = 0; sweep < 2; ++sweep) {
            uint32_t t0 = tie, count = rank;
            each_row([&](int i0, bool there, uint32_t key) {
                const int i = i0 + lane;
                const bool t = there && key == prefix;
                const uint64_t tb = __ballot(t);
                const bool stays = there && (key > prefix || (t && t0 + (uint32_t)__popcll(tb & lower) < want));
                t0 += (uint32_t)__popcll(tb);
                const bool listed = there && (c < ch.low ? !stays : stays);
                const uint64_t lb = __ballot(listed);
                if (sweep == 1) {
                    const uint32_t at = count + (uint32_t)__popcll(lb & lower);
                    if (listed) { if (c < ch.low) list[at].dst = i; else list[at].src = i; }
                    if (o && c < ch.low && stays) o[i] = i;
                }
                count += (uint32_t)__popcll(lb);
            });
            if (sweep == 0) {
                if (lane == 0) smove[wave] = count;
                __syncthreads();
                rank = base;
                for (int w = 0; w < wave; ++w) rank += smove[w];
            }
        }
    }
}

// One workgroup per row that may move, up to MOVE_GROUPS of them: its keys and values of all heads, 16 bytes a thread, and its position and weight (sources lie from `keep` on, places
// below it, so that no row is read after it was written)
constexpr int64_t MOVE_GROUPS = 1 << 20;
template <int NB>
__global__ void __launch_bounds__(256) kvp_move_kernel(u32x4* __restrict__ pk, u32x4* __restrict__ pv, uint32_t pages, int shift, EvictSeqs<NB> sq, const Move* __restrict__ moves,
                                                       const int32_t* __restrict__ n_moves, int32_t* __restrict__ old, int Hkv, int chunks) {
    const int b = blockIdx.y, n = n_moves[b];
    const int mask = (1 << shift) - 1;
    for (int i = blockIdx.x; i < n; i += gridDim.x) {
        const Move mv = moves[(int64_t)sq.list[b] + i];
        uint32_t from = (uint32_t)sq.table[b][mv.src >> shift];
        const uint32_t to = (uint32_t)sq.table[b][mv.dst >> shift];
        from = from < pages ? from : 0;
        if (threadIdx.x == 0) {
            sq.pos[b][mv.dst] = sq.pos[b][mv.src];
            sq.weight[b][mv.dst] = sq.weight[b][mv.src];
            if (old) old[(int64_t)sq.old[b] + mv.dst] = mv.src;
        }
        if (to >= pages) continue;
        for (int e = threadIdx.x; e < Hkv * chunks; e += 256) {
            const int g = e / chunks, ch = e % chunks;
            const int64_t f = ((((int64_t)from * Hkv + g) << shift) + (mv.src & mask)) * chunks + ch;
            const int64_t t = ((((int64_t)to * Hkv + g) << shift) + (mv.dst & mask)) * chunks + ch;
            const u32x4 kw = __builtin_nontemporal_load(pk + f), vw = __builtin_nontemporal_load(pv + f);
            pk[t] = kw;
            pv[t] = vw;
        }
    }
}

static int64_t most_moves(const PagedBatch& pb, const PagedEvict& ev, int b) {
    return pb.count[b] > ev.keep[b] ? std::min(ev.keep[b], pb.count[b] - ev.keep[b]) : 0;
}
// One workgroup per sequence as long as its registers hold the keys (us by one / over the chip: 8192 rows 13 / 23, 16384 17 / 26)
constexpr int64_t SELECT_ONE = 4096 * K4;
static int64_t longest_cut(const PagedBatch& pb, const PagedEvict& ev) {
    int64_t n = 0;
    for (int b = 0; b < pb.n; ++b)
        if (pb.count[b] > ev.keep[b] && ev.keep[b] > 0) n = std::max(n, pb.count[b]);
    return n;
}
static int64_t chunk_rows(int64_t longest) { return (longest + CHUNK * (MAX_CHUNKS - 4) - 1) / (CHUNK * (MAX_CHUNKS - 4)) * CHUNK; }   // both sides of `keep` end in a part of a chunk
static int chunk_room(int64_t longest) { return (int)(longest / chunk_rows(longest)) + 2; }
static size_t moves_bytes(const PagedBatch& pb, const PagedEvict& ev) {
    size_t n = 0;
    for (int b = 0; b < pb.n; ++b) n += (size_t)most_moves(pb, ev, b);
    return ((n * sizeof(Move) + DECODE_MAX_BATCH * sizeof(int32_t)) + 255) / 256 * 256;
}

size_t kvp_evict_scratch(const PagedBatch& pb, const PagedEvict& ev) {
    const int64_t longest = longest_cut(pb, ev);
    const size_t moves = moves_bytes(pb, ev);
    return longest <= SELECT_ONE ? moves : moves + (size_t)pb.n * (chunk_room(longest) * (3 * EBINS + 1) * sizeof(uint32_t) + 4 * sizeof(ChipState));
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
    const int64_t longest = longest_cut(pb, ev);
    if (longest <= SELECT_ONE) {
        kvp_select_kernel<NB><<<dim3((unsigned)pb.n), dim3(ET), 0, s>>>(sq, moves, n_moves, old);
    } else {
        ChipScratch cs{};
        cs.rows = chunk_rows(longest);
        cs.chunks = chunk_room(longest);
        cs.state = (ChipState*)((char*)scratch + moves_bytes(pb, ev));
        cs.hist = (uint32_t*)(cs.state + 4 * pb.n);
        cs.above = cs.hist + (size_t)3 * pb.n * cs.chunks * EBINS;
        const dim3 grid((unsigned)cs.chunks, (unsigned)pb.n);
        kvp_select_chip_kernel<NB, 0><<<grid, dim3(ET), 0, s>>>(sq, cs, pb.n, moves, n_moves, old);
        kvp_select_chip_kernel<NB, 1><<<grid, dim3(ET), 0, s>>>(sq, cs, pb.n, moves, n_moves, old);
        kvp_select_chip_kernel<NB, 2><<<grid, dim3(ET), 0, s>>>(sq, cs, pb.n, moves, n_moves, old);
        kvp_select_chip_kernel<NB, 3><<<grid, dim3(ET), 0, s>>>(sq, cs, pb.n, moves, n_moves, old);
    }
    if (most > 0) kvp_move_kernel<NB><<<dim3((unsigned)std::min(most, MOVE_GROUPS), (unsigned)pb.n), dim3(256), 0, s>>>((u32x4*)pool.k, (u32x4*)pool.v, (uint32_t)pool.pages, pool.shift, sq, moves, n_moves,
                                                                                               old, Hkv, chunks);
    return hipGetLastError();
}

hipError_t launch_kvp_evict(const PagedPool& pool, const PagedBatch& pb, const PagedEvict& ev, int32_t* old, int Hkv, int d, bool bf16, void* scratch, hipStream_t s) {
    if (pb.n < 1 || pb.n > DECODE_MAX_BATCH) return hipErrorInvalidValue;
    const int chunks = d * (bf16 ? 2 : 4) / 16;
    return pb.n == 1 ? launch_kvp_evict_n<1>(pool, pb, ev, old, Hkv, chunks, scratch, s) : launch_kvp_evict_n<DECODE_MAX_BATCH>(pool, pb, ev, old, Hkv, chunks, scratch, s);
}

}  // namespace spts
