// Log probabilities of given words, the entropy of their distributions and the words with the largest logits.
//
// One pass over a row with a running maximum m: s = sum e^(x - m), t = sum e^(x - m) (x - m).  Then log p(w) = (x_w - m) - log s and the entropy
// is log s - t / s; neither term is below zero, so nothing cancels.
// The row is bound by its bytes, so the largest words come out of the same pass: after the first tile of the row a bound is known that `top` words reach (the top-th largest of
// the maxima of 64 groups of the tile), and words above it are put into a list in LDS, some 200 of 128256 for top = 20.  Where a row (ascending logits, say) fills the list, it is cut down in
// the same way, by a bound from its own groups; at the end the words that are left are ranked.  Words are ordered by (logit, lower id), so that equals cannot fill the list either.
#include "spts_lanes.h"

namespace spts {

namespace {
constexpr int PT = 256, PWV = PT / 64;      // threads
constexpr int PCAP = 2048, PCUT = 512;      // places of the list; it is cut beyond PCUT words, for the better bound
constexpr int PGROUPS = 64;                 // of PT / 64 threads
constexpr float LOWEST = -3.402823466e38f;
constexpr float L2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int NOWORD = 0x7fffffff;

struct Word { float x; int id; };
__device__ inline bool before(Word a, Word b) { return a.x > b.x || (a.x == b.x && a.id < b.id); }
__device__ inline Word first_of(Word a, Word b) { return before(b, a) ? b : a; }

struct Sums { float m, s, t; };
// e^d for d <= 0
__device__ inline float exp_of(float d) { return __builtin_amdgcn_exp2f(d * L2E); }
// sums relative to a larger maximum (the clamps keep 0 * inf away: e^-1000 is 0)
__device__ inline Sums moved(Sums a, float m) {
    const float d = fmaxf(a.m - m, -1000.f), f = exp_of(d);
    return Sums{m, a.s * f, f * (a.t + d * a.s)};
}
__device__ inline Sums joined(Sums a, Sums b) {
    const float m = fmaxf(a.m, b.m);
    a = moved(a, m);
    b = moved(b, m);
    return Sums{m, a.s + b.s, a.t + b.t};
}

struct PartArgs {
    const void* logits; int64_t stride; int32_t V, span, parts, top; const int32_t* tokens; float* logprob; float* entropy; int32_t* ids; float* top_lp;
    Sums* psum; Word* pword;
};

__device__ inline float lse_of(Sums a) { return logf(a.s); }   // relative to m; -inf where no word is above -inf
__device__ inline void finish_row(const PartArgs& a, int64_t row, Sums z, float xt) {
    if (a.entropy) a.entropy[row] = z.s == 0.f ? 0.f : lse_of(z) - z.t / z.s;
    if (a.logprob) {
        const int32_t w = a.tokens[row];
        a.logprob[row] = w < 0 || w >= a.V ? __uint_as_float(0x7fc00000u) : z.s == 0.f ? -INFINITY : (xt - z.m) - lse_of(z);
    }
}
}  // namespace

template <typename T> __device__ inline float word_at(const T* row, int64_t i) { return to_f32(row[i]); }

// What a workgroup shares
struct ListLds {
    Word list[PCAP];
    Word gmax[PGROUPS];
    Word bound;
    int count;
    Sums sums[PWV];
};
static_assert(LOGPROBS_MAX_TOP <= PGROUPS && LOGPROBS_MAX_TOP * (PCAP / PGROUPS) + LOGPROBS_MAX_TOP * (4 * PT / PGROUPS) <= PCAP, "a list that was cut takes four words of every thread");

// The bound from the largest word of every thread: the top-th of the 64 groups' (groups are neighbouring threads), which `top` words of those that the threads have reach
__device__ inline void bound_of(ListLds& l, Word mx, int top, int tid) {
    constexpr int PER = PT / PGROUPS;
#pragma unroll
    for (int off = 1; off < PER; off <<= 1) mx = first_of(mx, Word{__shfl_xor(mx.x, off), __shfl_xor(mx.id, off)});
    if (tid % PER == 0) l.gmax[tid / PER] = mx;
    __syncthreads();
    if (tid < PGROUPS) {
        const Word w = l.gmax[tid];
        int rank = 0;
#pragma unroll 8
        for (int i = 0; i < PGROUPS; ++i) rank += before(l.gmax[i], w) ? 1 : 0;
        if (rank == top - 1) l.bound = first_of(l.bound, w);
    }
    __syncthreads();
}

// The list without the words below a bound that `top` of its own reach: at most top * PCAP / PGROUPS words stay
__device__ inline void cut_list(ListLds& l, int top, int tid) {
    __syncthreads();
    const int n = l.count;
    constexpr int PER = PCAP / PT;
    Word w[PER], mx{-INFINITY, NOWORD - tid};   // (groups without a word differ from each other)
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = tid + j * PT;
        w[j] = i < n ? l.list[i] : Word{-INFINITY, NOWORD};
        if (i < n) mx = first_of(mx, w[j]);
    }
    bound_of(l, mx, top, tid);
    if (tid == 0) l.count = 0;
    __syncthreads();
    const Word bd = l.bound;
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (tid + j * PT < n && !before(bd, w[j])) l.list[atomicAdd(&l.count, 1)] = w[j];
    __syncthreads();
}

// Ranks the words of the list: put(rank, word) for the best `top`, and for the places without a word
template <typename F> __device__ inline void rank_list(ListLds& l, int top, int tid, F put) {
    if (l.count > PGROUPS) cut_list(l, top, tid);
    const int n = l.count;
    for (int i = tid; i < n || i < top; i += PT) {
        if (i >= n) { put(i, Word{-INFINITY, NOWORD}); continue; }
        const Word w = l.list[i];
        int rank = 0;
#pragma unroll 4
        for (int o = 0; o < n; ++o) rank += before(l.list[o], w) ? 1 : 0;
        if (rank < top) put(rank, w);
    }
}

// Words [part * span, ..) of a row, a tile of PT * EPT at a time: pieces of up to 16 bytes at multiples of their size, of which the first begins at or before the part
template <typename T, int EPT>
__global__ void __launch_bounds__(PT) logprobs_kernel(PartArgs a) {
    constexpr int C = EPT < 16 / (int)sizeof(T) ? EPT : 16 / (int)sizeof(T), U = EPT / C;
    typedef uint32_t piece __attribute__((ext_vector_type(C * sizeof(T) / 4)));
    __shared__ ListLds l;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, top = a.top;
    const uint32_t row = blockIdx.x / (uint32_t)a.parts;
    const int part = (int)(blockIdx.x - row * (uint32_t)a.parts);
    const T* const x = (const T*)a.logits + row * a.stride;
    const int v0 = part * a.span, v1 = v0 + a.span < a.V ? v0 + a.span : a.V;
    const int start = v0 - (int)((reinterpret_cast<uintptr_t>(x + v0) / sizeof(T)) % C);
    auto load = [&](int base, piece (&raw)[U]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + (u * PT + tid) * C;
            if (i + C <= v1) {   // (the first piece may begin up to 15 bytes before the row, behind the one before it)
                raw[u] = *reinterpret_cast<const piece*>(x + i);
            } else {
                union { piece p; T e[C]; } z;
#pragma unroll
                for (int e = 0; e < C; ++e) {
                    z.e[e] = from_f32<T>(-INFINITY);
                    if (i + e < v1) z.e[e] = x[i + e];
                }
                raw[u] = z.p;
            }
        }
    };
    Sums z{LOWEST, 0.f, 0.f};
    if (tid == 0) { l.count = 0; l.bound = Word{-INFINITY, NOWORD}; }
    __syncthreads();
    piece next[U];
    load(start, next);
    for (int base = start; base < v1; base += PT * EPT) {
        float v[EPT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            union { piece p; T e[C]; } w;
            w.p = next[u];
#pragma unroll
            for (int e = 0; e < C; ++e) v[u * C + e] = base + (u * PT + tid) * C + e >= v0 ? to_f32(w.e[e]) : -INFINITY;
        }
        if (base + PT * EPT < v1) load(base + PT * EPT, next);
        auto id_of = [&](int j) { return base + ((j / C) * PT + tid) * C + j % C; };
        float m = z.m, big = -INFINITY;
#pragma unroll
        for (int j = 0; j < EPT; ++j) big = fmaxf(big, v[j]);
        m = fmaxf(m, big);
        if (m > z.m) z = moved(z, m);
#pragma unroll
        for (int j = 0; j < EPT; ++j) {
            const float d = v[j] - m, e = exp_of(d);
            z.s += e;
            z.t = fmaf(e, fmaxf(d, -1000.f), z.t);
        }
        if (top == 0) continue;
        auto largest = [&](int j0, int n) {
            Word mx{-INFINITY, NOWORD - tid};
#pragma unroll
            for (int j = 0; j < EPT; ++j)
                if (j >= j0 && j < j0 + n) mx = first_of(mx, Word{v[j], id_of(j)});
            return mx;
        };
        auto push = [&](int j0, int n) {
            const Word bd = l.bound;
            if (big >= bd.x) {
#pragma unroll
                for (int j = 0; j < EPT; ++j) {
                    const Word w{v[j], id_of(j)};
                    if (j >= j0 && j < j0 + n && w.x > -INFINITY && !before(bd, w)) {
                        const int at = atomicAdd(&l.count, 1);
                        if (at < PCAP) l.list[at] = w;
                    }
                }
            }
            __syncthreads();
        };
        if (base == start) bound_of(l, largest(0, EPT), top, tid);
        const int had = l.count;
        __syncthreads();
        push(0, EPT);
        if (l.count > PCAP) {   // more than the list holds: it is as before this tile again, and takes four words of every thread at a time, cut before by bounds from them and from itself
            __syncthreads();
            if (tid == 0) l.count = had;
            for (int j0 = 0; j0 < EPT; j0 += 4) {
                Word mx = largest(j0, 4);
                bound_of(l, mx, top, tid);
                cut_list(l, top, tid);
                push(j0, 4);
            }
        } else if (l.count > PCUT) {
            cut_list(l, top, tid);
        }
    }
    // the sums of the workgroup
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) z = joined(z, Sums{__shfl_xor(z.m, off), __shfl_xor(z.s, off), __shfl_xor(z.t, off)});
    if (lane == 0) l.sums[wave] = z;
    __syncthreads();
    z = l.sums[lane % PWV];
#pragma unroll
    for (int off = PWV / 2; off > 0; off >>= 1) z = joined(z, Sums{__shfl_xor(z.m, off), __shfl_xor(z.s, off), __shfl_xor(z.t, off)});
    if (tid == 0) {
        if (a.parts > 1) a.psum[blockIdx.x] = z;
        else {
            const int32_t w = a.tokens ? a.tokens[row] : -1;
            finish_row(a, row, z, w >= 0 && w < a.V ? word_at(x, w) : 0.f);
        }
    }
    if (top == 0) return;
    const float ls = lse_of(z);
    rank_list(l, top, tid, [&](int rank, Word w) {
        if (a.parts > 1) a.pword[(int64_t)blockIdx.x * top + rank] = w;
        else {
            a.ids[(int64_t)row * top + rank] = w.id == NOWORD ? -1 : w.id;
            a.top_lp[(int64_t)row * top + rank] = w.id == NOWORD ? -INFINITY : (w.x - z.m) - ls;
        }
    });
}

// The parts of a row: a lane has a part's sums, and the parts' words are a list
constexpr int PPARTS = 64;
static_assert(PPARTS * LOGPROBS_MAX_TOP <= PCAP, "the words of all parts fit the list");
template <typename T>
__global__ void __launch_bounds__(PT) logprobs_join_kernel(PartArgs a) {
    __shared__ ListLds l;
    const int tid = threadIdx.x, lane = tid & 63, top = a.top, n = a.parts * top;
    const int64_t row = blockIdx.x;
    Sums z = lane < a.parts ? a.psum[row * a.parts + lane] : Sums{LOWEST, 0.f, 0.f};
    float xt = 0.f;
    if (tid == 0) {
        const int32_t t = a.tokens ? a.tokens[row] : -1;
        if (t >= 0 && t < a.V) xt = word_at((const T*)a.logits + row * a.stride, t);
        l.count = 0;
        l.bound = Word{-INFINITY, NOWORD};
    }
    __syncthreads();
    for (int i = tid; i < n; i += PT) {
        const Word w = a.pword[row * n + i];
        if (w.id != NOWORD) l.list[atomicAdd(&l.count, 1)] = w;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) z = joined(z, Sums{__shfl_xor(z.m, off), __shfl_xor(z.s, off), __shfl_xor(z.t, off)});
    if (tid == 0) finish_row(a, row, z, xt);
    if (top == 0) return;
    __syncthreads();
    const float ls = lse_of(z);
    rank_list(l, top, tid, [&](int rank, Word w) {
        a.ids[row * top + rank] = w.id == NOWORD ? -1 : w.id;
        a.top_lp[row * top + rank] = w.id == NOWORD ? -INFINITY : (w.x - z.m) - ls;
    });
}

// Parts of a row: enough workgroups for the chip where rows are few
static int logprobs_parts(int64_t rows, int32_t V, int32_t* span) {
    constexpr int64_t WANT = 256;
    int64_t parts = rows >= WANT ? 1 : (WANT + rows - 1) / rows;
    parts = parts > PPARTS ? PPARTS : parts;
    const int64_t least = 8 * PT;   // words of a part
    if (parts > (V + least - 1) / least) parts = (V + least - 1) / least;
    *span = (int32_t)((V + parts - 1) / parts);
    return (int)((V + *span - 1) / *span);
}

size_t logprobs_scratch_bytes(int64_t rows, int32_t V, int32_t top) {
    int32_t span;
    const int parts = logprobs_parts(rows, V, &span);
    return parts == 1 ? 0 : (size_t)rows * parts * (sizeof(Sums) + top * sizeof(Word)) + 64;
}

template <typename T>
static hipError_t launch_logprobs_t(const PartArgs& a, int64_t rows, hipStream_t s) {
    if (rows * a.parts > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(rows * a.parts));
    if (a.span <= 8 * PT) logprobs_kernel<T, 8><<<grid, dim3(PT), 0, s>>>(a);
    else logprobs_kernel<T, 16><<<grid, dim3(PT), 0, s>>>(a);
    if (a.parts > 1) logprobs_join_kernel<T><<<dim3((unsigned)rows), dim3(a.top > 0 ? PT : 64), 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_token_logprobs(const LogprobArgs& g, bool bf16, void* scratch, hipStream_t s) {
    if (g.rows < 1 || g.V < 1 || g.top < 0 || g.top > LOGPROBS_MAX_TOP) return hipErrorInvalidValue;
    PartArgs a{g.logits, g.stride, g.V, 0, 1, g.top, g.tokens, g.logprob, g.entropy, g.ids, g.top_lp, nullptr, nullptr};
    a.parts = logprobs_parts(g.rows, g.V, &a.span);
    a.psum = (Sums*)scratch;
    a.pword = (Word*)((char*)scratch + ((size_t)g.rows * a.parts * sizeof(Sums) + 15) / 16 * 16);
    return bf16 ? launch_logprobs_t<bf16_t>(a, g.rows, s) : launch_logprobs_t<float>(a, g.rows, s);
}

}  // namespace spts
