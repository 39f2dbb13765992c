// Log probabilities of given words, the entropy of their distributions and the words with the largest logits.
//
// One pass over a row with a running maximum m: s = sum e^(x - m), t = sum e^(x - m) (x - m).  Then log p(w) = (x_w - m) - log s and the entropy
// is log s - t / s; neither term is below zero, so nothing cancels.
// The row is bound by its bytes, so the largest words come out of the same pass, and every wavefront keeps a list of its own in LDS, without a barrier: after its first 1024 words it has
// a bound that `top` of them reach (the top-th largest of its lanes' maxima), and puts words above it into the list.  A list that gets long is cut by a bound from its own
// words, which is a better one, and so is a list that a row (ascending logits, say) fills.  At the end the lists' words are ranked together.  Words are ordered by
// (logit, lower id), so that equals cannot fill a list either.
// Rows are read once, by loads that do not leave them in the caches (2048 rows of 128256 words in fp32, 20 of them listed: 177 us, 6.0 TB/s; by plain loads 191).
#include "spts_lanes.h"

namespace spts {

namespace {
constexpr int PT = 256, PWV = PT / 64;      // threads
constexpr int PCAP = 512, PCUT = 256;       // places of a wavefront's list; beyond PCUT it is cut
constexpr float LOWEST = -3.402823466e38f;
constexpr float L2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// A word as one number: its logit's bits in ascending order above its id's complement, so that the larger number is the word that comes first (-0 counts as 0)
typedef uint64_t Word;
constexpr Word NOTHING = 0;   // (below every word: the bits of -inf are 0x007fffff)
__device__ inline Word word_of(float x, int id) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (Word)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~id;
}
__device__ inline float logit_of(Word w) {
    const uint32_t u = (uint32_t)(w >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ inline int id_of_word(Word w) { return (int)~(uint32_t)w; }
__device__ inline Word first_of(Word a, Word b) { return a > b ? a : b; }

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

static_assert(LOGPROBS_MAX_TOP <= 64 && LOGPROBS_MAX_TOP * (PCAP / 64) <= PCAP - 64, "a list that was cut has room for a word of every lane");

// A wavefront's list: n and bound are the same in all lanes
struct List { Word* at; int n; Word bound; };

__device__ inline Word lane_word(Word w, int lane) {
    return (Word)(uint32_t)__builtin_amdgcn_readlane((int)(w >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)w, lane);
}
// A bound from the largest word of every lane (NOTHING: none): the top-th of them, which `top` words of those that the lanes have reach; none where fewer lanes have words
__device__ inline void raise_bound(List& l, Word mx, int top) {
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < 64; ++i) rank += lane_word(mx, i) > mx ? 1 : 0;
    const uint64_t m = __ballot(rank == top - 1 && mx != NOTHING);   // (words differ, so do ranks)
    if (m) l.bound = first_of(l.bound, lane_word(mx, __builtin_ctzll(m)));
}
__device__ inline int lanes_below(uint64_t m) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u)); }
__device__ inline void push(List& l, Word w, bool yes) {
    const uint64_t m = __ballot(yes);
    if (yes) l.at[l.n + lanes_below(m)] = w;
    l.n += (int)__popcll(m);
}
// Without the words below a bound that `top` of its own reach: at most top * PCAP / 64 stay
__device__ inline void cut(List& l, int top, int lane) {
    constexpr int PER = PCAP / 64;
    Word w[PER], mx = NOTHING;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = lane + 64 * j;
        w[j] = l.at[i];   // (whole lists are read; what is behind their ends does not count)
        w[j] = i < l.n ? w[j] : NOTHING;
        mx = first_of(mx, w[j]);
    }
    raise_bound(l, mx, top);
    const int n = l.n;
    l.n = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) push(l, w[j], lane + 64 * j < n && w[j] >= l.bound);
}

// What a workgroup shares
struct ListLds {
    Word list[PWV][PCAP];
    int n[PWV];
    Sums sums[PWV];
};
// Ranks the words of all lists: put(rank, word) for the best `top`, and for the places without a word
template <typename F> __device__ inline void rank_lists(ListLds& s, List& l, int top, int tid, F put) {
    const int lane = tid & 63, wave = tid >> 6;
    if (l.n > 24) cut(l, top, lane);   // (a cut costs less than ranking against the words that it leaves out: the join of 64 parts of five words 8.1 us with a cut beyond 64, 5.4 so)
    if (lane == 0) s.n[wave] = l.n;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < PWV; ++w) total += s.n[w];
    for (int i = lane; i < l.n; i += 64) {
        const Word me = l.at[i];
        int rank = 0;
        for (int w = 0; w < PWV; ++w) {
            const int n = s.n[w];
#pragma unroll 4
            for (int o = 0; o < n; ++o) rank += s.list[w][o] > me ? 1 : 0;
        }
        if (rank < top) put(rank, me);
    }
    for (int i = total + tid; i < top; i += PT) put(i, NOTHING);
}

// Words [part * span, ..) of a row, a tile of PT * EPT at a time: pieces of up to 16 bytes at multiples of their size, of which the first begins at or before the part
template <typename T, int EPT>
__global__ void __launch_bounds__(PT, 4) logprobs_kernel(PartArgs a) {
    constexpr int C = EPT < 16 / (int)sizeof(T) ? EPT : 16 / (int)sizeof(T), U = EPT / C;
    typedef uint32_t piece __attribute__((ext_vector_type(C * sizeof(T) / 4)));
    __shared__ ListLds s;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), top = a.top;
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
                raw[u] = __builtin_nontemporal_load(reinterpret_cast<const piece*>(x + i));
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
    List l{s.list[wave], 0, NOTHING};
    piece next[U];
    load(start, next);
    for (int base = start; base < v1; base += PT * EPT) {
        float v[EPT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            union { piece p; T e[C]; } w;
            w.p = next[u];
#pragma unroll
            for (int e = 0; e < C; ++e) v[u * C + e] = to_f32(w.e[e]);
        }
        if (base < v0) {   // words before the part
#pragma unroll
            for (int e = 0; e < C; ++e) v[e] = base + tid * C + e >= v0 ? v[e] : -INFINITY;
        }
        if (base + PT * EPT < v1) load(base + PT * EPT, next);
        auto id_of = [&](int j) { return base + ((j / C) * PT + tid) * C + j % C; };
        float big = -INFINITY;
#pragma unroll
        for (int j = 0; j < EPT; ++j) big = fmaxf(big, v[j]);
        const float m = fmaxf(z.m, big);
        if (m > z.m) z = moved(z, m);
#pragma unroll
        for (int j = 0; j < EPT; ++j) {
            const float d = v[j] - m, e = exp_of(d);
            z.s += e;
            z.t = fmaf(e, fmaxf(d, -1000.f), z.t);
        }
        if (top == 0) continue;
        if (base == start) {
            Word mx = NOTHING;
#pragma unroll
            for (int j = 0; j < EPT; ++j) mx = first_of(mx, v[j] > -INFINITY ? word_of(v[j], id_of(j)) : NOTHING);
            raise_bound(l, mx, top);
        }
        float least = l.bound == NOTHING ? -INFINITY : logit_of(l.bound);   // what a word's logit has to reach
        if (__ballot(big >= least) == 0) continue;
#pragma unroll
        for (int j = 0; j < EPT; ++j) {
            if (__ballot(v[j] >= least) == 0) continue;
            const Word w = word_of(v[j], id_of(j));
            if (l.n > PCAP - 64) {
                cut(l, top, lane);
                least = logit_of(l.bound);
            }
            push(l, w, v[j] > -INFINITY && w >= l.bound);
        }
        if (l.n > PCUT) cut(l, top, lane);
    }
    // the sums of the workgroup
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) z = joined(z, Sums{__shfl_xor(z.m, off), __shfl_xor(z.s, off), __shfl_xor(z.t, off)});
    if (lane == 0) s.sums[wave] = z;
    __syncthreads();
    z = s.sums[lane % PWV];
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
    rank_lists(s, l, top, tid, [&](int rank, Word w) {
        if (a.parts > 1) a.pword[(int64_t)blockIdx.x * top + rank] = w;
        else {
            a.ids[(int64_t)row * top + rank] = w == NOTHING ? -1 : id_of_word(w);
            a.top_lp[(int64_t)row * top + rank] = w == NOTHING ? -INFINITY : (logit_of(w) - z.m) - ls;
        }
    });
}

// The parts of a row: a lane has a part's sums, and the wavefronts share the parts' words
constexpr int PPARTS = 64;
static_assert(PPARTS * LOGPROBS_MAX_TOP <= PWV * PCAP, "the words of all parts fit the lists");
template <typename T>
__global__ void __launch_bounds__(PT) logprobs_join_kernel(PartArgs a) {
    __shared__ ListLds s;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), top = a.top, n = a.parts * top;
    const int64_t row = blockIdx.x;
    Sums z = lane < a.parts ? a.psum[row * a.parts + lane] : Sums{LOWEST, 0.f, 0.f};
    List l{s.list[wave], 0, NOTHING};
    Word w[PCAP / 64];
#pragma unroll
    for (int j = 0; j < PCAP / 64; ++j) {
        const int i = tid + j * PT;
        w[j] = top ? a.pword[row * n + (i < n ? i : n - 1)] : NOTHING;
        w[j] = i < n ? w[j] : NOTHING;
    }
    float xt = 0.f;
    if (tid == 0) {
        const int32_t t = a.tokens ? a.tokens[row] : -1;
        if (t >= 0 && t < a.V) xt = word_at((const T*)a.logits + row * a.stride, t);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) z = joined(z, Sums{__shfl_xor(z.m, off), __shfl_xor(z.s, off), __shfl_xor(z.t, off)});
    if (tid == 0) finish_row(a, row, z, xt);
    if (top == 0) return;
#pragma unroll
    for (int j = 0; j < PCAP / 64; ++j) push(l, w[j], w[j] != NOTHING);
    const float ls = lse_of(z);
    rank_lists(s, l, top, tid, [&](int rank, Word best) {
        a.ids[row * top + rank] = best == NOTHING ? -1 : id_of_word(best);
        a.top_lp[row * top + rank] = best == NOTHING ? -INFINITY : (logit_of(best) - z.m) - ls;
    });
}

// Parts of a row: enough workgroups for the chip where rows are few.  Rows in parts have fewer than 2 * WANT of them in all.
constexpr int64_t WANT = 256;
static_assert(2 * WANT * (sizeof(Sums) + LOGPROBS_MAX_TOP * sizeof(Word)) + 64 <= LOGPROBS_SCRATCH_BYTES, "sums and words of all parts");
static int logprobs_parts(int64_t rows, int32_t V, int32_t* span) {
    int64_t parts = rows >= WANT ? 1 : (WANT + rows - 1) / rows;
    parts = parts > PPARTS ? PPARTS : parts;
    const int64_t least = 8 * PT;   // words of a part
    if (parts > (V + least - 1) / least) parts = (V + least - 1) / least;
    *span = (int32_t)((V + parts - 1) / parts);
    return (int)((V + *span - 1) / *span);
}

template <typename T>
static hipError_t launch_logprobs_t(const PartArgs& a, int64_t rows, hipStream_t s) {
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
    constexpr int64_t MOST = 1 << 23;   // rows of a launch, which has fewer than 2^32 threads (so many are in one part each)
    for (int64_t r = 0; r < g.rows; r += MOST) {
        PartArgs z = a;
        z.logits = (const char*)a.logits + r * a.stride * (bf16 ? 2 : 4);
        if (a.tokens) { z.tokens += r; z.logprob += r; }
        if (a.entropy) z.entropy += r;
        if (a.top > 0) { z.ids += r * a.top; z.top_lp += r * a.top; }
        const int64_t n = g.rows - r < MOST ? g.rows - r : MOST;
        const hipError_t e = bf16 ? launch_logprobs_t<bf16_t>(z, n, s) : launch_logprobs_t<float>(z, n, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace spts
