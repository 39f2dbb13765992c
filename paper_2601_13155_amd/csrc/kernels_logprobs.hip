// Log probabilities of given words, the entropy of their distributions and the words with the largest logits.
//
// One pass over a row with a running maximum m: s = sum e^(x - m), t = sum e^(x - m) (x - m).  Then log p(w) = (x_w - m) - log s and the entropy
// is log s - t / s; neither term is below zero, so nothing cancels.
// The row is bound by its bytes, so the largest words come out of the same pass: after the first tile of the row a bound is known that `top` words reach (the top-th largest of
// the maxima of 256 groups of the tile), and words above it are put into a list in LDS, a few hundred of 128256.  The list is cut down in the same way where a row (ascending logits, say)
// fills it, and ranked at the end.  Words are ordered by (logit, lower id), so that equals cannot fill the list either.
#include "spts_lanes.h"

namespace spts {

namespace {
constexpr int PT = 1024, PWV = PT / 64;     // threads
constexpr int PCAP = 4096;                  // places of the list
constexpr int PGROUPS = 256;
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

template <typename T> __device__ inline float word_at(const T* row, int i) { return to_f32(row[i]); }

// What a workgroup shares
struct ListLds {
    Word list[PCAP];
    Word gmax[PGROUPS];
    Word bound;
    int count;
    Sums sums[PWV];
};

// The top-th of the 256 words in gmax (LOWEST's place if there are fewer): a word that `top` words of what the groups are of reach
__device__ inline void bound_of_groups(ListLds& l, int top, int tid) {
    __syncthreads();
    if (tid < PGROUPS) {
        const Word w = l.gmax[tid];
        int rank = 0;
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
    Word w[PER], mx{-INFINITY, NOWORD - tid};   // (empty groups differ from each other)
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = tid + j * PT;
        w[j] = i < n ? l.list[i] : Word{-INFINITY, NOWORD};
        if (i < n) mx = first_of(mx, w[j]);
    }
    // groups of four threads
#pragma unroll
    for (int off = 1; off < 4; off <<= 1) mx = first_of(mx, Word{__shfl_xor(mx.x, off), __shfl_xor(mx.id, off)});
    if ((tid & 3) == 0) l.gmax[tid >> 2] = mx;
    bound_of_groups(l, top, tid);
    if (tid == 0) l.count = 0;
    __syncthreads();
    const Word bd = l.bound;
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (tid + j * PT < n && !before(bd, w[j])) l.list[atomicAdd(&l.count, 1)] = w[j];
    __syncthreads();
}

// Words [part * span, ..) of a row, a tile of PT * EPT at a time
template <typename T, int EPT>
__global__ void __launch_bounds__(PT) logprobs_kernel(PartArgs a) {
    __shared__ ListLds l;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, top = a.top;
    const int64_t row = blockIdx.x / a.parts;
    const int part = (int)(blockIdx.x % a.parts);
    const T* const x = (const T*)a.logits + row * a.stride;
    const int v0 = part * a.span, v1 = v0 + a.span < a.V ? v0 + a.span : a.V;
    Sums z{LOWEST, 0.f, 0.f};
    if (tid == 0) { l.count = 0; l.bound = Word{-INFINITY, NOWORD}; }
    __syncthreads();
    for (int base = v0; base < v1; base += PT * EPT) {
        float v[EPT];
#pragma unroll
        for (int j = 0; j < EPT; ++j) {
            const int i = base + tid + j * PT;
            v[j] = i < v1 ? word_at(x, i) : -INFINITY;
        }
        float m = z.m;
#pragma unroll
        for (int j = 0; j < EPT; ++j) m = fmaxf(m, v[j]);
        if (m > z.m) z = moved(z, m);
#pragma unroll
        for (int j = 0; j < EPT; ++j) {
            const float d = v[j] - m, e = exp_of(d);
            z.s += e;
            z.t = fmaf(e, fmaxf(d, -1000.f), z.t);
        }
        if (top == 0) continue;
        auto group_bound = [&]() {
            Word mx{-INFINITY, NOWORD - tid};
#pragma unroll
            for (int j = 0; j < EPT; ++j) mx = first_of(mx, Word{v[j], base + tid + j * PT});
#pragma unroll
            for (int off = 1; off < 4; off <<= 1) mx = first_of(mx, Word{__shfl_xor(mx.x, off), __shfl_xor(mx.id, off)});
            if ((tid & 3) == 0) l.gmax[tid >> 2] = mx;
            bound_of_groups(l, top, tid);
        };
        auto push = [&]() {
            const Word bd = l.bound;
#pragma unroll
            for (int j = 0; j < EPT; ++j) {
                const Word w{v[j], base + tid + j * PT};
                if (w.x > -INFINITY && !before(bd, w)) {
                    const int at = atomicAdd(&l.count, 1);
                    if (at < PCAP) l.list[at] = w;
                }
            }
            __syncthreads();
        };
        if (base == v0) group_bound();
        const int had = l.count;
        __syncthreads();
        push();
        if (l.count > PCAP) {   // more than the list holds: a bound from this tile, and the list as it was before it cut by it
            __syncthreads();
            if (tid == 0) l.count = had;
            group_bound();
            cut_list(l, top, tid);
            push();
        }
        __syncthreads();
    }
    // the sums of the workgroup
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) z = joined(z, Sums{__shfl_xor(z.m, off), __shfl_xor(z.s, off), __shfl_xor(z.t, off)});
    if (lane == 0) l.sums[wave] = z;
    __syncthreads();
    z = l.sums[0];
    for (int w = 1; w < PWV; ++w) z = joined(z, l.sums[w]);
    if (tid == 0) {
        if (a.parts > 1) a.psum[blockIdx.x] = z;
        else {
            const int32_t w = a.tokens ? a.tokens[row] : -1;
            finish_row(a, row, z, w >= 0 && w < a.V ? word_at(x, w) : 0.f);
        }
    }
    if (top == 0) return;
    if (l.count > PGROUPS) cut_list(l, top, tid);
    const int n = l.count;
    const float ls = lse_of(z);
    for (int i = tid; i < n || i < top; i += PT) {
        int rank = i;
        Word w{-INFINITY, NOWORD};
        if (i < n) {
            w = l.list[i];
            rank = 0;
            for (int o = 0; o < n; ++o) rank += before(l.list[o], w) ? 1 : 0;
        }
        if (rank >= top) continue;
        if (a.parts > 1) a.pword[(int64_t)blockIdx.x * top + rank] = w;
        else {
            a.ids[row * top + rank] = i < n ? w.id : -1;
            a.top_lp[row * top + rank] = i < n ? (w.x - z.m) - ls : -INFINITY;
        }
    }
}

// The parts of a row: one workgroup of a wavefront's multiple per row; parts * top words are ranked in LDS
constexpr int PPARTS = 64;
template <typename T>
__global__ void __launch_bounds__(256) logprobs_join_kernel(PartArgs a) {
    __shared__ Word w[PPARTS * LOGPROBS_MAX_TOP];
    const int tid = threadIdx.x, top = a.top, n = a.parts * top;
    const int64_t row = blockIdx.x;
    Sums z = a.psum[row * a.parts];
    for (int p = 1; p < a.parts; ++p) z = joined(z, a.psum[row * a.parts + p]);
    if (tid == 0) {
        const int32_t t = a.tokens ? a.tokens[row] : -1;
        finish_row(a, row, z, t >= 0 && t < a.V ? word_at((const T*)a.logits + row * a.stride, t) : 0.f);
    }
    if (top == 0) return;
    for (int i = tid; i < n; i += 256) w[i] = a.pword[row * n + i];
    __syncthreads();
    const float ls = lse_of(z);
    for (int i = tid; i < n; i += 256) {
        const Word me = w[i];
        int rank = 0;
        for (int o = 0; o < n; ++o) rank += before(w[o], me) || (o < i && !before(me, w[o])) ? 1 : 0;   // (places without a word are equal)
        if (rank >= top) continue;
        a.ids[row * top + rank] = me.id == NOWORD ? -1 : me.id;
        a.top_lp[row * top + rank] = me.id == NOWORD ? -INFINITY : (me.x - z.m) - ls;
    }
}

// Parts of a row: enough workgroups for the chip where rows are few
static int logprobs_parts(int64_t rows, int32_t V, int32_t* span) {
    constexpr int64_t WANT = 256;
    int64_t parts = rows >= WANT ? 1 : (WANT + rows - 1) / rows;
    parts = parts > PPARTS ? PPARTS : parts;
    const int64_t least = 4 * PT;   // words of a part
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
    if (a.span <= 4 * PT) logprobs_kernel<T, 4><<<grid, dim3(PT), 0, s>>>(a);
    else logprobs_kernel<T, 16><<<grid, dim3(PT), 0, s>>>(a);
    if (a.parts > 1) logprobs_join_kernel<T><<<dim3((unsigned)rows), dim3(256), 0, s>>>(a);
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
