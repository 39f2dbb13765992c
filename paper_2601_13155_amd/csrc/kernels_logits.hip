// Penalties for repeated tokens, biases and masks on logits, and the token that is left on top.
#include "spts_internal.h"

#pragma clang fp contract(off)   // every product and sum of the rules is rounded on its own, as the formula reads

namespace spts {

namespace {
struct Best { float v; int i; };
constexpr int NONE = 0x7fffffff;
__device__ inline Best better(Best a, Best b) { return (b.v > a.v || (b.v == a.v && b.i < a.i)) ? b : a; }
__device__ inline Best wave_best(Best a) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) a = better(a, Best{__shfl_xor(a.v, off), __shfl_xor(a.i, off)});
    return a;
}
constexpr uint32_t IN_PROMPT = 0x80000000u;
}  // namespace

// A kernel's view of up to NB sequences' rules (few arguments make quick launches, hence one for a single sequence)
template <int NB> struct Rules {
    const int32_t* history; int64_t history_stride; const float* bias; int64_t bias_stride; const uint32_t* mask; int64_t mask_stride;
    int32_t len[NB], prompt[NB];
    float repetition[NB], frequency[NB], presence[NB];
};

// A workgroup owns 1024 LW words of one sequence: their logits, biases and mask words are asked for first, then it goes over the sequence's whole history (a few
// hundred KB at most, from the caches for all workgroups but one) and counts the ids that are its own in LDS; integers, so the order does not matter.  No
// table of counts is kept between calls or cleared in memory.  ONE: the workgroup has all words of a sequence without a history, and chooses the token itself.
constexpr int LT = 1024;
template <typename T, int LW, int NB, bool ONE>
__global__ void __launch_bounds__(LT) process_logits_kernel(const float* in, int V, Rules<NB> r, float* out, Best* __restrict__ part, int32_t* __restrict__ token,
                                                            const T* __restrict__ table, int D, T* __restrict__ x_next) {
    __shared__ uint32_t cnt[ONE ? 1 : LT * LW + LT];   // and a place for each thread that takes the ids of other words
    __shared__ Best sb[LT / 64];
    const int b = blockIdx.y, rb = NB > 1 ? b : 0, tid = threadIdx.x, v0 = (int)blockIdx.x * (LT * LW);
    const int n = V - v0 < LT * LW ? V - v0 : LT * LW;
    const int64_t row = (int64_t)b * V + v0;
    float x[LW];
#pragma unroll
    for (int j = 0; j < LW; ++j) {
        const int i = tid + j * LT;
        x[j] = i < n ? in[row + i] : 0.f;
    }
    if (!ONE && r.history) {
#pragma unroll
        for (int j = 0; j < LW; ++j) cnt[tid + j * LT] = 0;
        __syncthreads();
        const int32_t* const ids = r.history + b * r.history_stride;
        const int len = r.len[rb], prompt = r.prompt[rb];
        // Every id is an operation on LDS without a branch, ids of other words in the thread's own place; a wavefront's 256 ids of a load are as a rule all of the
        // prompt or all of the answer.  (A branch on whether the word is the workgroup's, and then on the part of the row: one sequence of 131072 ids 16.5 us, this way 14.7.)
        auto place = [&](uint32_t id) {
            const uint32_t w = id - (uint32_t)v0;
            return &cnt[w < (uint32_t)n ? w : (uint32_t)(LT * LW + tid)];
        };
        auto said = [&](uint32_t id) { atomicAdd(place(id), 1u); };
        auto given = [&](uint32_t id) { atomicOr(place(id), IN_PROMPT); };
        // whole 16-byte pieces of the row, and what is before and behind them one by one
        int head = (int)((4 - (reinterpret_cast<uintptr_t>(ids) / 4 & 3)) & 3);
        head = head < len ? head : len;
        const int quads = (len - head) / 4, tail = head + 4 * quads;
        if (tid < head) { if (tid < prompt) given((uint32_t)ids[tid]); else said((uint32_t)ids[tid]); }
        if (tid < len - tail) { if (tail + tid < prompt) given((uint32_t)ids[tail + tid]); else said((uint32_t)ids[tail + tid]); }
        const u32x4* const q = reinterpret_cast<const u32x4*>(ids + head);
        for (int i0 = tid; i0 < quads; i0 += 4 * LT) {
            u32x4 w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) w[u] = i0 + u * LT < quads ? q[i0 + u * LT] : u32x4{~0u, ~0u, ~0u, ~0u};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (i0 + u * LT >= quads) break;
                const int at = head + 4 * (i0 + u * LT), lo = __builtin_amdgcn_readfirstlane(at);
                if (lo >= prompt) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) said(w[u][e]);
                } else if (lo + 256 <= prompt) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) given(w[u][e]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) { if (at + e < prompt) given(w[u][e]); else said(w[u][e]); }
                }
            }
        }
        __syncthreads();
        const float rep = r.repetition[rb], freq = r.frequency[rb], pres = r.presence[rb];
#pragma unroll
        for (int j = 0; j < LW; ++j) {
            const uint32_t c = cnt[tid + j * LT], times = c & ~IN_PROMPT;
            if (c) x[j] = x[j] > 0.f ? x[j] / rep : x[j] * rep;
            if (times) {
                x[j] = x[j] - freq * (float)times;
                x[j] = x[j] - pres;
            }
        }
    }
    if (r.bias) {
        const float* const bias = r.bias + b * r.bias_stride + v0;
#pragma unroll
        for (int j = 0; j < LW; ++j) x[j] = x[j] + (tid + j * LT < n ? bias[tid + j * LT] : 0.f);
    }
    // Words of a mask that is not there are all ones, so that whether a word is allowed is one divergent condition.  Written as `!mask || bit`, a uniform branch around a divergent one,
    // it goes wrong in this compiler (AMD clang 22.0.0git, roc-7.2.0 26014): where both meet, the result of `allowed ? x : -inf` is copied on the uniform branch's way only, and
    // allowed words of a given mask get -inf.  The LLVM IR is right, the copy is missing in the machine code; no other kernel here selects a value by such a condition.
    uint32_t word[LW];
#pragma unroll
    for (int j = 0; j < LW; ++j) word[j] = ~0u;
    if (r.mask) {
        const uint32_t* const mask = r.mask + b * r.mask_stride + v0 / 32;   // (v0 is a multiple of 32)
#pragma unroll
        for (int j = 0; j < LW; ++j)
            if (tid + j * LT < n) word[j] = mask[(tid + j * LT) / 32];
    }
    Best best{-INFINITY, NONE};
#pragma unroll
    for (int j = 0; j < LW; ++j) {
        const int i = tid + j * LT;
        const bool allowed = i < n && (word[j] >> (i & 31) & 1u) != 0;
        x[j] = allowed ? x[j] : -INFINITY;
        if (i < n) out[row + i] = x[j];
        best = better(best, Best{x[j], allowed ? v0 + i : NONE});
    }
    if (ONE ? !token : !part) return;
    best = wave_best(best);
    if ((tid & 63) == 0) sb[tid >> 6] = best;
    __syncthreads();
    if (!ONE && tid >= 64) return;
    best = wave_best((tid & 63) < LT / 64 ? sb[tid & 63] : Best{-INFINITY, NONE});
    if (!ONE) {
        if (tid == 0) part[(int64_t)b * gridDim.x + blockIdx.x] = best;
        return;
    }
    const int tok = best.i == NONE ? -1 : best.i;
    if (tid == 0) token[b] = tok;
    if (x_next)
        for (int i = tid; i < D; i += LT) x_next[(int64_t)b * D + i] = tok < 0 ? T{} : table[(int64_t)tok * D + i];
}

template <typename T>
__global__ void __launch_bounds__(1024) pick_token_kernel(const Best* __restrict__ part, int nparts, int32_t* __restrict__ token, const T* __restrict__ table, int D,
                                                          T* __restrict__ x_next) {
    __shared__ int stok;
    const int b = blockIdx.x;
    if (threadIdx.x < 64) {
        Best best{-INFINITY, NONE};
        for (int i = threadIdx.x; i < nparts; i += 64) best = better(best, part[(int64_t)b * nparts + i]);
        best = wave_best(best);
        if (threadIdx.x == 0) {
            stok = best.i == NONE ? -1 : best.i;
            token[b] = stok;
        }
    }
    if (!x_next) return;
    __syncthreads();
    for (int i = threadIdx.x; i < D; i += blockDim.x) x_next[(int64_t)b * D + i] = stok < 0 ? T{} : table[(int64_t)stok * D + i];
}

// Words of a thread: without a history 32 where that makes one workgroup per sequence and saves the second launch (us for one sequence of 4000 / 32000 words 7.7 -> 6.7,
// 7.8 -> 7.2; with a history of 500 ids 8.1 -> 11.0, of 32768 9.7 -> 15.9), otherwise 4, so that the words are spread over the chip (16 sequences of
// 128256 words, histories of up to 32768 ids: 2 / 4 / 8 / 16 words 15.5 / 12.7 / 12.6 / 14.2; one sequence of 32768 ids 7.8 / 8.3 / 9.2 / 11.5)
constexpr int LW_ONE = 32, LW_MANY = 4;

size_t logits_scratch_bytes(int V, int nrows) { return (size_t)((V + LT * LW_MANY - 1) / (LT * LW_MANY)) * nrows * sizeof(Best); }

template <typename T, int NB>
static hipError_t launch_process_logits_n(const float* in, int V, int nrows, const LogitsRules& r, float* out, int32_t* token, const T* table, int D, T* x_next,
                                          Best* part, hipStream_t s) {
    Rules<NB> d{r.history, r.history_stride, r.bias, r.bias_stride, r.mask, r.mask_stride, {}, {}, {}, {}, {}};
    for (int b = 0; b < nrows; ++b) {
        d.len[b] = (int32_t)r.len[b]; d.prompt[b] = (int32_t)(r.prompt[b] < r.len[b] ? r.prompt[b] : r.len[b]);
        d.repetition[b] = r.repetition[b]; d.frequency[b] = r.frequency[b]; d.presence[b] = r.presence[b];
    }
    if (V <= LT * LW_ONE && !r.history) {
        process_logits_kernel<T, LW_ONE, NB, true><<<dim3(1, (unsigned)nrows), dim3(LT), 0, s>>>(in, V, d, out, nullptr, token, table, D, x_next);
        return hipGetLastError();
    }
    const int nparts = (V + LT * LW_MANY - 1) / (LT * LW_MANY);
    process_logits_kernel<T, LW_MANY, NB, false><<<dim3((unsigned)nparts, (unsigned)nrows), dim3(LT), 0, s>>>(
        in, V, d, out, token ? part : nullptr, nullptr, nullptr, 0, nullptr);
    if (token) pick_token_kernel<T><<<dim3((unsigned)nrows), dim3(x_next ? 1024 : 64), 0, s>>>(part, nparts, token, table, D, x_next);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_process_logits_t(const float* in, int V, int nrows, const LogitsRules& r, float* out, int32_t* token, const T* table, int D, T* x_next,
                                          Best* part, hipStream_t s) {
    return nrows == 1 ? launch_process_logits_n<T, 1>(in, V, nrows, r, out, token, table, D, x_next, part, s)
                      : launch_process_logits_n<T, DECODE_MAX_BATCH>(in, V, nrows, r, out, token, table, D, x_next, part, s);
}

hipError_t launch_process_logits(const float* in, int V, int nrows, const LogitsRules& r, float* out, int32_t* token, const void* table, int D,
                                 void* x_next, bool bf16, void* scratch, hipStream_t s) {
    if (nrows < 1 || nrows > DECODE_MAX_BATCH) return hipErrorInvalidValue;
    return bf16 ? launch_process_logits_t<bf16_t>(in, V, nrows, r, out, token, (const bf16_t*)table, D, (bf16_t*)x_next, (Best*)scratch, s)
                : launch_process_logits_t<float>(in, V, nrows, r, out, token, (const float*)table, D, (float*)x_next, (Best*)scratch, s);
}

}  // namespace spts
