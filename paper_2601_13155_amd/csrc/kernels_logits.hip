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

// A workgroup owns LOGITS_TILE words of one sequence, four of them a thread: their logits, biases and mask words are asked for first, then it goes over the
// sequence's whole history (a few hundred KB at most, from the caches for all workgroups but one) and counts the ids that are its own in LDS; integers, so
// the order does not matter.  No table of counts is kept between calls or cleared in memory.
constexpr int LT = 1024, LW = LOGITS_TILE / LT;   // threads, words of each
__global__ void __launch_bounds__(LT) process_logits_kernel(const float* in, int V, LogitsRules r, float* out, Best* __restrict__ part) {
    __shared__ uint32_t cnt[LOGITS_TILE];
    __shared__ Best sb[LT / 64];
    const int b = blockIdx.y, tid = threadIdx.x, v0 = (int)blockIdx.x * LOGITS_TILE;
    const int n = V - v0 < LOGITS_TILE ? V - v0 : LOGITS_TILE;
    const int64_t row = (int64_t)b * V + v0;
    float x[LW], bias[LW];
    uint32_t word[LW];
#pragma unroll
    for (int j = 0; j < LW; ++j) {
        const int i = tid + j * LT;
        x[j] = i < n ? in[row + i] : 0.f;
        bias[j] = 0.f;
        word[j] = ~0u;
    }
    if (r.bias) {
#pragma unroll
        for (int j = 0; j < LW; ++j)
            if (tid + j * LT < n) bias[j] = r.bias[b * r.bias_stride + v0 + tid + j * LT];
    }
    if (r.mask) {
#pragma unroll
        for (int j = 0; j < LW; ++j)
            if (tid + j * LT < n) word[j] = r.mask[b * r.mask_stride + (uint32_t)(v0 + tid + j * LT) / 32];
    }
    if (r.history) {
#pragma unroll
        for (int j = 0; j < LW; ++j) cnt[tid + j * LT] = 0;
        __syncthreads();
        const int32_t* const ids = r.history + b * r.history_stride;
        const int len = (int)r.len[b], prompt = (int)(r.prompt[b] < len ? r.prompt[b] : len);
        auto count = [&](int32_t id, int at) {
            const uint32_t w = (uint32_t)id - (uint32_t)v0;
            if (w < (uint32_t)n) {
                if (at < prompt) atomicOr(&cnt[w], IN_PROMPT);
                else atomicAdd(&cnt[w], 1u);
            }
        };
        // whole 16-byte pieces of the row, and what is before and behind them one by one
        int head = (int)((4 - (reinterpret_cast<uintptr_t>(ids) / 4 & 3)) & 3);
        head = head < len ? head : len;
        const int quads = (len - head) / 4;
        if (tid < head) count(ids[tid], tid);
        if (tid < len - head - 4 * quads) count(ids[head + 4 * quads + tid], head + 4 * quads + tid);
        const u32x4* const q = reinterpret_cast<const u32x4*>(ids + head);
        for (int i0 = tid; i0 < quads; i0 += 4 * LT) {
            u32x4 w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) w[u] = i0 + u * LT < quads ? q[i0 + u * LT] : u32x4{~0u, ~0u, ~0u, ~0u};
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) count((int32_t)w[u][e], head + 4 * (i0 + u * LT) + e);
        }
        __syncthreads();
        const float rep = r.repetition[b], freq = r.frequency[b], pres = r.presence[b];
#pragma unroll
        for (int j = 0; j < LW; ++j) {
            const uint32_t c = cnt[tid + j * LT], said = c & ~IN_PROMPT;
            if (c) x[j] = x[j] > 0.f ? x[j] / rep : x[j] * rep;
            if (said) {
                x[j] = x[j] - freq * (float)said;
                x[j] = x[j] - pres;
            }
        }
    }
    Best best{-INFINITY, NONE};
#pragma unroll
    for (int j = 0; j < LW; ++j) {
        const int i = tid + j * LT;
        if (r.bias) x[j] = x[j] + bias[j];   // (without a bias -0 stays -0)
        const bool allowed = i < n && (word[j] >> ((v0 + i) & 31) & 1u) != 0;
        x[j] = allowed ? x[j] : -INFINITY;
        if (i < n) out[row + i] = x[j];
        best = better(best, Best{x[j], allowed ? v0 + i : NONE});
    }
    if (!part) return;
    best = wave_best(best);
    if ((tid & 63) == 0) sb[tid >> 6] = best;
    __syncthreads();
    if (tid >= 64) return;
    best = wave_best(tid < LT / 64 ? sb[tid] : Best{-INFINITY, NONE});
    if (tid == 0) part[(int64_t)b * gridDim.x + blockIdx.x] = best;
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

size_t logits_scratch_bytes(int V, int nrows) { return (size_t)((V + LOGITS_TILE - 1) / LOGITS_TILE) * nrows * sizeof(Best); }

hipError_t launch_process_logits(const float* in, int V, int nrows, const LogitsRules& r, float* out, int32_t* token, const void* table, int D,
                                 void* x_next, bool bf16, void* scratch, hipStream_t s) {
    const int nparts = (V + LOGITS_TILE - 1) / LOGITS_TILE;
    Best* part = token ? (Best*)scratch : nullptr;
    process_logits_kernel<<<dim3((unsigned)nparts, (unsigned)nrows), dim3(LT), 0, s>>>(in, V, r, out, part);
    if (token) {
        const dim3 g((unsigned)nrows), t(x_next ? 1024 : 64);
        if (bf16) pick_token_kernel<bf16_t><<<g, t, 0, s>>>(part, nparts, token, (const bf16_t*)table, D, (bf16_t*)x_next);
        else pick_token_kernel<float><<<g, t, 0, s>>>(part, nparts, token, (const float*)table, D, (float*)x_next);
    }
    return hipGetLastError();
}

}  // namespace spts
