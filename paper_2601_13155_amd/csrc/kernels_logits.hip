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

// A workgroup owns LOGITS_TILE words of one sequence: it reads the sequence's whole history and counts those that are its own in LDS (integers: the
// order does not matter), then goes over its logits once.  Every rounding is one of fp32 (no fused multiply-add), so the result is that of the formula
// taken step by step.
__global__ void __launch_bounds__(256) process_logits_kernel(const float* in, int V, LogitsRules r, float* out, Best* __restrict__ part) {
    __shared__ uint32_t cnt[LOGITS_TILE];
    __shared__ Best sb[4];
    const int b = blockIdx.y, tid = threadIdx.x, v0 = (int)blockIdx.x * LOGITS_TILE;
    const int n = V - v0 < LOGITS_TILE ? V - v0 : LOGITS_TILE;
    if (r.history) {
        for (int i = tid; i < LOGITS_TILE; i += 256) cnt[i] = 0;
        __syncthreads();
        const int32_t* ids = r.history + b * r.history_stride;
        for (int64_t i = tid; i < r.len[b]; i += 256) {
            const uint32_t at = (uint32_t)ids[i] - (uint32_t)v0;
            if (at < (uint32_t)n) {
                if (i < r.prompt[b]) atomicOr(&cnt[at], IN_PROMPT);
                else atomicAdd(&cnt[at], 1u);
            }
        }
        __syncthreads();
    }
    Best best{-INFINITY, NONE};
    for (int i = tid; i < n; i += 256) {
        float x = in[(int64_t)b * V + v0 + i];
        if (r.history) {
            const uint32_t c = cnt[i], said = c & ~IN_PROMPT;
            if (c) x = x > 0.f ? x / r.repetition[b] : x * r.repetition[b];
            if (said) {
                x = x - r.frequency[b] * (float)said;
                x = x - r.presence[b];
            }
        }
        if (r.bias) x = x + r.bias[b * r.bias_stride + v0 + i];
        uint32_t word = ~0u;
        if (r.mask) word = r.mask[b * r.mask_stride + (uint32_t)(v0 + i) / 32];
        const bool allowed = (word >> ((v0 + i) & 31) & 1u) != 0;
        x = allowed ? x : -INFINITY;
        out[(int64_t)b * V + v0 + i] = x;
        best = better(best, Best{x, allowed ? v0 + i : NONE});
    }
    if (!part) return;
    best = wave_best(best);
    if ((tid & 63) == 0) sb[tid >> 6] = best;
    __syncthreads();
    if (tid == 0) part[(int64_t)b * gridDim.x + blockIdx.x] = better(better(sb[0], sb[1]), better(sb[2], sb[3]));
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
    for (int i = threadIdx.x; i < D; i += 1024) x_next[(int64_t)b * D + i] = stok < 0 ? T{} : table[(int64_t)stok * D + i];
}

size_t logits_scratch_bytes(int V, int nrows) { return (size_t)((V + LOGITS_TILE - 1) / LOGITS_TILE) * nrows * sizeof(Best); }

hipError_t launch_process_logits(const float* in, int V, int nrows, const LogitsRules& r, float* out, int32_t* token, const void* table, int D,
                                 void* x_next, bool bf16, void* scratch, hipStream_t s) {
    const int nparts = (V + LOGITS_TILE - 1) / LOGITS_TILE;
    Best* part = token ? (Best*)scratch : nullptr;
    process_logits_kernel<<<dim3((unsigned)nparts, (unsigned)nrows), dim3(256), 0, s>>>(in, V, r, out, part);
    if (token) {
        if (bf16) pick_token_kernel<bf16_t><<<dim3((unsigned)nrows), dim3(1024), 0, s>>>(part, nparts, token, (const bf16_t*)table, D, (bf16_t*)x_next);
        else pick_token_kernel<float><<<dim3((unsigned)nrows), dim3(1024), 0, s>>>(part, nparts, token, (const float*)table, D, (float*)x_next);
    }
    return hipGetLastError();
}

}  // namespace spts
