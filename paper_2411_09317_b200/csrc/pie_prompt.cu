// Causal attention over whole prompts, packed one after the other (Section 2.1: the prefill stage computes all prompt tokens at
// once): keys and values as the projection left them, nothing cached before them.
//
// One warp per (token, query head): a lane holds head_dim / 32 elements of the query and of the output, the scores are
// summed across the lanes, and one pass over the keys carries the running maximum and sum of the softmax.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "../../include/pie.h"
#include "pie_kernels.h"

namespace pie {

namespace {

template <bool BF16>
__device__ __forceinline__ float pr_load(const uint16_t *x) {
    return BF16 ? __uint_as_float((uint32_t)*x << 16) : __half2float(__ushort_as_half(*x));
}

template <int D, bool BF16>
__global__ void __launch_bounds__(256)
prompt_attn_kernel(const PromptLaunch a, int32_t n_q_heads, int32_t n_kv_heads) {
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t t = row / n_q_heads;
    if (t >= a.n_tokens) return;
    const int h = (int)(row - t * n_q_heads), kvh = h / (n_q_heads / n_kv_heads);
    int32_t lo = 0, hi = a.n_seqs;   // largest s with offsets[s] <= t
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (a.offsets[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int64_t t0 = a.offsets[lo];
    const uint16_t *q = (const uint16_t *)a.q + t * a.q_stride + (int64_t)h * D;
    float x[D / 32], o[D / 32], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        x[i] = pr_load<BF16>(q + 32 * i + lane);
        o[i] = 0.f;
    }
    for (int64_t j = t0; j <= t; ++j) {
        const uint16_t *k = (const uint16_t *)a.k + j * a.k_stride + (int64_t)kvh * D, *v = (const uint16_t *)a.v + j * a.v_stride + (int64_t)kvh * D;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) s += x[i] * pr_load<BF16>(k + 32 * i + lane);
#pragma unroll
        for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        s *= a.scale * 1.4426950408889634f;
        const float mn = fmaxf(m, s), f = m == -INFINITY ? 0.f : exp2f(m - mn), e = mn == -INFINITY ? 0.f : exp2f(s - mn);
        m = mn;
        l = l * f + e;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) o[i] = o[i] * f + e * pr_load<BF16>(v + 32 * i + lane);
    }
    uint16_t *out = (uint16_t *)a.out + (t * n_q_heads + h) * D;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const float r = o[i] / l;
        out[32 * i + lane] = BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(r)) : __half_as_ushort(__float2half_rn(r));
    }
}

}  // namespace

cudaError_t launch_prompt_attention(const AttnShape &sh, const PromptLaunch &a, cudaStream_t stream) {
    if (a.n_tokens <= 0) return cudaSuccess;
    const unsigned grid = (unsigned)((a.n_tokens * sh.n_q_heads + 7) / 8);
    if (sh.dtype == PIE_BF16) {
        if (sh.head_dim == 128) prompt_attn_kernel<128, true><<<grid, 256, 0, stream>>>(a, sh.n_q_heads, sh.n_kv_heads);
        else prompt_attn_kernel<64, true><<<grid, 256, 0, stream>>>(a, sh.n_q_heads, sh.n_kv_heads);
    } else {
        if (sh.head_dim == 128) prompt_attn_kernel<128, false><<<grid, 256, 0, stream>>>(a, sh.n_q_heads, sh.n_kv_heads);
        else prompt_attn_kernel<64, false><<<grid, 256, 0, stream>>>(a, sh.n_q_heads, sh.n_kv_heads);
    }
    return cudaGetLastError();
}

}  // namespace pie
