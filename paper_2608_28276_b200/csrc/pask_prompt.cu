// pask_prompt_attention_latent: causal attention of a ragged batch of prompts (or prompt chunks behind a history) with the
// latent rows expanded to keys and values per head.
#include <cuda_bf16.h>

#include "pask_internal.h"

namespace pask {

namespace {

constexpr int kNope = 128, kRope = 64, kQk = kNope + kRope, kV = 128;

// One warp per (query, head): lanes hold 6 query dims and 4 output dims.
__global__ void __launch_bounds__(256)
prompt_latent_kernel(int n_seqs, int total_q, int total_k, int n_heads, const int32_t *__restrict__ cu_q, const int32_t *__restrict__ cu_k,
                     const __nv_bfloat16 *__restrict__ q, const __nv_bfloat16 *__restrict__ kv, const __nv_bfloat16 *__restrict__ rope,
                     int rope_stride, float scale, __nv_bfloat16 *__restrict__ out, float *__restrict__ lse) {
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= (long long)total_q * n_heads) return;
    const int t = (int)(row / n_heads), head = (int)(row % n_heads);
    int i = -1;
    for (int s = 0; s < n_seqs; s++) if (t >= cu_q[s] && t < cu_q[s + 1]) { i = s; break; }
    if (i < 0 || cu_q[i] < 0 || cu_q[i + 1] > total_q || cu_k[i] < 0 || cu_k[i + 1] < cu_k[i] || cu_k[i + 1] > total_k) return;
    const int nq = cu_q[i + 1] - cu_q[i], nk = cu_k[i + 1] - cu_k[i], k0 = cu_k[i];
    const int visible = min(nk, t - cu_q[i] + nk - nq + 1);
    float qv[6], m = -INFINITY, l = 0.0f, o[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 6; e++) qv[e] = __bfloat162float(q[row * kQk + 32 * e + lane]) * scale;
    for (int j = 0; j < visible; j++) {
        const __nv_bfloat16 *kr = kv + ((size_t)(k0 + j) * n_heads + head) * (kNope + kV), *rr = rope + (size_t)(k0 + j) * rope_stride;
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; e++) s += qv[e] * __bfloat162float(kr[32 * e + lane]);
#pragma unroll
        for (int e = 0; e < 2; e++) s += qv[4 + e] * __bfloat162float(rr[32 * e + lane]);
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        const float mn = fmaxf(m, s), a = expf(m - mn), p = expf(s - mn);
        m = mn;
        l = l * a + p;
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] = o[e] * a + p * __bfloat162float(kr[kNope + 32 * e + lane]);
    }
#pragma unroll
    for (int e = 0; e < 4; e++) out[row * kV + 32 * e + lane] = __float2bfloat16_rn(visible > 0 ? o[e] / l : 0.0f);
    if (lane == 0 && lse) lse[row] = visible > 0 ? m + logf(l) : -INFINITY;
}

}  // namespace

pask_status_t launch_prompt_latent(int n_seqs, int total_q, int total_k, int n_heads, const int32_t *cu_q, const int32_t *cu_k,
                                   const void *q, const void *kv, const void *k_rope, int rope_stride, float scale, void *out,
                                   float *lse, cudaStream_t stream) {
    const long long ctas = ((long long)total_q * n_heads + 7) / 8;
    if (ctas > 0x7fffffffLL) return PASK_ERR_INVALID_ARG;
    prompt_latent_kernel<<<(int)ctas, 256, 0, stream>>>(n_seqs, total_q, total_k, n_heads, cu_q, cu_k, static_cast<const __nv_bfloat16 *>(q),
                                                        static_cast<const __nv_bfloat16 *>(kv), static_cast<const __nv_bfloat16 *>(k_rope),
                                                        rope_stride, scale, static_cast<__nv_bfloat16 *>(out), lse);
    return cudaGetLastError() == cudaSuccess ? PASK_OK : PASK_ERR_CUDA;
}

}  // namespace pask
