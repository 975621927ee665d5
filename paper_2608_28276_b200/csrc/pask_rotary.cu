// pask_rotary: rotary positions.  Pair i of a token's head, (a, b), becomes m (a cos x - b sin x, b cos x + a sin x) at the angle
// x = position times frequency i (the transpose: -x).
//
// Angles.  A frequency is kept as the fraction of a turn that a position turns it by, in units of 2^-64, and its product with the
// position is taken modulo 2^64: whole turns fall away by themselves (a product in fp32 would be off by 0.03 rad at position 500
// thousand).  For any 32-bit position the product is right to 2^-34 of a turn (the table's rounding, 2^-65, times 2^31); its upper 32 bits are
// rounded by 2^-33; quarter turns are taken off in whole numbers; what is left, an eighth of a turn at most, goes to sincospi as an
// fp32 number of half turns, off by another 2^-28 of a turn.
//
// Bound: memory, each value read and written once (rot dims of 128 and 40 heads: 20 KB a token).  A CTA works out the sines and
// cosines of its tokens once, in shared memory, for all their heads; then a thread has V pairs of a head (two 16-byte loads and
// stores), the heads of all tensors of the call one behind the other.  16-byte accesses need everything aligned to them; otherwise
// a thread has one pair.  17 thousand tokens x 40 heads of 128 in bf16: 58 us, 6.0 TB/s (92 % of a copy's); 16 thousand x 33 heads of 64
// cut out of wider rows 28 us, 4.8 TB/s.  Two rows of a thread at a time took 66 and 33 us (more registers, fewer CTAs an SM).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pask_internal.h"

namespace pask {

namespace {

constexpr int kThreads = 256, kMaxPairs = kRotaryMaxDim / 2, kMaxTokens = 8;

struct RotaryParams {
    pask_rotary_tensor_t t[kRotaryMaxTensors];
    int first[kRotaryMaxTensors + 1];              // heads of the tensors before
    int n_tensors, n_tokens, tokens;               // tokens: of a CTA
    int rot, tails;                                // tails: most pieces of a head behind its rotated dims
    const int32_t *positions;
    const uint64_t *table;
    float magnitude;
    int transpose;
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }

// V values, 16 bytes of them or one
template <typename T, int V>
struct Piece {
    T x[V];
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (V > 1) *reinterpret_cast<uint4 *>(x) = *reinterpret_cast<const uint4 *>(p);
        else x[0] = *p;
    }
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (V > 1) *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(x);
        else *p = x[0];
    }
};

template <typename T>
__device__ __forceinline__ void turn(T &first, T &second, float c, float z) {
    const float f = to_f(first), s = to_f(second);
    first = from_f<T>(f * c - s * z);
    second = from_f<T>(s * c + f * z);
}

template <typename T, int V, bool kNeighbours>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const __grid_constant__ RotaryParams p) {
    __shared__ float s_cos[kMaxTokens * kMaxPairs], s_sin[kMaxTokens * kMaxPairs];
    const int tid = threadIdx.x, pairs = p.rot / 2;
    pdl_launch_dependents();
    pdl_wait();
    const int t0 = blockIdx.x * p.tokens, n = min(p.tokens, p.n_tokens - t0);
    for (int e = tid; e < n * pairs; e += kThreads) {
        const int t = e / pairs;
        const uint64_t turn = (uint64_t)(int64_t)p.positions[t0 + t] * p.table[e - t * pairs];
        const uint32_t angle = (uint32_t)((turn + 0x80000000u) >> 32), quarters = (angle + 0x20000000u) >> 30;
        float s, c;
        sincospif((float)(int32_t)(angle - (quarters << 30)) * 0x1p-31f, &s, &c);
        const float cq = quarters & 1 ? -s : c, sq = quarters & 1 ? c : s;          // a quarter on: (c, s) to (-s, c); half a turn: both change sign
        s_cos[e] = (quarters & 2 ? -cq : cq) * p.magnitude;
        s_sin[e] = (((quarters & 2) != 0) != (p.transpose != 0) ? -sq : sq) * p.magnitude;
    }
    __syncthreads();
    // A row is a head of a token; a thread has unit u of the rows r, r + rows, ...: two pieces of V dims, one of either half of the rotated
    // ones (V 1 and neighbours: a pair), or one piece of the others
    const int units = pairs / V, per_row = units + p.tails, rows = kThreads / per_row, heads = p.first[p.n_tensors];
    const int u = tid % per_row;
    int t = 0, h = tid / per_row;
    if (h >= rows) return;
    for (;; h += rows) {
        while (h >= heads) { h -= heads; t++; }
        if (t >= n) return;
        int i = 0;
        while (h >= p.first[i + 1]) i++;
        const pask_rotary_tensor_t &x = p.t[i];
        const T *in = static_cast<const T *>(x.in) + (int64_t)(t0 + t) * x.in_token_stride + (int64_t)(h - p.first[i]) * x.in_head_stride;
        T *out = static_cast<T *>(x.out) + (int64_t)(t0 + t) * x.out_token_stride + (int64_t)(h - p.first[i]) * x.out_head_stride;
        if (u >= units) {                          // not rotated: copied, unless it is there already
            const int d = p.rot + (u - units) * V;
            if (d < x.head_dim && in != out) {
                Piece<T, V> y;
                y.load(in + d);
                y.store(out + d);
            }
            continue;
        }
        const int lo = kNeighbours && V == 1 ? 2 * u : V * u, hi = kNeighbours && V == 1 ? lo + 1 : lo + pairs;
        Piece<T, V> a, b;
        a.load(in + lo);
        b.load(in + hi);
        const float *cs = s_cos + t * pairs, *sn = s_sin + t * pairs;
        if constexpr (kNeighbours && V > 1) {
#pragma unroll
            for (int e = 0; e < V; e += 2) {
                const int j = (V * u + e) / 2;
                turn(a.x[e], a.x[e + 1], cs[j], sn[j]);
                turn(b.x[e], b.x[e + 1], cs[j + pairs / 2], sn[j + pairs / 2]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; e++) turn(a.x[e], b.x[e], cs[V * u + e], sn[V * u + e]);
        }
        a.store(out + lo);
        b.store(out + hi);
    }
}

// SMs of the current device (the tensors': the caller's to set), asked for once; 0 on an error
int sm_count() {
    static int n[64] = {};
    int dev = -1, found = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    if (n[dev]) return n[dev];
    if (cudaDeviceGetAttribute(&found, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return n[dev] = found;
}

template <typename T>
cudaError_t launch(RotaryParams &p, bool neighbours, cudaStream_t stream) {
    constexpr int V = 16 / sizeof(T);
    int tail = 0;
    bool wide = p.rot % (2 * V) == 0;
    for (int i = 0; i < p.n_tensors; i++) {
        const pask_rotary_tensor_t &x = p.t[i];
        tail = x.head_dim - p.rot > tail ? x.head_dim - p.rot : tail;
        wide = wide && x.head_dim % V == 0 && (((uintptr_t)x.in | (uintptr_t)x.out) & 15) == 0 &&
               (x.in_token_stride | x.in_head_stride | x.out_token_stride | x.out_head_stride) % V == 0;
    }
    const int v = wide ? V : 1;
    p.tails = (tail + v - 1) / v;
    // Tokens a CTA: several where there are enough of them to fill the GPU all the same, so that a thread has some four rows and
    // the sines are worked out beside other CTAs' copies; one in small calls.
    const int rows = kThreads / (p.rot / 2 / v + p.tails), heads = p.first[p.n_tensors];
    const int sms = sm_count();
    if (!sms) return cudaErrorInvalidDevice;
    p.tokens = 1;
    while (p.tokens < kMaxTokens && p.tokens * heads < 4 * rows && p.n_tokens >= p.tokens * 2 * sms * 4) p.tokens *= 2;
    const dim3 grid((p.n_tokens - 1) / p.tokens + 1);                  // (n_tokens + tokens may not be an int)
    if (wide)
        return neighbours ? launch_pdl(rotary_kernel<T, V, true>, grid, dim3(kThreads), 0, stream, p)
                          : launch_pdl(rotary_kernel<T, V, false>, grid, dim3(kThreads), 0, stream, p);
    return neighbours ? launch_pdl(rotary_kernel<T, 1, true>, grid, dim3(kThreads), 0, stream, p)
                      : launch_pdl(rotary_kernel<T, 1, false>, grid, dim3(kThreads), 0, stream, p);
}

}  // namespace

pask_status_t launch_rotary(int n_tokens, const int32_t *positions, const uint64_t *table, int rot_dim, bool neighbours, bool transpose,
                            float magnitude, int dtype, int n_tensors, const pask_rotary_tensor_t *tensors, cudaStream_t stream) {
    RotaryParams p{};
    for (int i = 0; i < n_tensors; i++) {
        p.t[i] = tensors[i];
        p.first[i + 1] = p.first[i] + tensors[i].n_heads;
    }
    p.n_tensors = n_tensors;
    p.n_tokens = n_tokens;
    p.rot = rot_dim;
    p.positions = positions;
    p.table = table;
    p.magnitude = magnitude;
    p.transpose = transpose ? 1 : 0;
    const cudaError_t e = dtype == PASK_TYPE_BF16   ? launch<__nv_bfloat16>(p, neighbours, stream)
                          : dtype == PASK_TYPE_FP16 ? launch<__half>(p, neighbours, stream)
                                                    : launch<float>(p, neighbours, stream);
    return e == cudaSuccess ? PASK_OK : PASK_ERR_CUDA;
}

}  // namespace pask
