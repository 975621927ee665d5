// Latent caches: models whose attention keeps one shared row a token (a 512-wide latent that every head expands to its own
// key and value, and 64 rotary key dims) instead of K and V per head.  The persistence path is the one of the other
// caches -- table lookup, two compacted streams, paging, budget state (Algorithm 2 steps 1, 2, 7, 8) -- with another payload.
//
//   append_latent    plan kernel of pask_append.cu, then one CTA per stream page the call writes into
//   read_latent      the two streams of a sequence as bf16 rows
//   decode_latent    attention of one new query per sequence, absorbed form
#include <cuda_bf16.h>

#include "pask_internal.h"

namespace pask {

namespace {

constexpr int kRowThreads = 288;                  // 18 groups x 16 tokens of a page
constexpr float kMinScale = 1.17549435e-38f;      // 2^-126: a smaller scale is stored as zero

template <int BITS> struct Codes;                 // levels on each side of zero; the offset that makes codes unsigned
template <> struct Codes<2> { static constexpr int kLevels = 1, kOffset = 2; };
template <> struct Codes<4> { static constexpr int kLevels = 7, kOffset = 8; };
template <> struct Codes<8> { static constexpr int kLevels = 127, kOffset = 128; };

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ uint32_t pages_touched(uint32_t old, uint32_t cnt) {
    return cnt ? ((old + cnt - 1) >> 4) - (old >> 4) + 1 : 0u;
}

// The 32 values of one group (16 bf16 pairs) -> BITS packed words and the scale's bf16 bits.
// scale = bf16(amax / levels) (zero unless a normal number), code = x / scale to the nearest integer, ties to even.
// x and scale have 8 significant bits each, so a quotient that is no tie is at least 2^-9 away from one: rounding
// x * (1 / scale) to a multiple of 2^-10 (the first addition, 1.5 * 2^13) removes the error of the reciprocal and leaves
// exact ties exact; the second addition (up to 1.5 * 2^23 + offset) rounds to the integer, ties to even.  |x / scale| is
// at most levels * (1 + 2^-8), which rounds to levels: no clamp.
template <int BITS>
__device__ __forceinline__ uint32_t quantise_group(const uint32_t (&xs)[16], uint32_t (&words)[BITS]) {
    constexpr int kLevels = Codes<BITS>::kLevels, kOffset = Codes<BITS>::kOffset;
    __nv_bfloat162 m2 = __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&xs[0]));
#pragma unroll
    for (int e = 1; e < 16; e++) m2 = __hmax2(m2, __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&xs[e])));
    const uint32_t m = *reinterpret_cast<const uint32_t *>(&m2);
    const float amax = fmaxf(bf16_lo(m), bf16_hi(m));
    __nv_bfloat16 sh = __float2bfloat16_rn(__fdiv_rn(amax, (float)kLevels));
    float s = __bfloat162float(sh);
    if (!(s >= kMinScale)) { s = 0.0f; sh = __ushort_as_bfloat16(0); }
    const float inv = s == 0.0f ? 0.0f : __fdiv_rn(1.0f, s);
    uint32_t code[32];
#pragma unroll
    for (int e = 0; e < 32; e++) {
        const float f = (e & 1) ? bf16_hi(xs[e >> 1]) : bf16_lo(xs[e >> 1]);
        const float grid = __fmaf_rn(f, inv, 12288.0f);
        code[e] = __float_as_uint(__fadd_rn(grid, 12582912.0f - 12288.0f + (float)kOffset)) & ((1u << BITS) - 1u);
    }
#pragma unroll
    for (int j = 0; j < BITS; j++) words[j] = 0;
#pragma unroll
    for (int e = 0; e < 32; e++) {
        if (BITS == 4) words[e >> 3] |= code[e] << (4 * ((e & 7) >> 1) + 16 * (e & 1));
        else if (BITS == 2) words[e >> 4] |= code[e] << ((e & 14) + 16 * (e & 1));
        else words[e >> 2] |= code[e] << (8 * (e & 3));
    }
    return (uint32_t)__bfloat16_as_ushort(sh);
}

// BITS packed words of a group and its scale -> 16 bf16 pairs: bf16((code - offset) * scale), one rounding each.
// Two- and four-bit codes: 0x4300 | code is the bf16 number 128 + code, the difference is exact and the product rounded
// once.  Eight-bit codes go through fp32 (0x4B000000 | code = 2^23 + code; the product of 7 and 8 bits is exact there).
template <int BITS>
__device__ __forceinline__ void dequantise_group(const uint32_t (&words)[BITS], uint32_t scale_bits, uint32_t (&xs)[16]) {
    constexpr int kOffset = Codes<BITS>::kOffset;
    if (BITS == 8) {
        const float s = __uint_as_float(scale_bits << 16);
#pragma unroll
        for (int p = 0; p < 16; p++) {
            const uint32_t w = words[(p >> 1) < BITS ? p >> 1 : 0];
            const float a = (__uint_as_float(__byte_perm(w, 0x4B000000u, (p & 1) ? 0x7442 : 0x7440)) - (8388608.0f + kOffset)) * s;
            const float b = (__uint_as_float(__byte_perm(w, 0x4B000000u, (p & 1) ? 0x7443 : 0x7441)) - (8388608.0f + kOffset)) * s;
            const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
            xs[p] = *reinterpret_cast<const uint32_t *>(&r);
        }
        return;
    }
    const __nv_bfloat162 s2 = __bfloat162bfloat162(__ushort_as_bfloat16((unsigned short)scale_bits));
    const __nv_bfloat162 off = __float2bfloat162_rn(128.0f + kOffset);
#pragma unroll
    for (int p = 0; p < 16; p++) {
        const uint32_t w = BITS == 4 ? words[(p >> 2) < BITS ? p >> 2 : 0] >> (4 * (p & 3)) : words[(p >> 3) < BITS ? p >> 3 : 0] >> (2 * (p & 7));
        const uint32_t v = (w & (BITS == 4 ? 0x000F000Fu : 0x00030003u)) | 0x43004300u;
        const __nv_bfloat162 r = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&v), off), s2);
        xs[p] = *reinterpret_cast<const uint32_t *>(&r);
    }
}

// the packed codes of (token, group) of a LOW page
template <int BITS>
__device__ __forceinline__ void load_codes(const uint8_t *page, int tau, int group, uint32_t (&words)[BITS]) {
    const uint8_t *p = page + latent_code_off(tau, group, BITS);
    if (BITS == 2) {
        const uint2 a = *reinterpret_cast<const uint2 *>(p);
        words[0] = a.x; words[1] = a.y;
    } else {
#pragma unroll
        for (int h = 0; h < BITS / 4; h++) {
            const uint4 a = *reinterpret_cast<const uint4 *>(p + h * kPageTokens * 16);
            words[(4 * h) % BITS] = a.x; words[(4 * h + 1) % BITS] = a.y; words[(4 * h + 2) % BITS] = a.z; words[(4 * h + 3) % BITS] = a.w;
        }
    }
}
template <int BITS>
__device__ __forceinline__ void store_codes(uint8_t *page, int tau, int group, const uint32_t (&words)[BITS], uint32_t scale_bits) {
    uint8_t *p = page + latent_code_off(tau, group, BITS);
    if (BITS == 2) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(words[0], words[1]);
    } else {
#pragma unroll
        for (int h = 0; h < BITS / 4; h++)
            *reinterpret_cast<uint4 *>(p + h * kPageTokens * 16) =
                make_uint4(words[(4 * h) % BITS], words[(4 * h + 1) % BITS], words[(4 * h + 2) % BITS], words[(4 * h + 3) % BITS]);
    }
    *reinterpret_cast<uint16_t *>(page + latent_scale_off(tau, group, BITS)) = (uint16_t)scale_bits;
}

// Second kernel of an append: a work item is a stream page the call writes into (AppendPlan, tok_list and item_base of the
// plan kernel); CTA b takes items b, b + grid, ...  A thread moves four 16-byte chunks of a HIGH page, or quantises one
// (token, group) of a LOW page.  When the call is the first to touch a page, the rows behind its last token are written
// as zeros: decode attention multiplies whole pages, and a row that has never been written could hold NaN patterns.
template <int BITS>
__global__ void __launch_bounds__(kRowThreads)
append_latent_kernel(DevCache c, int layer, int n_seqs, const uint4 *__restrict__ latent) {
    __shared__ uint32_t s_tok[kPageTokens];
    __shared__ uint32_t s_base[PASK_MAX_SEQS_PER_CALL + 1];
    if (c.ctrl[kCtrlPlanOk] == 0) return;
    const int tid = threadIdx.x;
    const uint32_t n_items = c.ctrl[kCtrlItems];
    if (blockIdx.x >= n_items) return;
    for (int x = tid; x <= n_seqs; x += kRowThreads) s_base[x] = c.item_base[x];
    __syncthreads();
    for (uint32_t item = blockIdx.x; item < n_items; item += gridDim.x) {
        int lo = 0, hi = n_seqs - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s_base[mid] <= item) lo = mid; else hi = mid - 1;
        }
        const AppendPlan p = c.plan[lo];
        const uint32_t in_seq = item - s_base[lo];
        const uint32_t items_h = pages_touched(p.old_high, p.cnt_high);
        const bool high = in_seq < items_h;
        const uint32_t old = high ? p.old_high : p.old_low, cnt = high ? p.cnt_high : p.cnt_low;
        const uint32_t pg = (old >> 4) + (high ? in_seq : in_seq - items_h);
        const uint32_t first = 16u * pg, at0 = old > first ? old - first : 0u;                 // tokens of the page: [at0, at1) written,
        const uint32_t at1 = old + cnt < first + 16u ? old + cnt - first : 16u;                 // the rest zeroed if the page is new
        const uint32_t end = at0 == 0 ? 16u : at1;
        const size_t sl = (size_t)p.seq * c.n_layers + layer;
        const uint32_t page = (high ? c.tbl_high : c.tbl_low)[sl * c.max_pages + pg];
        __syncthreads();                          // the previous item is done with s_tok
        if ((uint32_t)tid >= at0 && (uint32_t)tid < at1) {
            const uint32_t r = first + tid - old;
            s_tok[tid] = c.tok_list[high ? p.tok0 + r : p.tok1 - 1 - r];
        }
        __syncthreads();
        if (page >= (high ? c.cap_high : c.cap_low)) {   // never expected: refuse, do not write
            if (tid == 0) atomicOr(&c.ctrl[kCtrlStatus], PASK_DEV_INTERNAL);
            continue;
        }
        if (high) {
            uint8_t *dst = c.pool_high + (size_t)page * kLatentHighPageBytes;
            uint4 x[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t at = (uint32_t)(tid / kLatentChunks + 4 * i), ch = tid % kLatentChunks;
                x[i] = make_uint4(0, 0, 0, 0);
                if (at >= at0 && at < at1) x[i] = __ldcs(&latent[(size_t)s_tok[at] * kLatentChunks + ch]);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t at = (uint32_t)(tid / kLatentChunks + 4 * i), ch = tid % kLatentChunks;
                if (at >= at0 && at < end) *reinterpret_cast<uint4 *>(dst + latent_chunk_off((int)at, (int)ch)) = x[i];
            }
        } else {
            uint8_t *dst = c.pool_low + (size_t)page * c.low_page_bytes;
            const uint32_t at = tid & 15, g = tid >> 4;
            if (at >= at0 && at < end) {
                uint32_t words[BITS];
                uint32_t sb = 0;
                if (at < at1) {
                    uint32_t xs[16];
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const uint4 x = latent[(size_t)s_tok[at] * kLatentChunks + 4 * g + i];
                        xs[4 * i] = x.x; xs[4 * i + 1] = x.y; xs[4 * i + 2] = x.z; xs[4 * i + 3] = x.w;
                    }
                    sb = quantise_group<BITS>(xs, words);
                } else {
#pragma unroll
                    for (int j = 0; j < BITS; j++) words[j] = 0;
                }
                store_codes<BITS>(dst, (int)at, (int)g, words, sb);
            }
        }
    }
}

// pask_read_latent: a work item is a page of a sequence; sequence i owns items cu_rows[i] / 16 + 2 i .. (at least as many as
// it can have pages), so an item finds its sequence without a prefix over page counts.
template <int BITS>
__global__ void __launch_bounds__(kRowThreads)
read_latent_kernel(DevCache c, int layer, int n_seqs, int total_rows, const int32_t *__restrict__ seq_ids,
                   const int32_t *__restrict__ cu_rows, uint4 *__restrict__ out, int32_t *__restrict__ lens_out) {
    __shared__ __align__(16) uint8_t s_rows[kPageTokens * (kLatentDim * 2 + 16)];
    constexpr int kStride = kLatentDim * 2 + 16;
    const int tid = threadIdx.x;
    if (lens_out)
        for (int i = blockIdx.x * kRowThreads + tid; i < n_seqs; i += gridDim.x * kRowThreads) {
            const int seq = seq_ids[i];
            const bool ok = seq >= 0 && seq < c.max_seqs;
            const size_t sl = (size_t)(ok ? seq : 0) * c.n_layers + layer;
            lens_out[2 * i] = ok ? (int32_t)c.n_high[sl] : 0;
            lens_out[2 * i + 1] = ok ? (int32_t)c.n_low[sl] : 0;
        }
    const uint32_t n_items = (uint32_t)(total_rows >> 4) + 2u * (uint32_t)n_seqs;
    for (uint32_t item = blockIdx.x; item < n_items; item += gridDim.x) {
        // the sequence: the last one whose first item is not behind this one
        int cnt = 0;
        for (int x = 0; x < n_seqs; x += kRowThreads) {
            bool before = false;
            if (x + tid < n_seqs) {
                const int r = cu_rows[x + tid];
                before = (uint32_t)(max(0, min(r, total_rows)) >> 4) + 2u * (uint32_t)(x + tid) <= item;
            }
            cnt += __syncthreads_count(before);
        }
        const int i = cnt - 1;
        if (i < 0) continue;
        const int seq = seq_ids[i], r0 = cu_rows[i], r1 = cu_rows[i + 1];
        uint32_t err = 0;
        if (seq < 0 || seq >= c.max_seqs) err |= PASK_DEV_BAD_SEQ;
        if (r0 < 0 || r1 < r0 || r1 > total_rows) err |= PASK_DEV_BAD_RAGGED;
        const size_t sl = (size_t)(err ? 0 : seq) * c.n_layers + layer;
        const uint32_t nh = c.n_high[sl], nl = c.n_low[sl];
        if (!err && nh + nl > (uint32_t)(r1 - r0)) err |= PASK_DEV_BAD_RAGGED;
        if (err) {                                 // this sequence's rows are not written
            if (tid == 0) atomicOr(&c.ctrl[kCtrlStatus], err);
            continue;
        }
        const uint32_t in_seq = item - ((uint32_t)(r0 >> 4) + 2u * (uint32_t)i);
        const uint32_t ph = (nh + 15) >> 4, pl = (nl + 15) >> 4;
        if (in_seq >= ph + pl) continue;
        const bool high = in_seq < ph;
        const uint32_t pg = high ? in_seq : in_seq - ph;
        const uint32_t valid = min(16u, (high ? nh : nl) - 16u * pg);
        const uint32_t page = (high ? c.tbl_high : c.tbl_low)[sl * c.max_pages + pg];
        if (page >= (high ? c.cap_high : c.cap_low)) {
            if (tid == 0) atomicOr(&c.ctrl[kCtrlStatus], PASK_DEV_INTERNAL);
            continue;
        }
        uint4 *dst = out + (size_t)((uint32_t)r0 + (high ? 0u : nh) + 16u * pg) * kLatentChunks;
        if (high) {
            const uint8_t *src = c.pool_high + (size_t)page * kLatentHighPageBytes;
            uint4 x[4];
#pragma unroll
            for (int k = 0; k < 4; k++)
                x[k] = __ldcs(reinterpret_cast<const uint4 *>(src + latent_chunk_off(tid / kLatentChunks + 4 * k, tid % kLatentChunks)));
#pragma unroll
            for (int k = 0; k < 4; k++)
                if ((uint32_t)(tid / kLatentChunks + 4 * k) < valid) dst[tid + k * kRowThreads] = x[k];
        } else {
            const uint8_t *src = c.pool_low + (size_t)page * c.low_page_bytes;
            const int tau = tid & 15, g = tid >> 4;
            uint32_t words[BITS], xs[16];
            load_codes<BITS>(src, tau, g, words);
            dequantise_group<BITS>(words, *reinterpret_cast<const uint16_t *>(src + latent_scale_off(tau, g, BITS)), xs);
            __syncthreads();                       // the previous item has left s_rows
#pragma unroll
            for (int k = 0; k < 4; k++)
                *reinterpret_cast<uint4 *>(s_rows + tau * kStride + g * 64 + k * 16) = make_uint4(xs[4 * k], xs[4 * k + 1], xs[4 * k + 2], xs[4 * k + 3]);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const int row = tid / kLatentChunks + 4 * k;
                if ((uint32_t)row < valid) dst[tid + k * kRowThreads] = *reinterpret_cast<const uint4 *>(s_rows + row * kStride + (tid % kLatentChunks) * 16);
            }
        }
    }
}

// ---------------------------------------------------------------- decode attention

// One CTA per (query head, sequence); a warp takes every eighth row, lanes take the row's 18 groups' dims.
template <int BITS>
__global__ void __launch_bounds__(256)
decode_latent_kernel(DevCache c, int layer, const int32_t *__restrict__ seq_ids, const __nv_bfloat16 *__restrict__ q, float scale,
                     __nv_bfloat16 *__restrict__ out, float *__restrict__ lse) {
    __shared__ float s_q[kLatentDim], s_m[8], s_l[8], s_o[8][kLatentValueDim];
    const int head = blockIdx.x, i = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int seq = seq_ids[i];
    const bool ok = seq >= 0 && seq < c.max_seqs;
    if (!ok && tid == 0) atomicOr(&c.ctrl[kCtrlStatus], PASK_DEV_BAD_SEQ);
    const size_t sl = (size_t)(ok ? seq : 0) * c.n_layers + layer;
    const uint32_t nh = ok ? c.n_high[sl] : 0u, nl = ok ? c.n_low[sl] : 0u;
    for (int d = tid; d < kLatentDim; d += 256) s_q[d] = __bfloat162float(q[((size_t)i * c.n_q + head) * kLatentDim + d]) * scale;
    __syncthreads();
    float m = -INFINITY, l = 0.0f, o[16];          // lane g < 18 holds group g: its 32 dims as two halves of 16 in turn
    float o2[16];
#pragma unroll
    for (int e = 0; e < 16; e++) o[e] = o2[e] = 0.0f;
    for (uint32_t r = warp; r < nh + nl; r += 8) {
        const bool high = r < nh;
        const uint32_t at = high ? r : r - nh;
        const uint32_t page = (high ? c.tbl_high : c.tbl_low)[sl * c.max_pages + (at >> 4)];
        if (page >= (high ? c.cap_high : c.cap_low)) {
            if (lane == 0) atomicOr(&c.ctrl[kCtrlStatus], PASK_DEV_INTERNAL);
            continue;
        }
        uint32_t xs[16];
#pragma unroll
        for (int e = 0; e < 16; e++) xs[e] = 0;
        if (lane < kLatentGroups) {
            if (high) {
                const uint8_t *src = c.pool_high + (size_t)page * kLatentHighPageBytes;
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(src + latent_chunk_off((int)(at & 15), 4 * lane + k));
                    xs[4 * k] = x.x; xs[4 * k + 1] = x.y; xs[4 * k + 2] = x.z; xs[4 * k + 3] = x.w;
                }
            } else {
                const uint8_t *src = c.pool_low + (size_t)page * c.low_page_bytes;
                uint32_t words[BITS];
                load_codes<BITS>(src, (int)(at & 15), lane, words);
                dequantise_group<BITS>(words, *reinterpret_cast<const uint16_t *>(src + latent_scale_off((int)(at & 15), lane, BITS)), xs);
            }
        }
        float s = 0.0f;
        if (lane < kLatentGroups)
#pragma unroll
            for (int e = 0; e < 16; e++) s += bf16_lo(xs[e]) * s_q[32 * lane + 2 * e] + bf16_hi(xs[e]) * s_q[32 * lane + 2 * e + 1];
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        const float mn = fmaxf(m, s), a = expf(m - mn), p = expf(s - mn);
        m = mn;
        l = l * a + p;
#pragma unroll
        for (int e = 0; e < 16; e++) { o[e] = o[e] * a + p * bf16_lo(xs[e]); o2[e] = o2[e] * a + p * bf16_hi(xs[e]); }
    }
    if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
    if (lane < 16)
#pragma unroll
        for (int e = 0; e < 16; e++) { s_o[warp][32 * lane + 2 * e] = o[e]; s_o[warp][32 * lane + 2 * e + 1] = o2[e]; }
    __syncthreads();
    float mm = -INFINITY, ll = 0.0f;
    for (int w = 0; w < 8; w++) mm = fmaxf(mm, s_m[w]);
    for (int w = 0; w < 8; w++) ll += s_l[w] != 0.0f ? s_l[w] * expf(s_m[w] - mm) : 0.0f;
    for (int d = tid; d < kLatentValueDim; d += 256) {
        float acc = 0.0f;
        for (int w = 0; w < 8; w++) if (s_l[w] != 0.0f) acc += s_o[w][d] * expf(s_m[w] - mm);
        out[((size_t)i * c.n_q + head) * kLatentValueDim + d] = __float2bfloat16_rn(ll != 0.0f ? acc / ll : 0.0f);
    }
    if (tid == 0 && lse) lse[(size_t)i * c.n_q + head] = ll != 0.0f ? mm + logf(ll) : -INFINITY;
}

}  // namespace

pask_status_t launch_append_latent(pask_cache *c, int layer, int n_seqs, int total_tokens, const int32_t *seq_ids,
                                   const int32_t *cu_tokens, const void *latent, const uint8_t *tags, const uint8_t *decided,
                                   uint8_t *actions_out, cudaStream_t stream) {
    if (total_tokens == 0) return PASK_OK;
    const pask_status_t rc = launch_append_plan(c, layer, n_seqs, total_tokens, seq_ids, cu_tokens, tags, decided, actions_out, stream);
    if (rc != PASK_OK) return rc;
    // at most one item per 16 tokens plus two partly filled pages per stream
    const long long bound = (long long)total_tokens / 16 + 4LL * n_seqs;
    const int ctas = (int)(bound < (long long)c->sm_count * 6 ? bound : c->sm_count * 6);
    auto kern = c->dev.low_bits == 8 ? append_latent_kernel<8> : c->dev.low_bits == 2 ? append_latent_kernel<2> : append_latent_kernel<4>;
    kern<<<ctas, kRowThreads, 0, stream>>>(c->dev, layer, n_seqs, static_cast<const uint4 *>(latent));
    return cudaGetLastError() == cudaSuccess ? PASK_OK : PASK_ERR_CUDA;
}

pask_status_t launch_read_latent(pask_cache *c, int layer, int n_seqs, int total_rows, const int32_t *seq_ids,
                                 const int32_t *cu_rows, void *rows_out, int32_t *lens_out, cudaStream_t stream) {
    const long long items = (long long)(total_rows >> 4) + 2LL * n_seqs;
    const int ctas = (int)(items < (long long)c->sm_count * 6 ? items : c->sm_count * 6);
    auto kern = c->dev.low_bits == 8 ? read_latent_kernel<8> : c->dev.low_bits == 2 ? read_latent_kernel<2> : read_latent_kernel<4>;
    kern<<<ctas, kRowThreads, 0, stream>>>(c->dev, layer, n_seqs, total_rows, seq_ids, cu_rows, static_cast<uint4 *>(rows_out), lens_out);
    return cudaGetLastError() == cudaSuccess ? PASK_OK : PASK_ERR_CUDA;
}

size_t latent_workspace_bytes(const pask_cache *c, int n_seqs) { (void)c; (void)n_seqs; return 256; }

pask_status_t launch_decode_latent(pask_cache *c, int layer, int n_seqs, const int32_t *seq_ids, const void *q, float scale,
                                   void *out, float *lse, void *workspace, cudaStream_t stream) {
    (void)workspace;
    auto kern = c->dev.low_bits == 8 ? decode_latent_kernel<8> : c->dev.low_bits == 2 ? decode_latent_kernel<2> : decode_latent_kernel<4>;
    kern<<<dim3(c->desc.n_q_heads, n_seqs), 256, 0, stream>>>(c->dev, layer, seq_ids, static_cast<const __nv_bfloat16 *>(q), scale,
                                                              static_cast<__nv_bfloat16 *>(out), lse);
    return cudaGetLastError() == cudaSuccess ? PASK_OK : PASK_ERR_CUDA;
}

}  // namespace pask
