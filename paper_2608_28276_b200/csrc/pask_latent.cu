// Latent caches: models whose attention keeps one shared row a token (a 512-wide latent that every head expands to its own
// key and value, and 64 rotary key dims) instead of K and V per head.  The persistence path is the one of the other
// caches -- table lookup, two compacted streams, paging, budget state (Algorithm 2 steps 1, 2, 7, 8) -- with another payload.
//
//   append_latent    plan kernel of pask_append.cu, then one CTA per stream page the call writes into
//   read_latent      the two streams of a sequence as bf16 rows
//   decode_latent    attention of one new query per sequence, absorbed form
#include <cuda_bf16.h>

#include <cstddef>

#include "pask_internal.h"
#include "pask_latent.h"
#include "pask_umma.h"

namespace pask {

namespace {

constexpr int kRowThreads = 288;                  // 18 groups x 16 tokens of a page
constexpr int kReadCtas = 6;                      // CTAs of the read-back an SM has at a time
__device__ __forceinline__ uint32_t pages_touched(uint32_t old, uint32_t cnt) {
    return cnt ? ((old + cnt - 1) >> 4) - (old >> 4) + 1 : 0u;
}

// Second kernel of a bulk append: a work item is a stream page the call writes into (AppendPlan, tok_list and item_base of the
// plan kernel); a CTA takes consecutive items, so that plan, table and token list are mostly at hand, and looks up the next
// item's page and tokens while the rows of the current one are on their way.  A thread moves four 16-byte chunks of a HIGH
// page, or quantises one (token, group) of a LOW page.  When the call is the first to touch a page, the rows behind its last
// token are written as zeros: decode attention multiplies whole pages, and a row that has never been written could hold
// NaN patterns.  Bound by memory: 326 K tokens, a quarter HIGH, 0.4 LOW at 4 bits, 77 us behind the plan's 20 (383 MB: 5.0 TB/s;
// five CTAs an SM and the look-ahead hide the table and list lookups: 85 us with three).
template <int BITS>
__global__ void __launch_bounds__(kRowThreads, 5)
append_latent_kernel(DevCache c, int layer, int n_seqs, const uint4 *__restrict__ latent) {
    __shared__ uint32_t s_tok[2][kPageTokens];
    __shared__ uint32_t s_base[PASK_MAX_SEQS_PER_CALL + 1];
    __shared__ uint32_t s_items;
    const int tid = threadIdx.x;
    if (tid == 0) s_items = c.ctrl[kCtrlPlanOk] ? c.ctrl[kCtrlItems] : 0u;
    __syncthreads();
    const uint32_t n_items = s_items;
    const uint32_t item0 = (uint32_t)((uint64_t)n_items * blockIdx.x / gridDim.x), item1 = (uint32_t)((uint64_t)n_items * (blockIdx.x + 1) / gridDim.x);
    if (item0 >= item1) return;
    for (int x = tid; x <= n_seqs; x += kRowThreads) s_base[x] = c.item_base[x];
    __syncthreads();
    int j = 0;
    for (int hi = n_seqs - 1; j < hi;) {
        const int mid = (j + hi + 1) >> 1;
        if (s_base[mid] <= item0) j = mid; else hi = mid - 1;
    }
    AppendPlan p = c.plan[j];
    struct Page { bool high; uint32_t at0, at1, id; } now, then;
    uint32_t tok = 0;
    auto look_up = [&](uint32_t item, Page &g) {
        bool moved = false;
        while (j + 1 < n_seqs && item >= s_base[j + 1]) { j++; moved = true; }
        if (moved) p = c.plan[j];
        const uint32_t in_seq = item - s_base[j], items_h = pages_touched(p.old_high, p.cnt_high);
        g.high = in_seq < items_h;
        const uint32_t old = g.high ? p.old_high : p.old_low, cnt = g.high ? p.cnt_high : p.cnt_low;
        const uint32_t pg = (old >> 4) + (g.high ? in_seq : in_seq - items_h), first = 16u * pg;
        g.at0 = old > first ? old - first : 0u;                    // tokens [at0, at1) of the page are written, the rest zeroed if it is new
        g.at1 = min(old + cnt - first, 16u);
        g.id = (g.high ? c.tbl_high : c.tbl_low)[((size_t)p.seq * c.n_layers + layer) * c.max_pages + pg];
        if ((uint32_t)tid >= g.at0 && (uint32_t)tid < g.at1) {
            const uint32_t r = first + tid - old;
            tok = c.tok_list[g.high ? p.tok0 + r : p.tok1 - 1 - r];
        }
    };
    look_up(item0, now);
    for (uint32_t item = item0; item < item1; item++) {
        uint32_t *toks = s_tok[item & 1];
        if (tid < kPageTokens) toks[tid] = tok;
        __syncthreads();                           // (two buffers: nobody still reads the one before last)
        const uint32_t at0 = now.at0, at1 = now.at1, end = at0 == 0 ? 16u : at1;
        const bool fits = now.id < (now.high ? c.cap_high : c.cap_low);          // never expected not to: refuse, do not write
        if (!fits && tid == 0) atomicOr(&c.ctrl[kCtrlStatus], PASK_DEV_INTERNAL);
        if (now.high) {
            uint8_t *dst = c.pool_high + (size_t)now.id * kLatentHighPageBytes;
            uint4 x[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t at = (uint32_t)(tid / kLatentChunks + 4 * i), ch = tid % kLatentChunks;
                x[i] = make_uint4(0, 0, 0, 0);
                if (at >= at0 && at < at1) x[i] = __ldcs(&latent[(size_t)toks[at] * kLatentChunks + ch]);
            }
            if (item + 1 < item1) look_up(item + 1, then);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t at = (uint32_t)(tid / kLatentChunks + 4 * i), ch = tid % kLatentChunks;
                if (fits && at >= at0 && at < end) *reinterpret_cast<uint4 *>(dst + latent_chunk_off((int)at, (int)ch)) = x[i];
            }
        } else {
            uint8_t *dst = c.pool_low + (size_t)now.id * c.low_page_bytes;
            const uint32_t at = tid & 15, g = tid >> 4;
            uint32_t xs[16], words[BITS], sb = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (at >= at0 && at < at1) x = latent[(size_t)toks[at] * kLatentChunks + 4 * g + i];
                xs[4 * i] = x.x; xs[4 * i + 1] = x.y; xs[4 * i + 2] = x.z; xs[4 * i + 3] = x.w;
            }
            if (item + 1 < item1) look_up(item + 1, then);
            if (at < at1) {
                sb = quantise_group<BITS>(xs, words);
            } else {
#pragma unroll
                for (int i = 0; i < BITS; i++) words[i] = 0;
            }
            if (fits && at >= at0 && at < end) store_codes<BITS>(dst, (int)at, (int)g, words, sb);
        }
        now = then;
    }
}

// pask_read_latent: a work item is a page of a sequence.  Every CTA first counts the pages of the sequences that have a range to
// go to (a prefix over the batch, a sequence a thread) and then finds an item's sequence in it: the order of the ranges, and
// what a malformed one says, does not come into it.  Bound by memory: 213 K rows of the same batch in 67 us (382 MB: 5.7 TB/s).
template <int BITS>
__global__ void __launch_bounds__(kRowThreads, kReadCtas)
read_latent_kernel(DevCache c, int layer, int n_seqs, int total_rows, const int32_t *__restrict__ seq_ids,
                   const int32_t *__restrict__ cu_rows, uint4 *__restrict__ out, int32_t *__restrict__ lens_out) {
    __shared__ __align__(16) uint8_t s_rows[kPageTokens * (kLatentDim * 2 + 16)];
    __shared__ uint32_t s_base[PASK_MAX_SEQS_PER_CALL], s_warp[kRowThreads / 32];
    constexpr int kStride = kLatentDim * 2 + 16;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t n_items = 0;
    for (int x = 0; x < n_seqs; x += kRowThreads) {
        const int i = x + tid;
        uint32_t pages = 0;
        if (i < n_seqs) {
            const int seq = seq_ids[i], r0 = cu_rows[i], r1 = cu_rows[i + 1];
            uint32_t err = 0, nh = 0, nl = 0;
            if (seq < 0 || seq >= c.max_seqs) {
                err = PASK_DEV_BAD_SEQ;
            } else {
                const size_t sl = (size_t)seq * c.n_layers + layer;
                nh = c.n_high[sl];
                nl = c.n_low[sl];
            }
            if (r0 < 0 || r1 < r0 || r1 > total_rows || nh + nl > (uint32_t)(r1 - r0)) err |= PASK_DEV_BAD_RAGGED;
            if (!err) pages = ((nh + 15) >> 4) + ((nl + 15) >> 4);
            if (blockIdx.x == 0) {
                if (err) atomicOr(&c.ctrl[kCtrlStatus], err);      // this sequence's rows are not written
                if (lens_out) {
                    lens_out[2 * i] = (int32_t)nh;
                    lens_out[2 * i + 1] = (int32_t)nl;
                }
            }
        }
        uint32_t inc = pages;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, inc, d);
            if (lane >= d) inc += o;
        }
        if (x > 0) __syncthreads();                // s_warp has been read
        if (lane == 31) s_warp[warp] = inc;
        __syncthreads();
        uint32_t base = n_items + inc - pages;
#pragma unroll
        for (int w = 0; w < kRowThreads / 32; w++) {
            if (w < warp) base += s_warp[w];
            n_items += s_warp[w];
        }
        if (i < n_seqs) s_base[i] = base;
    }
    __syncthreads();
    for (uint32_t item = blockIdx.x; item < n_items; item += gridDim.x) {
        int i = 0;                                 // the last sequence that does not begin behind the item (its pages: the item's)
        for (int hi = n_seqs - 1; i < hi;) {
            const int mid = (i + hi + 1) >> 1;
            if (s_base[mid] <= item) i = mid; else hi = mid - 1;
        }
        const uint32_t r0 = (uint32_t)cu_rows[i], in_seq = item - s_base[i];
        const size_t sl = (size_t)seq_ids[i] * c.n_layers + layer;
        const uint32_t nh = c.n_high[sl], nl = c.n_low[sl], ph = (nh + 15) >> 4, pl = (nl + 15) >> 4;
        if (in_seq >= ph + pl) continue;           // (more than 2^32 pages: ranges that overlap many times over)
        const bool high = in_seq < ph;
        const uint32_t pg = high ? in_seq : in_seq - ph;
        const uint32_t valid = min(16u, (high ? nh : nl) - 16u * pg);
        const uint32_t page = (high ? c.tbl_high : c.tbl_low)[sl * c.max_pages + pg];
        if (page >= (high ? c.cap_high : c.cap_low)) {
            if (tid == 0) atomicOr(&c.ctrl[kCtrlStatus], PASK_DEV_INTERNAL);
            continue;
        }
        uint4 *dst = out + (size_t)(r0 + (high ? 0u : nh) + 16u * pg) * kLatentChunks;
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
//
// out_h = sum_j softmax_j(scale q_h . x_j) x_j[0:512] over a sequence's rows x_j (576 values): every head reads every row, so a
// row is fetched once and used as key and value by all heads -- 2 n_q (576 + 512) operations for 1152 bytes, 121 (n_q = 64)
// or 242 (n_q = 128) a byte, around the ratio of the tensor core's rate to the memory's.  Matrix products, then, on tcgen05:
//
//   S^T [64 tokens x heads] = X Q^T       X K-major from shared memory (M = 64), Q K-major (N = heads)
//   O^T [512 dims x heads] += X^T P^T     X MN-major, the very same bytes (M = 128, four blocks), P [token][head] MN-major
//
// Rows on the M side and heads on the N side: a CTA takes up to 64 heads (kHeads = 16, 32 or 64, the next size up) and the
// accumulators of all 512 value dims fit tensor memory (4 x 64 columns, beside two S tiles).  More than 64 heads are split
// over that many CTAs that walk the same tiles side by side and find each other's rows in L2.
//
// A CTA is one of `slots` equal shares of the batch's tiles: 64 rows = four pages of one stream, a sequence's HIGH and LOW tiles
// visited in turn, evenly mixed.  (A LOW tile is a quarter of the bytes but as much work on chip: 2.5 us against 2.0
// at 32 heads, so a tile counts as a tile.)  Roles:
//   warp 13     HIGH tiles: one linear bulk copy a page (pages are stored in the operand layout) into its place in one of two
//               stages, as soon as the product that last read the place is done, and a prefetch into L2 some tiles ahead
//   warps 4-12  LOW tiles: a thread takes one (token, group) of each page, codes in registers one tile ahead, values as bf16 into
//               the stage; and the queries of a sequence.  (The loop over pages is rolled, its codes move up a place instead:
//               straight-line code for a whole tile waited for its instructions, 18 % a tile.)
//   warp 14     the products for S, two tiles ahead at most;  warp 15  those for O.  (One warp for both had to poll: waiting on a
//               barrier wakes it 70 cycles after the arrival, polling two of them sees it after 150 to 350.)
//   warps 0-3   softmax of a tile's S (warp w: page w of the tile), P to shared memory, and a sequence's end
// The reference maximum of a head moves only when a score exceeds it by more than 2^8 (the sums have room for that), so that
// the rescaling of O leaves the common path.  A share that covers a whole sequence writes its result; otherwise partial sums
// go to the workspace and decode_latent_merge joins them in a fixed order: results do not depend on timing.
//
// Rounding: S is fp32; a weight is rounded to bf16 once, as an operand of the product with bf16 rows (its sum is taken before),
// which is off by half a step at most, 2^-8 of each weight, as the rounding of the result is.  A second product with what the
// rounding left would add 768 cycles to the 1920 of a tile's products.
//
// HIGH tiles are bound by memory up to 32 heads (148 sequences of 2048 rows, 16 / 32 heads, the captured call replayed back to back,
// merge included: 64 / 69 us, 5.5 / 5.1 TB/s; the call alone, L2 flushed: 81 / 85).  At 64 heads (82 us replayed; 128 heads in two
// groups 148) some 4500 cycles a tile are the chain copy - S - softmax - O over two stages of a whole tile and one place for P;
// shared memory's own bandwidth accounts for 2555 of them (327 KB a tile: copy, X twice, Q, P; 128 B a cycle).  LOW tiles are
// bound by the fill, 2.2 us for 16 heads and 3.0 for 64: of 4070 cycles the codes' requests take 1250, four pages 2030.  Replayed /
// called: 64 sequences of 2 to 8 thousand rows, 128 heads, all HIGH 159 / 175 us; 128 of 16 thousand tokens, 64 heads, a fifth HIGH
// and 0.3 LOW at 4 bits 260 / 281; one of 1023 rows, 16 heads 12.4 / 11.4.
constexpr int kTile = 64, kTilePages = 4;
constexpr int kTileBytes = kTilePages * kLatentHighPageBytes;      // 73728
constexpr int kDecThreads = 512, kFillThreads = kPageTokens * kLatentGroups;      // 288: nine warps
constexpr uint32_t kMaxSlots = 1024;
// first, last tile of a sequence's part; the part is the whole sequence; last tile of the share; the sequence began in an earlier one
enum : uint32_t { kInfoFirst = 1, kInfoLast = 2, kInfoWhole = 4, kInfoFinal = 8, kInfoGoesOn = 16 };
constexpr float kLazy = 8.0f;                      // log2 of how far a score may exceed the reference maximum

struct DecParams {
    DevCache c;
    int layer, n_seqs, groups, heads;              // groups of `heads` heads each (the last one may have fewer)
    uint32_t slots;
    const int32_t *seq_ids;
    const uint4 *q;
    float scale_log2;
    __nv_bfloat16 *out;
    float *lse;
    uint4 *meta;                                   // [n_seqs] {tiles before it, its tiles, first share, end of its shares}
    // A share leaves at most two partial results, those of its first sequence (if that began in an earlier share) and of its
    // last: part 2 share, and 2 share + 1.
    float2 *part_ml;                               // [2 slots][n_q] (reference maximum in log2 units, sum)
    float *part_o;                                 // [2 slots][n_q][512]
    long long wait_cycles;
    uint32_t surplus;
    unsigned long long *span;
};

__device__ __forceinline__ uint32_t tiles_of(uint32_t tokens) { return (tokens + kTile - 1) / kTile; }
// floor(a b / c), in 32 bits where the product fits (a 64-bit division is some 200 cycles of the set-up)
__device__ __forceinline__ uint32_t mul_div(uint32_t a, uint32_t b, uint32_t c) {
    const uint64_t x = (uint64_t)a * b;
    return (x >> 32) == 0 ? (uint32_t)x / c : (uint32_t)(x / c);
}
// share b of `slots` is tiles [start(b), start(b + 1)) of all
__device__ __forceinline__ uint32_t slot_start(uint32_t total, uint32_t slot, uint32_t slots) { return mul_div(total, slot, slots); }

// The tiles of one share, in order; the roles walk their own copies.
struct TileWalk {
    const DevCache *c;
    const int32_t *seq_ids;
    int layer, n_seqs, s;
    uint32_t lo, hi, base;                         // the share; tiles of the sequences before s
    uint32_t nh, nl, th, n, v, v0, v1;             // rows of the streams; HIGH tiles, tiles, position and range of it
    uint32_t h0, rem;                              // v * th = h0 * n + rem (page_at of pask_layout.h without its divisions)
    size_t sl;

    __device__ __forceinline__ void enter(uint32_t high_rows, uint32_t low_rows) {
        nh = high_rows;
        nl = low_rows;
        th = tiles_of(nh);
        n = th + tiles_of(nl);
        v = v0 = lo > base ? lo - base : 0u;
        v1 = min(n, hi - base);
        h0 = rem = 0;
        if (v0) {
            h0 = mul_div(v0, th, n);
            rem = (uint32_t)((uint64_t)v0 * th - (uint64_t)h0 * n);
        }
    }
    __device__ __forceinline__ bool settle() {     // on to a sequence with tiles in the share
        while (v >= v1) {
            base += n;
            if (++s >= n_seqs || base >= hi) return false;
            const int seq = seq_ids[s];
            const bool ok = seq >= 0 && seq < c->max_seqs;
            sl = (size_t)(ok ? seq : 0) * c->n_layers + layer;
            enter(ok ? c->n_high[sl] : 0u, ok ? c->n_low[sl] : 0u);
        }
        return true;
    }
    __device__ __forceinline__ bool next() {
        v++;
        rem += th;
        if (rem >= n) { rem -= n; h0++; }
        return v < v1 || settle();
    }
    __device__ __forceinline__ bool high() const { return rem + th >= n; }
    __device__ __forceinline__ uint32_t tile() const { return high() ? h0 : v - h0; }
    __device__ __forceinline__ uint32_t valid() const { return min((uint32_t)kTile, (high() ? nh : nl) - kTile * tile()); }
    __device__ __forceinline__ uint32_t pages() const { return (valid() + kPageTokens - 1) / kPageTokens; }
    __device__ __forceinline__ bool first() const { return v == v0; }
    __device__ __forceinline__ bool last() const { return v + 1 == v1; }
    __device__ __forceinline__ bool goes_on() const { return v0 > 0; }
    __device__ __forceinline__ bool whole() const { return v0 == 0 && v1 == n; }
    // where the tile's page p lies, from its id (read a tile before it is looked at); an id the pools cannot hold is never
    // dereferenced
    __device__ __forceinline__ uint32_t page_id(uint32_t p) const {
        return p < pages() ? (high() ? c->tbl_high : c->tbl_low)[sl * c->max_pages + kTilePages * tile() + p] : 0u;
    }
    __device__ __forceinline__ uint32_t page_bytes() const { return high() ? (uint32_t)kLatentHighPageBytes : c->low_page_bytes; }
    __device__ __forceinline__ const uint8_t *page(uint32_t id) const {
        if (id >= (high() ? c->cap_high : c->cap_low)) {
            if (pages()) atomicOr(&c->ctrl[kCtrlStatus], PASK_DEV_INTERNAL);
            id = 0;
        }
        return (high() ? c->pool_high : c->pool_low) + (size_t)id * page_bytes();
    }
};

template <int kHeads>
struct DecSmem {
    static constexpr int kQ = 2 * kTileBytes, kP = kQ + kHeads * 1152, kMisc = kP + kTile * 128;
    struct Misc {
        uint64_t full[2], empty[2][2], s_full[2], s_empty[2], q_full, q_empty, q_first, p_full, p_empty, o_free, drain[2];
        uint4 info[2];                             // of the tile whose S a stage holds: valid rows, flags, sequence
        uint32_t tmem;
        int first;                                 // the sequence of the share's first tile: index, tiles before it, rows, place
        uint32_t first_base, first_high, first_low;
        size_t first_sl;
        uint32_t warp_sum[kDecThreads / 32];
        alignas(16) float red[4][kHeads];
        alignas(16) float fac[kHeads], mref[kHeads];           // read in pairs
    };
    static_assert(offsetof(Misc, fac) % 8 == 0 && offsetof(Misc, mref) % 8 == 0 && offsetof(Misc, info) % 16 == 0 && kMisc % 16 == 0, "vector loads");
    static constexpr int kBytes = kMisc + (int)sizeof(Misc) + 1024;
};

template <int kHeads, int BITS>
__global__ void __launch_bounds__(kDecThreads, 1)
decode_latent_kernel(const __grid_constant__ DecParams p) {
    using namespace umma;
    using Sm = DecSmem<kHeads>;
    extern __shared__ uint8_t s_raw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>(((uintptr_t)s_raw + 1023) & ~(uintptr_t)1023);
    typename Sm::Misc &ms = *reinterpret_cast<typename Sm::Misc *>(sm + Sm::kMisc);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t slot = blockIdx.x / p.groups, group = blockIdx.x % p.groups;
    const int h0 = (int)group * p.heads, nh_here = min(p.heads, p.c.n_q - h0);       // this CTA's query heads
    if (tid == 0) {
        for (int i = 0; i < 2; i++) {
            bar_init(smem_u32(&ms.full[i]), 2 + kFillThreads / 32);
            bar_init(smem_u32(&ms.empty[i][0]), 1);
            bar_init(smem_u32(&ms.empty[i][1]), 1);
            bar_init(smem_u32(&ms.s_full[i]), 2);
            bar_init(smem_u32(&ms.s_empty[i]), 4);
            bar_init(smem_u32(&ms.drain[i]), 1);
        }
        bar_init(smem_u32(&ms.q_full), kFillThreads / 32);
        bar_init(smem_u32(&ms.q_empty), 1);
        bar_init(smem_u32(&ms.q_first), kFillThreads / 32);    // completes once, with the first queries
        bar_init(smem_u32(&ms.p_full), 4);
        bar_init(smem_u32(&ms.p_empty), 1);
        bar_init(smem_u32(&ms.o_free), 4);
        bar_init_fence();
    }
    pdl_launch_dependents();
    pdl_wait();
    unsigned long long t_start = 0;
    if (p.span && tid == 0) asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t_start));

    // ---- the share: prefix of tiles over the sequences (1024 at most, kPer a thread)
    constexpr int kPer = (PASK_MAX_SEQS_PER_CALL + kDecThreads - 1) / kDecThreads;
    uint32_t nh[kPer], nl[kPer], tiles[kPer], sum = 0;
    size_t sl[kPer];
#pragma unroll
    for (int r = 0; r < kPer; r++) {
        const int s = tid * kPer + r;
        nh[r] = nl[r] = 0;
        sl[r] = 0;
        if (s < p.n_seqs) {
            const int seq = p.seq_ids[s];
            if (seq >= 0 && seq < p.c.max_seqs) {
                sl[r] = (size_t)seq * p.c.n_layers + p.layer;
                nh[r] = p.c.n_high[sl[r]];
                nl[r] = p.c.n_low[sl[r]];
            } else if (blockIdx.x == 0) {
                atomicOr(&p.c.ctrl[kCtrlStatus], PASK_DEV_BAD_SEQ);
            }
        }
        tiles[r] = tiles_of(nh[r]) + tiles_of(nl[r]);
        sum += tiles[r];
    }
    uint32_t inc = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, inc, d);
        if (lane >= d) inc += o;
    }
    if (lane == 31) ms.warp_sum[warp] = inc;
    __syncthreads();
    uint32_t at = inc - sum, total = 0;
#pragma unroll
    for (int w = 0; w < kDecThreads / 32; w++) {
        if (w < warp) at += ms.warp_sum[w];
        total += ms.warp_sum[w];
    }
    const uint32_t slots = min(total, p.slots);    // no more shares than tiles
    const uint32_t lo = slot < slots ? slot_start(total, slot, slots) : 0u, hi = slot < slots ? slot_start(total, slot + 1, slots) : 0u;
    uint32_t base = at;
#pragma unroll
    for (int r = 0; r < kPer; r++) {
        if (base <= lo && lo < base + tiles[r] && lo < hi) {
            ms.first = tid * kPer + r;
            ms.first_base = base;
            ms.first_high = nh[r];
            ms.first_low = nl[r];
            ms.first_sl = sl[r];
        }
        base += tiles[r];
    }
    if (blockIdx.x == 0) {                         // what the merge needs to know
        base = at;
#pragma unroll
        for (int r = 0; r < kPer; r++) {
            const int s = tid * kPer + r;
            if (s < p.n_seqs) {
                uint32_t b0 = 0, b1 = 0;
                if (tiles[r]) {                    // shares [b0, b1): the one its first tile is in .. the one its last is in
                    b0 = mul_div(base, slots, total);
                    while (slot_start(total, b0 + 1, slots) <= base) b0++;
                    b1 = mul_div(base + tiles[r] - 1, slots, total) + 1;
                    while (slot_start(total, b1, slots) < base + tiles[r]) b1++;
                }
                p.meta[s] = make_uint4(base, tiles[r], b0, b1);
            }
            base += tiles[r];
        }
    }
    if (lo >= hi) return;                          // nothing for this CTA
    if (warp == 14) tmem_alloc(smem_u32(&ms.tmem), 512);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = ms.tmem;
    constexpr uint32_t kO = 128;                   // columns: S tiles at 0 and 64, O blocks from 128
    const uint32_t kv0 = smem_u32(sm), qs = smem_u32(sm + Sm::kQ), ps = smem_u32(sm + Sm::kP);
    const long long limit = p.wait_cycles;
    TileWalk w;
    w.c = &p.c; w.seq_ids = p.seq_ids; w.layer = p.layer; w.n_seqs = p.n_seqs;
    w.lo = lo; w.hi = hi; w.s = ms.first; w.base = ms.first_base; w.sl = ms.first_sl;
    w.enter(ms.first_high, ms.first_low);
    bool more = true, ok = true;

    if (warp == 13) {
        // ================================================= copies
        // (page ids are read an iteration before they are used: the read's way to L2 would otherwise sit between a freed
        // place and the copy into it)
        uint32_t i = 0, id = more ? w.page_id(lane) : 0u, ahead_id = 0, copied = 0, phase[2] = {0, 0};
        TileWalk ahead = w;
        bool ahead_more = more;
        // Tiles between a prefetch into L2 and the copy.  What is on its way may not crowd itself out: 4 x 148 tiles (43 MB) in all
        // of the 126 MB, whose halves may both hold a line.  One group, all HIGH, 148 sequences of 2048 rows, 16 / 64 heads: 83 /
        // 100 us with six tiles, 66 / 87 with two, 68 / 90 with one; two groups share their tiles: six 3 % before two.
        const int look_ahead = 4 * p.groups - 2;
        for (; more; i++) {
            const uint32_t st = i & 1, np = w.pages();
            const bool high = w.high();
            const uint8_t *src = high && (uint32_t)lane < np ? w.page(id) : nullptr;
            more = w.next();
            if (more) id = w.page_id(lane);
            const uint32_t full = smem_u32(&ms.full[st]), extra = i == 0 ? p.surplus : 0u;
            const uint32_t dst = kv0 + st * kTileBytes + lane * kLatentHighPageBytes;
#pragma unroll
            for (int half = 0; half < 2; half++) {            // two pages at a time: a copy's way through the issue is long
                // (both producers wait for every tile's stage and report to its barrier, whoever fills it: a phase's parity only
                // tells it from its neighbours, so nobody may fall two phases behind)
                ok = ok && (i < 2 || bar_wait(smem_u32(&ms.empty[st][half]), ((i >> 1) - 1) & 1, limit));
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (!high) {
                    if (lane == 0) bar_arrive(full);
                    continue;
                }
                const uint32_t here = np > 2u * half ? min(2u, np - 2u * half) : 0u;      // pages of this half
                if (lane == 0) bar_expect(full, here * kLatentHighPageBytes + (half == 0 ? extra : 0u));
                __syncwarp();
                if ((lane >> 1) == half && (uint32_t)lane < np) bulk_load(dst, src, kLatentHighPageBytes, full);
                copied |= 1u << st;
                if (st) phase[1] = (i >> 1) & 1; else phase[0] = (i >> 1) & 1;
            }
            if (!ok) break;
            if (i == 0) {
                for (int k = 0; k < look_ahead; k++) ahead_more = ahead_more && ahead.next();
                if (ahead_more) ahead_id = ahead.page_id(lane);
                continue;
            }
            if (i == 1) {                          // the first queries go before rows that are not needed yet
                ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&ms.q_first), 0, limit));
                if (!ok) break;
            }
            if (ahead_more) {
                if ((uint32_t)lane < ahead.pages()) bulk_prefetch(ahead.page(ahead_id), ahead.page_bytes());
                ahead_more = ahead.next();
                if (ahead_more) ahead_id = ahead.page_id(lane);
            }
        }
        if (!ok || p.surplus) {                    // gave up: let the copies in flight land (bounded) before the CTA ends
            if (copied & 1u) bar_wait(smem_u32(&ms.full[0]), phase[0], limit);
            if (copied & 2u) bar_wait(smem_u32(&ms.full[1]), phase[1], limit);
        }
    } else if (warp == 14) {
        // ================================================= products for S
        constexpr uint32_t kIdS = instr(kTile, kHeads, false, false);
        const bool mine = elect_one();
        uint32_t n_seg = 0;
        TileWalk wn = w;                           // one tile ahead of w, moved on behind the products: nothing waits for its loads
        bool after = more && wn.next();
        for (uint32_t i = 0; more; i++) {
            const uint32_t st = __shfl_sync(0xffffffffu, i & 1, 0), ph = (i >> 1) & 1;
            const bool is_first = w.first(), is_last = w.last();
            if (is_first) ok = bar_wait(smem_u32(&ms.q_full), n_seg++ & 1, limit);
            if (i >= 2) ok = ok && bar_wait(smem_u32(&ms.s_empty[st]), ph ^ 1, limit);
            ok = ok && bar_wait(smem_u32(&ms.full[st]), ph, limit);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            fence_after();
            const uint64_t dk = desc(kv0 + st * kTileBytes, 0, kLatentHalfPage), dq = desc(qs, 0, kLatentHalfPage);
#pragma unroll
            for (int k = 0; k < kLatentDim / 16; k++) {
                const uint64_t off = (uint64_t)(((k >> 2) * 1024 + (k & 3) * 32) >> 4);
                mma_ss(tmem + st * 64, dk + off, dq + off, kIdS, k > 0, mine);
            }
            if (mine) {
                commit(smem_u32(&ms.s_full[st]));
                if (is_last) commit(smem_u32(&ms.q_empty));
                const uint32_t flags = (is_first ? kInfoFirst : 0u) | (is_last ? kInfoLast : 0u) | (w.whole() ? kInfoWhole : 0u) |
                                       (w.goes_on() ? kInfoGoesOn : 0u);
                ms.info[st] = make_uint4(w.valid(), flags | (after ? 0u : kInfoFinal), (uint32_t)w.s, 0);
                bar_arrive(smem_u32(&ms.s_full[st]));
            }
            more = after;
            if (more) {
                w = wn;
                after = wn.next();
            }
        }
        if (!ok) {                                 // gave up: the products in flight end before tensor memory is freed
            if (mine) commit(smem_u32(&ms.drain[0]));
            bar_wait(smem_u32(&ms.drain[0]), 0, limit);
        }
        __syncwarp();
    } else if (warp == 15) {
        // ================================================= products for O
        constexpr uint32_t kIdO = instr(128, kHeads, true, true);
        const bool mine = elect_one();
        uint32_t n_seg = 0;
        for (uint32_t i = 0; more; i++) {
            const uint32_t st = __shfl_sync(0xffffffffu, i & 1, 0), np = __shfl_sync(0xffffffffu, w.pages(), 0);
            const bool fresh = __shfl_sync(0xffffffffu, (int)w.first(), 0) != 0;
            // (the segment before has been read out of O)
            if (fresh && n_seg++ > 0) ok = bar_wait(smem_u32(&ms.o_free), (n_seg - 2) & 1, limit);
            ok = ok && bar_wait(smem_u32(&ms.p_full), i & 1, limit);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            fence_after();
            const uint64_t dv = desc(kv0 + st * kTileBytes, 1024, kLatentHalfPage), dp = desc(ps, 0, 1024);
#pragma unroll
            for (int k = 0; k < kTilePages; k++) {
                if ((uint32_t)k < np) {
#pragma unroll
                    for (int b = 0; b < 4; b++)
                        mma_ss(tmem + kO + b * 64, dv + (uint64_t)((k * kLatentHighPageBytes + b * 2048) >> 4), dp + (uint64_t)(k * 2048 >> 4),
                               kIdO, k > 0 || !fresh, mine);
                }
                if ((k & 1) && mine) commit(smem_u32(&ms.empty[st][k >> 1]));
            }
            if (mine) commit(smem_u32(&ms.p_empty));
            more = w.next();
        }
        if (!ok) {
            if (mine) commit(smem_u32(&ms.drain[1]));
            bar_wait(smem_u32(&ms.drain[1]), 0, limit);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ================================================= queries and LOW tiles
        const int t = tid - 128, tau = t & 15, g = t >> 4;     // token and group of every page
        uint32_t codes[kTilePages][BITS], scales[kTilePages], ids[kTilePages];
        TileWalk ahead = w;                        // codes: of the next LOW tile; ahead, ids: the one behind it
        auto to_low = [&](bool here) { while (here && ahead.high()) here = ahead.next(); return here; };
        // (no branch around the loads, pages that are not there read their last neighbour's: a load under a condition was waited
        // for where the paths join, 2500 cycles a tile)
        auto fetch_ids = [&]() {
            const uint32_t *tbl = p.c.tbl_low + ahead.sl * p.c.max_pages + kTilePages * ahead.tile();
            const uint32_t last = ahead.pages() - 1;
#pragma unroll
            for (int k = 0; k < kTilePages; k++) ids[k] = tbl[min((uint32_t)k, last)];
        };
        auto fetch_codes = [&]() {
            uint32_t most = 0;
#pragma unroll
            for (int k = 0; k < kTilePages; k++) most = max(most, ids[k]);
            if (most >= p.c.cap_low) atomicOr(&p.c.ctrl[kCtrlStatus], PASK_DEV_INTERNAL);      // never expected, never dereferenced
#pragma unroll
            for (int k = 0; k < kTilePages; k++) {
                const uint8_t *src = p.c.pool_low + (size_t)(ids[k] < p.c.cap_low ? ids[k] : 0u) * p.c.low_page_bytes;
                load_codes<BITS>(src, tau, g, codes[k]);
                scales[k] = *reinterpret_cast<const uint16_t *>(src + latent_scale_off(tau, g, BITS));
            }
        };
        bool ahead_more = to_low(more);
        if (ahead_more) fetch_ids();
        bool primed = false;                       // the first codes are asked for behind the first queries
        auto advance = [&]() {
            if (ahead_more) {
                fetch_codes();
                ahead_more = to_low(ahead.next());
                if (ahead_more) fetch_ids();
            }
        };
        uint32_t n_seg = 0;
        for (uint32_t i = 0; more; i++, more = w.next()) {
            const uint32_t st = i & 1;
            if (w.first()) {
                if (n_seg > 0) ok = bar_wait(smem_u32(&ms.q_empty), (n_seg - 1) & 1, ok ? limit : 0) && ok;
                n_seg++;
                const uint4 *src = p.q + ((size_t)w.s * p.c.n_q + h0) * kLatentChunks;
#pragma unroll
                for (int k = 0; k < (kHeads + 8) / 9; k++) {   // a warp takes every ninth head, all in flight at once; heads this
                    const int row = 9 * k + warp - 4;          // CTA does not have are zeros
                    if (row >= kHeads) break;
                    const bool there = row < nh_here;
#pragma unroll
                    for (int ch = lane; ch < kLatentChunks; ch += 32)
                        copy16(qs + (row >> 4) * kLatentHighPageBytes + latent_chunk_off(row & 15, ch), there ? src + row * kLatentChunks + ch : src,
                               there ? 16 : 0);
                }
                if (!primed) { advance(); primed = true; }
                copy16_wait();
                fence_async_shared();
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) bar_arrive(smem_u32(&ms.q_full));
                if (lane == 0 && n_seg == 1) bar_arrive(smem_u32(&ms.q_first));
            }
            const bool low = !w.high();
            const uint32_t np = w.pages();
            uint8_t *dst = sm + st * kTileBytes;
            auto fill = [&](int k0, int k1) {      // pages [k0, k1) of the tile
#pragma unroll 1
                for (int k = k0; k < k1; k++) {
                    if ((uint32_t)k < np) {
                        uint32_t xs[16];
                        dequantise_group<BITS>(codes[0], scales[0], xs);
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            *reinterpret_cast<uint4 *>(dst + k * kLatentHighPageBytes + latent_chunk_off(tau, 4 * g + e)) =
                                make_uint4(xs[4 * e], xs[4 * e + 1], xs[4 * e + 2], xs[4 * e + 3]);
                    }
#pragma unroll
                    for (int j = 0; j + 1 < kTilePages; j++) {
                        scales[j] = scales[j + 1];
#pragma unroll
                        for (int e = 0; e < BITS; e++) codes[j][e] = codes[j + 1][e];
                    }
                }
            };
            if (i >= 2) ok = bar_wait(smem_u32(&ms.empty[st][0]), ((i >> 1) - 1) & 1, ok ? limit : 0) && ok;
            if (low && ok) fill(0, 2);
            if (i >= 2) ok = bar_wait(smem_u32(&ms.empty[st][1]), ((i >> 1) - 1) & 1, ok ? limit : 0) && ok;
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (low) {
                fill(2, kTilePages);
                fence_async_shared();
                __syncwarp();
            }
            if (lane == 0) bar_arrive(smem_u32(&ms.full[st]));
            if (low) advance();
        }
    } else {
        // ================================================= softmax; warp = page of the tile, rows lane / 4 and lane / 4 + 8
        constexpr int kJ = kHeads / 8;             // blocks of 8 heads; this lane's heads: 8 j + 2 (lane % 4) + {0, 1}
        float l[2 * kJ];                           // sums of this lane's rows; the reference maxima are in ms.mref
        const int r0 = lane >> 2, hc = 2 * (lane & 3);
        const uint32_t row8 = (uint32_t)(lane & 7), p_row = ps + (2 * warp + ((lane >> 3) & 1)) * 1024 + row8 * 128;
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
#pragma unroll
        for (int k = 0; k < 2 * kJ; k++) l[k] = 0.0f;
        for (uint32_t i = 0; more; i++) {
            const uint32_t st = i & 1;
            ok = bar_wait(smem_u32(&ms.s_full[st]), (i >> 1) & 1, ok ? limit : 0) && ok;
            __syncwarp();
            fence_after();
            const uint4 info = ms.info[st];
            const bool is_first = info.y & kInfoFirst;
            float x[4 * kJ];                       // scores in log2 units, relative to the reference maximum
            {
                uint32_t sr[4 * kJ];
                tmem_ld_frag(tmem + lanes + st * 64, sr);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 4 * kJ; k++) x[k] = __uint_as_float(sr[k]);
            }
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(&ms.s_empty[st]));
            const int vp = (int)info.x - 16 * warp;
            if (vp < 16) {                         // rows behind the stream's end
#pragma unroll
                for (int k = 0; k < 4 * kJ; k++)
                    if (!((k & 2) ? r0 + 8 < vp : r0 < vp)) x[k] = -INFINITY;
            }
            float most = -INFINITY;
#pragma unroll
            for (int j = 0; j < kJ; j++) {
                float2 m = *reinterpret_cast<const float2 *>(&ms.mref[8 * j + hc]);
                if (is_first) m = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int e = 0; e < 4; e++) x[4 * j + e] = __fmaf_rn(x[4 * j + e], p.scale_log2, -((e & 1) ? m.y : m.x));
                most = fmaxf(most, fmaxf(fmaxf(x[4 * j], x[4 * j + 1]), fmaxf(x[4 * j + 2], x[4 * j + 3])));
            }
            if (group_any(1, 128, is_first || most > kLazy || !ok)) {
                if (group_any(1, 128, !ok)) break;
                // a new reference maximum for the heads that need one
#pragma unroll
                for (int j = 0; j < kJ; j++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        float a = fmaxf(x[4 * j + e], x[4 * j + 2 + e]);
                        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 4));
                        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 8));
                        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 16));
                        if (lane < 4) ms.red[warp][8 * j + hc + e] = a;
                    }
                group_sync(1, 128);
                if (tid < kHeads) {                // red: largest score above the reference
                    const float a = fmaxf(fmaxf(ms.red[0][tid], ms.red[1][tid]), fmaxf(ms.red[2][tid], ms.red[3][tid]));
                    const bool raise = is_first || a > kLazy;
                    ms.fac[tid] = raise ? a : 0.0f;
                    if (raise) ms.mref[tid] = is_first ? a : ms.mref[tid] + a;
                }
                group_sync(1, 128);
#pragma unroll
                for (int j = 0; j < kJ; j++) {
                    const float2 f = *reinterpret_cast<const float2 *>(&ms.fac[8 * j + hc]);
#pragma unroll
                    for (int e = 0; e < 4; e++) x[4 * j + e] -= (e & 1) ? f.y : f.x;
                    l[2 * j] = is_first ? 0.0f : l[2 * j] * ex2(-f.x);
                    l[2 * j + 1] = is_first ? 0.0f : l[2 * j + 1] * ex2(-f.y);
                }
                if (!is_first) {                   // O so far, in the new reference
                    ok = bar_wait(smem_u32(&ms.p_empty), (i - 1) & 1, ok ? limit : 0) && ok;
                    __syncwarp();
                    fence_after();
#pragma unroll 1
                    for (int b = 0; b < 4; b++)
#pragma unroll 1
                        for (int cc = 0; cc < kHeads; cc += 16) {
                            uint32_t o[16];
                            tmem_ld16(tmem + lanes + kO + b * 64 + cc, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; e++) o[e] = __float_as_uint(__uint_as_float(o[e]) * ex2(-ms.fac[cc + e]));
                            tmem_st16(tmem + lanes + kO + b * 64 + cc, o);
                        }
                    tmem_wait_st();
                    fence_before();
                }
            }
            uint32_t pk[2 * kJ];                   // weights as pairs of heads: row 0 in [2j], row 1 in [2j + 1]
#pragma unroll
            for (int j = 0; j < kJ; j++) {
                const float a0 = ex2(x[4 * j]), a1 = ex2(x[4 * j + 1]), b0 = ex2(x[4 * j + 2]), b1 = ex2(x[4 * j + 3]);
                l[2 * j] += a0 + b0;
                l[2 * j + 1] += a1 + b1;
                pk[2 * j] = pack_bf16(a0, a1);
                pk[2 * j + 1] = pack_bf16(b0, b1);
            }
            if (i > 0) ok = bar_wait(smem_u32(&ms.p_empty), (i - 1) & 1, ok ? limit : 0) && ok;     // P is free
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kJ; j += 2)
                stmatrix4(p_row + ((((uint32_t)j + (uint32_t)(lane >> 4)) ^ row8) << 4), pk[2 * j], pk[2 * j + 1], pk[2 * j + 2], pk[2 * j + 3]);
            fence_async_shared();
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(&ms.p_full));
            if (info.y & kInfoLast) {
                // ---- the sequence's part ends: sums over the rows, then O out of tensor memory
#pragma unroll
                for (int j = 0; j < kJ; j++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        float a = l[2 * j + e];
                        a += __shfl_xor_sync(0xffffffffu, a, 4);
                        a += __shfl_xor_sync(0xffffffffu, a, 8);
                        a += __shfl_xor_sync(0xffffffffu, a, 16);
                        if (lane < 4) ms.red[warp][8 * j + hc + e] = a;
                    }
                const bool whole = info.y & kInfoWhole;
                const size_t row0 = (size_t)(whole ? info.z : 2 * slot + (info.y & kInfoGoesOn ? 0u : 1u)) * p.c.n_q + h0;
                group_sync(1, 128);
                if (tid < kHeads) {
                    const float ls = (ms.red[0][tid] + ms.red[1][tid]) + (ms.red[2][tid] + ms.red[3][tid]);
                    ms.fac[tid] = whole ? 1.0f / ls : 1.0f;
                    if (tid < nh_here) {
                        if (!whole) p.part_ml[row0 + tid] = make_float2(ms.mref[tid], ls);
                        else if (p.lse) p.lse[row0 + tid] = (ms.mref[tid] + log2f(ls)) * 0.69314718055994531f;
                    }
                }
                group_sync(1, 128);
                ok = bar_wait(smem_u32(&ms.p_empty), i & 1, ok ? limit : 0) && ok;
                __syncwarp();
                fence_after();
#pragma unroll 1
                for (int b = 0; b < 4; b++)
#pragma unroll 1
                    for (int cc = 0; cc < kHeads; cc += 16) {
                        uint32_t o[16];
                        tmem_ld16(tmem + lanes + kO + b * 64 + cc, o);
                        tmem_wait_ld();
                        const size_t at = (row0 + cc) * kLatentValueDim + 128 * b + 32 * warp + lane;
                        const int left = nh_here - cc;
                        if (whole) {
#pragma unroll
                            for (int e = 0; e < 16; e++)
                                if (e < left) p.out[at + e * kLatentValueDim] = __float2bfloat16_rn(__uint_as_float(o[e]) * ms.fac[cc + e]);
                        } else {
#pragma unroll
                            for (int e = 0; e < 16; e++)
                                if (e < left) p.part_o[at + e * kLatentValueDim] = __uint_as_float(o[e]);
                        }
                    }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_u32(&ms.o_free));
            }
            if (info.y & kInfoFinal) break;
        }
    }
    if (!ok) atomicOr(&p.c.ctrl[kCtrlStatus], PASK_DEV_TIMEOUT);
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == 14) tmem_free(tmem, 512);
    if (p.span && tid == 0) {
        unsigned long long t_end;
        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t_end));
        atomicMin(p.span, t_start);
        atomicMax(p.span + 1, t_end);
    }
}

// Joins the partial sums of a sequence: a CTA takes kRows heads of it (few sequences: one, with the partials split over kSplit
// groups of threads), a thread four of the 512 dims.  Two trips to L2: what the sequence's shares are, and their partials
// (the first ones of every head fetched before their weights are known).  Sequences that one share covered are left alone;
// empty ones are written here.
template <int kSplit, int kRows>
__global__ void __launch_bounds__(128 * kSplit)
decode_latent_merge(int n_seqs, int n_q, const uint4 *__restrict__ meta, const float2 *__restrict__ part_ml,
                    const float *__restrict__ part_o, __nv_bfloat16 *__restrict__ out, float *__restrict__ lse) {
    constexpr int kAhead = kRows > 1 ? 3 : 8;      // partials of a head fetched at once
    __shared__ float s_w[kRows][kMaxSlots], s_l[kRows], s_top[kRows];
    __shared__ float4 s_o[kSplit > 1 ? (kSplit - 1) * 128 : 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int groups = (n_q + kRows - 1) / kRows, s = blockIdx.x / groups, h0 = (blockIdx.x % groups) * kRows;
    const int rows = min(kRows, n_q - h0);
    pdl_launch_dependents();
    pdl_wait();
    const uint4 ms = meta[s];
    const uint32_t b0 = ms.z, count = ms.w - ms.z;
    const size_t row0 = (size_t)s * n_q + h0;
    if (ms.y == 0) {
        for (int d = tid; d < rows * (kLatentValueDim / 8); d += 128 * kSplit)
            reinterpret_cast<uint4 *>(out)[row0 * (kLatentValueDim / 8) + d] = make_uint4(0, 0, 0, 0);
        if (tid < rows && lse) lse[row0 + tid] = -INFINITY;
        return;
    }
    if (count == 1) return;                        // the share has written the result
    const int part = tid >> 7, d4 = tid & 127;
    auto row_of = [&](uint32_t k) { return (size_t)(2 * (b0 + k) + (k == 0 ? 1u : 0u)) * n_q + h0; };   // of the k-th partial
    const float4 *src = reinterpret_cast<const float4 *>(part_o) + d4;
    float4 v[kRows][kAhead];
#pragma unroll
    for (int r = 0; r < kRows; r++)
#pragma unroll
        for (int k = 0; k < kAhead; k++) {
            v[r][k] = make_float4(0, 0, 0, 0);
            if (r < rows && part + (uint32_t)k * kSplit < count) v[r][k] = src[(row_of(part + k * kSplit) + r) * (kLatentValueDim / 4)];
        }
    // weights: a warp per head
    for (int r = warp; r < rows; r += 4 * kSplit) {
        float top = -INFINITY, sum = 0.0f;
        for (uint32_t k = lane; k < count; k += 32) top = fmaxf(top, part_ml[row_of(k) + r].x);
#pragma unroll
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        for (uint32_t k = lane; k < count; k += 32) {
            const float2 ml = part_ml[row_of(k) + r];
            const float wgt = umma::ex2(ml.x - top);
            sum += wgt * ml.y;
            s_w[r][k] = ml.y == ml.y ? wgt : ml.y; // a NaN stays one
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) { s_l[r] = sum; s_top[r] = top; }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRows; r++) {
        if (r >= rows) break;
        float4 acc = make_float4(0, 0, 0, 0);
        auto add = [&](const float4 &x, float wgt) { acc.x += wgt * x.x; acc.y += wgt * x.y; acc.z += wgt * x.z; acc.w += wgt * x.w; };
#pragma unroll
        for (int k = 0; k < kAhead; k++)
            if (part + (uint32_t)k * kSplit < count) add(v[r][k], s_w[r][part + k * kSplit]);
#pragma unroll 8
        for (uint32_t k = part + kAhead * kSplit; k < count; k += kSplit) add(src[(row_of(k) + r) * (kLatentValueDim / 4)], s_w[r][k]);
        if (kSplit > 1) {
            if (part > 0) s_o[(part - 1) * 128 + d4] = acc;
            __syncthreads();
            if (part > 0) return;
#pragma unroll
            for (int k = 0; k < kSplit - 1; k++) {
                const float4 x = s_o[k * 128 + d4];
                acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
            }
        }
        const float inv = 1.0f / s_l[r];
        reinterpret_cast<uint2 *>(out)[(row0 + r) * (kLatentValueDim / 4) + d4] =
            make_uint2(umma::pack_bf16(acc.x * inv, acc.y * inv), umma::pack_bf16(acc.z * inv, acc.w * inv));
        if (tid == 0 && lse) lse[row0 + r] = (s_top[r] + log2f(s_l[r])) * 0.69314718055994531f;
    }
}

}  // namespace

pask_status_t launch_append_latent(pask_cache *c, int layer, int n_seqs, int total_tokens, const int32_t *seq_ids,
                                   const int32_t *cu_tokens, const void *latent, const uint8_t *tags, const uint8_t *decided,
                                   uint8_t *actions_out, cudaStream_t stream) {
    if (total_tokens == 0) return PASK_OK;
    bool done = false;
    pask_status_t rc = launch_append_small_latent(c, layer, n_seqs, total_tokens, seq_ids, cu_tokens, latent, tags, decided, actions_out, stream, &done);
    if (done || rc != PASK_OK) return rc;
    rc = launch_append_plan(c, layer, n_seqs, total_tokens, seq_ids, cu_tokens, tags, decided, actions_out, stream);
    if (rc != PASK_OK) return rc;
    // at most one item per 16 tokens plus two partly filled pages per stream; twice the resident CTAs, since HIGH and LOW
    // pages do not take the same time
    const long long bound = (long long)total_tokens / 16 + 4LL * n_seqs;
    const int ctas = (int)(bound < (long long)c->sm_count * 14 ? bound : c->sm_count * 14);
    auto kern = c->dev.low_bits == 8 ? append_latent_kernel<8> : c->dev.low_bits == 2 ? append_latent_kernel<2> : append_latent_kernel<4>;
    kern<<<ctas, kRowThreads, 0, stream>>>(c->dev, layer, n_seqs, static_cast<const uint4 *>(latent));
    return cudaGetLastError() == cudaSuccess ? PASK_OK : PASK_ERR_CUDA;
}

pask_status_t launch_read_latent(pask_cache *c, int layer, int n_seqs, int total_rows, const int32_t *seq_ids,
                                 const int32_t *cu_rows, void *rows_out, int32_t *lens_out, cudaStream_t stream) {
    const long long items = (long long)(total_rows >> 4) + 2LL * n_seqs;
    const int ctas = (int)(items < (long long)c->sm_count * kReadCtas ? items : c->sm_count * kReadCtas);
    auto kern = c->dev.low_bits == 8 ? read_latent_kernel<8> : c->dev.low_bits == 2 ? read_latent_kernel<2> : read_latent_kernel<4>;
    kern<<<ctas, kRowThreads, 0, stream>>>(c->dev, layer, n_seqs, total_rows, seq_ids, cu_rows, static_cast<uint4 *>(rows_out), lens_out);
    return cudaGetLastError() == cudaSuccess ? PASK_OK : PASK_ERR_CUDA;
}

// heads are taken in groups of at most 64, evenly
static void latent_shares(const pask_cache *c, int *groups, int *heads, uint32_t *slots) {
    *groups = (c->desc.n_q_heads + 63) / 64;
    *heads = (c->desc.n_q_heads + *groups - 1) / *groups;
    const uint32_t n = (uint32_t)(c->attn_ctas / *groups);
    *slots = n < 1 ? 1 : n > kMaxSlots ? kMaxSlots : n;
}

static size_t carve_latent(const pask_cache *c, int n_seqs, uint8_t *base, DecParams *p) {
    int groups, heads;
    uint32_t slots;
    latent_shares(c, &groups, &heads, &slots);
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off = (off + bytes + 255) / 256 * 256; return at; };
    const size_t rows = (size_t)2 * slots * c->desc.n_q_heads;
    const size_t o_meta = take((size_t)n_seqs * sizeof(uint4)), o_ml = take(rows * sizeof(float2)), o_o = take(rows * kLatentValueDim * sizeof(float));
    if (p) {
        p->groups = groups;
        p->heads = heads;
        p->slots = slots;
        p->meta = reinterpret_cast<uint4 *>(base + o_meta);
        p->part_ml = reinterpret_cast<float2 *>(base + o_ml);
        p->part_o = reinterpret_cast<float *>(base + o_o);
    }
    return off;
}

size_t latent_workspace_bytes(const pask_cache *c, int n_seqs) { return carve_latent(c, n_seqs, nullptr, nullptr); }

template <int kHeads, int BITS>
static cudaError_t launch_decode_kernel(const DecParams &p, cudaStream_t stream) {
    static bool granted[64] = {};                  // the shared-memory opt-in, asked for once per device
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    constexpr int kSmem = DecSmem<kHeads>::kBytes;
    static_assert(kSmem <= 232448, "shared memory of a CTA");
    if (!granted[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(decode_latent_kernel<kHeads, BITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return e;
        granted[dev] = true;
    }
    return launch_pdl(decode_latent_kernel<kHeads, BITS>, dim3(p.slots * (uint32_t)p.groups), dim3(kDecThreads), kSmem, stream, p);
}
template <int BITS>
static cudaError_t launch_decode_heads(const DecParams &p, cudaStream_t stream) {
    return p.heads <= 16 ? launch_decode_kernel<16, BITS>(p, stream) : p.heads <= 32 ? launch_decode_kernel<32, BITS>(p, stream)
                                                                     : launch_decode_kernel<64, BITS>(p, stream);
}

pask_status_t launch_decode_latent(pask_cache *c, int layer, int n_seqs, const int32_t *seq_ids, const void *q, float scale,
                                   void *out, float *lse, void *workspace, cudaStream_t stream) {
    DecParams p;
    carve_latent(c, n_seqs, static_cast<uint8_t *>(workspace), &p);
    p.c = c->dev;
    p.layer = layer;
    p.n_seqs = n_seqs;
    p.seq_ids = seq_ids;
    p.q = static_cast<const uint4 *>(q);
    p.scale_log2 = scale * 1.4426950408889634f;
    p.out = static_cast<__nv_bfloat16 *>(out);
    p.lse = lse;
    p.wait_cycles = c->wait_cycles;
    p.surplus = c->wait_test_surplus;
    p.span = c->span;
    if (c->ev_start) cudaEventRecord(c->ev_start, stream);
    cudaError_t e = c->dev.low_bits == 8 ? launch_decode_heads<8>(p, stream)
                  : c->dev.low_bits == 2 ? launch_decode_heads<2>(p, stream) : launch_decode_heads<4>(p, stream);
    if (c->ev_stop) cudaEventRecord(c->ev_stop, stream);
    c->ev_start = c->ev_stop = nullptr;
    c->span = nullptr;
    if (e != cudaSuccess) return PASK_ERR_CUDA;
    const int n_q = c->desc.n_q_heads;
    // few sequences have many partials to a head, which four groups of threads share; many sequences have a few, and a CTA takes
    // four heads so that all of them are resident at once
    if (p.slots >= 16u * (uint32_t)n_seqs)
        e = launch_pdl(decode_latent_merge<4, 1>, dim3(n_seqs * n_q), dim3(512), 0, stream, n_seqs, n_q, p.meta, p.part_ml, p.part_o, p.out, lse);
    else
        e = launch_pdl(decode_latent_merge<1, 4>, dim3(n_seqs * ((n_q + 3) / 4)), dim3(128), 0, stream, n_seqs, n_q, p.meta, p.part_ml, p.part_o,
                       p.out, lse);
    return e == cudaSuccess ? PASK_OK : PASK_ERR_CUDA;
}

}  // namespace pask
