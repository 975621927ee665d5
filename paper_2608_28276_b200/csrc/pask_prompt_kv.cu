// pask_prompt_attention: causal attention of the tokens of a ragged batch behind what a cache retains of their sequences.
//
// Per query head: S = Q K^T over 128 dims, P = softmax(S / sqrt(128)), O = P V, where K and V are the history (pages of bf16 rows and of
// 2, 4 or 8-bit rows, the protected window's ring) and the call's own tokens up to the query's.  The four query heads of a
// key / value head are rows of one product: a tile is 32 tokens x 4 heads = 128 rows.
//
// Work.  An item is a block of tokens and a key / value head; its keys are blocks of 128: eight pages of the history, or 128 tokens of
// the call.  prompt_plan_kernel lays all items end to end on a line of their costs (key blocks, and two more for the beginning and the
// result) and every CTA of the grid, one an SM, takes an equal stretch: cuts fall inside items, at any key block.  No more items than
// CTAs: each gets whole CTAs of its own instead.  An item's parts leave unscaled outputs, maxima and sums in the workspace;
// prompt_join_kernel adds them up in the order of the parts, so that the result does not depend on which CTA was done first.
//
// In a CTA (one tile of 128 rows of S, or two)
//   softmax          four warps a tile, a thread a row; P back to tensor memory in bf16, as the left operand of P V.  128 scores go in two
//                    halves, so that the product over the first 64 keys runs beside the exponentials of the others.  The reference maximum
//                    moves only when a score exceeds it by more than 2^8: O is rarely rescaled
//   products         one warp.  Two tiles: P V of tile t, block j;  Q K^T of tile t, block j + 1;  the other tile.  One: Q K^T of block j + 1 into
//                    the other place of S while the softmax has block j, then P V of block j
//   copies           queries; the call's own keys and values (TMA)
//   fill             history pages: read as they are stored, expanded to bf16 and laid out as the tensor core reads them.  Sixteen warps; they leave
//                    where the plan finds no history in the whole call, and a variant without them is launched beside for long sequences
//   items            which items, and which parts of them, are this CTA's
// Few tokens do not fill 128 rows with 4 heads each.  Then the rows of Q stand kCopies times in the tile, and copy c of a row takes the
// softmax of keys 128 / kCopies c on, with zero weights for the others: the exponentials, the chain that bounds short items, are spread
// over all threads; the copies' O are summed at the end.
// Shared memory: Q 32 KB a tile, stages of 64 KB (128 keys and values).  Tensor memory: two tiles, S (P over it) and O, 128 columns
// each; one tile, two places of S, two of P, O.
//
// What bounds it, at 6539 GB/s and 1643 TFLOP/s (1394 sustained) measured:
//   prompts without history (4 of 4096 - 8192, 32 heads) 1400 - 1435 us, 942 at the sustained rate: some 3500 cycles for two tiles and 128
//       keys, of which the products need 2048 and the exponentials as many, beside them; the rest is waits between the two (a row's halves are
//       loaded, waited for and worked on one after the other), at 1.34 GHz under the power limit
//   chunks of 512 behind 9K rows in 8 bits 726 - 738 us (377): the same chain, 580 with no page read or expanded; expansion in its issue slots
//   5 drafted tokens of 64 sequences of 2K - 8K 180 - 184 us (75: the pages once): 104 with no page read or expanded, 110 with expansion
//       alone: a fill warp's chain for a page (its pieces from memory, expansion, the block's hand-over) does not overlap with itself
//   one prompt of 131: 14.4 us; three launches in a row: plan 4, items 8, join 3
//
// Rounding: S, O and the sums are fp32; a weight is rounded to bf16 once, as an operand of a product with bf16 values; a low-precision
// row enters as bf16(code * scale), rounded once from the exact product.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pask_internal.h"
#include "pask_tensormap.h"
#include "pask_umma.h"

namespace pask {

namespace {

constexpr int kDim = kHeadDim, kGqa = 4;
constexpr int kTileRows = 128, kTileTokens = kTileRows / kGqa, kBlockK = 128, kBlockPages = kBlockK / kPageTokens;
constexpr int kSub = kBlockK * 128;                // 128 rows x 64 dims: 16 KB
constexpr int kTileBytes = 2 * kSub;               // 128 rows x 128 dims
constexpr int kItemCost = 2;                       // of an item's beginning and end, in key blocks
constexpr int kMinPiece = 2;                       // no part of an item is shorter, in key blocks
constexpr float kLazy = 8.0f;
constexpr float kScaleLog2 = 0.08838834764831845f * 1.4426950408889634f;       // 1 / sqrt(128), log2 e

// What the plan says of a sequence of the call.
struct __align__(16) PromptSeq {
    int q0, nq;                                    // its rows; none if its range is malformed or its id is out of range
    uint32_t slot;                                 // sequence * layers + layer
    uint32_t nh, nl, nw;                           // tokens attended from the two streams and from the window's ring
    int blocks;                                    // key blocks of its history
    int parts;                                     // CTAs an item of it has for itself (0: the line is cut evenly)
};
static_assert(sizeof(PromptSeq) == 32, "two 16-byte loads");

// An item in parts: its rows (none: there is no such item), the CTAs that have one.
struct Join { int row, rows, head, first, last; };

struct PromptWorkspace {
    uint64_t *prefix;                              // [n_seqs + 1] cost (or CTAs) of the sequences before
    int *paged;                                    // whether any sequence with tokens has a history
    PromptSeq *seqs;                               // [n_seqs]
    Join *joins;                                   // [grid] the item in parts that begins with this CTA's part
    float2 *ml;                                    // [2 grid][rows] reference maximum in log2 units, sum
    float4 *o;                                     // [2 grid][rows][32] unscaled outputs, four dims a piece
};

size_t carve(int n_seqs, int grid, int rows, uint8_t *base, PromptWorkspace *ws) {
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t at = off; off = (off + bytes + 255) / 256 * 256; return at; };
    const size_t o_prefix = take((size_t)(n_seqs + 1) * 8), o_seqs = take((size_t)n_seqs * sizeof(PromptSeq)), o_join = take((size_t)grid * sizeof(Join));
    const size_t o_paged = take(sizeof(int));
    const size_t o_ml = take((size_t)2 * grid * rows * sizeof(float2)), o_o = take((size_t)2 * grid * rows * kDim * 4);
    if (ws) {
        ws->prefix = reinterpret_cast<uint64_t *>(base + o_prefix);
        ws->paged = reinterpret_cast<int *>(base + o_paged);
        ws->seqs = reinterpret_cast<PromptSeq *>(base + o_seqs);
        ws->joins = reinterpret_cast<Join *>(base + o_join);
        ws->ml = reinterpret_cast<float2 *>(base + o_ml);
        ws->o = reinterpret_cast<float4 *>(base + o_o);
    }
    return off;
}

struct PromptParams {
    PromptWorkspace ws;
    const uint8_t *pool_high, *pool_low;
    const uint32_t *tbl_high, *tbl_low;
    uint32_t *status;
    uint32_t high_page_bytes, low_page_bytes, low_head_bytes, cap_low, high_limit, ring_first, ring_pages;
    int max_pages, n_kv, n_seqs, grid;
    int only;                                      // 0, 1: nothing to do where `paged` is something else;  -1: always
    __nv_bfloat16 *out;
    float *lse;
    long long wait_cycles;
    uint32_t surplus;
};

PASK_HD int pages_of(uint32_t tokens) { return (int)((tokens + kPageTokens - 1) / kPageTokens); }
// key blocks of the call's own tokens that token block j (of `tokens`) looks at, and the sum of that over blocks 0 .. j - 1
__host__ __device__ __forceinline__ int own_blocks(int j, int tokens) { return j * tokens / kBlockK + 1; }
__host__ __device__ __forceinline__ long long own_blocks_before(int j, int tokens) {
    const long long r = kBlockK / tokens, m = j / r, k = j % r;
    return r * m * (m + 1) / 2 + k * (m + 1);
}

// ------------------------------------------------------------------------------------------------ plan

constexpr int kPlanThreads = 1024;

// One CTA, a sequence a thread: what each has to attend, the line of costs.  (A CTA of as few warps as there are sequences for: its
// barriers are most of its time.)
__global__ void __launch_bounds__(kPlanThreads)
prompt_plan_kernel(DevCache c, int layer, int n_seqs, int total, const int32_t *__restrict__ seq_ids, const int32_t *__restrict__ cu,
                   PromptWorkspace ws, int grid, int block_tokens, uint4 *__restrict__ out, float *__restrict__ lse) {
    __shared__ uint64_t s_sum[32];
    __shared__ uint32_t s_part, s_items, s_longest, s_bad, s_paged;
    __shared__ int2 s_seq[kPlanThreads];           // items and key blocks of the longest, of each sequence
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
    pdl_launch_dependents();
    pdl_wait();
    if (tid == 0) s_items = s_longest = s_bad = s_paged = 0;
    __syncthreads();
    PromptSeq s{};
    uint32_t bad = 0;
    bool unknown = false;
    if (tid < n_seqs) {
        const int id = seq_ids[tid], q0 = cu[tid], q1 = cu[tid + 1];
        unknown = id < 0 || id >= c.max_seqs;
        if (q0 < 0 || q1 < q0 || q1 > total) bad |= PASK_DEV_BAD_RAGGED;
        else { s.q0 = q0; s.nq = q1 - q0; }
        if (unknown) bad |= PASK_DEV_BAD_SEQ;
        else {
            s.slot = (uint32_t)id * (uint32_t)c.n_layers + (uint32_t)layer;
            s.nh = c.n_high[s.slot];
            s.nl = c.n_low[s.slot];
            if (c.window) {
                // The last min(W, tokens seen) tokens come from the ring, whatever their action; the streams are in arrival order, so
                // that their members among those are the streams' last entries.
                const uint32_t seen = c.n_tok[s.slot];
                s.nw = min(seen, c.window);
                const uint4 *act = reinterpret_cast<const uint4 *>(c.win_act + (size_t)s.slot * c.window);
                for (uint32_t i = 0; 16 * i < s.nw; i++) {
                    const uint4 a = act[i];
                    const uint32_t w[4] = {a.x, a.y, a.z, a.w}, in = min(16u, s.nw - 16 * i);
#pragma unroll
                    for (uint32_t e = 0; e < 4; e++) {         // actions are 0, 1, 2: bit 0 of a byte says LOW, bit 1 HIGH
                        const uint32_t have = in > 4 * e ? in - 4 * e : 0, member = have >= 4 ? 0xFFFFFFFFu : (1u << (8 * have)) - 1u;
                        s.nl -= __popc(w[e] & member & 0x01010101u);
                        s.nh -= __popc(w[e] & member & 0x02020202u);
                    }
                }
            }
        }
        if (bad) { atomicOr(&s_bad, bad); }
        s.blocks = (pages_of(s.nh) + pages_of(s.nl) + pages_of(s.nw) + kBlockPages - 1) / kBlockPages;
    }
    const int named = s.nq;                        // rows of an unknown sequence: cleared below, no item
    if (unknown) s.nq = 0;
    const int nqb = (s.nq + block_tokens - 1) / block_tokens, longest = nqb ? s.blocks + own_blocks(nqb - 1, block_tokens) : 0;
    if (nqb && s.blocks) s_paged = 1;
    if (nqb && nqb <= grid) {                      // (more: no need to count)
        atomicAdd(&s_items, (uint32_t)(nqb * c.n_kv));
        atomicMax(&s_longest, (uint32_t)longest);
    }
    s_seq[tid] = make_int2(nqb ? min(nqb, grid + 1) * c.n_kv : 0, longest);
    const bool many = __syncthreads_or(nqb > grid);
    if (tid == 0 && s_bad) atomicOr(&c.ctrl[kCtrlStatus], s_bad);
    uint64_t cost = (uint64_t)c.n_kv * ((uint64_t)nqb * (uint64_t)(s.blocks + kItemCost) + (uint64_t)own_blocks_before(nqb, block_tokens));
    if (!many && s_items <= (uint32_t)grid) {
        // Whole CTAs for each item: the shortest part length for which the grid has enough of them
        if (warp == 0) {
            uint32_t lo = kMinPiece, hi = max(s_longest, (uint32_t)kMinPiece);
            while (lo < hi) {
                const uint32_t mid = (lo + hi) / 2;
                uint32_t need = 0;
                for (int i = lane; i < n_seqs; i += 32) need += s_seq[i].x * ((s_seq[i].y + mid - 1) / mid);
                if (__reduce_add_sync(0xffffffffu, need) <= (uint32_t)grid) hi = mid; else lo = mid + 1;
            }
            if (lane == 0) s_part = lo;
        }
        __syncthreads();
        s.parts = max(1, (int)((longest + s_part - 1) / s_part));          // (at least one: says that items have CTAs of their own)
        cost = (uint64_t)c.n_kv * nqb * s.parts;
    }
    // prefix over the sequences
    uint64_t inc = cost;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint64_t o = __shfl_up_sync(0xffffffffu, inc, d);
        if (lane >= d) inc += o;
    }
    if (lane == 31) s_sum[warp] = inc;
    __syncthreads();
    uint64_t before = 0;
    for (int w = 0; w < warp; w++) before += s_sum[w];
    if (tid < n_seqs) {
        ws.prefix[tid + 1] = before + inc;
        ws.seqs[tid] = s;
    }
    if (tid == 0) {
        ws.prefix[0] = 0;
        *ws.paged = (int)s_paged;
    }
    // rows of sequences that are none
    if (s_bad & PASK_DEV_BAD_SEQ) {
        __shared__ int s_q0, s_n;
        for (int i = 0; i < n_seqs; i++) {
            __syncthreads();
            if (tid == i) { s_q0 = s.q0; s_n = unknown ? named : 0; }
            __syncthreads();
            const size_t heads = (size_t)kGqa * c.n_kv, from = (size_t)s_q0 * heads, count = (size_t)s_n * heads;
            for (size_t e = tid; e < count * (kDim / 8); e += threads) out[from * (kDim / 8) + e] = make_uint4(0, 0, 0, 0);
            if (lse)
                for (size_t e = tid; e < count; e += threads) lse[from + e] = -INFINITY;
        }
    }
}

// ------------------------------------------------------------------------------------------------ items

struct Item {
    int q0, nq, head, block;                       // rows of the sequence; key / value head; token block; block -1: no further item
    uint32_t slot, nh, nl, nw;
    int hist, blocks;                              // key blocks: of the history, in all
    int b0, b1;                                    // this CTA's
    int first, last;                               // the CTAs that have a part
};

// Walks over a CTA's items; all lanes of a warp hold the same.
struct Walker {
    uint64_t x0, x1, at;                           // the CTA's stretch of the line, beginning of the item to come
    int cta, grid, n_seqs, tokens, n_kv, s, head, block;
    PromptSeq q;
    bool whole;                                    // whole CTAs for each item
    const PromptWorkspace *ws;
    int step;                                      // sequences a lane stands for
    uint64_t mine;                                 // where the last of them ends

    __device__ __forceinline__ uint64_t edge(uint64_t total, int b) const { return total * (uint64_t)b / (uint64_t)grid; }
    // sequences that end at or before x
    __device__ __forceinline__ int seqs_before(uint64_t x, int lane) const {
        const int n = __popc(__ballot_sync(0xffffffffu, (lane + 1) * step <= n_seqs && mine <= x)) * step;
        if (step == 1) return n;
        const int k = n + lane + 1;
        return n + __popc(__ballot_sync(0xffffffffu, lane < step && k <= n_seqs && ws->prefix[min(k, n_seqs)] <= x));
    }
    __device__ __forceinline__ int token_blocks() const { return (q.nq + tokens - 1) / tokens; }
    __device__ __forceinline__ int key_blocks() const { return q.blocks + own_blocks(block, tokens); }

    __device__ __forceinline__ void load_seq() { q = ws->seqs[s]; }

    __device__ __forceinline__ void init(const PromptParams &p, int block_tokens, int lane) {
        ws = &p.ws;
        cta = blockIdx.x; grid = p.grid; n_seqs = p.n_seqs; tokens = block_tokens; n_kv = p.n_kv;
        step = (n_seqs + 31) / 32;
        mine = ws->prefix[min((lane + 1) * step, n_seqs)];
        const uint64_t total = ws->prefix[n_seqs];
        whole = ws->seqs[0].parts > 0;
        if (whole) { x0 = cta; x1 = (uint64_t)cta + 1 <= total ? (uint64_t)cta + 1 : (uint64_t)cta; }
        else { x0 = edge(total, cta); x1 = edge(total, cta + 1); }
        if (x0 >= x1) { s = n_seqs; return; }
        s = seqs_before(x0, lane);
        if (s >= n_seqs) return;
        load_seq();
        uint64_t rest = x0 - ws->prefix[s];
        if (whole) {
            const int item = (int)(rest / q.parts), nb = token_blocks();
            head = item / nb;
            block = item % nb;
            return;
        }
        const int nb = token_blocks();
        const uint64_t per = (uint64_t)nb * (q.blocks + kItemCost) + own_blocks_before(nb, tokens);
        head = (int)(rest / per);
        rest -= per * head;
        int lo = 0, hi = nb - 1;                   // the last block that begins at or before rest
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if ((uint64_t)mid * (q.blocks + kItemCost) + own_blocks_before(mid, tokens) <= rest) lo = mid; else hi = mid - 1;
        }
        block = lo;
        at = x0 - rest + (uint64_t)block * (q.blocks + kItemCost) + own_blocks_before(block, tokens);
    }
    // key blocks of the item at `at` before point x of the line.  Both sides of a cut ask the same.
    __device__ __forceinline__ int cut(uint64_t x, int nb) const {
        if (x <= at + kItemCost) return 0;
        if (x >= at + kItemCost + nb) return nb;
        const int y = (int)(x - at - kItemCost);
        return y < kMinPiece ? 0 : nb - y < kMinPiece ? nb : y;
    }
    __device__ __forceinline__ bool next(Item &it, int lane) {
        while (s < n_seqs) {
            const int nb = key_blocks();
            it.q0 = q.q0; it.nq = q.nq; it.head = head; it.block = block;
            it.slot = q.slot; it.nh = q.nh; it.nl = q.nl; it.nw = q.nw;
            it.hist = q.blocks; it.blocks = nb;
            if (whole) {
                const int rest = (int)(x0 - ws->prefix[s]), part = rest % q.parts, parts = min(q.parts, nb);
                s = n_seqs;
                if (part >= parts) return false;
                it.b0 = (int)((long long)nb * part / parts);
                it.b1 = (int)((long long)nb * (part + 1) / parts);
                it.first = cta - part;
                it.last = it.first + parts - 1;
                return true;
            }
            if (at >= x1) { s = n_seqs; return false; }
            it.b0 = cut(x0, nb);
            it.b1 = cut(x1, nb);
            it.first = it.last = cta;
            if (it.b0 < it.b1 && it.b1 - it.b0 < nb) {
                // Who has the rest: the CTAs whose stretches meet the item's, a lane each
                const uint64_t total = ws->prefix[n_seqs];
                const double per = (double)grid / (double)total;
                const int from = max(0, (int)((double)at * per) - 1), to = min(grid - 1, (int)((double)(at + kItemCost + nb) * per) + 1);
                int lo = grid, hi = -1;
                for (int b = from + lane; b <= to; b += 32)
                    if (cut(edge(total, b), nb) < cut(edge(total, b + 1), nb)) { lo = min(lo, b); hi = max(hi, b); }
                it.first = __reduce_min_sync(0xffffffffu, lo);
                it.last = __reduce_max_sync(0xffffffffu, hi);
            }
            at += kItemCost + nb;
            if (++block >= token_blocks()) {
                block = 0;
                if (++head >= n_kv) {
                    head = 0;
                    s = seqs_before(at, lane);
                    if (s < n_seqs) load_seq();
                }
            }
            if (it.b0 < it.b1) return true;
        }
        return false;
    }
};

// ------------------------------------------------------------------------------------------------ pages to operands

constexpr uint32_t kPageLow = 0, kPageBad = 1, kPageHigh = 2, kPageNone = 3;       // kinds of a page: the low bits of its place

// A lane's share of what is expanded at a time, in registers: half of a bf16 page's keys or values of one head, or the codes of a
// low-precision page's and two of its scales.
struct Raw { uint4 x[4]; uint32_t s0, s1; };

// (code - kZero) * scale for two codes, as bf16, rounded once: the difference is exact, the scale is the sum of two bf16 numbers of which the
// smaller has three bits, so that its product with a code is exact and one fma rounds the sum of both products.
__device__ __forceinline__ uint32_t scaled_codes(uint32_t codes, uint32_t offset, uint32_t s_hi, uint32_t s_lo) {
    uint32_t r;
    asm("{\n\t.reg .b32 c, m;\n\tsub.rn.bf16x2 c, %1, %2;\n\tmul.rn.bf16x2 m, c, %4;\n\tfma.rn.bf16x2 %0, c, %3, m;\n\t}"
        : "=r"(r) : "r"(codes | 0x43004300u), "r"(offset), "r"(s_hi), "r"(s_lo));
    return r;
}
__device__ __forceinline__ float half_bits(uint32_t h) { return __half2float(__ushort_as_half((unsigned short)h)); }
// two scales as pairs of two bf16 numbers whose sums they are
__device__ __forceinline__ void split_scales(float a, float b, uint32_t &hi, uint32_t &lo) {
    hi = umma::pack_bf16(a, b);
    lo = umma::pack_bf16(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xFFFF0000u));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float x;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(x) : "f"(a), "f"(b), "f"(c));
    return x;
}
// bytes k0 and k1 of w, less 128, times s: as bf16, rounded once from exact products (codes of 8 bits, scales of 11)
__device__ __forceinline__ uint32_t scaled_bytes(uint32_t w, uint32_t k0, uint32_t k1, float s) {
    const uint64_t c = umma::pair(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440u | k0)), __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440u | k1)));
    uint64_t x;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(umma::add2(c, umma::pair(-8388736.0f, -8388736.0f))), "l"(umma::pair(s, s)));
    float lo, hi;
    umma::unpair(x, lo, hi);
    return umma::pack_bf16(lo, hi);
}
__device__ __forceinline__ void store16(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void store8(uint32_t a, uint32_t x, uint32_t y) {
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(a), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void store4(uint32_t a, uint32_t x) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(x) : "memory"); }

// Lanes of the fragment packing (g = token or dims, t): keys are stored 16 bytes a lane, eight lanes at a time, and rows g and g + 4 side by
// side have their pieces in different banks; values 8 bytes, sixteen lanes at a time, in the packing's own order.
struct Lanes {
    int g, t;
    bool keys;
    __device__ __forceinline__ Lanes(bool k, int lane) : keys(k) {
        g = k ? (lane >> 3) | (lane & 4) : lane >> 2;
        t = lane & 3;
    }
    __device__ __forceinline__ int source() const { return 4 * g + t; }
};

template <int kBits>
constexpr int kLowRounds = kBits / 2 < 1 ? 1 : kBits / 2;                       // 512-byte rounds of codes of a page's keys or values: 1, 2, 4
template <int kBits>
constexpr int kLowHalf = 512 * kLowRounds<kBits> + kLowScalesBytes;

// half 0: dims 0 .. 63, 1: 64 .. 127 (keys: rounds 2 j + h of dims 32 j ..; values: rounds 4 e + k of dims 64 e ..)
template <bool kKeys>
__device__ __forceinline__ void load_high(Raw &r, const uint8_t *tile, int half, int lane) {
    const uint4 *src = reinterpret_cast<const uint4 *>(tile + half * (kHighTileBytes / 2)) + Lanes(kKeys, lane).source();
#pragma unroll
    for (int i = 0; i < 4; i++) r.x[i] = __ldg(src + 32 * i);
}
// `row`: first row of the page in its block; the block is two pieces of 64 dims, 128 rows of 128 bytes with the 128-byte swizzle
template <bool kKeys>
__device__ __forceinline__ void store_high(const Raw &r, uint32_t block, int row, int half, int lane) {
    const Lanes l(kKeys, lane);
    block += half * kSub;
    if (kKeys) {
        const uint32_t base = block + (uint32_t)(row + l.g) * 128;
#pragma unroll
        for (int j = 0; j < 2; j++) {              // dims 64 half + 32 j + 8 t .. + 7 of tokens g and g + 8
            const uint4 a = r.x[2 * j], b = r.x[2 * j + 1];
            const uint32_t at = base + (((4 * j + l.t) ^ l.g) << 4);
            store16(at, a.x, a.z, b.x, b.z);
            store16(at + 1024, a.y, a.w, b.y, b.w);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; k++) {              // token 2 t + (k & 1) + 8 (k >> 1), dims 64 half + 4 g .. and 32 on
            const int tok = 2 * l.t + (k & 1), sw = tok & 7;
            const uint32_t base = block + (uint32_t)(row + tok + 8 * (k >> 1)) * 128 + 8 * (l.g & 1);
            store8(base + (((l.g >> 1) ^ sw) << 4), r.x[k].x, r.x[k].y);
            store8(base + (((4 + (l.g >> 1)) ^ sw) << 4), r.x[k].z, r.x[k].w);
        }
    }
}

template <int kBits, bool kKeys>
__device__ __forceinline__ void load_low(Raw &r, const uint8_t *half, int lane) {
    const Lanes l(kKeys, lane);
    const uint4 *src = reinterpret_cast<const uint4 *>(half) + l.source();
#pragma unroll
    for (int i = 0; i < kLowRounds<kBits>; i++) r.x[i] = __ldg(src + 32 * i);
    // Of the 64 scales a lane fetches two, and they go around: keys those of tokens g and g + 8 in group t; values those of tokens 2 t
    // and 2 t + 1, 8 on for g > 3, in group g & 3.
    const unsigned short *scales = reinterpret_cast<const unsigned short *>(half + 512 * kLowRounds<kBits>) + (kKeys ? 4 * l.g + l.t : 8 * l.t + 32 * (l.g >> 2) + (l.g & 3));
    r.s0 = __ldg(scales);
    r.s1 = __ldg(scales + (kKeys ? 32 : 4));
}

__device__ __forceinline__ uint32_t word_of(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

template <int kBits, bool kKeys>
__device__ __forceinline__ void store_low(const Raw &r, uint32_t block, int row, int lane) {
    const Lanes l(kKeys, lane);
    constexpr uint32_t kOffset = kBits == 4 ? 0x43084308u : 0x43024302u;         // bf16 136 or 130, twice: 128 + the code of zero
    constexpr uint32_t kMask = kBits == 4 ? 0x000F000Fu : 0x00030003u;
    const float f0 = half_bits(r.s0), f1 = half_bits(r.s1);
    if constexpr (kKeys) {
        uint32_t s_hi[2], s_lo[2];
        if constexpr (kBits < 8) {
            split_scales(f0, f0, s_hi[0], s_lo[0]);
            split_scales(f1, f1, s_hi[1], s_lo[1]);
        }
#pragma unroll
        for (int hi = 0; hi < 2; hi++) {           // tokens g, g + 8
            const uint32_t base = block + (uint32_t)(row + l.g + 8 * hi) * 128;
#pragma unroll
            for (int w = 0; w < 4; w++) {          // group w
                const int from = (lane & ~3) | w;
                if constexpr (kBits == 8) {        // dims 32 w + 8 k + 2 t, + 1
                    const float s = __shfl_sync(0xffffffffu, hi ? f1 : f0, from);
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const uint32_t c = word_of(r.x[w], k);
                        store4(base + (w >> 1) * kSub + (((4 * (w & 1) + k) ^ l.g) << 4) + 4 * l.t,
                               scaled_bytes(c, 2 * hi, 2 * hi + 1, s));
                    }
                } else {                           // dims 32 w + 8 t .. + 7
                    const uint32_t h = __shfl_sync(0xffffffffu, s_hi[hi], from), o = __shfl_sync(0xffffffffu, s_lo[hi], from);
                    const uint32_t c = kBits == 4 ? word_of(r.x[hi], w) : word_of(r.x[0], w) >> (8 * hi);
                    store16(base + (w >> 1) * kSub + (((4 * (w & 1) + l.t) ^ l.g) << 4), scaled_codes(c & kMask, kOffset, h, o),
                            scaled_codes((c >> kBits) & kMask, kOffset, h, o), scaled_codes((c >> 2 * kBits) & kMask, kOffset, h, o),
                            scaled_codes((c >> 3 * kBits) & kMask, kOffset, h, o));
                }
            }
        }
    } else {
        uint32_t s_hi, s_lo;
        if constexpr (kBits < 8) split_scales(f0, f1, s_hi, s_lo);
        // tokens 2 t (`even`) and 2 t + 1, 8 on for ps, dims 32 q + 4 g .. + 3
        const uint32_t even = block + (uint32_t)(row + 2 * l.t) * 128 + 8 * (l.g & 1);
#pragma unroll
        for (int ps = 0; ps < 2; ps++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const int from = 4 * (4 * ps + q) + l.t;
                const uint32_t to = even + (q >> 1) * kSub + 1024 * ps, chunk = 4 * (q & 1) + (l.g >> 1);
                const uint32_t at0 = to + ((chunk ^ (2 * l.t)) << 4), at1 = to + 128 + ((chunk ^ (2 * l.t + 1)) << 4);
                if constexpr (kBits == 8) {
                    const float s = __shfl_sync(0xffffffffu, f0, from), z = __shfl_sync(0xffffffffu, f1, from);
                    const uint32_t c = ps ? r.x[q].y : r.x[q].x, d = ps ? r.x[q].w : r.x[q].z;
                    store8(at0, scaled_bytes(c, 0, 2, s), scaled_bytes(d, 0, 2, s));
                    store8(at1, scaled_bytes(c, 1, 3, z), scaled_bytes(d, 1, 3, z));
                } else {                           // a dim of both tokens at a time, then sorted by token
                    const uint32_t h = __shfl_sync(0xffffffffu, s_hi, from), o = __shfl_sync(0xffffffffu, s_lo, from);
                    const uint32_t c = kBits == 4 ? word_of(r.x[ps], q) : word_of(r.x[0], q) >> (8 * ps);
                    uint32_t v[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) v[i] = scaled_codes((c >> kBits * i) & kMask, kOffset, h, o);
                    store8(at0, __byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410));
                    store8(at1, __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
                }
            }
    }
}

// ------------------------------------------------------------------------------------------------ attention

// kTiles 2: 64 tokens an item.  1: 32 / kCopies tokens, each row of S kCopies times in the tile.
// kPaged false: for calls in which no sequence has a history (kBits is not looked at).
template <int kTiles, int kCopies, bool kPaged>
struct __align__(16) PromptSmem {
    // Warps: softmax, four for control, fill (one for the keys and one for the values of each page of a block)
    static constexpr int kStages = 2, kSoft = 4 * kTiles, kFill = kPaged ? 2 * kBlockPages : 0, kThreads = 32 * (kSoft + 4 + kFill);
    uint8_t q[kTiles][kTileBytes], k[kStages][kTileBytes], v[kStages][kTileBytes];
    float share[kCopies > 1 ? 32 : 1][kTileRows];  // 32 dims of the copies' results on their way to one another
    float2 ml[kTileRows];
    uint64_t q_full, q_empty, k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
    // Of a tile; one tile: the first five of a place of S (pv_done: one tile only), so that whoever holds S of a block knows the phase before
    // to be over on the barriers of its place, and a wait by parity cannot take that phase, two blocks ago, for its own.
    uint64_t s_full[2], p_half[2], p_full[2], pv_half[2], pv_done[2], o_full[2], o_free[2];
    uint64_t item_full[2], item_empty[2], copies, drain;
    Item item[2];
    uint32_t tmem;
};

// Which of a block's key slots hold a token: pages 8 b .. of the history, of which the last of each kind may be partly filled.
struct Filled {
    int ph, pl, pages;
    uint32_t nh, nl, nw;
    __device__ __forceinline__ Filled(const volatile Item &it) : nh(it.nh), nl(it.nl), nw(it.nw) {
        ph = pages_of(nh);
        pl = pages_of(nl);
        pages = ph + pl + pages_of(nw);
    }
    __device__ __forceinline__ int of_page(int page) const {
        const int left = page < ph ? (int)nh - 16 * page : page < ph + pl ? (int)nl - 16 * (page - ph) : (int)nw - 16 * (page - ph - pl);
        return min(16, max(0, left));
    }
};

template <int kBits, int kTiles, int kCopies, bool kPaged>
__global__ void __launch_bounds__(PromptSmem<kTiles, kCopies, kPaged>::kThreads, 1)
prompt_kernel(const __grid_constant__ PromptParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
              const __grid_constant__ CUtensorMap map_v) {
    using namespace umma;
    using Smem = PromptSmem<kTiles, kCopies, kPaged>;
    constexpr int kStages = Smem::kStages, kSoft = Smem::kSoft, kFill = Smem::kFill;
    constexpr int kTokens = kTiles * kTileTokens / kCopies, kRows = kTokens * kGqa;
    extern __shared__ __align__(1024) uint8_t s_raw[];
    Smem &sm = *reinterpret_cast<Smem *>(s_raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    if (p.only >= 0) {
        pdl_wait();
        if (*p.ws.paged != p.only) return;         // the other variant's call
    }
    if (tid == 0) {
        bar_init(smem_u32(&sm.q_full), 1);
        bar_init(smem_u32(&sm.q_empty), 1);
        bar_init(smem_u32(&sm.copies), kSoft);
        bar_init(smem_u32(&sm.drain), 1);
        for (int i = 0; i < kStages; i++) {
            bar_init(smem_u32(&sm.k_full[i]), 1 + kFill / 2);
            bar_init(smem_u32(&sm.k_empty[i]), 1);
            bar_init(smem_u32(&sm.v_full[i]), 1 + kFill / 2);
            bar_init(smem_u32(&sm.v_empty[i]), 1);
        }
        for (int i = 0; i < 2; i++) {
            bar_init(smem_u32(&sm.s_full[i]), 1);
            bar_init(smem_u32(&sm.p_half[i]), 4);
            bar_init(smem_u32(&sm.p_full[i]), 4);
            bar_init(smem_u32(&sm.pv_half[i]), 1);
            bar_init(smem_u32(&sm.pv_done[i]), 1);
            bar_init(smem_u32(&sm.o_full[i]), 1);
            bar_init(smem_u32(&sm.o_free[i]), 4);
        }
        for (int i = 0; i < 2; i++) {
            bar_init(smem_u32(&sm.item_full[i]), 1);
            bar_init(smem_u32(&sm.item_empty[i]), kSoft + 2 + kFill);
        }
        bar_init_fence();
    }
    // Columns.  Two tiles: S (P over it) and O of tile 0, those of tile 1 128 behind.  One tile: two places of S, two of P, O
    constexpr uint32_t kS = 0, kP = kTiles == 2 ? 0 : 256, kO = kTiles == 2 ? 256 : 384;
    if (warp == kSoft) tmem_alloc(smem_u32(&sm.tmem), 512);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = sm.tmem;
    const long long limit = p.wait_cycles;
    bool ok = true;
    pdl_wait();                                    // the plan; and what came before it
    pdl_launch_dependents();
    if (tid == 0) p.ws.joins[blockIdx.x].rows = 0;
    // No history in the whole call: the fill warps leave, and the copies arrive in their place.
    const bool fills = kPaged && *p.ws.paged != 0;
    // the CTA's n-th item; false behind the last one or after a wait ran out
    auto next_item = [&](uint32_t n, Item &it) {
        const uint32_t slot = n & 1;
        ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.item_full[slot]), (n >> 1) & 1, limit)) && ok;
        if (!ok) return false;
        it = sm.item[slot];
        __syncwarp();
        if (lane == 0) bar_arrive(smem_u32(&sm.item_empty[slot]));
        return it.block >= 0;
    };
    auto tiles_of = [&](const Item &it) { return kTiles == 2 && it.block * kTokens + kTileTokens < it.nq ? 2 : 1; };

    // ================================================= fill
    auto fill = [&](int me) {                      // me: of the fill warps: page `slot` of each block, its keys or its values
        const int slot = me % kBlockPages, kv0 = me / kBlockPages;
        Item it;
        uint32_t g = 0;                            // blocks so far
        for (uint32_t n = 0; next_item(n, it); n++) {
            const Filled f(it);
            const uint32_t *tbl_high = p.tbl_high + (size_t)it.slot * p.max_pages, *tbl_low = p.tbl_low + (size_t)it.slot * p.max_pages;
            const uint32_t ring = p.ring_first + it.slot * p.ring_pages;
            const int b1 = min(it.b1, it.hist);
            // the pages of four blocks at a time, a lane each: their ids, then where this head's keys or values lie, and the kind
            auto ids = [&](int b) {
                const int page = 8 * b + lane;
                if (page >= f.pages || b >= b1) return 0u;
                return page < f.ph ? __ldg(tbl_high + page) : page < f.ph + f.pl ? __ldg(tbl_low + page - f.ph) : ring + (uint32_t)(page - f.ph - f.pl);
            };
            auto places = [&](int b, uint32_t id) {
                const int page = 8 * b + lane;
                if (page >= f.pages || b >= b1) return (uint64_t)kPageNone;
                const bool low = page >= f.ph && page < f.ph + f.pl;
                if (id >= (low ? p.cap_low : p.high_limit)) {  // never expected
                    atomicOr(p.status, PASK_DEV_INTERNAL);
                    return (uint64_t)kPageBad;
                }
                const uint8_t *at = low ? p.pool_low + (size_t)id * p.low_page_bytes + (size_t)it.head * p.low_head_bytes + kv0 * kLowHalf<kBits>
                                        : p.pool_high + (size_t)id * p.high_page_bytes + (size_t)it.head * kHighHeadBytes + kv0 * kHighTileBytes;
                return reinterpret_cast<uint64_t>(at) | (low ? kPageLow : kPageHigh);          // (16-byte aligned: the kind fits)
            };
            uint64_t window = places(it.b0, ids(it.b0));
            uint32_t ids_next = ids(it.b0 + 4);
            // What was stored makes room for the next page's pieces, which travel while its place in the block is waited for: two pieces of a
            // bf16 page, one of a low-precision one.
            Raw x, y;
            uint32_t kind = kPageNone;
            auto load = [&](int b, int kv) {       // the warp's page of block b
                const uint64_t e = __shfl_sync(0xffffffffu, window, 8 * ((b - it.b0) & 3) + slot);
                const uint8_t *at = reinterpret_cast<const uint8_t *>(e & ~(uint64_t)15);
                kind = (uint32_t)e & 15u;
                if (kind == kPageHigh) {
                    if (kv) { load_high<false>(x, at, 0, lane); load_high<false>(y, at, 1, lane); }
                    else { load_high<true>(x, at, 0, lane); load_high<true>(y, at, 1, lane); }
                } else if (kind == kPageLow) {
                    if (kv) load_low<kBits, false>(x, at, lane); else load_low<kBits, true>(x, at, lane);
                }
            };
            if (it.b0 < b1) load(it.b0, kv0);
            // (The warps pass through every block, those that are copied too: a barrier's phase is only told from the next but one
            // by who has to arrive on it.)
            for (int b = it.b0; b < it.b1; b++, g++) {
                const uint32_t st = g % kStages;
                // (A loop of one pass: with `kv` plainly the same throughout, keys and values get a loop each over all blocks, whose addresses do not
                // fit the registers: 5 drafted tokens of 64 sequences in 8 bits 173 us, 183 so.)
#pragma unroll 1
                for (int kv = kv0; kv < kv0 + 1; kv++) {
                    const uint32_t block = smem_u32(kv ? sm.v[st] : sm.k[st]);
                    if (g >= kStages) ok = __all_sync(0xffffffffu, bar_wait(smem_u32(kv ? &sm.v_empty[st] : &sm.k_empty[st]), (g / kStages - 1) & 1, limit));
                    if (!ok) break;
                    if (b < b1) {
                        if (kind == kPageHigh) {
                            if (kv) { store_high<false>(x, block, 16 * slot, 0, lane); store_high<false>(y, block, 16 * slot, 1, lane); }
                            else { store_high<true>(x, block, 16 * slot, 0, lane); store_high<true>(y, block, 16 * slot, 1, lane); }
                        } else if (kind == kPageLow) {
                            if (kv) store_low<kBits, false>(x, block, 16 * slot, lane); else store_low<kBits, true>(x, block, 16 * slot, lane);
                        }
                        // slots without a token: whatever the page holds there counts as zero
                        const int have = kind == kPageNone ? 16 : kind == kPageBad ? 0 : f.of_page(8 * b + slot);
                        if (have < 16) {
                            __syncwarp();
                            for (int e = lane; e < (16 - have) * 16; e += 32)
                                store16(block + ((e >> 3) & 1) * kSub + (uint32_t)(16 * slot + have + (e >> 4)) * 128 + (e & 7) * 16, 0, 0, 0, 0);
                        }
                        if (((b + 1 - it.b0) & 3) == 0) {
                            window = places(b + 1, ids_next);
                            ids_next = ids(b + 5);
                        }
                        if (b + 1 < b1) load(b + 1, kv);
                        fence_async_shared();
                        __syncwarp();
                    }
                    if (lane == 0) bar_arrive(smem_u32(kv ? &sm.v_full[st] : &sm.k_full[st]));
                }
                if (!ok) break;
            }
            if (!ok) break;
        }
    };

    // 384 threads x 168 registers at launch = 128 x (2 x 200 + 104) (more than a softmax thread needs, since rows go in halves); with fill warps 896 x 72 = 128 x (2 x 104 + 72 + 4 x 56), one tile: 768 x 80 =
    // 128 x (120 + 72 + 4 x 72)
    if (kPaged && warp >= kSoft + 4) {
        if constexpr (kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if constexpr (kPaged) if (fills) fill(warp - kSoft - 4);
    } else if (warp >= kSoft) {
        if constexpr (kPaged) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        if (warp == kSoft + 2) {
            // ================================================= items
            Walker walk;
            walk.init(p, kTokens, lane);
            bool live = true;
            for (uint32_t n = 0; live; n++) {
                const uint32_t slot = n & 1;
                Item it;
                live = walk.next(it, lane);
                if (!live) it.block = -1;
                if (n >= 2) ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.item_empty[slot]), ((n >> 1) - 1) & 1, limit));
                if (!ok) break;
                if (lane == 0) {
                    sm.item[slot] = it;
                    bar_arrive(smem_u32(&sm.item_full[slot]));
                }
                __syncwarp();
            }
        } else if (warp == kSoft + 1) {
            // ================================================= copies
            Item it;
            uint32_t g = 0, qc = 0;                // blocks, items so far
            const uint32_t qf = smem_u32(&sm.q_full);
            for (uint32_t n = 0; next_item(n, it); n++) {
                if (kPaged && !fills && lane == 0) bar_arrive(smem_u32(&sm.item_empty[n & 1]), kFill);
                if (qc > 0) ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.q_empty), (qc - 1) & 1, limit));
                if (!ok) break;
                const bool mine = elect_one();
                const int nt = tiles_of(it), first = it.q0 + it.block * kTokens;
                if (mine) {
                    bar_expect(qf, nt * kTileBytes + (qc == 0 ? p.surplus : 0u));
                    for (int t = 0; t < nt; t++)
                        for (int c = 0; c < 2 * kCopies; c++)
                            tile_load3(smem_u32(sm.q[t]) + (c & 1) * kSub + (c >> 1) * (kSub / kCopies), &map_q, 64 * (c & 1), kGqa * it.head,
                                       first + t * kTileTokens, qf);
                }
                qc++;
                for (int b = it.b0; b < it.b1; b++, g++) {
                    const uint32_t st = g % kStages, round = g / kStages;
                    const int row = it.q0 + (b - it.hist) * kBlockK;
#pragma unroll
                    for (int kv = 0; kv < 2; kv++) {
                        if (g >= kStages)
                            ok = __all_sync(0xffffffffu, bar_wait(smem_u32(kv ? &sm.v_empty[st] : &sm.k_empty[st]), (round - 1) & 1, limit));
                        if (!ok) break;
                        const uint32_t full = smem_u32(kv ? &sm.v_full[st] : &sm.k_full[st]), dst = smem_u32(kv ? sm.v[st] : sm.k[st]);
                        if (!mine) continue;
                        if (b < it.hist) { bar_arrive(full); continue; }
                        bar_expect(full, kTileBytes);
                        if (kPaged && !fills) bar_arrive(full, kFill / 2);
                        for (int c = 0; c < 2; c++) tile_load3(dst + c * kSub, kv ? &map_v : &map_k, 64 * c, it.head, row, full);
                    }
                    if (!ok) break;
                }
                if (!ok) break;
            }
            if (!ok) {                             // gave up: let the copies in flight land (bounded) before the CTA ends
                if (qc) bar_wait(qf, (qc - 1) & 1, limit);
                for (uint32_t b = g >= kStages ? g - kStages + 1 : 0; b <= g; b++) {
                    bar_wait(smem_u32(&sm.k_full[b % kStages]), (b / kStages) & 1, limit);
                    bar_wait(smem_u32(&sm.v_full[b % kStages]), (b / kStages) & 1, limit);
                }
            }
        } else if (warp == kSoft) {
            // ================================================= products
            constexpr uint32_t kIdS = instr(kTileRows, kBlockK, false, false), kIdO = instr(kTileRows, kDim, false, true);
            const bool mine = elect_one();
            const uint64_t dq = desc(smem_u32(sm.q[0]), 0, 1024), dk = desc(smem_u32(sm.k[0]), 0, 1024), dv = desc(smem_u32(sm.v[0]), kSub, 1024);
            Item it;
            uint32_t g = 0, qc = 0, pc[2] = {}, oc[2] = {};            // blocks, items, weights and items of each tile so far
            // (One thread issues: a branch around it, not a predicate on each product.  The predicate is taken for uniform over the warp and
            // looked at once; where the warp was not together, as behind a wait, products were issued once for each part of it.)
            auto scores = [&](int t, uint32_t st) {            // one tile: t is the place of S
                __syncwarp();
                if (mine) {
                    const uint64_t a = dq + (uint64_t)(kTiles == 2 ? t * kTileBytes >> 4 : 0), b = dk + (uint64_t)(st * (kTileBytes >> 4));
#pragma unroll
                    for (int k = 0; k < 8; k++)
                        mma_ss(tmem + kS + t * 128, a + (k >> 2) * (kSub >> 4) + 2 * (k & 3), b + (k >> 2) * (kSub >> 4) + 2 * (k & 3), kIdS, k > 0, true);
                    commit(smem_u32(&sm.s_full[t]));
                }
                __syncwarp();
            };
            auto values = [&](int t, uint32_t st, bool fresh, int from, int to) {          // keys 16 from .. 16 to - 1
                __syncwarp();
                if (mine) {
                    const uint64_t b = dv + (uint64_t)(st * (kTileBytes >> 4));
#pragma unroll
                    for (int k = 0; k < 8; k++)
                        if (k >= from && k < to)
                            mma_ts(tmem + kO + (kTiles == 2 ? t * 128 : 0), tmem + kP + t * (kTiles == 2 ? 128 : 64) + k * 8, b + 128 * k, kIdO,
                                   k > 0 || !fresh, true);
                }
                __syncwarp();
            };
            // the call's own rows behind the last token in its step of 16 count as zero
            auto zero_rows = [&](uint32_t st, int left, int steps) {
                if (16 * steps <= left) return;
                for (int e = lane; e < (16 * steps - left) * 16; e += 32)
                    *reinterpret_cast<uint4 *>(sm.v[st] + ((e >> 3) & 1) * kSub + (left + (e >> 4)) * 128 + (e & 7) * 16) = make_uint4(0, 0, 0, 0);
                fence_async_shared();
                __syncwarp();
            };
            for (uint32_t n = 0; next_item(n, it); n++) {
                const int nt = __shfl_sync(0xffffffffu, tiles_of(it), 0), nb = __shfl_sync(0xffffffffu, it.b1 - it.b0, 0);
                ok = bar_wait(smem_u32(&sm.q_full), qc & 1, limit);
                qc++;
                ok = bar_wait(smem_u32(&sm.k_full[g % kStages]), (g / kStages) & 1, limit) && ok;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                fence_after();
                {
                    const uint32_t st = __shfl_sync(0xffffffffu, g % kStages, 0);
                    scores(kTiles == 2 ? 0 : __shfl_sync(0xffffffffu, g & 1, 0), st);
                    if (kTiles == 2 && nt == 2) scores(1, st);
                    if (mine) {
                        commit(smem_u32(&sm.k_empty[st]));
                        if (nb == 1) commit(smem_u32(&sm.q_empty));
                    }
                    __syncwarp();
                }
                const int pages = pages_of(it.nh) + pages_of(it.nl) + pages_of(it.nw);
                for (int j = 0; j < nb; j++, g++) {
                    // slots of the block with a token, and of those the ones that the item looks at
                    const int b = it.b0 + j, left = b < it.hist ? (pages - kBlockPages * b) * kPageTokens : it.nq - (b - it.hist) * kBlockK;
                    const int seen = b < it.hist ? left : min(it.nq, (it.block + 1) * kTokens) - (b - it.hist) * kBlockK;
                    const int steps = __shfl_sync(0xffffffffu, (min(kBlockK, seen) + 15) / 16, 0);
                    const uint32_t st = __shfl_sync(0xffffffffu, g % kStages, 0), ph = (g / kStages) & 1;
                    const uint32_t st1 = __shfl_sync(0xffffffffu, (g + 1) % kStages, 0), ph1 = ((g + 1) / kStages) & 1;
                    if constexpr (kTiles == 1) {
                        // S of the next block goes to the other place while the softmax has this one
                        const int at = __shfl_sync(0xffffffffu, g & 1, 0);
                        if (j + 1 < nb) {
                            ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.k_full[st1]), ph1, limit));
                            if (!ok) break;
                            fence_after();
                            scores(at ^ 1, st1);
                            if (mine) {
                                commit(smem_u32(&sm.k_empty[st1]));
                                if (j + 2 == nb) commit(smem_u32(&sm.q_empty));
                            }
                            __syncwarp();
                        }
                        if (j == 0) {
                            if (oc[0] > 0) ok = bar_wait(smem_u32(&sm.o_free[0]), (oc[0] - 1) & 1, limit);
                            oc[0]++;
                        }
                        ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.v_full[st]), ph, limit) && ok);
                        if (!ok) break;
                        zero_rows(st, left, steps);
                        if constexpr (kCopies == 1) {
                            ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.p_half[at]), (g >> 1) & 1, limit));
                            if (!ok) break;
                            fence_after();
                            values(at, st, j == 0, 0, min(4, steps));
                            if (mine) commit(smem_u32(&sm.pv_half[at]));
                        }
                        ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.p_full[at]), (g >> 1) & 1, limit));
                        if (!ok) break;
                        fence_after();
                        values(at, st, j == 0, kCopies == 1 ? 4 : 0, steps);
                        if (mine) {
                            commit(smem_u32(&sm.v_empty[st]));
                            commit(smem_u32(&sm.pv_done[at]));
                            if (j + 1 == nb) commit(smem_u32(&sm.o_full[0]));
                        }
                        __syncwarp();
                        continue;
                    }
                    bool have_k = false;
                    ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.v_full[st]), ph, limit));
                    if (!ok) break;
                    zero_rows(st, left, steps);
#pragma unroll
                    for (int t = 0; t < kTiles; t++) {
                        if (t >= nt) continue;
                        if (j == 0) {              // the item before has been read out of O
                            if (oc[t] > 0) ok = bar_wait(smem_u32(&sm.o_free[t]), (oc[t] - 1) & 1, limit) && ok;
                            oc[t]++;
                        }
                        ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.p_half[t]), pc[t] & 1, limit) && ok);
                        if (!ok) break;
                        fence_after();
                        values(t, st, j == 0, 0, min(4, steps));
                        if (mine) commit(smem_u32(&sm.pv_half[t]));
                        ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.p_full[t]), pc[t] & 1, limit));
                        if (!ok) break;
                        pc[t]++;
                        fence_after();
                        values(t, st, false, 4, steps);
                        if (mine) {
                            if (t + 1 == nt) commit(smem_u32(&sm.v_empty[st]));
                            if (j + 1 == nb) commit(smem_u32(&sm.o_full[t]));
                        }
                        __syncwarp();
                        if (j + 1 < nb) {
                            if (!have_k) {
                                ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.k_full[st1]), ph1, limit));
                                if (!ok) break;
                                fence_after();
                                have_k = true;
                            }
                            scores(t, st1);
                        }
                    }
                    if (!ok) break;
                    if (mine) {
                        if (j + 1 < nb) commit(smem_u32(&sm.k_empty[st1]));
                        if (j + 2 == nb) commit(smem_u32(&sm.q_empty));
                    }
                    __syncwarp();
                }
                if (!ok) break;
            }
            if (!ok) {                             // gave up: the products in flight end before tensor memory is freed
                if (mine) commit(smem_u32(&sm.drain));
                bar_wait(smem_u32(&sm.drain), 0, limit);
            }
            __syncwarp();
        }
    } else {
        if constexpr (!kPaged) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        else if constexpr (kTiles == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 120;");
        // ================================================= softmax: thread = row, or one of a row's copies with its share of the keys
        constexpr int kCols = kBlockK / kCopies, kCopyRows = kTileRows / kCopies, kPart = kCols < 64 ? kCols : 64, kParts = kCols / kPart;
        const int t = warp >> 2, copy = (tid & (kTileRows - 1)) / kCopyRows;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, base = tmem + lanes + (kTiles == 2 ? t * 128 : copy * kCols);
        const uint32_t p_base = tmem + lanes + kP + (kTiles == 2 ? t * 128 : copy * (kCols / 2)), o_base = tmem + lanes + kO + t * 128;
        const uint32_t s_full = smem_u32(&sm.s_full[t]);
        const int row_in = t * kTileRows + (tid & (kCopyRows - 1));
        uint32_t sc = 0, ic = 0, cc = 0;           // blocks of this tile (S, P and P V alike), items, exchanges between copies so far
        // a row's copies among themselves (all softmax warps)
        auto meet = [&] {
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(&sm.copies));
            ok = __all_sync(0xffffffffu, ok && bar_wait(smem_u32(&sm.copies), cc++ & 1, limit));
            return ok;
        };
        if constexpr (kCopies > 1) {               // weights of the other copies' keys: zero for good
            const uint32_t zero[16] = {};
#pragma unroll
            for (int c = 0; c < 8; c++) tmem_st16(tmem + lanes + kP + 16 * c, zero);
            tmem_wait_st();
        }
        // (the item stays in shared memory until its end: a copy of it and the row of S do not fit the registers)
        for (uint32_t n = 0;; n++) {
            if (n > 0) {
                __syncwarp();
                if (lane == 0) bar_arrive(smem_u32(&sm.item_empty[(n - 1) & 1]));
            }
            ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.item_full[n & 1]), (n >> 1) & 1, limit)) && ok;
            const volatile Item &it = sm.item[n & 1];
            if (!ok || it.block < 0) break;
            const int i = it.block * kTokens + row_in / kGqa, hist = it.hist, b0 = it.b0;
            const bool here = t == 0 || it.block * kTokens + kTileTokens < it.nq, live = i < it.nq;
            const int nb = here ? it.b1 - b0 : 0;
            const bool idle = !__any_sync(0xffffffffu, live);          // no row of this warp is one
            int pages, own = min((int)it.nq, (it.block + 1) * kTokens);            // pages of the history, own tokens that the item looks at
            int part_h, part_l, part_w;            // the blocks with slots without a token (-1: none): ends of the streams and of the history
            {
                const Filled f(it);
                part_h = f.nh & 15 ? (f.ph - 1) >> 3 : -1;
                part_l = f.nl & 15 ? (f.ph + f.pl - 1) >> 3 : -1;
                part_w = f.nw & 15 || f.pages & 7 ? (f.pages - 1) >> 3 : -1;
                pages = f.pages;
            }
            float m = -INFINITY, l = 0.0f;
            for (int j = 0; j < nb; j++, sc++) {
                const int b = b0 + j;
                const uint32_t place = kTiles == 2 ? 0 : sc & 1;
                ok = kTiles == 2 ? bar_wait(s_full, sc & 1, limit) : bar_wait(smem_u32(&sm.s_full[place]), (sc >> 1) & 1, limit);
                if (!__all_sync(0xffffffffu, ok)) break;
                const uint32_t at = kTiles == 2 ? t : place;               // of p_half, p_full
                if (idle) {
                    if (lane == 0) {
                        if (kParts == 2) bar_arrive(smem_u32(&sm.p_half[at]));
                        bar_arrive(smem_u32(&sm.p_full[at]));
                    }
                    continue;
                }
                fence_after();
                const bool causal = b >= hist;     // the call's own tokens: those up to the row's
                const int left = !causal ? kCols : live ? i + 1 - (b - hist) * kBlockK - copy * kCols : 0;
                uint32_t filled = 0xFFFFu;         // of page lane & 7 of the block
                bool masked = __any_sync(0xffffffffu, left < kCols);
                if (b == part_h || b == part_l || b == part_w) {
                    masked = true;
                    filled = (1u << Filled(it).of_page(8 * b + (lane & 7))) - 1u;
                }
                // 128 columns go in two halves: the product over the first 64 keys runs beside the exponentials of the others
                const int seen = causal ? own - (b - hist) * kBlockK : (pages - kBlockPages * b) * kPageTokens;
#pragma unroll 1
                for (int part = 0; part < kParts; part++) {
                    const int from = part * kPart;
                    if (kParts == 2 && from >= seen) {         // no row looks at the second half: no product takes it
                        __syncwarp();
                        if (lane == 0) bar_arrive(smem_u32(&sm.p_full[at]));
                        break;
                    }
                    float x[kPart];
#pragma unroll
                    for (int c = 0; c < kPart / 32; c++) {
                        uint32_t r[32];
                        tmem_ld32(base + kS + place * 128 + from + 32 * c, r);
#pragma unroll
                        for (int e = 0; e < 32; e++) x[32 * c + e] = __uint_as_float(r[e]);
                    }
                    tmem_wait_ld();
                    if (masked) {
#pragma unroll
                        for (int pg = 0; pg < kPart / 16; pg++) {
                            const uint32_t bits = __shfl_sync(0xffffffffu, filled, pg + (copy * kCols + from) / 16);
#pragma unroll
                            for (int e = 0; e < 16; e++) if (16 * pg + e >= left - from || !((bits >> e) & 1)) x[16 * pg + e] = -INFINITY;
                        }
                    }
                    float a0 = max3(x[0], x[1], x[2]), a1 = max3(x[3], x[4], x[5]), a2 = fmaxf(x[6], x[7]);
#pragma unroll
                    for (int e = 8; e < kPart; e += 6) {
                        a0 = max3(a0, x[e], x[e + 1]);
                        if (e + 2 < kPart) a1 = max3(a1, x[e + 2], x[e + 3]);
                        if (e + 4 < kPart) a2 = max3(a2, x[e + 4], x[e + 5]);
                    }
                    const float top = max3(a0, a1, a2) * kScaleLog2;
                    const bool raise = top > m + kLazy;
                    if (__any_sync(0xffffffffu, raise)) {
                        const float d = raise ? ex2(m - top) : 1.0f;
                        if (raise) { m = top; l *= d; }
                        if (j > 0 || part > 0) {   // O so far, in the new reference, when the last product into it is done
                            // (two tiles: this S was issued behind P V of the block before.  One: behind that of two blocks ago)
                            if (part > 0) ok = kTiles == 2 ? bar_wait(smem_u32(&sm.pv_half[t]), sc & 1, limit) : bar_wait(smem_u32(&sm.pv_half[place]), (sc >> 1) & 1, limit);
                            else if (kTiles == 1) ok = bar_wait(smem_u32(&sm.pv_done[place ^ 1]), ((sc - 1) >> 1) & 1, limit);
                            ok = __all_sync(0xffffffffu, ok);
                            if (!ok) break;
                            fence_after();
#pragma unroll 1
                            for (int c = 0; c < 8; c++) {
                                uint32_t r[16];
                                tmem_ld16(o_base + 16 * c, r);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 16; e++) r[e] = __float_as_uint(__uint_as_float(r[e]) * d);
                                tmem_st16(o_base + 16 * c, r);
                            }
                        }
                    }
                    const float ref = m == -INFINITY ? 0.0f : m;           // a row that has seen no key yet
                    const uint64_t scale2 = pair(kScaleLog2, kScaleLog2), ref2 = pair(-ref, -ref);
                    uint64_t l2 = pair(0.0f, 0.0f);
#pragma unroll
                    for (int c = 0; c < kPart / 32; c++) {
                        uint32_t r[16];
#pragma unroll
                        for (int e = 0; e < 16; e++) {
                            float u, v;
                            unpair(fma2(pair(x[32 * c + 2 * e], x[32 * c + 2 * e + 1]), scale2, ref2), u, v);
                            u = ex2(u);
                            v = ex2(v);
                            l2 = add2(l2, pair(u, v));
                            r[e] = pack_bf16(u, v);
                        }
                        tmem_st16(p_base + place * 64 + from / 2 + 16 * c, r);
                    }
                    tmem_wait_st();
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_u32(part + 1 < kParts ? &sm.p_half[at] : &sm.p_full[at]));
                    float l0, l1;
                    unpair(l2, l0, l1);
                    l += l0 + l1;
                }
                if (!ok) break;
            }
            ok = __all_sync(0xffffffffu, ok);
            if (ok && here) ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.o_full[t]), ic++ & 1, limit));
            if (!ok) break;
            fence_after();
            const size_t heads = (size_t)kGqa * p.n_kv, row = (size_t)(it.q0 + i) * heads + kGqa * it.head + (row_in & 3);
            const bool whole = it.first == it.last;
            const size_t part = 2 * (size_t)blockIdx.x + (it.first == (int)blockIdx.x);      // the place of a CTA's part of an item
            if constexpr (kCopies > 1) {
                // Each copy brings its sums to the row's reference; 32 dims at a time they meet in shared memory.
                sm.ml[tid] = make_float2(m, l);
                if (!meet()) break;
                float top = -INFINITY, sum = 0.0f;
#pragma unroll
                for (int c = 0; c < kCopies; c++) top = fmaxf(top, sm.ml[c * kCopyRows + row_in].x);
                const float ref = top == -INFINITY ? 0.0f : top, mine = ex2(m - ref);
#pragma unroll
                for (int c = 0; c < kCopies; c++) {
                    const float2 y = sm.ml[c * kCopyRows + row_in];
                    sum += y.y * ex2(y.x - ref);
                }
                const float inv = live ? 1.0f / sum : 0.0f;
#pragma unroll 1
                for (int d0 = 0; d0 < kDim; d0 += 32) {
                    __syncwarp();
                    uint32_t r[32];
                    tmem_ld32(o_base + d0, r);
                    tmem_wait_ld();
                    if (d0 > 0 && !meet()) break;
#pragma unroll
                    for (int e = 0; e < 32; e++) sm.share[e][tid] = __uint_as_float(r[e]) * mine;
                    if (!meet()) break;
                    constexpr int kOwn = 32 / kCopies;         // dims of the row that this copy writes
                    float y[kOwn];
#pragma unroll
                    for (int e = 0; e < kOwn; e++) {
                        y[e] = 0.0f;
#pragma unroll
                        for (int c = 0; c < kCopies; c++) y[e] += sm.share[copy * kOwn + e][c * kCopyRows + row_in];
                    }
                    const int d = d0 + copy * kOwn;
                    if (whole && live) {
#pragma unroll
                        for (int e = 0; e < kOwn; e += 8)
                            *reinterpret_cast<uint4 *>(p.out + row * kDim + d + e) =
                                make_uint4(pack_bf16(y[e] * inv, y[e + 1] * inv), pack_bf16(y[e + 2] * inv, y[e + 3] * inv),
                                           pack_bf16(y[e + 4] * inv, y[e + 5] * inv), pack_bf16(y[e + 6] * inv, y[e + 7] * inv));
                    } else if (live) {
#pragma unroll
                        for (int e = 0; e < kOwn; e += 4)
                            __stcg(p.ws.o + (part * kRows + row_in) * (kDim / 4) + (d + e) / 4, make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]));
                    }
                }
                if (!ok) break;
                if (live && copy == 0) {
                    if (!whole) __stcg(p.ws.ml + part * kRows + row_in, make_float2(top, sum));
                    else if (p.lse) p.lse[row] = (top + log2f(sum)) * 0.69314718055994531f;
                }
            } else
            if (here && !idle) {
                const float inv = live ? 1.0f / l : 0.0f;
#pragma unroll
                for (int c = 0; c < 8; c++) {
                    uint32_t r[16];
                    tmem_ld16(o_base + 16 * c, r);
                    tmem_wait_ld();
                    if (whole && live) {
                        uint4 *dst = reinterpret_cast<uint4 *>(p.out + row * kDim + 16 * c);
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            uint32_t y[4];
#pragma unroll
                            for (int e = 0; e < 4; e++)
                                y[e] = pack_bf16(__uint_as_float(r[8 * h + 2 * e]) * inv, __uint_as_float(r[8 * h + 2 * e + 1]) * inv);
                            dst[h] = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                    } else if (live) {
#pragma unroll
                        for (int h = 0; h < 4; h++)
                            __stcg(p.ws.o + (part * kRows + row_in) * (kDim / 4) + 4 * c + h,
                                   make_float4(__uint_as_float(r[4 * h]), __uint_as_float(r[4 * h + 1]), __uint_as_float(r[4 * h + 2]), __uint_as_float(r[4 * h + 3])));
                    }
                }
                if (live) {
                    if (!whole) __stcg(p.ws.ml + part * kRows + row_in, make_float2(m, l));
                    else if (p.lse) p.lse[row] = (m + log2f(l)) * 0.69314718055994531f;
                }
            }
            if (here) {
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_u32(&sm.o_free[t]));
            }
            if (tid == 0 && !whole && it.first == (int)blockIdx.x) {
                Join &to = p.ws.joins[blockIdx.x];
                to.row = it.q0 + it.block * kTokens;
                to.rows = min(kRows, (it.nq - it.block * kTokens) * kGqa);
                to.head = it.head; to.first = it.first; to.last = it.last;
            }
        }
    }
    if (!ok && lane == 0) atomicOr(p.status, PASK_DEV_TIMEOUT);
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == kSoft) tmem_free(tmem, 512);
}

// The rows of the items in parts, a warp each in turn: the parts' weights (a lane a part), then the sums, four dims a lane, over the parts
// in order.
constexpr int kJoinThreads = 512, kJoinCtas = 2, kMaxGrid = 256;
__global__ void __launch_bounds__(kJoinThreads)
prompt_join_kernel(PromptWorkspace ws, int grid, int rows_max, int n_kv, __nv_bfloat16 *__restrict__ out, float *__restrict__ lse) {
    using namespace umma;
    __shared__ int s_end[kMaxGrid];                // rows of the items up to this one
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_launch_dependents();
    pdl_wait();
    if (warp == 0) {
        int carry = 0;
        for (int b = 0; b < grid; b += 32) {
            int inc = b + lane < grid ? ws.joins[b + lane].rows : 0;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, inc, d);
                if (lane >= d) inc += o;
            }
            if (b + lane < grid) s_end[b + lane] = carry + inc;
            carry += __shfl_sync(0xffffffffu, inc, 31);
        }
    }
    __syncthreads();
    const size_t heads = (size_t)kGqa * n_kv;
    for (int at = blockIdx.x * (kJoinThreads / 32) + warp; at < s_end[grid - 1]; at += gridDim.x * (kJoinThreads / 32)) {
        int lo = 0, hi = grid - 1;                 // the first item that ends behind row `at`
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (s_end[mid] > at) hi = mid; else lo = mid + 1;
        }
        const Join j = ws.joins[lo];
        const int r = at - (lo ? s_end[lo - 1] : 0), parts = j.last - j.first + 1;
        // a CTA's part of the item: place 2 c, the first one's 2 c + 1
        auto place = [&](int c) { return (2 * (size_t)(j.first + c) + (c == 0)) * rows_max + r; };
        float top = -INFINITY, sum = 0.0f;
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int c0 = 0; c0 < parts; c0 += 32) {
            const int n = min(32, parts - c0);
            const float2 ml = lane < n ? __ldcg(ws.ml + place(c0 + lane)) : make_float2(-INFINITY, 0.0f);
            float next = ml.x;
#pragma unroll
            for (int d = 16; d; d >>= 1) next = fmaxf(next, __shfl_xor_sync(0xffffffffu, next, d));
            next = fmaxf(next, top);
            const float ref = next == -INFINITY ? 0.0f : next, old = ex2(top - ref), w = ex2(ml.x - ref);
            float share = ml.y * w;
#pragma unroll
            for (int d = 16; d; d >>= 1) share += __shfl_xor_sync(0xffffffffu, share, d);
            top = next;
            sum = sum * old + share;
            x.x *= old; x.y *= old; x.z *= old; x.w *= old;
#pragma unroll 8
            for (int c = 0; c < n; c++) {
                const float4 y = __ldcg(ws.o + place(c0 + c) * (kDim / 4) + lane);
                const float v = __shfl_sync(0xffffffffu, w, c);
                x.x += y.x * v; x.y += y.y * v; x.z += y.z * v; x.w += y.w * v;
            }
        }
        const float inv = 1.0f / sum;
        const size_t to = (size_t)(j.row + r / kGqa) * heads + kGqa * j.head + (r & 3);
        *reinterpret_cast<uint2 *>(out + to * kDim + 4 * lane) = make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
        if (lane == 0 && lse) lse[to] = (top + log2f(sum)) * 0.69314718055994531f;
    }
}

template <int kBits, int kTiles, int kCopies, bool kPaged>
pask_status_t launch(const PromptParams &p, const CUtensorMap &map_q, const CUtensorMap &map_k, const CUtensorMap &map_v, int dev, cudaStream_t stream) {
    constexpr int kSmem = (int)sizeof(PromptSmem<kTiles, kCopies, kPaged>);
    static_assert(kSmem <= 232448, "shared memory of a CTA");
    static bool granted[64] = {};                  // a property of (device, kernel)
    if (!granted[dev]) {
        if (cudaFuncSetAttribute(prompt_kernel<kBits, kTiles, kCopies, kPaged>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) return PASK_ERR_CUDA;
        granted[dev] = true;
    }
    return launch_pdl(prompt_kernel<kBits, kTiles, kCopies, kPaged>, dim3(p.grid), dim3(PromptSmem<kTiles, kCopies, kPaged>::kThreads), kSmem, stream, p, map_q,
                      map_k, map_v) == cudaSuccess
               ? PASK_OK
               : PASK_ERR_CUDA;
}

template <int kTiles, int kCopies>
pask_status_t launch_bits(uint32_t bits, const PromptParams &p, const CUtensorMap &map_q, const CUtensorMap &map_k, const CUtensorMap &map_v, int dev,
                          cudaStream_t stream) {
    return bits == 8 ? launch<8, kTiles, kCopies, true>(p, map_q, map_k, map_v, dev, stream)
           : bits == 2 ? launch<2, kTiles, kCopies, true>(p, map_q, map_k, map_v, dev, stream)
                       : launch<4, kTiles, kCopies, true>(p, map_q, map_k, map_v, dev, stream);
}

// Tokens of an item: 64 (two tiles), or 32, 16, 8 (one tile, its rows once, twice, four times), by the mean of a sequence: the pages are read
// and expanded once an item, so that one item holds all of its tokens, and the fewer there are, the more threads share a row.  With 8, 16, 32, 64
// tokens: 5 tokens of 64 sequences 182, 194, 209, 228 us; 17 tokens behind 32K rows 58, 48, 38, 41; chunks of 33 - 120 behind 3K 70, 56, 47,
// 47; of 512 behind 9K 3022, 1606, 961, 733; prompts of 8K without history 5208, 2767, 1771, 1426.
int tokens_for(int n_seqs, int total_tokens) {
    const long long n = ((long long)total_tokens + n_seqs - 1) / n_seqs;
    return n <= 8 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : 64;
}

// Mean tokens of a sequence from which the variant without fill warps is launched beside the other.  Without history, the one with fill warps
// alone and both: one prompt of 1024 tokens 36, 39 us; of 2048 79, 78; four of 1400 112, 112; of 2048 191, 187; of 4096 - 8192 1470, 1415.  With a
// history, with fill warps and with one of the control warps in their place: chunks of 512 behind 9K 733, 3894.
constexpr int kBothFrom = 2048;

}  // namespace

static int prompt_grid(const pask_cache *c) { return c->sm_count < kMaxGrid ? c->sm_count : kMaxGrid; }

size_t prompt_workspace_bytes(const pask_cache *c, int n_seqs, int total_tokens) {
    return carve(n_seqs, prompt_grid(c), tokens_for(n_seqs, total_tokens) * kGqa, nullptr, nullptr);
}

pask_status_t launch_prompt(pask_cache *c, int layer, int n_seqs, int total_tokens, const int32_t *seq_ids, const int32_t *cu_tokens, const void *q,
                            const void *k, const void *v, void *out, float *lse, void *workspace, cudaStream_t stream) {
    const int n_kv = c->desc.n_kv_heads, tokens = tokens_for(n_seqs, total_tokens);
    CUtensorMap map_q{}, map_k{}, map_v{};
    const size_t head = kDim * 2;
    if (!encode_heads(&map_q, q, kDim, kGqa * n_kv, total_tokens, head, head * kGqa * n_kv, kGqa, tokens < kTileTokens ? tokens : kTileTokens) ||
        !encode_heads(&map_k, k, kDim, n_kv, total_tokens, head, head * n_kv, 1, kBlockK) ||
        !encode_heads(&map_v, v, kDim, n_kv, total_tokens, head, head * n_kv, 1, kBlockK))
        return PASK_ERR_CUDA;
    const DevCache &d = c->dev;
    PromptParams p{};
    carve(n_seqs, prompt_grid(c), tokens * kGqa, static_cast<uint8_t *>(workspace), &p.ws);
    p.pool_high = d.pool_high;
    p.pool_low = d.pool_low;
    p.tbl_high = d.tbl_high;
    p.tbl_low = d.tbl_low;
    p.status = d.ctrl + kCtrlStatus;
    p.high_page_bytes = d.high_page_bytes;
    p.low_page_bytes = d.low_page_bytes;
    p.low_head_bytes = d.low_head_bytes;
    p.cap_low = d.cap_low;
    p.high_limit = d.high_limit;
    p.ring_first = d.cap_high;
    p.ring_pages = d.window / kPageTokens;
    p.max_pages = d.max_pages;
    p.n_kv = n_kv;
    p.n_seqs = n_seqs;
    p.grid = prompt_grid(c);
    p.out = static_cast<__nv_bfloat16 *>(out);
    p.lse = lse;
    p.wait_cycles = c->wait_cycles;
    p.surplus = c->wait_test_surplus;
    if (launch_pdl(prompt_plan_kernel, dim3(1), dim3((n_seqs + 31) / 32 * 32), 0, stream, d, layer, n_seqs, total_tokens, seq_ids, cu_tokens, p.ws, p.grid,
                   tokens, static_cast<uint4 *>(out), lse) != cudaSuccess)
        return PASK_ERR_CUDA;
    // Long sequences: with fill warps and without, and the one that the plan's finding is not for leaves at once (the host knows neither
    // what the cache holds nor what it will hold when a graph is replayed).
    const bool both = tokens == 64 && total_tokens / n_seqs >= kBothFrom;
    p.only = both ? 0 : -1;
    pask_status_t ok = both ? launch<4, 2, 1, false>(p, map_q, map_k, map_v, c->device, stream) : PASK_OK;
    if (ok != PASK_OK) return ok;
    p.only = both ? 1 : -1;
    const auto fn = tokens == 64 ? launch_bits<2, 1> : tokens == 32 ? launch_bits<1, 1> : tokens == 16 ? launch_bits<1, 2> : launch_bits<1, 4>;
    ok = fn(d.low_bits, p, map_q, map_k, map_v, c->device, stream);
    if (ok != PASK_OK) return ok;
    return launch_pdl(prompt_join_kernel, dim3(kJoinCtas * c->sm_count), dim3(kJoinThreads), 0, stream, p.ws, p.grid, tokens * kGqa, n_kv, p.out, lse) ==
                   cudaSuccess
               ? PASK_OK
               : PASK_ERR_CUDA;
}

}  // namespace pask
