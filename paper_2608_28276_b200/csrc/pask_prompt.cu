// pask_prompt_attention_latent: causal attention of a ragged batch of prompts (or prompt chunks behind a history) with the
// latent rows expanded to keys and values per head.
//
// Per head: S = Q K^T over 192 dims (128 expanded + 64 rotary that all heads share), P = softmax(scale S), O = P V over 128
// dims: 640 operations per (query, visible key), and a key block of 128 keys (80 KB) serves 256 queries, so the tensor core
// bounds it: per block 2 x 12 products of 128 x 128 x 16 for S and 2 x 8 for O, 40 x 64 = 2560 cycles (tcgen05, fp32 sums in
// tensor memory; see pask_umma.h).  The 32768 exponentials of a block take the special-function units 2048 cycles.
//
// A CTA works on 256 queries of one head as two tiles of 128 rows, in turn: while the softmax warps of one tile turn its S into
// P, the tensor core works for the other.
//   warps 0-3, 4-7   softmax of tile 0, 1: a thread has a query (its row of S in registers, no exchange between lanes); P goes
//                    back to tensor memory over S, in bf16, as the left operand of P V.  The reference maximum of a row moves
//                    only when a score exceeds it by more than 2^8, so that O is rarely rescaled.  Then the row's result.
//   warp 8           products, in the order  P V of tile t, block j;  Q K^T of tile t, block j + 1;  the other tile
//   warp 9           copies: queries; key blocks (three pieces of 16 KB: 128 expanded and 64 rotary dims) and value blocks (two
//                    pieces of 64 keys) in turn into a ring of eight pieces: a block's keys and values and the next one's keys
//   warp 10          the next item: blocks of 256 queries with the most visible keys first; a CTA that is done takes over one
//                    that has not started (cluster launch control), so the tail evens out without a counter in memory
// Shared memory: Q 96 KB + ring 128 KB.  (Two stages of keys and one of values in the same space let P V wait for the copy of
// its values, which can only start when the product before it is done.)  Tensor memory: S 2 x 128 columns, O 2 x 128 columns.
//
// Measured: 4123 cycles for a block of 128 keys, 1.6 of the bound; the chain S - exponentials - P - P V of a tile is longer than
// the other tile's products.  Two threads a query (16 softmax warps) took as long: 155 us against 150 for 4 x 500 queries
// behind 3333 keys, 32 heads (the captured call replayed back to back; called on its own, L2 flushed, 180).  4 prompts of 4 to 8
// thousand, 16 heads: 750 to 820 us, replayed or called, 1.0 to 1.1 PFLOP/s at the clock that the power limit leaves (681 at
// 1.6 GHz, in a short burst).
//
// Rounding: S, O and the sums are fp32; a weight is rounded to bf16 once (half a step, 2^-8 of it), as an operand of a product with
// bf16 values.  What the rounding left would take a second P V, 1024 cycles more a block of keys.
//
// kSplit > 1: a cluster of kSplit CTAs shares an item, each a range of its key blocks; the unscaled results meet in shared
// memory, each CTA joining the rows of 256 / kSplit queries (no workspace, a fixed order).  No stealing there.
#include <cuda.h>
#include <cuda_bf16.h>

#include <atomic>
#include <cmath>

#include "pask_internal.h"
#include "pask_umma.h"

namespace pask {

namespace {

constexpr int kNope = 128, kRope = 64, kQk = kNope + kRope, kV = 128;
constexpr int kTileQ = 128, kBlockQ = 2 * kTileQ, kBlockK = 128;
constexpr int kSub = kBlockK * 128;                // 128 rows x 64 dims: 16 KB
constexpr int kQBytes = 3 * kSub, kKBytes = 3 * kSub, kVBytes = 2 * kSub, kRing = 8;
constexpr int kThreads = 384;
constexpr float kLazy = 8.0f;
// pask_debug_set_prompt_wait: bound of a wait in SM clock cycles (about two seconds), bytes a copy announces and does not bring
std::atomic<long long> g_wait_cycles{4000000000LL};
std::atomic<uint32_t> g_surplus{0};

struct PromptParams {
    int n_seqs, total_q, total_k, n_heads;
    const int32_t *cu_q, *cu_k;
    float scale_log2;
    uint32_t surplus;
    __nv_bfloat16 *out;
    float *lse;
    uint32_t wait_kcycles;
    __device__ __forceinline__ long long wait_cycles() const { return (long long)wait_kcycles << 10; }
};
// (another 64 bytes of parameters are another miss of the constant cache: 1 us a call)
static_assert(sizeof(PromptParams) <= 64, "one line of the constant cache");

struct Item {
    int q0, nq, k0, nk, head;                      // first row of the sequence, rows; the same of its keys
    int block;                                     // 256-query block of the sequence; -1: no further item
};

struct __align__(16) PromptSmem {
    uint8_t q[2][kQBytes], ring[kRing * kSub];     // block g of the CTA: keys in pieces 5 g .. + 2, values in 5 g + 3, 5 g + 4 (mod 8)
    uint64_t q_full, q_empty, k_full[2], k_empty[2], v_full[2], v_half[2], v_empty[2], s_full[2], p_half[2], p_full[2], pv_done[2], o_free[2];
    uint64_t item_full[2], item_empty[2], steal, drain;
    uint4 answer;
    Item item[2];
    uint32_t tmem, failed;                         // failed: a softmax warp's wait has run out
    float m[kBlockQ], l[kBlockQ];                  // kSplit > 1: reference maximum and sum of each query over this CTA's keys
};

// visible keys of the query at position i of its sequence
__device__ __forceinline__ int visible(const Item &it, int i) { return max(0, min(it.nk, i + 1 + it.nk - it.nq)); }
// key blocks tile t of the item looks at
__device__ __forceinline__ int key_blocks(const Item &it, int t) {
    const int i0 = it.block * kBlockQ + t * kTileQ;
    if (i0 >= it.nq) return 0;
    return (visible(it, min(it.nq, i0 + kTileQ) - 1) + kBlockK - 1) / kBlockK;
}

// The blocks of keys CTA `part` of `split` looks at: [first, first + max(n[0], n[1])), tile t the first n[t] of them.
struct Part { int first, n[2]; };
__device__ __forceinline__ Part part_of(const Item &it, int part, int split) {
    const int n0 = key_blocks(it, 0), n1 = key_blocks(it, 1), nb = max(n0, n1);
    Part r;
    r.first = split > 1 ? nb * part / split : 0;
    const int mine = (split > 1 ? nb * (part + 1) / split : nb) - r.first;
    r.n[0] = max(0, min(n0 - r.first, mine));
    r.n[1] = max(0, min(n1 - r.first, mine));
    return r;
}

// The item of grid position x, worked out by a warp: position r = x / heads among the blocks of 256 queries, head x % heads.
// Up to 32 sequences (one a lane): blocks in the order of their visible keys, most first.  More: in the order of the batch.
struct Ranker {
    int nq = 0, nk = 0, q0 = 0, k0 = 0;            // of sequence `lane`
    __device__ __forceinline__ static bool load(const PromptParams &p, int s, int &q0, int &nq, int &k0, int &nk) {
        q0 = p.cu_q[s]; k0 = p.cu_k[s];
        nq = p.cu_q[s + 1] - q0; nk = p.cu_k[s + 1] - k0;
        if (q0 >= 0 && nq >= 0 && q0 + nq <= p.total_q && k0 >= 0 && nk >= 0 && k0 + nk <= p.total_k) return true;
        nq = nk = 0;                               // malformed: not written
        return false;
    }
    __device__ __forceinline__ void init(const PromptParams &p, int lane) {
        if (p.n_seqs <= 32 && lane < p.n_seqs) load(p, lane, q0, nq, k0, nk);
    }
    // blocks of this lane's sequence with at least t key blocks
    __device__ __forceinline__ int at_least(int t) const {
        const int nb = (nq + kBlockQ - 1) / kBlockQ;
        if (t <= 0) return nb;
        const long long y = 128LL * (t - 1) - (nk - nq);
        if (y < 0) return nb;
        return y >= nq ? 0 : nb - (int)(y / kBlockQ);
    }
    __device__ __forceinline__ bool find(const PromptParams &p, int x, int lane, Item &it) const {
        const int r = x / p.n_heads;
        it.head = x - r * p.n_heads;
        if (p.n_seqs <= 32) {
            if (r >= __reduce_add_sync(0xffffffffu, at_least(0))) return false;
            int lo = 0, hi = (p.total_k + kBlockK - 1) / kBlockK;      // the largest t that more than r blocks reach
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (__reduce_add_sync(0xffffffffu, at_least(mid)) > r) lo = mid; else hi = mid - 1;
            }
            const int above = at_least(lo + 1), here = at_least(lo) - above;
            const int skip = r - __reduce_add_sync(0xffffffffu, above);
            int inc = here;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, inc, d);
                if (lane >= d) inc += o;
            }
            const int owner = __ffs(__ballot_sync(0xffffffffu, inc > skip)) - 1;
            // fewer keys come first in a sequence: its blocks with lo key blocks are the ones before those with more
            const int block = (nq + kBlockQ - 1) / kBlockQ - above - 1 - (skip - (inc - here));
            it.block = __shfl_sync(0xffffffffu, block, owner);
            it.q0 = __shfl_sync(0xffffffffu, q0, owner);
            it.nq = __shfl_sync(0xffffffffu, nq, owner);
            it.k0 = __shfl_sync(0xffffffffu, k0, owner);
            it.nk = __shfl_sync(0xffffffffu, nk, owner);
            return true;
        }
        const int per = (p.n_seqs + 31) / 32, s0 = min(lane * per, p.n_seqs), s1 = min(s0 + per, p.n_seqs);
        int a, b, c, d, sum = 0;
        for (int s = s0; s < s1; s++) { load(p, s, a, b, c, d); sum += (b + kBlockQ - 1) / kBlockQ; }
        int inc = sum;
#pragma unroll
        for (int e = 1; e < 32; e <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, inc, e);
            if (lane >= e) inc += o;
        }
        const uint32_t reach = __ballot_sync(0xffffffffu, inc > r);
        if (!reach) return false;
        const int owner = __ffs(reach) - 1;
        Item mine = {};
        if (lane == owner) {
            int left = r - (inc - sum);
            for (int s = s0; s < s1; s++) {
                load(p, s, a, b, c, d);
                const int nb = (b + kBlockQ - 1) / kBlockQ;
                if (left < nb) { mine.q0 = a; mine.nq = b; mine.k0 = c; mine.nk = d; mine.block = left; break; }
                left -= nb;
            }
        }
        it.block = __shfl_sync(0xffffffffu, mine.block, owner);
        it.q0 = __shfl_sync(0xffffffffu, mine.q0, owner);
        it.nq = __shfl_sync(0xffffffffu, mine.nq, owner);
        it.k0 = __shfl_sync(0xffffffffu, mine.k0, owner);
        it.nk = __shfl_sync(0xffffffffu, mine.nk, owner);
        return true;
    }
};

// A softmax warp's wait ran out (never expected): its rows of item n and of those that the CTA has accepted behind it say so.  The
// next one, or the -1 at their end, comes at most a wait for the other warps and one for an answer later, and an item's place is
// not filled again before every softmax warp has read the next item.  begun: items this warp has read.  Out of line: inlined,
// it cost 1 us of a call of 150.
__device__ __noinline__ void give_up(const PromptParams &p, PromptSmem &sm, uint32_t n, uint32_t begun, int row_in, int lane) {
    using namespace umma;
    if (lane == 0) *(volatile uint32_t *)&sm.failed = 1;
    for (; __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.item_full[n & 1]), (n >> 1) & 1, 4 * p.wait_cycles())); n++) {
        const Item it = sm.item[n & 1];
        __syncwarp();
        if (lane == 0 && n >= begun) bar_arrive(smem_u32(&sm.item_empty[n & 1]));
        if (it.block < 0) break;
        const int i = it.block * kBlockQ + row_in;
        if (i < it.nq) {
            const size_t row = (size_t)(it.q0 + i) * p.n_heads + it.head;
            for (int d = 0; d < kV; d++) p.out[row * kV + d] = __ushort_as_bfloat16((unsigned short)0x7FC0);
            if (p.lse) p.lse[row] = __int_as_float(0x7FC00000);
        }
        __syncwarp();
    }
}

template <int kSplit>
__global__ void __launch_bounds__(kThreads, 1)
prompt_latent_kernel(const __grid_constant__ PromptParams p, const __grid_constant__ CUtensorMap map_q,
                     const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ CUtensorMap map_v,
                     const __grid_constant__ CUtensorMap map_rope) {
    using namespace umma;
    extern __shared__ __align__(1024) uint8_t s_raw[];
    PromptSmem &sm = *reinterpret_cast<PromptSmem *>(s_raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    if (tid == 0) {
        sm.failed = 0;
        bar_init(smem_u32(&sm.q_full), 1);
        bar_init(smem_u32(&sm.q_empty), 1);
        bar_init(smem_u32(&sm.steal), 1);
        bar_init(smem_u32(&sm.drain), 1);
        for (int i = 0; i < 2; i++) {
            bar_init(smem_u32(&sm.k_full[i]), 1);
            bar_init(smem_u32(&sm.k_empty[i]), 1);
            bar_init(smem_u32(&sm.v_full[i]), 1);
            bar_init(smem_u32(&sm.v_half[i]), 1);
            bar_init(smem_u32(&sm.v_empty[i]), 1);
            bar_init(smem_u32(&sm.s_full[i]), 1);
            bar_init(smem_u32(&sm.p_half[i]), 4);
            bar_init(smem_u32(&sm.p_full[i]), 4);
            bar_init(smem_u32(&sm.pv_done[i]), 1);
            bar_init(smem_u32(&sm.o_free[i]), 4);
            bar_init(smem_u32(&sm.item_full[i]), 1);
            bar_init(smem_u32(&sm.item_empty[i]), 10);
        }
        bar_init_fence();
    }
    if (warp == 8) tmem_alloc(smem_u32(&sm.tmem), 512);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = sm.tmem;
    constexpr uint32_t kS = 0, kO = 256;           // columns of tile 0; tile 1 is 128 behind
    const int part = kSplit > 1 ? (int)blockIdx.x % kSplit : 0;      // = rank in the cluster
    const long long limit = p.wait_cycles();
    bool ok = true;
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

    // 384 threads x 168 registers at launch = 128 x (2 x 200 + 104): the rows of S in the softmax threads need the larger share
    if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (warp == 10) {
        // ================================================= items
        Ranker rank;
        rank.init(p, lane);
        int x = (int)blockIdx.x / kSplit;
        uint32_t asked = 0;
        bool live = true;
        for (uint32_t n = 0; live; n++) {
            const uint32_t slot = n & 1;
            Item it;
            live = x >= 0 && rank.find(p, x, lane, it);
            if (!live) it.block = -1;
            if (lane == 0) {
                sm.item[slot] = it;
                bar_arrive(smem_u32(&sm.item_full[slot]));
            }
            if (!live) break;
            if constexpr (kSplit > 1) { x = -1; continue; }
            // The next one only when the softmax has begun with this one: items held back behind others
            // make the tail longer (4 prompts of 4 to 8 thousand: 833 us with up to three ahead, 820 with one).
            ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.item_empty[slot]), (n >> 1) & 1, limit));
            if (!ok) break;
            if (*(volatile uint32_t *)&sm.failed) { x = -1; continue; }    // no further one
            if (lane == 0) {
                bar_expect(smem_u32(&sm.steal), 16);
                steal_ask(smem_u32(&sm.answer), smem_u32(&sm.steal));
            }
            // (longer than other waits: a CTA that has been taken over is nobody else's any more)
            ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.steal), asked++ & 1, 2 * limit));
            if (!ok) break;
            x = steal_answer(smem_u32(&sm.answer));
            __syncwarp();
            fence_async_shared();                  // the answer has been read before the next one is asked for
        }
    } else if (warp == 9) {
        // ================================================= copies
        Item it;
        uint32_t g = 0, qc = 0;                    // blocks, items with queries copied so far
        const uint32_t qf = smem_u32(&sm.q_full), ring = smem_u32(sm.ring);
        for (uint32_t n = 0; next_item(n, it); n++) {
            const Part in = part_of(it, part, kSplit);
            const int n0 = in.n[0], n1 = in.n[1], nb = max(n0, n1);
            if (nb == 0) continue;
            if (qc > 0) ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.q_empty), (qc - 1) & 1, limit));
            if (!ok) break;
            qc++;
            const bool mine = elect_one();
            if (mine) {
                const uint32_t extra = qc == 1 && part == 0 && ((blockIdx.x / kSplit) & 1) ? p.surplus : 0u;
                bar_expect(qf, (n0 ? kQBytes : 0) + (n1 ? kQBytes : 0) + extra);
                for (int t = 0; t < 2; t++)
                    if (t ? n1 : n0)
                        for (int c = 0; c < 3; c++)
                            tile_load3(smem_u32(sm.q[t]) + c * kSub, &map_q, 64 * c, it.head, it.q0 + it.block * kBlockQ + t * kTileQ, qf);
            }
            for (int j = 0; j < nb; j++, g++) {
                // keys, piece by piece: over the last piece of the keys two blocks before, over that block's values as their halves
                // are done with (one piece takes 16 KB of copy time from a freed place to the product that waits for it, not 48)
                const uint32_t st = g & 1, row = (uint32_t)(it.k0 + (in.first + j) * kBlockK), kf = smem_u32(&sm.k_full[st]), ph = ((g >> 1) - 1) & 1;
                if (g >= 2) ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.k_empty[st]), ph, limit));
                if (!ok) break;
                if (mine) {
                    bar_expect(kf, kKBytes);
                    tile_load3(ring + ((5 * g) & 7) * kSub, &map_kv, 0, it.head, row, kf);
                }
                if (g >= 2) ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.v_half[st]), ph, limit));
                if (!ok) break;
                if (mine) tile_load3(ring + ((5 * g + 1) & 7) * kSub, &map_kv, 64, it.head, row, kf);
                if (g >= 2) ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.v_empty[st]), ph, limit));
                if (!ok) break;
                if (mine) tile_load2(ring + ((5 * g + 2) & 7) * kSub, &map_rope, 0, row, kf);
                // values: over the first two pieces of the keys one block before
                if (g >= 1) ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.k_empty[st ^ 1]), ((g - 1) >> 1) & 1, limit));
                if (!ok) break;
                if (mine) {
                    const uint32_t vf = smem_u32(&sm.v_full[st]);
                    bar_expect(vf, kVBytes);
#pragma unroll
                    for (int c = 0; c < 4; c++)
                        tile_load3(ring + ((5 * g + 3 + (c >> 1)) & 7) * kSub + (c & 1) * (kSub / 2), &map_v, kNope + 64 * (c & 1), it.head,
                                   row + 64 * (c >> 1), vf);
                }
            }
            if (!ok) break;
        }
        if (!ok) {                                 // gave up: let the copies in flight land (bounded) before the CTA ends
            if (qc) bar_wait(qf, (qc - 1) & 1, limit);
            for (uint32_t b = g > 1 ? g - 1 : 0; b <= g; b++) {
                bar_wait(smem_u32(&sm.k_full[b & 1]), (b >> 1) & 1, b < g ? limit : 1000000);
                bar_wait(smem_u32(&sm.v_full[b & 1]), (b >> 1) & 1, b < g ? limit : 1000000);
            }
        }
    } else if (warp == 8) {
        // ================================================= products
        constexpr uint32_t kIdS = instr(kTileQ, kBlockK, false, false), kIdO = instr(kTileQ, kV, false, true);
        const bool mine = elect_one();
        const uint64_t dq = desc(smem_u32(sm.q[0]), 0, 1024), dk = desc(smem_u32(sm.ring), 0, 1024), dv = desc(smem_u32(sm.ring), kSub / 2, 1024);
        Item it;
        uint32_t g = 0, qc = 0, pc[2] = {0, 0}, oc[2] = {0, 0};            // blocks, items, weights and items of each tile so far
        auto scores = [&](int t, uint32_t first) { // first: piece of the ring the keys start at
            uint64_t a = dq + (uint64_t)(t * kQBytes >> 4);
#pragma unroll 1
            for (int c = 0; c < 3; c++, a += kSub >> 4) {      // (rolled: 24 descriptors kept apart would cost 100 registers)
                const uint64_t b = dk + (uint64_t)(((first + c) & 7) * kSub >> 4);
#pragma unroll
                for (int k = 0; k < 4; k++) mma_ss(tmem + kS + t * 128, a + 2 * k, b + 2 * k, kIdS, c > 0 || k > 0, mine);
            }
            if (mine) commit(smem_u32(&sm.s_full[t]));
        };
        auto values = [&](int t, uint32_t first, bool fresh, int from, int steps) {        // half of the keys
            const uint64_t b = dv + (uint64_t)(((first + (from >> 2)) & 7) * kSub >> 4);
#pragma unroll
            for (int k = 0; k < 4; k++)
                if (from + k < steps)
                    mma_ts(tmem + kO + t * 128, tmem + kS + t * 128 + (from + k) * 8, b + 128 * k, kIdO, from + k > 0 || !fresh, mine);
        };
        for (uint32_t n = 0; next_item(n, it); n++) {
            const Part in = part_of(it, part, kSplit);
            const int nt[2] = {in.n[0], in.n[1]}, nb = max(nt[0], nt[1]);
            if (nb == 0) continue;
            ok = bar_wait(smem_u32(&sm.q_full), qc & 1, limit);
            qc++;
            ok = bar_wait(smem_u32(&sm.k_full[g & 1]), (g >> 1) & 1, limit) && ok;
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            fence_after();
            {
                const uint32_t first = __shfl_sync(0xffffffffu, (5 * g) & 7, 0);
                if (nt[0]) scores(0, first);
                if (nt[1]) scores(1, first);
                if (mine) {
                    commit(smem_u32(&sm.k_empty[g & 1]));
                    if (nb == 1) commit(smem_u32(&sm.q_empty));
                }
            }
            for (int j = 0; j < nb; j++, g++) {
                const int valid = __shfl_sync(0xffffffffu, min(kBlockK, it.nk - (in.first + j) * kBlockK), 0), steps = (valid + 15) / 16;
                const uint32_t at = __shfl_sync(0xffffffffu, (5 * g) & 7, 0), ph = (g >> 1) & 1;
                const int last_t = j < nt[1] ? 1 : 0;       // the tile whose product is the last to use the block's values
                bool have_k = false;
                ok = bar_wait(smem_u32(&sm.v_full[g & 1]), ph, limit) && ok;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (valid & 15) {                  // rows behind the last key in its step of 16: whatever they hold counts as zero
                    uint8_t *v = sm.ring + ((at + 3 + (valid >> 6)) & 7) * kSub;
                    const int rows = 16 * steps - valid;
                    for (int e = lane; e < rows * 16; e += 32)
                        *reinterpret_cast<uint4 *>(v + ((e >> 3) & 1) * (kSub / 2) + ((valid & 63) + (e >> 4)) * 128 + (e & 7) * 16) =
                            make_uint4(0, 0, 0, 0);
                    fence_async_shared();
                    __syncwarp();
                }
#pragma unroll
                for (int t = 0; t < 2; t++) {
                    if (j < nt[t]) {
                        if (j == 0) {              // the item before has been read out of O
                            if (oc[t] > 0) ok = bar_wait(smem_u32(&sm.o_free[t]), (oc[t] - 1) & 1, limit) && ok;
                            oc[t]++;
                        }
                        ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.p_half[t]), pc[t] & 1, limit) && ok);
                        if (!ok) break;
                        fence_after();
                        values(t, at + 3, j == 0, 0, steps);
                        if (t == last_t && mine) commit(smem_u32(&sm.v_half[g & 1]));
                        ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.p_full[t]), pc[t] & 1, limit));
                        if (!ok) break;
                        pc[t]++;
                        fence_after();
                        values(t, at + 3, false, 4, steps);
                        if (mine) {
                            if (t == last_t) commit(smem_u32(&sm.v_empty[g & 1]));
                            if (j + 1 == nt[t]) commit(smem_u32(&sm.pv_done[t]));
                        }
                    }
                    if (j + 1 < nt[t]) {
                        if (!have_k) {
                            ok = __all_sync(0xffffffffu, bar_wait(smem_u32(&sm.k_full[(g + 1) & 1]), ((g + 1) >> 1) & 1, limit));
                            if (!ok) break;
                            fence_after();
                            have_k = true;
                        }
                        scores(t, at + 5);
                    }
                }
                if (!ok) break;
                if (mine) {
                    if (j + 1 < nb) commit(smem_u32(&sm.k_empty[(g + 1) & 1]));
                    if (j + 2 == nb) commit(smem_u32(&sm.q_empty));
                }
            }
            if (!ok) break;
        }
        if (!ok) {                                 // gave up: the products in flight end before tensor memory is freed
            if (mine) commit(smem_u32(&sm.drain));
            bar_wait(smem_u32(&sm.drain), 0, limit);
        }
        __syncwarp();
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        // ================================================= softmax: thread = query
        const int t = warp >> 2;
        const uint32_t base = tmem + ((uint32_t)((warp & 3) * 32) << 16) + t * 128;
        const uint32_t s_full = smem_u32(&sm.s_full[t]), p_half = smem_u32(&sm.p_half[t]), p_full = smem_u32(&sm.p_full[t]),
                       pv_done = smem_u32(&sm.pv_done[t]);
        const int row_in = t * kTileQ + (warp & 3) * 32 + lane;
        Item it;
        it.block = -1;
        float m = -INFINITY, l = 0.0f;
        bool none = true;                          // no keys here
        uint32_t sc = 0, ic = 0;                   // blocks of this tile so far (S, P and P V alike), items with any
        uint32_t n = 0, begun = 0;                 // the item at hand, items read so far
        for (; next_item(n, it); n++) {
            begun = n + 1;
            const Part in = part_of(it, part, kSplit);
            const int nb = in.n[t], i = it.block * kBlockQ + row_in;
            const int vis = i < it.nq ? visible(it, i) : 0;
            m = -INFINITY;
            l = 0.0f;
            for (int j = 0; j < nb; j++, sc++) {
                ok = bar_wait(s_full, sc & 1, limit);
                if (!__all_sync(0xffffffffu, ok)) break;
                fence_after();
                float x[128];
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    uint32_t r[32];
                    tmem_ld32(base + kS + 32 * c, r);
#pragma unroll
                    for (int e = 0; e < 32; e++) x[32 * c + e] = __uint_as_float(r[e]);
                }
                tmem_wait_ld();
                const int left = vis - (in.first + j) * kBlockK;
                if (__any_sync(0xffffffffu, left < kBlockK)) {
#pragma unroll
                    for (int e = 0; e < 128; e++) if (e >= left) x[e] = -INFINITY;
                }
                float top = -INFINITY;
                {
                    float a = x[0], b = x[1], c = x[2], d = x[3];
#pragma unroll
                    for (int e = 4; e < 128; e += 4) {
                        a = fmaxf(a, x[e]); b = fmaxf(b, x[e + 1]); c = fmaxf(c, x[e + 2]); d = fmaxf(d, x[e + 3]);
                    }
                    top = fmaxf(fmaxf(a, b), fmaxf(c, d)) * p.scale_log2;
                }
                const bool raise = top > m + kLazy;
                if (__any_sync(0xffffffffu, raise)) {
                    const float f = raise ? ex2(m - top) : 1.0f;
                    if (raise) { m = top; l *= f; }
                    if (j > 0) {                   // O so far, in the new reference (complete: this S was issued behind it)
#pragma unroll 1
                        for (int c = 0; c < 8; c++) {
                            uint32_t r[16];
                            tmem_ld16(base + kO + 16 * c, r);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; e++) r[e] = __float_as_uint(__uint_as_float(r[e]) * f);
                            tmem_st16(base + kO + 16 * c, r);
                        }
                    }
                }
                const float ref = m == -INFINITY ? 0.0f : m;               // a row that has seen no key yet
                const uint64_t scale2 = pair(p.scale_log2, p.scale_log2), ref2 = pair(-ref, -ref);
                uint64_t l2 = pair(0.0f, 0.0f);
                // Weights go out in two halves: the product over the first 64 keys runs beside the other exponentials.
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    uint32_t r[16];
#pragma unroll
                    for (int e = 0; e < 16; e++) {
                        float a, b;
                        unpair(fma2(pair(x[32 * c + 2 * e], x[32 * c + 2 * e + 1]), scale2, ref2), a, b);
                        a = ex2(a);
                        b = ex2(b);
                        l2 = add2(l2, pair(a, b));
                        r[e] = pack_bf16(a, b);
                    }
                    tmem_st16(base + kS + 16 * c, r);
                    if (c & 1) {
                        tmem_wait_st();
                        fence_before();
                        __syncwarp();
                        if (lane == 0) bar_arrive(c == 1 ? p_half : p_full);
                    }
                }
                float l0, l1;
                unpair(l2, l0, l1);
                l += l0 + l1;
            }
            if constexpr (kSplit > 1) {            // one item: its parts are joined below
                if (nb > 0 && ok) ok = bar_wait(pv_done, 0, limit);
                none = nb == 0;
                break;
            }
            // ---- the row's result
            ok = __all_sync(0xffffffffu, ok);
            if (ok && nb > 0) ok = __all_sync(0xffffffffu, bar_wait(pv_done, ic++ & 1, limit));
            if (!ok) break;
            fence_after();
            const size_t row = (size_t)(it.q0 + i) * p.n_heads + it.head;
            const float inv = vis > 0 ? 1.0f / l : 0.0f;
#pragma unroll
            for (int c = 0; c < 8; c++) {
                uint32_t r[16];
#pragma unroll
                for (int e = 0; e < 16; e++) r[e] = 0;
                if (nb > 0) {
                    tmem_ld16(base + kO + 16 * c, r);
                    tmem_wait_ld();
                }
                if (i < it.nq) {
                    uint4 *dst = reinterpret_cast<uint4 *>(p.out + row * kV + 16 * c);
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            const float a = __uint_as_float(r[8 * h + 2 * e]) * inv, b = __uint_as_float(r[8 * h + 2 * e + 1]) * inv;
                            w[e] = vis > 0 ? pack_bf16(a, b) : 0u;
                        }
                        dst[h] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            if (i < it.nq && p.lse) p.lse[row] = vis > 0 ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
            if (nb > 0) {
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_u32(&sm.o_free[t]));
            }
        }
        if constexpr (kSplit == 1) {
            if (!ok) give_up(p, sm, n, begun, row_in, lane);
        } else {
            // All products of this CTA are done, so that nothing reads or fills its tiles any more: [dim][query] over them.
            const bool good = !group_any(1, 2 * kTileQ, !ok);
            fence_after();
            sm.m[row_in] = good ? m : __int_as_float(0x7FC00000);
            sm.l[row_in] = l;
            float *o = reinterpret_cast<float *>(sm.q);
            if (good && it.block >= 0)
#pragma unroll
                for (int c = 0; c < 8; c++) {
                    uint32_t r[16];
#pragma unroll
                    for (int e = 0; e < 16; e++) r[e] = 0;
                    if (!none) {
                        tmem_ld16(base + kO + 16 * c, r);
                        tmem_wait_ld();
                    }
#pragma unroll
                    for (int e = 0; e < 16; e++) o[(16 * c + e) * kBlockQ + row_in] = __uint_as_float(r[e]);
                }
        }
    }
    fence_before();
    if constexpr (kSplit > 1) cluster_sync(); else __syncthreads();
    fence_after();
    if (warp == 8) tmem_free(tmem, 512);
    if constexpr (kSplit > 1) {
        const Item item = sm.item[0];              // (from here and not from a wait that may have run out)
        // Each CTA joins the parts of 256 / kSplit queries, a thread 128 / kSplit dims of one, in the order of the parts.
        constexpr int kRows = kBlockQ / kSplit, kDims = kV / kSplit;
        const int r = part * kRows + tid % kRows, d0 = tid / kRows * kDims, i = item.block * kBlockQ + r;
        if (warp < 8 && item.block >= 0 && i < item.nq) {
            float w[kSplit], top = -INFINITY, l = 0.0f;
#pragma unroll
            for (int s = 0; s < kSplit; s++) { w[s] = peer_load(smem_u32(&sm.m[r]), s); top = fmaxf(top, w[s]); }
            const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int s = 0; s < kSplit; s++) { w[s] = ex2(w[s] - ref); l += w[s] * peer_load(smem_u32(&sm.l[r]), s); }
            const int vis = visible(item, i);
            const float inv = vis > 0 ? 1.0f / l : 0.0f;
            const size_t row = (size_t)(item.q0 + i) * p.n_heads + item.head;
            const uint32_t o = smem_u32(sm.q) + (d0 * kBlockQ + r) * 4;
#pragma unroll 2
            for (int d = 0; d < kDims; d += 8) {
                float x[8] = {};
#pragma unroll
                for (int s = 0; s < kSplit; s++)
#pragma unroll
                    for (int e = 0; e < 8; e++) x[e] += w[s] * peer_load(o + (d + e) * kBlockQ * 4, s);
                uint32_t y[4];
#pragma unroll
                for (int e = 0; e < 4; e++) y[e] = vis > 0 ? pack_bf16(x[2 * e] * inv, x[2 * e + 1] * inv) : 0u;
                *reinterpret_cast<uint4 *>(p.out + row * kV + d0 + d) = make_uint4(y[0], y[1], y[2], y[3]);
            }
            if (d0 == 0 && p.lse) p.lse[row] = vis > 0 ? (top + log2f(l)) * 0.69314718055994531f : -INFINITY;
        }
        cluster_sync();                            // the others may still be reading here
    }
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// rows of 64-dim pieces: dims {inner, heads, rows} (or {inner, rows}), a box of 64 x 1 x box_rows with the 128-byte swizzle
bool encode(EncodeTiled fn, CUtensorMap *map, const void *base, int inner, int heads, int rows, size_t head_stride, size_t row_stride,
            int box_rows) {
    const int rank = heads ? 3 : 2;
    const cuuint64_t dims3[3] = {(cuuint64_t)inner, (cuuint64_t)heads, (cuuint64_t)rows}, dims2[2] = {(cuuint64_t)inner, (cuuint64_t)rows};
    const cuuint64_t str3[2] = {head_stride, row_stride}, str2[1] = {row_stride};
    const cuuint32_t box3[3] = {64, 1, (cuuint32_t)box_rows}, box2[2] = {64, (cuuint32_t)box_rows}, one[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void *>(base), rank == 3 ? dims3 : dims2,
              rank == 3 ? str3 : str2, rank == 3 ? box3 : box2, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kSplit>
void config(cudaLaunchConfig_t &cfg, cudaLaunchAttribute &attr, int items, cudaStream_t stream) {
    constexpr int kSmem = (int)sizeof(PromptSmem);
    static_assert(kSmem <= 232448, "shared memory of a CTA");
    static_assert(kBlockQ * kV * 4 <= sizeof(PromptSmem::q) + sizeof(PromptSmem::ring), "partial results over the tiles");
    attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = kSplit;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg = {};
    cfg.gridDim = dim3(items * kSplit);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = kSplit > 1 ? 1 : 0;
}

// Once per device: the right to the shared memory, and how many clusters of kSplit CTAs run at a time; 0 on an error.
template <int kSplit>
int places(int dev) {
    static int n[64] = {};
    if (n[dev]) return n[dev];
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr;
    config<kSplit>(cfg, attr, 1, nullptr);
    if (cudaFuncSetAttribute(prompt_latent_kernel<kSplit>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes) != cudaSuccess)
        return 0;
    int found = 0;
    if (kSplit > 1 ? cudaOccupancyMaxActiveClusters(&found, prompt_latent_kernel<kSplit>, &cfg) != cudaSuccess
                   : cudaDeviceGetAttribute(&found, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return 0;
    return n[dev] = found;
}

template <int kSplit>
pask_status_t launch(const PromptParams &p, const CUtensorMap &map_q, const CUtensorMap &map_kv, const CUtensorMap &map_v,
                     const CUtensorMap &map_rope, int items, cudaStream_t stream) {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr;
    config<kSplit>(cfg, attr, items, stream);
    return cudaLaunchKernelEx(&cfg, prompt_latent_kernel<kSplit>, p, map_q, map_kv, map_v, map_rope) == cudaSuccess ? PASK_OK : PASK_ERR_CUDA;
}

// Time of n items on p places in key blocks: the longest item has `longest`, the others go evenly down to longest - spread.
double makespan(double n, double p, double longest, double spread) {
    if (n <= p) return longest;
    return fmax(longest, n <= 2 * p ? 2 * longest - 2 * spread * p / n : (longest - spread / 2) * n / p);
}

// CTAs an item's keys are split over.  Few blocks of queries would leave SMs idle while one walks all its keys (16 heads, 200
// queries, 6000 keys: 101.7 us in 16 CTAs, 35.8 us in 64).  Each round of clusters costs some two key blocks more than the
// unsplit kernel (queries read by every part, the joining, no overlap from item to item), so 128 keys stay whole: 10.4 against
// 12.4 us.  Four and eight only while all items run at once (32 heads x 2 blocks, 3000 keys: 38.2 us by two, 51.5 by four).  Two
// also where causal blocks of different lengths fill further rounds (5 heads, 8000 queries of 8000 keys: 136 -> 108 us) and the
// estimate gains a tenth.  The host knows sums only: the rule takes a batch for one of equal sequences.
int split_of(int n_seqs, int total_q, int total_k, int n_heads, int dev) {
    const int nq = max(1, total_q / n_seqs), nk = total_k / n_seqs;
    const double n = (double)n_seqs * ((nq + kBlockQ - 1) / kBlockQ) * n_heads, longest = (nk + kBlockK - 1) / kBlockK;
    const double spread = fmin(longest, fmax(0.0, (double)(nq - kBlockQ) / kBlockK));
    const double whole = makespan(n, places<1>(dev), longest, spread);
    int split = 1;
    double best = whole;
    const int p2 = places<2>(dev), p4 = places<4>(dev), p8 = places<8>(dev);
    if (p2 > 0) {
        const double t = makespan(n, p2, longest / 2, spread / 2) + 2 * ceil(n / p2);
        if (t < (n <= p2 ? best : 0.9 * best)) { best = t; split = 2; }
    }
    if (n <= p4 && longest / 4 + 2 < best) { best = longest / 4 + 2; split = 4; }
    if (n <= p8 && longest / 8 + 2 < best) split = 8;
    return split;
}

}  // namespace

void set_prompt_wait(long long limit_cycles, uint32_t surplus_bytes) {
    g_wait_cycles = limit_cycles;
    g_surplus = surplus_bytes;
}

pask_status_t launch_prompt_latent(int n_seqs, int total_q, int total_k, int n_heads, const int32_t *cu_q, const int32_t *cu_k,
                                   const void *q, const void *kv, const void *k_rope, int rope_stride, float scale, void *out,
                                   float *lse, cudaStream_t stream) {
    static EncodeTiled encode_fn = nullptr;
    if (!encode_fn) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess || !fn ||
            found != cudaDriverEntryPointSuccess)
            return PASK_ERR_CUDA;
        encode_fn = reinterpret_cast<EncodeTiled>(fn);
    }
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return PASK_ERR_CUDA;
    if (!places<1>(dev)) return PASK_ERR_CUDA;
    CUtensorMap map_q{}, map_kv{}, map_v{}, map_rope{};
    const size_t q_row = (size_t)n_heads * kQk * 2, kv_head = (kNope + kV) * 2, kv_row = (size_t)n_heads * kv_head;
    if (!encode(encode_fn, &map_q, q, kQk, n_heads, total_q, kQk * 2, q_row, kTileQ)) return PASK_ERR_CUDA;
    if (total_k > 0 && (!encode(encode_fn, &map_kv, kv, kNope + kV, n_heads, total_k, kv_head, kv_row, kBlockK) ||
                        !encode(encode_fn, &map_v, kv, kNope + kV, n_heads, total_k, kv_head, kv_row, kBlockK / 2) ||
                        !encode(encode_fn, &map_rope, k_rope, kRope, 0, total_k, 0, (size_t)rope_stride * 2, kBlockK)))
        return PASK_ERR_CUDA;
    const long long items = ((long long)total_q / kBlockQ + n_seqs) * n_heads;
    if (items > 0x7fffffffLL) return PASK_ERR_INVALID_ARG;
    const PromptParams p{n_seqs, total_q, total_k, n_heads, cu_q, cu_k, scale * 1.4426950408889634f, g_surplus.load(),
                         static_cast<__nv_bfloat16 *>(out), lse, (uint32_t)(g_wait_cycles.load() >> 10)};
    const int split = split_of(n_seqs, total_q, total_k, n_heads, dev);
    if (items * split > 0x7fffffffLL) return PASK_ERR_INVALID_ARG;
    const auto fn = split == 8 ? launch<8> : split == 4 ? launch<4> : split == 2 ? launch<2> : launch<1>;
    return fn(p, map_q, map_kv, map_v, map_rope, (int)items, stream);
}

}  // namespace pask
