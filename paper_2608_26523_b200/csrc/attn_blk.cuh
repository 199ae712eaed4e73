// Attention over listed pages (block-sparse), head_dim 128: a token of a kv-head sees the keys of the pages in its own list, at or
// before its position.
//
// Two kernels:
//  * block_lists_kernel: the rows of a query tile are (token, q-head) pairs, as in attn_ws.cuh: the `group` q-heads of a kv-head
//    over tile_tokens = 128 / group consecutive tokens.  A block forms the union of a tile's lists, ascending, with a mask
//    of its tokens for every page, from a bitmap in shared memory (pages x tokens), a window of pages at a time.
//  * attn_blk_kernel (persistent, a CTA per SM): runs over the union's pages, 128 keys a step, with the mask applied to the scores.
//    Neighbours' lists mostly agree, so the union is little longer than a list; one of few tokens stays so where they agree less
//    (that is why a tile is one accumulator tile, not two as in the dense kernel: 8 tokens of groups of 16, not 16).
//
// One Q tile, two softmax groups of four warps: of every step's 128 keys group 0 takes the first 64 and group 1 the others, each an online softmax of its
// own with an accumulator of its own.  Scores have two buffers in tensor memory (S 128 columns | S 128 | O_0 | O_1), so that the groups work on
// one step's while the tensor core runs P V of the last and forms the next.  The scores of both groups are one MMA chain of 128 keys, and a step has two commits: "scores"
// (also: the K stage and Q are free) and "P V" (also: the V stage is free, O is quiet).  4096 tokens of 64/4 heads, lists of
// 32 pages of 64, unions of 68, 34 steps a tile: 557 us in a captured graph, 1048 TFLOP/s over the unions; as calls one after the other, at the power limit, 648 us, 900.  Tried before:
// whole steps in turn, one buffer a group, 690 us (a group waits 1900 clk for its next scores); a chain of 64 keys and commits of its own for each
// group, 690 us (2500 clk a step, 1800 of them the issue of 24 MMAs and 4 commits).  At the end both join the two results, half the features
// each.  Q has two buffers, so that the next item's first scores are formed under the join.
// A page is listed or not by a token as a whole, so the mask of most steps is a bit per row and 16 columns: it is applied to the weights' words, the sums
// and the maxima of 16 columns, not to every score; the own page, which is seen in part, goes through the scores.
//   warp 0      scheduler, K producer      warp 1  the thread that issues the MMAs
//   warp 2      V producer, tensor memory  warps 4-7, 8-11  softmax groups
// Scores, maxima, sums and accumulators are in 32 bits; the weights are rounded to bf16, half a step of 2^-8 each, because the tensor core takes both operands of P V in one type and
// V is bf16 (two parts of a weight would double that product).  The result's error against 64 bits is 2.3e-3 (relative 2-norm), of which its own rounding is 1.7e-3.
// Every wait is bounded, as in attn_ws.cuh, whose lazy rescale and packed fma this kernel has too.
// (A quarter of the exponentials as polynomials by fused multiply-adds: 551 -> 560 us; half: 592.)
#pragma once
#include <cstdint>

#include "attn_ws.cuh"
#include "common.cuh"
#include "lengths.cuh"
#include "ptx.cuh"

namespace vpp {

constexpr int kBlkListThreads = 128;
constexpr int kBlkWindow = 8192;              // mask words of a window of pages, at most
constexpr int kBlkHalfPages = 4;              // pages of a group's 64 keys, at most (pages of 16)

// One query tile and kv-head.
struct __align__(16) BlkItem {
    int32_t row0;       // first packed query row (token)
    int32_t tokens;     // tokens of the tile
    int32_t pos0;       // position of the first
    int32_t pages;      // pages of the union
    int32_t last_keys;  // keys that exist in its last page, if that is the context's last and not full; else 0
    int32_t bad;        // an entry of the block table was out of range (its page is left out)
    int32_t pad[2];
};

struct BlkListParams {
    const int32_t* indices;       // [total_q, Hkv, topk]
    const int32_t* block_table;
    const int32_t* prefix_len;
    const int32_t* chunk_len;
    int num_reqs, max_blocks_per_req, block_shift, num_blocks;
    long long capacity;
    int total_q, num_kv_heads, topk;
    int tile_tokens, words;       // mask words of a page
    int max_tiles, max_pages;     // tiles of the launch and pages of a union, at most
    int window;                   // pages whose masks are in shared memory at a time
    WorkHeader* header;           // num_units: tiles; error; counter
    BlkItem* items;               // [Hkv, max_tiles]
    int32_t* pages;               // [Hkv, max_tiles, max_pages]: physical
    uint2* masks;                 // [Hkv, max_tiles, max_pages, words]: logical, tokens
    int32_t* status;
};

__global__ void __launch_bounds__(kBlkListThreads) block_lists_kernel(const BlkListParams p) {
    extern __shared__ int32_t cu[];           // cu[num_reqs + 1], tiles before request r [num_reqs + 1], masks [window, words], pages [window]
    __shared__ int s_count[kBlkListThreads / 32], s_pages, s_last;
    __shared__ int s_bad;
    int32_t* const first_tile = cu + p.num_reqs + 1;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        s_bad = 0;
        s_pages = 0;
        s_last = -1;
    }
    pdl_launch_dependents();
    pdl_wait();
    const bool ok = scan_lengths<kBlkListThreads>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu, p.tile_tokens, first_tile);
    if (!ok) {
        if (blockIdx.x == 0 && tid == 0) {
            *p.header = WorkHeader{0, 0, 0, 1 /* VPP_DEV_BAD_LENGTHS */, 0, 0, 0, 0, {}};
            if (p.status) *p.status = 1;
        }
        return;
    }
    const int tiles = first_tile[p.num_reqs];
    if (blockIdx.x == 0 && tid == 0) {
        *p.header = WorkHeader{tiles, 0, 0, 0, 0, 0, 0, 0, {}};
        if (p.status) *p.status = 0;
    }
    const int tile = blockIdx.x / p.num_kv_heads, g = blockIdx.x % p.num_kv_heads;
    if (tile >= tiles) return;
    const int r = request_of(first_tile, p.num_reqs, tile);
    const int t0 = (tile - first_tile[r]) * p.tile_tokens, row0 = cu[r] + t0;
    const int tokens = min(p.tile_tokens, cu[r + 1] - row0);
    const int pos0 = p.prefix_len[r] + t0, kv_len = p.prefix_len[r] + (cu[r + 1] - cu[r]);
    const int used = ((pos0 + tokens - 1) >> p.block_shift) + 1;         // pages that some token may see
    const int32_t* const lists = p.indices + (static_cast<long long>(row0) * p.num_kv_heads + g) * p.topk;
    const int32_t* const table = p.block_table + static_cast<long long>(r) * p.max_blocks_per_req;
    const long long item = static_cast<long long>(g) * p.max_tiles + tile;
    int32_t* const pages = p.pages + item * p.max_pages;
    uint2* const masks = p.masks + item * p.max_pages * p.words;
    const int W = p.words;
    // Page `e` is the k-th of the union, seen by the tokens of masks word(w).
    auto put = [&](int k, int e, auto word) {
        const int phys = __ldg(table + e);
        const bool fine = phys >= 0 && phys < p.num_blocks;
        if (!fine) s_bad = 1;
        pages[k] = fine ? phys : p.num_blocks;       // (num_blocks: reads as zero)
        for (int w = 0; w < W; ++w) masks[static_cast<long long>(k) * W + w] = make_uint2(e, fine ? word(w) : 0u);
    };
    int count = 0;
    bool done = false;
    if (tokens == 1) {
        // A decode row's list, as a selection gives it: ascending, what is no page behind.  It is the union as it is.
        bool sorted = true;
        for (int i = tid; i < p.topk; i += kBlkListThreads) {
            const int e = lists[i], last = i > 0 ? lists[i - 1] : -1, next = i + 1 < p.topk ? lists[i + 1] : -1;
            const bool valid = e >= 0 && e < used;
            if (valid && (i > 0 && (last < 0 || last >= e))) sorted = false;
            if (valid && (next < 0 || next >= used)) {
                s_pages = i + 1;
                s_last = e;
            }
        }
        done = __syncthreads_and(sorted);
        if (done) {
            count = s_pages;
            for (int i = tid; i < count; i += kBlkListThreads) put(i, lists[i], [](int w) { return w == 0 ? 1u : 0u; });
        }
    }
    if (!done) {
        uint32_t* const s_mask = reinterpret_cast<uint32_t*>(first_tile + p.num_reqs + 1);
        int32_t* const s_page = reinterpret_cast<int32_t*>(s_mask + p.window * W);
        const int entries = tokens * p.topk;
        int last = -1;            // of this warp's pages
        for (int w0 = 0; w0 < used; w0 += p.window) {
            const int n = min(p.window, used - w0);
            for (int i = tid; i < n * W; i += kBlkListThreads) s_mask[i] = 0;
            __syncthreads();
            for (int i = tid; i < entries; i += kBlkListThreads) {
                const int t = i / p.topk;
                const int e = lists[static_cast<long long>(t) * p.num_kv_heads * p.topk + (i - t * p.topk)];
                if (e >= w0 && e < w0 + n && e <= ((pos0 + t) >> p.block_shift)) atomicOr(&s_mask[(e - w0) * W + (t >> 5)], 1u << (t & 31));
            }
            __syncthreads();
            // a run of pages a warp: count, then place
            const int run = (n + kBlkListThreads - 1) / kBlkListThreads * 32, a = min(n, warp * run), b = min(n, a + run);
            auto listed = [&](int i) {
                uint32_t m = 0;
                if (i < b)
                    for (int w = 0; w < W; ++w) m |= s_mask[i * W + w];
                return m != 0;
            };
            int mine = 0;
            for (int i0 = a; i0 < b; i0 += 32) mine += __popc(__ballot_sync(0xffffffffu, listed(i0 + lane)));
            if (lane == 0) s_count[warp] = mine;
            __syncthreads();
            int at = 0, found = 0;
            for (int w = 0; w < kBlkListThreads / 32; ++w) {
                if (w < warp) at += s_count[w];
                found += s_count[w];
            }
            for (int i0 = a; i0 < b; i0 += 32) {
                const bool in = listed(i0 + lane);
                const uint32_t m = __ballot_sync(0xffffffffu, in);
                if (in) s_page[at + __popc(m & ((1u << lane) - 1))] = i0 + lane;
                at += __popc(m);
                if (m) last = w0 + i0 + 31 - __clz(m);
            }
            __syncthreads();
            for (int k = tid; k < found; k += kBlkListThreads) {
                const int i = s_page[k];
                put(count + k, w0 + i, [&](int w) { return s_mask[i * W + w]; });
            }
            count += found;
            __syncthreads();
        }
        if (lane == 0 && last >= 0) atomicMax(&s_last, last);
    }
    __syncthreads();
    const int tail = kv_len & ((1 << p.block_shift) - 1);
    if (tid == 0) p.items[item] = BlkItem{row0, tokens, pos0, count, s_last == (kv_len - 1) >> p.block_shift ? tail : 0, s_bad, {0, 0}};
}

struct BlkParams {
    const WorkHeader* header_ro;
    WorkHeader* header;
    const BlkItem* items;
    const int32_t* pages;
    const uint2* masks;
    int max_tiles, max_pages, words;
    int block_shift, num_blocks;
    int num_q_heads, num_kv_heads, group;
    long long total_q;
    int tile_tokens;
    int splits;                   // parts of every union, each an item
    int k_block_units, k_head_units, k_end;
    int v_block_units, v_head_units, v_end;
    int box_rows;                 // keys a copy brings (a page, or 8 where the maps are the exact ones)
    int k_exact, v_exact;
    float scale_log2e;
    uint8_t* out;                 // bf16 [total_q, Hq, 128]
    float* lse;
    float* o_parts;               // [splits, total_q, Hq, 128]
    float* lse_parts;
    int32_t* status;
};

struct BlkWork {
    int32_t valid, row0, tokens, pos0, g;
    int32_t begin, end;           // steps of 128 keys
    int32_t pages;                // of the whole union
    int32_t last_keys;            // of the last page; 0: nothing to mend
    int32_t split;
    long long list;               // first page of the union
};

constexpr int kBlkBars = 6 * kTileBytes;      // offset of what follows the tiles: two of Q, two stages of K and V each
constexpr int kBlkOffStat = 512, kBlkOffStage = kBlkOffStat + 2 * 2 * 128 * 4, kBlkStageBytes = 2048;
constexpr int kBlkSmem = kBlkBars + kBlkOffStage + 8 * kBlkStageBytes + 1024 /* alignment */;
static_assert(kBlkSmem <= 232448, "shared memory of one CTA");

// What a token sees of a group's 64 keys: a bit for each 16 of them (bits 0 .. 3), and `lim`, the last key seen where the own page is among them (else >= 63).
// f: the group's pages of the step, logical number and the word of the mask that has the token.
__device__ __forceinline__ uint32_t blk_visible(const uint2 (&f)[kBlkHalfPages], int t, int shift, int bit, int own, int own_off, int& lim) {
    lim = 64;
    if (shift >= 6) {                        // one page
        if (static_cast<int>(f[0].x) == own) lim = own_off - ((t * 64) & ((1 << shift) - 1));
        return (f[0].y >> bit) & 1 && lim >= 0 ? 15u : 0u;
    }
    uint32_t v = 0;
    const int n = 64 >> shift;               // two or four pages
#pragma unroll
    for (int i = 0; i < kBlkHalfPages; ++i) {
        if (i >= n || !((f[i].y >> bit) & 1)) continue;
        v |= (shift == 5 ? 3u : 1u) << (shift == 5 ? 2 * i : i);
        if (static_cast<int>(f[i].x) == own) lim = (i << shift) + own_off;      // (the last page that the token lists: none behind it)
    }
    return v;
}
// A warp's 32 rows x 64 bytes (lane l holds row l) to global memory, whole runs of 64 bytes, through 2 KB of the warp's own.  (Straight from the registers a
// store of 16 bytes a lane touches 32 lines: 4000 clk for the join of an item.)
template <typename RowOf>
__device__ __forceinline__ void blk_flush(uint8_t* stage, const uint4 (&v)[4], RowOf row_of) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 4; ++q) *reinterpret_cast<uint4*>(stage + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) = v[q];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2), q = lane & 3;
        uint8_t* const dst = row_of(r);
        if (dst) *reinterpret_cast<uint4*>(dst + q * 16) = *reinterpret_cast<const uint4*>(stage + r * 64 + ((q ^ ((r >> 1) & 3)) << 4));
    }
}

__global__ void __launch_bounds__(kWsThreads, 1)
attn_blk_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_q1, const __grid_constant__ CUtensorMap tm_k,
                const __grid_constant__ CUtensorMap tm_v, const BlkParams p) {
    // tm_q / tm_q1: q with a box of (64 features, group heads, tile_tokens tokens / one token)
    // tm_k / tm_v: as in attn_ws.cuh, a page per copy (or, k_exact / v_exact, eight keys)
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const gen = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t sQ = base, sKV = base + 2 * kTileBytes, sBar = base + kBlkBars;
    const uint32_t bar_item_full = sBar, bar_item_empty = sBar + 16;       // [2]
    const uint32_t bar_q_full = sBar + 32, bar_q_empty = sBar + 48;        // [2]
    const uint32_t bar_s = sBar + 64;                                      // [2] scores of a buffer
    const uint32_t bar_p = sBar + 80;                                      // [2] weights of a buffer, of both groups
    const uint32_t bar_pv = sBar + 112;                                    // [2] both groups' products of a step, by its buffer
    const uint32_t bar_kv_full = sBar + 144;                               // [2][K, V]
    const uint32_t bar_vfix = sBar + 208;                                  // [2]
    const uint32_t bar_stat = sBar + 288, bar_done = sBar + 296;
    uint8_t* const gen_bar = gen + kBlkBars;
    volatile int* const s_abort = reinterpret_cast<volatile int*>(gen_bar + 304);
    volatile uint32_t* const s_tmem = reinterpret_cast<volatile uint32_t*>(gen_bar + 308);
    BlkWork* const ring = reinterpret_cast<BlkWork*>(gen_bar + 320);       // [2]
    static_assert(320 + 2 * sizeof(BlkWork) <= kBlkOffStat, "item ring");
    float* const stat = reinterpret_cast<float*>(gen_bar + kBlkOffStat);   // [group][m, l][128]

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_item_full + 8 * i, 1);
            mbar_init(bar_item_empty + 8 * i, 10);      // 8 softmax warps, the MMA thread, the V producer
            mbar_init(bar_q_full + 8 * i, 1);
            mbar_init(bar_q_empty + 8 * i, 1);
            mbar_init(bar_s + 8 * i, 1);
            mbar_init(bar_pv + 8 * i, 1);
            mbar_init(bar_p + 8 * i, 8);
            mbar_init(bar_kv_full + 8 * i, 1);
            mbar_init(bar_kv_full + 16 + 8 * i, 1);
            mbar_init(bar_vfix + 8 * i, 1);
        }
        mbar_init(bar_stat, 8);
        mbar_init(bar_done, 8);
        fence_mbar_init();
        *s_abort = 0;
        prefetch_tmap(&tm_q);
        prefetch_tmap(&tm_q1);
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
    }
    __syncthreads();
    if (warp == 2) {
        tmem_alloc(smem_u32(const_cast<uint32_t*>(s_tmem)), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;

    pdl_wait();                  // the lists come from the kernel launched just before
    pdl_launch_dependents();
    const WorkList head = read_header(p.header_ro);
    const int tiles = head.num_units, shift = p.block_shift, per_step = 128 >> shift;
    const int total = tiles * p.num_kv_heads * p.splits;

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kWsRegsLow));
        // The K (which = 0) or V tile of step `step` (counted over all items): `phys` is the page of the lane's copy.
        auto load_tile = [&](int which, uint32_t step, int g, int phys) -> bool {
            const uint32_t st = 2 * (step & 1) + which, full = bar_kv_full + 8 * st;
            const bool exact = which == 0 ? p.k_exact : p.v_exact;
            const int rows = exact ? kExactRows : p.box_rows, off = lane * rows;
            bool ok = true;
            if (lane == 0) {
                // the stage's last user: the scores, or the products, of two steps ago
                // (neither barrier can be a phase further: that takes this very tile)
                if (step >= 2) ok = mbar_wait((which == 0 ? bar_s : bar_pv) + 8 * (step & 1), ((step - 2) >> 1) & 1, s_abort, 603 + which);
                if (ok) mbar_arrive_expect_tx(full, kTileBytes);
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) return false;
            if (off < kTileN) {
                const uint32_t dst = sKV + st * kTileBytes + static_cast<uint32_t>(off) * (kGroupBytes / 8);
                const CUtensorMap* const tm = which == 0 ? &tm_k : &tm_v;
                if (exact) {
                    tma_load_5d(dst, tm, full, 0, off & ((1 << shift) - 1), 0, g, phys);
                } else {
                    const int at = phys == p.num_blocks ? (which == 0 ? p.k_end : p.v_end)
                                   : which == 0 ? phys * p.k_block_units + g * p.k_head_units : phys * p.v_block_units + g * p.v_head_units;
                    tma_load_5d(dst, tm, full, 0, 0, 0, 0, at);
                }
            }
            __syncwarp();
            return true;
        };
        if (warp == 0) {
            // ============================ scheduler, K producer ============================
            uint32_t n_item = 0, step = 0, n_q = 0;
            const int copy_rows = p.k_exact ? kExactRows : p.box_rows;
            while (true) {
                int k = blockIdx.x;
                if (n_item > 0) {
                    if (lane == 0) k = gridDim.x + atomicAdd(&p.header->counter, 1);
                    k = __shfl_sync(0xffffffffu, k, 0);
                }
                const bool have = k < total;
                BlkWork w{};
                if (have) {
                    // kv-head by kv-head, so that CTAs running at the same time read the same pages
                    const int tg = k / p.splits;
                    w.split = k - tg * p.splits;
                    w.g = tg / tiles;
                    const long long item = static_cast<long long>(w.g) * p.max_tiles + (tg - w.g * tiles);
                    const BlkItem x = p.items[item];
                    w.valid = 1;
                    w.row0 = x.row0;
                    w.tokens = x.tokens;
                    w.pos0 = x.pos0;
                    w.pages = x.pages;
                    w.last_keys = x.last_keys;
                    w.list = item * p.max_pages;
                    const int steps = (x.pages + per_step - 1) / per_step;
                    w.begin = static_cast<int>(static_cast<long long>(steps) * w.split / p.splits);
                    w.end = static_cast<int>(static_cast<long long>(steps) * (w.split + 1) / p.splits);
                    if (x.bad && lane == 0 && p.status) atomicMax(p.status, 2 /* VPP_DEV_BAD_BLOCK */);
                }
                const uint32_t slot = n_item & 1;
                bool ok = true;
                if (lane == 0) {
                    ok = mbar_wait(bar_item_empty + 8 * slot, ((n_item >> 1) & 1) ^ 1, s_abort, 601);
                    if (ok) {
                        ring[slot] = w;
                        mbar_arrive(bar_item_full + 8 * slot);
                    }
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                ++n_item;
                if (!have) break;
                if (w.begin == w.end) continue;      // (nobody waits for its queries)
                const uint32_t qb = n_q & 1;
                if (lane == 0) {
                    ok = mbar_wait(bar_q_empty + 8 * qb, ((n_q >> 1) & 1) ^ 1, s_abort, 602);
                    if (ok) {
                        const bool one = w.tokens == 1;
                        const CUtensorMap* const tm = one ? &tm_q1 : &tm_q;
                        mbar_arrive_expect_tx(bar_q_full + 8 * qb, 2 * p.group * (one ? 1 : p.tile_tokens) * 128);
                        tma_load_3d(sQ + qb * kTileBytes, tm, bar_q_full + 8 * qb, 0, w.g * p.group, w.row0);
                        tma_load_3d(sQ + qb * kTileBytes + kSlabBytes, tm, bar_q_full + 8 * qb, 64, w.g * p.group, w.row0);
                    }
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                ++n_q;
                // pages 32 at a time, a lane each
                int phys_mine = 0;
                const int e0 = w.begin * per_step;
                for (int j = w.begin; j < w.end && ok; ++j, ++step) {
                    const int k0 = j * per_step, in = (k0 - e0) & 31;
                    if (in == 0) phys_mine = k0 + lane < w.pages ? p.pages[w.list + k0 + lane] : p.num_blocks;
                    ok = load_tile(0, step, w.g, __shfl_sync(0xffffffffu, phys_mine, in + ((lane * copy_rows) >> shift)));
                }
                if (!ok) break;
            }
        } else if (warp == 2) {
            // ============================ V producer ============================
            uint32_t n_item = 0, step = 0, fixes = 0;
            const int copy_rows = p.v_exact ? kExactRows : p.box_rows;
            while (true) {
                const uint32_t slot = n_item & 1;
                bool ok = true;
                if (lane == 0) ok = mbar_wait(bar_item_full + 8 * slot, (n_item >> 1) & 1, s_abort, 611);
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                const BlkWork w = ring[slot];
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_item_empty + 8 * slot);
                ++n_item;
                if (!w.valid) break;
                int phys_mine = 0;
                const int e0 = w.begin * per_step, steps = (w.pages + per_step - 1) / per_step;
                for (int j = w.begin; j < w.end && ok; ++j) {
                    const int k0 = j * per_step, in = (k0 - e0) & 31;
                    if (in == 0) phys_mine = k0 + lane < w.pages ? p.pages[w.list + k0 + lane] : p.num_blocks;
                    ok = load_tile(1, step, w.g, __shfl_sync(0xffffffffu, phys_mine, in + ((lane * copy_rows) >> shift)));
                    if (!ok) break;
                    if (w.last_keys != 0 && j == steps - 1) {
                        // slots past the end hold anything: their values become 0, so that 0 * garbage cannot reach O.  The MMA thread waits for it.
                        const uint32_t st = 2 * (step & 1) + 1;
                        if (lane == 0) ok = mbar_wait(bar_kv_full + 8 * st, (step >> 1) & 1, s_abort, 612);
                        ok = __shfl_sync(0xffffffffu, ok, 0);
                        if (!ok) break;
                        uint8_t* const vb = gen + 2 * kTileBytes + st * kTileBytes;
                        const int first = ((w.pages - 1 - k0) << shift) + w.last_keys;
                        const uint4 z = make_uint4(0, 0, 0, 0);
                        for (int r = first + lane; r < kTileN; r += 32) {
                            uint4* const a = reinterpret_cast<uint4*>(vb + (r >> 3) * kGroupBytes + (r & 7) * 128);
                            uint4* const b = a + kHalfBytes / 16;
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                a[c] = z;
                                b[c] = z;
                            }
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar_vfix + 8 * (fixes & 1));
                        ++fixes;
                    }
                    ++step;
                }
                if (!ok) break;
            }
        } else if (warp == 1 && lane == 0) {
            // ============================ MMA issuer (a single thread) ============================
            constexpr uint32_t kIdescQK = idesc_bf16(128, 128, false, false), kIdescPV = idesc_bf16(128, 128, false, true);
            constexpr uint32_t kHiQ = desc_hi_sw128(1024), kHiKV = desc_hi_sw128(kGroupBytes);
            uint32_t n_item = 0, n_q = 0, step = 0, fixes = 0;
            auto wait = [&](uint32_t bar, uint32_t parity, int where) { return mbar_wait(bar, parity, s_abort, where); };
            while (true) {
                const uint32_t slot = n_item & 1;
                if (!wait(bar_item_full + 8 * slot, (n_item >> 1) & 1, 621)) break;
                const int valid = ring[slot].valid, n = ring[slot].end - ring[slot].begin;
                const bool mend = ring[slot].last_keys != 0 && ring[slot].end == (ring[slot].pages + per_step - 1) / per_step;
                mbar_arrive(bar_item_empty + 8 * slot);
                ++n_item;
                if (!valid) break;
                if (n == 0) continue;
                const uint32_t qb = n_q & 1;
                if (!wait(bar_q_full + 8 * qb, (n_q >> 1) & 1, 622)) break;
                ++n_q;
                const uint32_t q_lo = desc_lo_sw128(sQ + qb * kTileBytes, 16), first = step;
                auto have_k = [&](int j) { return wait(bar_kv_full + 16 * ((first + j) & 1), ((first + j) >> 1) & 1, 623); };
                auto scores = [&](int j) {
                    const uint32_t buf = (first + j) & 1, st = 2 * buf;
                    const uint32_t k_lo = desc_lo_sw128(sKV + st * kTileBytes, 16), tS = tmem + buf * 128;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint32_t qoff = ((k >> 2) * kSlabBytes + (k & 3) * 32) >> 4, koff = ((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4;
                        mma_ss_lhh(tS, q_lo + qoff, kHiQ, k_lo + koff, kHiKV, kIdescQK, k > 0);
                    }
                    tc_commit(bar_s + 8 * buf);
                    if (j + 1 == n) tc_commit(bar_q_empty + 8 * qb);
                };
                bool ok = have_k(0);
                if (!ok) break;
                tc_fence_after();
                scores(0);
                if (n > 1) {
                    ok = have_k(1);
                    if (!ok) break;
                    scores(1);
                }
                for (int j = 0; j < n && ok; ++j) {
                    const uint32_t buf = (first + j) & 1, parity = ((first + j) >> 1) & 1, st = 2 * buf + 1;
                    ok = wait(bar_kv_full + 8 * st, parity, 624);
                    if (!ok) break;
                    if (mend && j == n - 1) {
                        ok = wait(bar_vfix + 8 * (fixes & 1), (fixes >> 1) & 1, 625);
                        if (!ok) break;
                        ++fixes;
                    }
                    if (j + 2 < n) ok = have_k(j + 2);      // (before the waits for P: a wait that is over takes 90 clk too)
                    if (!ok) break;
                    ok = wait(bar_p + 8 * buf, parity, 626);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t tP = tmem + buf * 128, v_lo = desc_lo_sw128(sKV + st * kTileBytes, kHalfBytes);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        mma_ts_lh(tmem + 256 + (k >> 2) * 128, tP + (k >> 2) * 64 + (k & 3) * 8, v_lo + k * (2 * kGroupBytes >> 4), kHiKV, kIdescPV,
                                  (j > 0 || (k & 3) > 0) ? 1u : 0u);
                    tc_commit(bar_pv + 8 * buf);
                    if (j + 2 < n) scores(j + 2);
                }
                if (!ok) break;
                step = first + n;
            }
        }
        // warp 3 has nothing to do until teardown
    } else {
        // ===================================== softmax groups =====================================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kWsRegsHigh));
        const int t = (warp - 4) >> 2, row = ((warp & 3) << 5) | lane;
        const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t tS0 = tmem + t * 64 + lane_off, tO = tmem + 256 + t * 128 + lane_off;
        const float sc = p.scale_log2e;
        const int my_tok = row / p.group, my_head = row - my_tok * p.group;
        uint32_t n_item = 0, x_it = 0, step = 0;      // step: those of all items
        while (true) {
            const uint32_t slot = n_item & 1;
            if (!mbar_wait(bar_item_full + 8 * slot, (n_item >> 1) & 1, s_abort, 631)) break;
            const BlkWork w = ring[slot];
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_item_empty + 8 * slot);
            ++n_item;
            if (!w.valid) break;
            const int n = w.end - w.begin;
            const bool live = my_tok < w.tokens;
            const int pos = w.pos0 + my_tok, own = live ? pos >> shift : -2, own_off = pos & ((1 << shift) - 1);
            const int tok = live ? my_tok : 0;
            float m_ref = -INFINITY, l_run = 0.f;
            bool ok = true, seen = false;
            // the pages and masks of a step are requested a step ahead
            uint2 next[kBlkHalfPages];
            const uint2* at = p.masks + (w.list + static_cast<long long>(w.begin) * per_step + ((t * 64) >> shift)) * p.words + (tok >> 5);
            int left = w.pages - w.begin * per_step - ((t * 64) >> shift);      // pages of the union from `at` on
            const int stride = per_step * p.words;
            auto request = [&]() {
                next[0] = make_uint2(0, 0);
                if (left > 0) next[0] = __ldg(at);
                if (shift < 6) {
#pragma unroll
                    for (int i = 1; i < kBlkHalfPages; ++i) {
                        next[i] = make_uint2(0, 0);
                        if (i < (64 >> shift) && left > i) next[i] = __ldg(at + i * p.words);
                    }
                }
                at += stride;
                left -= per_step;
            };
            request();
            for (int j = 0; j < n && ok; ++j, ++step) {
                const uint32_t buf = step & 1, parity = (step >> 1) & 1, tS = tS0 + buf * 128;
                int now_lim = 64;
                const uint32_t now = live ? blk_visible(next, t, shift, tok & 31, own, own_off, now_lim) : 0u;
                request();
                const bool mine = now != 0;
                seen |= mine;
                const bool none = !__any_sync(0xffffffffu, mine);
                ok = mbar_wait(bar_s + 8 * buf, parity, s_abort, 633);
                if (!ok) break;
                if (j == 0 && x_it > 0) {      // the last item's accumulators are read by both groups before P V overwrites them
                    ok = mbar_wait(bar_done, (x_it - 1) & 1, s_abort, 638);
                    if (!ok) break;
                }
                tc_fence_after();
                if (none) {
                    // no row of this warp sees a key of this step
                    uint32_t z[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) z[i] = 0;
                    tmem_st32(tS, z);
                } else {
                    uint32_t s[64];
                    tmem_ld32(tS, reinterpret_cast<uint32_t(&)[32]>(s[0]));
                    tmem_ld32(tS + 32, reinterpret_cast<uint32_t(&)[32]>(s[32]));
                    tc_wait_ld(reinterpret_cast<uint32_t(&)[32]>(s[0]));
                    tc_wait_ld(reinterpret_cast<uint32_t(&)[32]>(s[32]));
                    if (__any_sync(0xffffffffu, mine && now_lim < 63)) {
#pragma unroll
                        for (int i = 0; i < 64; ++i)
                            if (mine && i > now_lim) s[i] = 0xff800000u;  // -inf
                    }
                    // the largest of the 16-column pieces that are seen
                    float mxa = -INFINITY;
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        float mx[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) mx[k] = fmax3(__uint_as_float(s[u * 16 + k]), __uint_as_float(s[u * 16 + 4 + k]), __uint_as_float(s[u * 16 + 8 + k]));
#pragma unroll
                        for (int k = 0; k < 2; ++k) mx[k] = fmax3(mx[k], mx[k + 2], __uint_as_float(s[u * 16 + 12 + k]));
                        const float x = fmax3(fmaxf(mx[0], mx[1]), __uint_as_float(s[u * 16 + 14]), __uint_as_float(s[u * 16 + 15]));
                        mxa = (now >> u) & 1 ? fmaxf(mxa, x) : mxa;
                    }
                    const float m_new = fmaxf(mxa * sc, m_ref);
                    const bool grow = (m_new - m_ref > kRescaleThreshold) || (m_ref == -INFINITY && m_new != -INFINITY);
                    if (__any_sync(0xffffffffu, grow)) {
                        const float alpha = grow ? ex2(m_ref - m_new) : 1.f;  // m_ref = -inf gives 0
                        if (grow) m_ref = m_new;
                        l_run *= alpha;
                        if (j > 0) {   // O of this group already holds something
                            ok = mbar_wait(bar_pv + 8 * (buf ^ 1), ((step - 1) >> 1) & 1, s_abort, 635);      // (the last step's products are still under way)
                            if (!ok) break;
                            tc_fence_after();
                            uint32_t o[32];
#pragma unroll 1
                            for (int c = 0; c < 4; ++c) {
                                tmem_ld32(tO + c * 32, o);
                                tc_wait_ld(o);
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                tmem_st32(tO + c * 32, o);
                            }
                        }
                    }
                    const float m_use = (m_ref == -INFINITY) ? 0.f : m_ref;
                    const uint64_t sc2 = pack_f32x2(sc, sc), neg_m2 = pack_f32x2(-m_use, -m_use);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t pk[16];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t keep = (now >> (2 * c + h)) & 1 ? 0xffffffffu : 0u;
                            float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
                            for (int i = 0; i < 16; i += 2) {
                                const int a = c * 32 + h * 16 + i;
                                float x0, x1;
                                unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[a]), __uint_as_float(s[a + 1])), sc2, neg_m2), x0, x1);
                                const float p0 = ex2(x0), p1 = ex2(x1);
                                sum0 += p0;
                                sum1 += p1;
                                pk[h * 8 + (i >> 1)] = pack_bf16x2(p0, p1) & keep;
                            }
                            l_run += keep ? sum0 + sum1 : 0.f;
                        }
                        tmem_st16(tS + c * 16, pk);
                    }
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_p + 8 * buf);
            }
            if (!ok) break;
            // ---- the two groups' results joined, half the features each ----
            if (n > 0) {
                ok = mbar_wait(bar_pv + 8 * ((step - 1) & 1), ((step - 1) >> 1) & 1, s_abort, 636);
                if (!ok) break;
            }
            tc_fence_after();
            if (seen && m_ref == -INFINITY && l_run == 0.f) l_run = NAN;        // keys, but all scores -inf: 0 / 0, as the definition has it
            if (n == 0 && x_it > 0) {          // (an item without steps: as above, before the statistics are overwritten)
                ok = mbar_wait(bar_done, (x_it - 1) & 1, s_abort, 639);
                if (!ok) break;
            }
            stat[t * 256 + row] = m_ref;
            stat[t * 256 + 128 + row] = l_run;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_stat);
            ok = mbar_wait(bar_stat, x_it & 1, s_abort, 637);
            if (!ok) break;
            tc_fence_after();
            const float m0 = stat[row], l0 = stat[128 + row], m1 = stat[256 + row], l1 = stat[256 + 128 + row];
            const float M = fmaxf(m0, m1);
            float a0 = 0.f, a1 = 0.f, L = 0.f, s0 = 0.f, s1 = 0.f;
            if (M != -INFINITY) {
                a0 = m0 == -INFINITY ? 0.f : ex2(m0 - M);
                a1 = m1 == -INFINITY ? 0.f : ex2(m1 - M);
                L = (m0 == -INFINITY && l0 == l0 ? 0.f : a0 * l0) + (m1 == -INFINITY && l1 == l1 ? 0.f : a1 * l1);
                s0 = a0 / L;
                s1 = a1 / L;
            } else {
                L = l0 + l1;                     // 0: no key at all; NaN: keys, but no finite score
                if (!(L == L)) s0 = s1 = NAN;
            }
            const uint32_t tH = tmem + 256 + lane_off + t * 64;      // this group's features of O_0; O_1's are 128 columns further
            const long long orow = (static_cast<long long>(w.row0) + my_tok) * p.num_q_heads + w.g * p.group + my_head;
            uint8_t* const stage = gen_bar + kBlkOffStage + (warp - 4) * kBlkStageBytes;
            const long long prow = static_cast<long long>(w.split) * p.total_q * p.num_q_heads + orow;
#pragma unroll
            for (int c = 0; c < 2; ++c) {        // 32 features at a time
                uint32_t r0[32], r1[32];
                if (n > 0) {
                    tmem_ld32(tH + c * 32, r0);
                    tmem_ld32(tH + 128 + c * 32, r1);
                    tc_wait_ld(r0);
                    tc_wait_ld(r1);
                }
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) {   // (an accumulator without weight is not looked at: 0 * inf)
                    v[i] = s0 != 0.f && n > 0 ? __uint_as_float(r0[i]) * s0 : s0;
                    if (s1 != 0.f && n > 0) v[i] = fmaf(__uint_as_float(r1[i]), s1, v[i]);
                }
                if (p.splits == 1) {
                    uint4 pk[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        pk[i] = make_uint4(pack_bf16x2(v[8 * i], v[8 * i + 1]), pack_bf16x2(v[8 * i + 2], v[8 * i + 3]), pack_bf16x2(v[8 * i + 4], v[8 * i + 5]),
                                           pack_bf16x2(v[8 * i + 6], v[8 * i + 7]));
                    blk_flush(stage, pk, [&](int r) -> uint8_t* {
                        const long long to = __shfl_sync(0xffffffffu, live ? orow : -1ll, r);
                        return to < 0 ? nullptr : p.out + (to * 128 + t * 64 + c * 32) * 2;
                    });
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint4 f[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            f[i] = make_uint4(__float_as_uint(v[h * 16 + 4 * i]), __float_as_uint(v[h * 16 + 4 * i + 1]), __float_as_uint(v[h * 16 + 4 * i + 2]),
                                              __float_as_uint(v[h * 16 + 4 * i + 3]));
                        blk_flush(stage, f, [&](int r) -> uint8_t* {
                            const long long to = __shfl_sync(0xffffffffu, live ? prow : -1ll, r);
                            return to < 0 ? nullptr : reinterpret_cast<uint8_t*>(p.o_parts + to * 128 + t * 64 + c * 32 + h * 16);
                        });
                    }
                }
            }
            if (live && t == 0) {
                const float lse = (M + log2f(L)) * 0.6931471805599453f;      // (no key: -inf + -inf)
                if (p.splits == 1) {
                    if (p.lse) p.lse[orow] = lse;
                } else {
                    p.lse_parts[prow] = lse == lse ? lse : INFINITY;      // (the merge takes the largest: a NaN would be lost beside parts without keys)
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_done);
            ++x_it;
        }
    }

    // ---- teardown ----
    __syncthreads();
    if (*s_abort != 0) {
        if (tid == 0 && p.status) atomicMax(p.status, 3 /* VPP_DEV_TIMEOUT */);
        for (int i = 0; i < 64; ++i) __nanosleep(1000);  // let copies and MMAs in flight drain
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2) tmem_dealloc(tmem, 512);
}

}  // namespace vpp
