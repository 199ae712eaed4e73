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
// One Q tile, two softmax groups of four warps that take the KV steps in turn, each an online softmax of its own with its own scores
// and accumulator in tensor memory (S_0 | S_1 | O_0 | O_1): while one group works on its scores the tensor core runs the other's products.
// At the end both join the two results, half the features each.  Q has two buffers, so that the next item's first scores are
// formed under the join.
//   warp 0      scheduler, K producer      warp 1  the thread that issues the MMAs
//   warp 2      V producer, tensor memory  warps 4-7, 8-11  softmax groups
// Every wait is bounded, as in attn_ws.cuh, whose hand-overs of P in parts, lazy rescale and packed fma this kernel has too.
#pragma once
#include <cstdint>

#include "attn_ws.cuh"
#include "common.cuh"
#include "lengths.cuh"
#include "ptx.cuh"

namespace vpp {

constexpr int kBlkListThreads = 128;
constexpr int kBlkWindow = 8192;              // mask words of a window of pages
constexpr int kBlkMaxPages = 8;               // pages of a step (128 keys, pages of 16)
constexpr int kBlkInfo = 8;                   // steps whose masks are in shared memory

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
    WorkHeader* header;           // num_units: tiles; error; counter
    BlkItem* items;               // [Hkv, max_tiles]
    int2* pages;                  // [Hkv, max_tiles, max_pages]: physical, logical
    uint32_t* masks;              // [Hkv, max_tiles, max_pages, words]
    int32_t* status;
};

__global__ void __launch_bounds__(kBlkListThreads) block_lists_kernel(const BlkListParams p) {
    extern __shared__ int32_t cu[];           // cu[num_reqs + 1], then tiles before request r [num_reqs + 1]
    __shared__ uint32_t s_mask[kBlkWindow];
    __shared__ int s_count[kBlkListThreads / 32];
    __shared__ int s_bad;
    int32_t* const first_tile = cu + p.num_reqs + 1;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_launch_dependents();
    pdl_wait();
    const bool ok = scan_lengths<kBlkListThreads>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu);
    if (!ok) {
        if (blockIdx.x == 0 && tid == 0) {
            *p.header = WorkHeader{0, 0, 0, 1 /* VPP_DEV_BAD_LENGTHS */, 0, 0, 0, 0, {}};
            if (p.status) *p.status = 1;
        }
        return;
    }
    if (warp == 0) {
        int carry = 0;
        for (int b = 0; b < p.num_reqs; b += 32) {
            const int r = b + lane;
            const int n = r < p.num_reqs ? (cu[r + 1] - cu[r] + p.tile_tokens - 1) / p.tile_tokens : 0;
            int x = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            if (r < p.num_reqs) first_tile[r] = carry + x - n;
            carry += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) first_tile[p.num_reqs] = carry;
    }
    if (tid == 0) s_bad = 0;
    __syncthreads();
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
    int2* const pages = p.pages + item * p.max_pages;
    uint32_t* const masks = p.masks + item * p.max_pages * p.words;
    const int W = p.words, window = kBlkWindow / W, entries = tokens * p.topk;
    int count = 0;            // pages so far
    int last = -1;            // the last of them
    for (int w0 = 0; w0 < used; w0 += window) {
        const int n = min(window, used - w0);
        for (int i = tid; i < n * W; i += kBlkListThreads) s_mask[i] = 0;
        __syncthreads();
        for (int i = tid; i < entries; i += kBlkListThreads) {
            const int t = i / p.topk;
            const int e = lists[static_cast<long long>(t) * p.num_kv_heads * p.topk + (i - t * p.topk)];
            if (e >= w0 && e < w0 + n && e <= ((pos0 + t) >> p.block_shift)) atomicOr(&s_mask[(e - w0) * W + (t >> 5)], 1u << (t & 31));
        }
        __syncthreads();
        // a run of pages a warp: count, then write
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
        int at = count;
        for (int w = 0; w < kBlkListThreads / 32; ++w) {
            if (w < warp) at += s_count[w];
            count += s_count[w];
        }
        for (int i0 = a; i0 < b; i0 += 32) {
            const int i = i0 + lane;
            const bool in = listed(i);
            const uint32_t m = __ballot_sync(0xffffffffu, in);
            if (in) {
                const int k = at + __popc(m & ((1u << lane) - 1));
                const int e = __ldg(table + w0 + i);
                const bool fine = e >= 0 && e < p.num_blocks;
                if (!fine) s_bad = 1;
                pages[k] = make_int2(fine ? e : p.num_blocks, w0 + i);       // (num_blocks: reads as zero)
                for (int w = 0; w < W; ++w) masks[static_cast<long long>(k) * W + w] = fine ? s_mask[i * W + w] : 0;
            }
            at += __popc(m);
            if (m) last = w0 + i0 + 31 - __clz(m);
        }
        __syncthreads();
    }
    // (the last page of the context is in the last window, in the last run with pages)
    const int tail = kv_len & ((1 << p.block_shift) - 1);
    const int has_last = __syncthreads_or(last == (kv_len - 1) >> p.block_shift);
    if (tid == 0) p.items[item] = BlkItem{row0, tokens, pos0, count, has_last ? tail : 0, s_bad, {0, 0}};
}

struct BlkParams {
    const WorkHeader* header_ro;
    WorkHeader* header;
    const BlkItem* items;
    const int2* pages;
    const uint32_t* masks;
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

// masks of a step: pages' logical numbers and tokens
struct BlkInfo {
    int32_t page[kBlkMaxPages];
    uint32_t mask[kBlkMaxPages][4];
};

constexpr int kBlkStages = 4;
constexpr int kBlkBars = (2 + kBlkStages) * kTileBytes;        // offset of what follows the tiles
constexpr int kBlkOffInfo = 512, kBlkOffStat = kBlkOffInfo + kBlkInfo * static_cast<int>(sizeof(BlkInfo));
constexpr int kBlkSmem = kBlkBars + kBlkOffStat + 2 * 2 * 128 * 4 + 1024 /* alignment */;
static_assert(kBlkSmem <= 232448, "shared memory of one CTA");

// The keys of columns 32 w .. 32 w + 31 of a step that a token sees.
__device__ __forceinline__ uint32_t blk_visible(const BlkInfo& f, int w, int shift, int tok, int own, int own_off) {
    const int word = tok >> 5, bit = tok & 31;
    if (shift >= 5) {
        const int s = (w * 32) >> shift, first = (w * 32) & ((1 << shift) - 1);
        if (!((f.mask[s][word] >> bit) & 1)) return 0;
        const int lim = f.page[s] == own ? own_off - first : 31;
        return lim >= 31 ? 0xffffffffu : lim < 0 ? 0u : (2u << lim) - 1;
    }
    uint32_t v = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int s = 2 * w + h;
        if (!((f.mask[s][word] >> bit) & 1)) continue;
        const int lim = f.page[s] == own ? own_off : 15;
        v |= ((2u << lim) - 1) << (16 * h);
    }
    return v;
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
    const uint32_t bar_s_full = sBar + 64, bar_p_full = sBar + 80;         // [2]
    const uint32_t bar_o_full = sBar + 96;                                 // [2]
    const uint32_t bar_p_part = sBar + 112;                                // [2][2]: after 32 and after 64 columns
    const uint32_t bar_kv_full = sBar + 144, bar_kv_empty = sBar + 176;    // [kBlkStages]
    const uint32_t bar_vfix = sBar + 208;                                  // [2]
    const uint32_t bar_info = sBar + 224;                                  // [kBlkInfo]
    const uint32_t bar_stat = sBar + 288, bar_done = sBar + 296;
    uint8_t* const gen_bar = gen + kBlkBars;
    volatile int* const s_abort = reinterpret_cast<volatile int*>(gen_bar + 304);
    volatile uint32_t* const s_tmem = reinterpret_cast<volatile uint32_t*>(gen_bar + 308);
    BlkWork* const ring = reinterpret_cast<BlkWork*>(gen_bar + 320);       // [2]
    static_assert(320 + 2 * sizeof(BlkWork) <= kBlkOffInfo, "item ring");
    BlkInfo* const info = reinterpret_cast<BlkInfo*>(gen_bar + kBlkOffInfo);
    float* const stat = reinterpret_cast<float*>(gen_bar + kBlkOffStat);   // [group][m, l][128]

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_item_full + 8 * i, 1);
            mbar_init(bar_item_empty + 8 * i, 10);      // 8 softmax warps, the MMA thread, the V producer
            mbar_init(bar_q_full + 8 * i, 1);
            mbar_init(bar_q_empty + 8 * i, 1);
            mbar_init(bar_s_full + 8 * i, 1);
            mbar_init(bar_p_full + 8 * i, 4);
            mbar_init(bar_o_full + 8 * i, 1);
            mbar_init(bar_p_part + 8 * i, 4);
            mbar_init(bar_p_part + 16 + 8 * i, 4);
            mbar_init(bar_vfix + 8 * i, 1);
        }
        for (int i = 0; i < kBlkStages; ++i) {
            mbar_init(bar_kv_full + 8 * i, 1);
            mbar_init(bar_kv_empty + 8 * i, 1);
        }
        for (int i = 0; i < kBlkInfo; ++i) mbar_init(bar_info + 8 * i, 1);
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
        // One K (which = 0) or V tile into ring stage it % kBlkStages: `phys` is the page of the lane's copy.
        auto load_tile = [&](int which, uint32_t it, int g, int phys) -> bool {
            const uint32_t st = it % kBlkStages, full = bar_kv_full + 8 * st;
            const bool exact = which == 0 ? p.k_exact : p.v_exact;
            const int rows = exact ? kExactRows : p.box_rows, off = lane * rows;
            bool ok = true;
            if (lane == 0) {
                ok = mbar_wait(bar_kv_empty + 8 * st, ((it / kBlkStages) & 1) ^ 1, s_abort, 603 + which);
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
            uint32_t n_item = 0, it = 0, n_q = 0;
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
                // entries 32 at a time, a lane each
                int2 e = make_int2(0, 0);
                uint32_t m[4] = {};
                const int e0 = w.begin * per_step;
                for (int j = w.begin; j < w.end && ok; ++j) {
                    const int k0 = j * per_step, in = (k0 - e0) & 31;
                    if (in == 0) {
                        const int i = k0 + lane;
                        e = make_int2(p.num_blocks, -1);
#pragma unroll
                        for (int x = 0; x < 4; ++x) m[x] = 0;
                        if (i < w.pages) {
                            e = p.pages[w.list + i];
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                if (x < p.words) m[x] = p.masks[(w.list + i) * p.words + x];
                        }
                    }
                    const int phys = __shfl_sync(0xffffffffu, e.x, in + ((lane * copy_rows) >> shift));
                    ok = load_tile(0, it, w.g, phys);
                    if (!ok) break;
                    // (the stage is free, so the softmax has read the masks of four steps ago)
                    const uint32_t s = (it >> 1) % kBlkInfo;
                    if (lane >= in && lane < in + per_step) {
                        info[s].page[lane - in] = e.y;
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            if (x < p.words) info[s].mask[lane - in][x] = m[x];
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_info + 8 * s);
                    it += 2;
                }
                if (!ok) break;
            }
        } else if (warp == 2) {
            // ============================ V producer ============================
            uint32_t n_item = 0, it = 0, fixes = 0;
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
                    if (in == 0) phys_mine = k0 + lane < w.pages ? p.pages[w.list + k0 + lane].x : p.num_blocks;
                    const int phys = __shfl_sync(0xffffffffu, phys_mine, in + ((lane * copy_rows) >> shift));
                    ok = load_tile(1, it + 1, w.g, phys);
                    if (!ok) break;
                    if (w.last_keys != 0 && j == steps - 1) {
                        // slots past the end hold anything: their values become 0, so that 0 * garbage cannot reach O.  The MMA thread waits for it.
                        const uint32_t st = (it + 1) % kBlkStages;
                        if (lane == 0) ok = mbar_wait(bar_kv_full + 8 * st, ((it + 1) / kBlkStages) & 1, s_abort, 612);
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
                    it += 2;
                }
                if (!ok) break;
            }
        } else if (warp == 1 && lane == 0) {
            // ============================ MMA issuer (a single thread) ============================
            constexpr uint32_t kIdescQK = idesc_bf16(128, 128, false, false), kIdescPV = idesc_bf16(128, 128, false, true);
            constexpr uint32_t kHiQ = desc_hi_sw128(1024), kHiKV = desc_hi_sw128(kGroupBytes);
            uint32_t n_item = 0, n_q = 0, it = 0, fixes = 0, p_it0 = 0, p_it1 = 0;
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
                const uint32_t q_lo = desc_lo_sw128(sQ + qb * kTileBytes, 16), first = it;
                // step j takes ring entries first + 2 j (K) and first + 2 j + 1 (V), and group j & 1
                auto scores = [&](int j) -> bool {
                    const uint32_t idx = first + 2 * j, st = idx % kBlkStages;
                    if (!wait(bar_kv_full + 8 * st, (idx / kBlkStages) & 1, 623)) return false;
                    tc_fence_after();
                    const uint32_t k_lo = desc_lo_sw128(sKV + st * kTileBytes, 16), tS = tmem + (j & 1) * 128;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint32_t qoff = ((k >> 2) * kSlabBytes + (k & 3) * 32) >> 4, koff = ((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4;
                        mma_ss_lhh(tS, q_lo + qoff, kHiQ, k_lo + koff, kHiKV, kIdescQK, k > 0);
                    }
                    tc_commit(bar_s_full + 8 * (j & 1));
                    tc_commit(bar_kv_empty + 8 * st);
                    if (j + 1 == n) tc_commit(bar_q_empty + 8 * qb);
                    return true;
                };
                bool ok = scores(0);
                if (ok && n > 1) ok = scores(1);
                for (int j = 0; j < n && ok; ++j) {
                    const int t = j & 1;
                    const uint32_t idx = first + 2 * j + 1, st = idx % kBlkStages, pit = t ? p_it1 : p_it0;
                    ok = wait(bar_kv_full + 8 * st, (idx / kBlkStages) & 1, 624);
                    if (!ok) break;
                    if (mend && j == n - 1) {
                        ok = wait(bar_vfix + 8 * (fixes & 1), (fixes >> 1) & 1, 625);
                        if (!ok) break;
                        ++fixes;
                    }
                    const uint32_t tP = tmem + t * 128, tO = tmem + 256 + t * 128, v_lo = desc_lo_sw128(sKV + st * kTileBytes, kHalfBytes);
                    int k0 = 0;
#pragma unroll
                    for (int c = 0; c < 3; ++c) {
                        ok = wait(c < 2 ? bar_p_part + 16 * c + 8 * t : bar_p_full + 8 * t, pit & 1, 626 + c);
                        if (!ok) break;
                        tc_fence_after();
                        const int k1 = c < 2 ? 2 * (c + 1) : 8;
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (k >= k0 && k < k1) mma_ts_lh(tO, tP + k * 8, v_lo + k * (2 * kGroupBytes >> 4), kHiKV, kIdescPV, (j >= 2 || k > 0) ? 1u : 0u);
                        k0 = k1;
                    }
                    if (!ok) break;
                    tc_commit(bar_kv_empty + 8 * st);
                    if (t) ++p_it1; else ++p_it0;
                    if (j + 2 < n) ok = scores(j + 2);
                    else tc_commit(bar_o_full + 8 * t);
                }
                if (!ok) break;
                it = first + 2 * n;
            }
        }
        // warp 3 has nothing to do until teardown
    } else {
        // ===================================== softmax groups =====================================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kWsRegsHigh));
        const int t = (warp - 4) >> 2, row = ((warp & 3) << 5) | lane;
        const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + t * 128 + lane_off, tO = tmem + 256 + t * 128 + lane_off;
        const float sc = p.scale_log2e;
        const int my_tok = row / p.group, my_head = row - my_tok * p.group;
        uint32_t n_item = 0, s_it = 0, o_it = 0, x_it = 0, step0 = 0;      // step0: steps of the items before
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
            for (int j = t; j < n; j += 2) {
                const uint32_t step = step0 + j, slot_i = step % kBlkInfo;
                ok = mbar_wait(bar_info + 8 * slot_i, (step / kBlkInfo) & 1, s_abort, 632);
                if (!ok) break;
                uint32_t vis[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) vis[c] = live ? blk_visible(info[slot_i], c, shift, tok, own, own_off) : 0u;
                const bool mine = (vis[0] | vis[1] | vis[2] | vis[3]) != 0;
                seen |= mine;
                const bool none = !__any_sync(0xffffffffu, mine);
                ok = mbar_wait(bar_s_full + 8 * t, s_it & 1, s_abort, 633);
                if (!ok) break;
                ++s_it;
                tc_fence_after();
                if (none) {
                    // no row of this warp sees a key of this step
                    uint32_t z[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) z[i] = 0;
                    tmem_st32(tS, z);
                    tmem_st32(tS + 32, z);
                    tc_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(bar_p_part + 8 * t);
                        mbar_arrive(bar_p_part + 16 + 8 * t);
                        mbar_arrive(bar_p_full + 8 * t);
                    }
                    continue;
                }
                uint32_t s[128];
                float mx[8];
                tmem_ld32(tS, reinterpret_cast<uint32_t(&)[32]>(s[0]));
                tmem_ld32(tS + 32, reinterpret_cast<uint32_t(&)[32]>(s[32]));
                tc_wait_ld(reinterpret_cast<uint32_t(&)[32]>(s[0]));
                tc_wait_ld(reinterpret_cast<uint32_t(&)[32]>(s[32]));
                tmem_ld32(tS + 64, reinterpret_cast<uint32_t(&)[32]>(s[64]));
                tmem_ld32(tS + 96, reinterpret_cast<uint32_t(&)[32]>(s[96]));
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    if (hh == 1) {
                        tc_wait_ld(reinterpret_cast<uint32_t(&)[32]>(s[64]));
                        tc_wait_ld(reinterpret_cast<uint32_t(&)[32]>(s[96]));
                    }
#pragma unroll
                    for (int c = 2 * hh; c < 2 * hh + 2; ++c)
                        if (__any_sync(0xffffffffu, vis[c] != 0xffffffffu)) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (!((vis[c] >> i) & 1)) s[c * 32 + i] = 0xff800000u;  // -inf
                        }
#pragma unroll
                    for (int i = 0; i < 64; i += 16)
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float v0 = __uint_as_float(s[hh * 64 + i + k]), v1 = __uint_as_float(s[hh * 64 + i + 8 + k]);
                            mx[k] = (hh == 0 && i == 0) ? fmaxf(v0, v1) : fmax3(mx[k], v0, v1);
                        }
                }
                const float mxa = fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), fmaxf(fmaxf(mx[4], mx[5]), fmaxf(mx[6], mx[7])));
                const float m_new = fmaxf(mxa * sc, m_ref);
                const bool grow = (m_new - m_ref > kRescaleThreshold) || (m_ref == -INFINITY && m_new != -INFINITY);
                if (__any_sync(0xffffffffu, grow)) {
                    const float alpha = grow ? ex2(m_ref - m_new) : 1.f;  // m_ref = -inf gives 0
                    if (grow) m_ref = m_new;
                    l_run *= alpha;
                    if (j >= 2) {   // O of this group already holds something
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
                float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t pk[16];
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        float x0, x1;
                        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[c * 32 + i]), __uint_as_float(s[c * 32 + i + 1])), sc2, neg_m2), x0, x1);
                        const float p0 = ex2(x0), p1 = ex2(x1);
                        sum0 += p0;
                        sum1 += p1;
                        pk[i >> 1] = pack_bf16x2(p0, p1);
                        if ((c == 1 || c == 2) && (i >> 1) == kPartWaitDefer - 1) {
                            tc_wait_st();
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(bar_p_part + 16 * (c - 1) + 8 * t);
                        }
                    }
                    tmem_st16(tS + c * 16, pk);
                }
                l_run += sum0 + sum1;
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_p_full + 8 * t);
            }
            if (!ok) break;
            step0 += n;
            // ---- the two groups' results joined, half the features each ----
            if (t < n) {
                ok = mbar_wait(bar_o_full + 8 * t, o_it & 1, s_abort, 634);
                if (!ok) break;
                ++o_it;
            }
            tc_fence_after();
            if (seen && m_ref == -INFINITY && l_run == 0.f) l_run = NAN;        // keys, but all scores -inf: 0 / 0, as the definition has it
            stat[t * 256 + row] = m_ref;
            stat[t * 256 + 128 + row] = l_run;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_stat);
            ok = mbar_wait(bar_stat, x_it & 1, s_abort, 635);
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
            const long long prow = static_cast<long long>(w.split) * p.total_q * p.num_q_heads + orow;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {        // 16 features at a time
                uint32_t r[32];                  // (O_0's, O_1's)
                float v[16];
                if (n > 0) tmem_ld16(tH + c * 16, reinterpret_cast<uint32_t(&)[16]>(r[0]));
                if (n > 1) tmem_ld16(tH + 128 + c * 16, reinterpret_cast<uint32_t(&)[16]>(r[16]));
                tc_wait_ld(r);
#pragma unroll
                for (int i = 0; i < 16; ++i) {   // (an accumulator without weight is not looked at: 0 * inf)
                    v[i] = s0 != 0.f && n > 0 ? __uint_as_float(r[i]) * s0 : s0;
                    if (s1 != 0.f && n > 1) v[i] = fmaf(__uint_as_float(r[16 + i]), s1, v[i]);
                }
                if (!live) continue;
                if (p.splits == 1) {
                    uint32_t pk[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) pk[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
                    uint4* const dst = reinterpret_cast<uint4*>(p.out + (orow * 128 + t * 64 + c * 16) * 2);
                    dst[0] = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                    dst[1] = make_uint4(pk[4], pk[5], pk[6], pk[7]);
                } else {
                    float4* const dst = reinterpret_cast<float4*>(p.o_parts + prow * 128 + t * 64 + c * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) dst[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
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
            ok = mbar_wait(bar_done, x_it & 1, s_abort, 636);      // (both accumulators and the statistics are read)
            if (!ok) break;
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
