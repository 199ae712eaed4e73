// Page selection: which cache pages each token's attention should read, from a score that is cheap to form.
//
// For token t of request r at position p, kv-head g and page b (b < p / block_size + 1):
//     s(t, g, b) = sum over the q-heads h of g of <q_h(t), mean_b,g>  =  < sum_h q_h(t), mean_b,g >
// The first `num_first` pages and the last `num_last` (the token's own among them) are always taken, the rest of the topk by
// score, ties to the lowest index, and NaN below everything.  The list comes out ascending, -1 behind it where fewer pages exist.
//
// The selection is that of exact arithmetic.  Scores are formed in 32 bits with a bound on their error, and where two pages near
// the border are closer than the bound allows to tell, theirs are formed again in 64 bits (products of bf16 are exact there).
//
// Kernels of a slab of tokens (one slab unless their candidates take more than kSelectSlabBytes):
//  * block_filter_kernel: an item is (up to 256 tokens of one request, kv-head, a run of pages), a block of 16 warps and four that issue the MMAs.  The group's
//    queries are summed first, in 32 bits, and the sum split in two bf16 (hi + rest), so that the tensor cores do 2 / group
//    of the work of all q-heads; scores of 128 tokens x 128 pages are one accumulator, and an item has two of those a step, with two buffers: the next step's
//    products run under this one's scores.  They are formed twice: the first time the maxima of groups
//    of pages are kept, whose need-th largest bounds a token's border from below; the second time what is not below that by more than the error
//    bound -- a few more pages than needed -- is written down, a thread a token and half of the pages.
//  * block_few_kernel: tokens of requests of up to kSelectFew in the slab -- decode rows, a last rest -- multiplied by warps from the registers that the loads fill, the scores in
//    shared memory: there reading the means is all.
//  * block_pick_kernel: a warp a (token, kv-head) ranks the candidates and settles the border.
// 8192 tokens of 64/4 heads, 1152 pages, lists of 32: 125 us in a captured graph (132 as calls one after the other), of which the filter takes 88: 26 reading 134 MB of q (21 at the copy rate), then 18 steps of 2.4 (maxima)
// and 4.4 thousand clk (lists), where the products take 2.05; of its issue slots 48 %, of the tensor pipe 24 %.  One row of twenty has pages too close for 32 bits (8 us).
// An infinite or NaN mean, or more than `cap` pages of one half within the bound of the border (zero or repeated keys), send every row that scores them through 64 bits, a page after the other
// (pick_thorough): the same call takes 5.6 to 7.1 ms then, 16 decode rows 0.15 to 1.0 ms instead of 27 us.
// Before: all scores written down once, 4.6 KB a token and kv-head, and picked from there, 420 us; items of 128 tokens, eight warps that do one thing after the
// other, two an SM, 195; items of 224 tokens, 148 of them, 130; means fetched and bounded by the four other warps alone, 3900 clk a step for 64 copies.
#pragma once
#include <cuda_bf16.h>

#include <cstdint>

#include "device_status.h"
#include "lengths.cuh"
#include "ptx.cuh"
#include "rope.cuh"

namespace vpp {

constexpr int kSelectTile = 128;              // tokens of an accumulator, pages of a step
constexpr int kSelectItem = 256;              // tokens of an item
constexpr int kSelectThreads = 512;           // of block_filter_kernel, beside the warp that issues and three that make it a group of four
// Registers a thread after the roles split: the launch gives 96 (five warps a sub-partition), of which the last four warps hand back 32 (72: the thread that issues spills, 132 us instead of 128).
constexpr int kSelectRegsLow = 64, kSelectRegsHigh = 104;
static_assert(4 * kSelectRegsHigh + kSelectRegsLow <= 5 * 96, "register budget");
constexpr int kSelectFew = 4;
constexpr int kFewThreads = 512;
constexpr int kSelectSlabBytes = 128 << 20;
constexpr int kSelectMaxTopk = 256;
constexpr int kSelectMaxRun = 4096;           // pages of an item: their scores, or their places, are kept in shared memory
constexpr int kSelectA = 2 * 2 * kSelectTile * 128;   // an accumulator's operand: two bf16 parts of 128 x 128, two 64-feature slabs each
constexpr int kSelectB = 2 * kSelectTile * 128;
constexpr int kSelectSmem = 2 * kSelectA + 2 * kSelectB + 1024 /* alignment */ + 4096 /* barriers, borders */;      // and the pages
static_assert(kSelectSmem + 4 * kSelectMaxRun <= 232448 - 8 * 1024, "shared memory of one CTA");
static_assert(2 * 4 * (kLengthsMaxReqs + 1) <= 2 * kSelectA, "the lengths fit where the operands come");

// A page that may be among a token's best.
struct __align__(8) SelectCandidate {
    float score;
    int32_t page;
};

struct SelectParams {
    const uint8_t* q;             // [total_q, Hq, 128] bf16
    const uint8_t* means;         // [num_blocks, Hkv, 128] bf16
    const int32_t* block_table;
    const int32_t* prefix_len;
    const int32_t* chunk_len;
    int num_reqs, max_blocks_per_req, block_shift, num_blocks;
    long long capacity;
    int total_q, num_q_heads, num_kv_heads;
    int topk, num_first, num_last;
    int row0, row1;               // this slab's tokens
    int run_pages, runs;          // pages of an item (a multiple of 128), items along a row (0: nothing is scored)
    int group_pages;              // pages of a group of which the maximum is kept (4, 2, 1; 0: 64 groups of every 64th page or so, in registers)
    int item_tokens;              // of an item, at most
    int cap;                      // candidates of half an item's pages, at most
    SelectCandidate* found;       // [row1 - row0, Hkv, runs, 2, cap]
    int32_t* counts;              // [row1 - row0, Hkv, runs, 2] (past cap: more than fit)
    float* bounds;                // [row1 - row0, Hkv, runs]: error bound of the row's scores of a run
    float* maxima;                // [many_items, 256, run_pages / group_pages] (group_pages > 0)
    int32_t* bad;                 // one word an item of the slab, of both kernels
    int many_items, items;        // of block_filter_kernel, of both
    int32_t* indices;             // [total_q, Hkv, topk]
    int32_t* status;
};

// Candidates of a token whose own page is `own`: pages [num_first, end).
__device__ __forceinline__ int select_end(const SelectParams& p, int own) { return own + 1 - p.num_last; }

// Bound on the error of an item's scores, formed by the tensor cores from the two parts of the summed query:
//
//     |fp32 score - exact score| <= (13 2^-19 |s| + G 2^-23 |a|) |mean|          s = sum_h q_h,  a = sum_h |q_h| (features);  |.|: 2-norms
//
// by Cauchy and Schwarz.  The split leaves 2^-17 of s.  16 products and the sum so far are added a step, with at most 2^-23 of their absolute sum lost each: 8 steps of the
// part that is small come first and lose 2^-8 of 2^-16 of |s| |mean|, 8 of the other 17 2^-20.  (4 + 8.5 + 0.04) 2^-19.
// Forming s is G - 1 additions of at most 2^-24 of a feature's a each.  token_weight is what stands before |mean|: 0 where the queries are 0, infinite where anything is or
// where products could overflow.  (Squares may vanish: below 1e-30 the sum of a is taken, which is no less than either norm.)
// (With the largest feature of the means and the sum of all |q| in place of the norms two thirds of all rows had pages too close to tell.)
__device__ __forceinline__ float token_weight(int group, float sum_a, float square_a, float square_s) {
    if (!(sum_a < 1e38f)) return INFINITY;
    const float s = square_s > 1e-30f ? sqrtf(square_s) * 1.001f : sum_a, a = square_a > 1e-30f ? sqrtf(square_a) * 1.001f : sum_a;
    return 2.4795532e-5f * s + static_cast<float>(group) * 1.1920929e-7f * a;
}
// square: the largest sum of squares of a page's features as mean_square forms it (bits; NaN above infinity above everything finite).
__device__ __forceinline__ float select_bound(float weight, uint32_t square) {
    const float norm = sqrtf(__uint_as_float(square) * 1.02f) * 1.001f + 2e-18f;
    if (weight == 0.f && norm < INFINITY) return 0.f;
    return weight * norm + 1e-35f;
}
// Sum of squares of 8 features, at least 0.98 of it (four roundings to bf16); features below 1e-19 may be lost.
__device__ __forceinline__ float mean_square(uint4 v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    __nv_bfloat162 acc = __floats2bfloat162_rn(0.f, 0.f);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&w[e]);
        acc = __hfma2(x, x, acc);
    }
    return __low2float(acc) + __high2float(acc);
}

// Unsigned integers in the order of floats; NaN below everything.
__device__ __forceinline__ uint32_t order_key(float f) {
    if (!(f == f)) return 0;
    const uint32_t u = __float_as_uint(f + 0.f);          // (-0 becomes 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// A value that at least `need` of n numbers reach, and not many more: the need-th largest of 32 * kKeys maxima over value(i), i = lane + 32 k, by a warp.
// -inf where there are fewer maxima.
template <int kKeys, typename Value>
__device__ __forceinline__ float border_below(int n, int need, Value value) {
    const int lane = threadIdx.x & 31;
    float mx[kKeys];
#pragma unroll
    for (int k = 0; k < kKeys; ++k) mx[k] = -INFINITY;
    for (int i = lane; i < n; i += 32 * kKeys) {
#pragma unroll
        for (int k = 0; k < kKeys; ++k)
            if (i + 32 * k < n) mx[k] = fmaxf(mx[k], value(i + 32 * k));
    }
    uint32_t key[kKeys], t = 0;
#pragma unroll
    for (int k = 0; k < kKeys; ++k) key[k] = order_key(mx[k]);
    for (int b = 31; b >= 8; --b) {              // (a little below will do)
        const uint32_t c = t | (1u << b);
        int k = 0;
#pragma unroll
        for (int e = 0; e < kKeys; ++e) k += key[e] >= c;
        const int all = static_cast<int>(__reduce_add_sync(0xffffffffu, k));
        if (all >= need) t = c;
        if (all == need) break;
    }
    return t < 0x00800000u ? -INFINITY : key_value(t);      // (maxima of nothing)
}
template <typename Value>
__device__ __forceinline__ float border_of(int n, int need, Value value) {
    return need <= 64 ? border_below<8>(n, need, value) : border_below<16>(n, need, value);
}

// Rows of request r inside the slab: their number, and the first.
__device__ __forceinline__ int slab_rows(const SelectParams& p, const int32_t* cu, int r, int& lo) {
    lo = max(cu[r], p.row0);
    const int n = min(cu[r + 1], p.row1) - lo;
    return n > 0 ? n : 0;
}

// D += A B, 16 x 8 += 16 x 16 times 16 x 8, bf16, by a warp
__device__ __forceinline__ void mma_16x8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Few tokens: a block a (token, kv-head, run of pages); by_token 1: any token of the slab (launches of decode rows: however the tokens lie in the requests), 0: one of
// kSelectFew places of every request, of which those with more tokens are left to block_filter_kernel.  Reading the means is all that takes time, if it goes
// with few instructions: 16 pages a warp and round, multiplied by small matrix instructions straight from the registers that the loads fill (each lane's features are a
// permutation of the product's inner index that the other operand shares).  The columns of that operand are the two parts of the summed query, and for the absolute
// products that bound the error -- the same registers without signs -- those of the parts and of sum_h |q_h|.  (Dot products in registers, eight lanes a page: 400 instructions
// for 16 pages instead of 70; 16 rows of 64/8 heads, up to 2048 pages, took 32 us with block_pick_kernel behind it, and take 26.)
__global__ void __launch_bounds__(kFewThreads) block_few_kernel(const SelectParams p, const int by_token) {
    extern __shared__ float s_score[];                              // [run_pages], then cu [num_reqs + 1]
    constexpr int kWarps = kFewThreads / 32;
    __shared__ __align__(16) __nv_bfloat16 s_ask[3][128];           // the summed query's parts, sum_h |q_h|
    __shared__ uint32_t s_product, s_forming;                       // largest sums of absolute products (bits)
    __shared__ float s_largest[kFewThreads], s_floor;
    __shared__ int s_count[kWarps], s_bad;
    int32_t* const cu = reinterpret_cast<int32_t*>(s_score + p.run_pages);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gr = lane >> 2, tq = lane & 3;
    if (tid == 0) s_bad = 0;
    pdl_launch_dependents();
    pdl_wait();
    const bool ok = scan_lengths<kFewThreads>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu);
    int32_t* const flag = p.bad + p.many_items + blockIdx.x;
    int id = blockIdx.x;
    const int run = id % p.runs, g = (id /= p.runs) % p.num_kv_heads;
    id /= p.num_kv_heads;
    int r = 0, row = p.row0 + id;
    bool mine = ok && row < p.row1;
    if (ok && by_token) {
        if (mine) r = request_of(cu, p.num_reqs, row);
    } else if (ok) {
        int lo;
        r = id / kSelectFew;
        const int rows = slab_rows(p, cu, r, lo);
        row = lo + id % kSelectFew;
        mine = rows <= kSelectFew && row < lo + rows;
    }
    const int own = mine ? (p.prefix_len[r] + (row - cu[r])) >> p.block_shift : 0;
    // a page run that nobody needs: below the first candidate, past the last, or the token has no more pages than it may list
    const int page0 = run * p.run_pages, page1 = min(page0 + p.run_pages, select_end(p, own)), begin = max(page0, p.num_first);
    if (!mine || page1 <= begin || own + 1 <= p.topk) {
        if (tid == 0) *flag = ok ? 0 : 1 /* VPP_DEV_BAD_LENGTHS */;
        return;
    }
    const int G = p.num_q_heads / p.num_kv_heads, need = p.topk - p.num_first - p.num_last;
    const int32_t* const table = p.block_table + static_cast<long long>(r) * p.max_blocks_per_req;
    const uint8_t* const means = p.means + g * 256 + tq * 16;
    const long long mean_stride = static_cast<long long>(p.num_kv_heads) * 256;
    bool bad = false;
    // rows gr and gr + 8 of a round's 16 pages; -1: counts as 0 (pages that are taken anyway: what theirs hold must not widen the bound)
    int e[2];
    auto look = [&](int j0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = j0 + gr + 8 * i;
            e[i] = j >= begin && j < page1 ? __ldg(table + j) : -1;
            bad |= j >= begin && j < page1 && (e[i] < 0 || e[i] >= p.num_blocks);
        }
    };
    uint4 x[2][8];
    auto fetch = [&](uint4 (&to)[8]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool fine = e[i] >= 0 && e[i] < p.num_blocks;
            const uint8_t* const from = means + (fine ? e[i] : 0) * mean_stride;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                to[4 * i + v] = make_uint4(0, 0, 0, 0);
                if (fine) to[4 * i + v] = ld_once(from + v * 64);
            }
        }
    };
    const int first = page0 + warp * 16;
    constexpr int kStep = kWarps * 16;
    look(first);
    fetch(x[0]);
    look(first + kStep);
    fetch(x[1]);
    look(first + 2 * kStep);
    bool some = false;
    if (tid < 128) {
        float s = 0.f, a = 0.f;
        const __nv_bfloat16* const q = reinterpret_cast<const __nv_bfloat16*>(p.q) + (static_cast<long long>(row) * p.num_q_heads + g * G) * 128 + tid;
#pragma unroll 8
        for (int h = 0; h < G; ++h) {
            const float y = __bfloat162float(q[h * 128]);
            s += y;
            a += fabsf(y);
        }
        const __nv_bfloat16 hi = __float2bfloat16(s);
        s_ask[0][tid] = hi;
        s_ask[1][tid] = __float2bfloat16(s - __bfloat162float(hi));
        s_ask[2][tid] = __float2bfloat16(fmaxf(a, 1e-30f));      // (parts below 2^-126 are cut at 2^-134: less than 2^-23 of that.  NaN and infinity show in the parts)
        some = a != 0.f;
    }
    if (tid == 0) s_product = s_forming = 0;
    const bool zero = !__syncthreads_or(some);
    // column gr of the operands: vector tq + 4 v of the features, two steps of the product in each
    uint32_t ask[16];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        uint4 y = make_uint4(0, 0, 0, 0);
        if (gr < 3) y = *reinterpret_cast<const uint4*>(&s_ask[gr][(tq + 4 * v) * 8]);
        ask[4 * v] = y.x;
        ask[4 * v + 1] = y.y;
        ask[4 * v + 2] = y.z;
        ask[4 * v + 3] = y.w;
    }
    uint32_t product = 0, forming = 0;
    auto multiply = [&](const uint4 (&y)[8], int j0) {
        float d[4] = {}, n[4] = {};
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const uint4 a = y[v], b = y[4 + v];
            constexpr uint32_t kAbs = 0x7fff7fffu;
            mma_16x8(d, a.x, b.x, a.y, b.y, ask[4 * v], ask[4 * v + 1]);
            mma_16x8(n, a.x & kAbs, b.x & kAbs, a.y & kAbs, b.y & kAbs, ask[4 * v] & kAbs, ask[4 * v + 1] & kAbs);
            mma_16x8(d, a.z, b.z, a.w, b.w, ask[4 * v + 2], ask[4 * v + 3]);
            mma_16x8(n, a.z & kAbs, b.z & kAbs, a.w & kAbs, b.w & kAbs, ask[4 * v + 2] & kAbs, ask[4 * v + 3] & kAbs);
        }
        if (tq == 0) {                // columns 0 and 1: the parts
            if (j0 + gr < page1) s_score[j0 + gr - page0] = d[0] + d[1];
            if (j0 + gr + 8 < page1) s_score[j0 + gr + 8 - page0] = d[2] + d[3];
            product = max(product, max(__float_as_uint(n[0] + n[1]) & 0x7fffffffu, __float_as_uint(n[2] + n[3]) & 0x7fffffffu));
        } else if (tq == 1) {         // column 2
            forming = max(forming, max(__float_as_uint(n[0]) & 0x7fffffffu, __float_as_uint(n[2]) & 0x7fffffffu));
        }
    };
    for (int j0 = first; j0 < page1; j0 += 2 * kStep) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            multiply(x[k], j0 + k * kStep);
            fetch(x[k]);
            look(j0 + (k + 3) * kStep);
        }
    }
    product = __reduce_max_sync(0xffffffffu, product);
    forming = __reduce_max_sync(0xffffffffu, forming);
    if (lane == 0) {
        atomicMax(&s_product, product);
        atomicMax(&s_forming, forming);
    }
    __syncthreads();                  // (the scores are there)
    // The border: a warp's part of the pages, a maximum a lane; the first warp takes the need-th largest of them all.  (One warp through all pages: 5 us of 2048.)
    const float* const scores = s_score - page0;
    const int part = (page1 - begin + 32 * kWarps - 1) / (32 * kWarps) * 32, from = min(page1, begin + warp * part), to = min(page1, from + part);
    float largest = -INFINITY;
    for (int j = from + lane; j < to; j += 32) largest = fmaxf(largest, scores[j]);
    s_largest[tid] = largest;
    __syncthreads();
    // as token_weight, from the absolute products themselves: the split leaves 2^-17 of s, 128 products of either part are accumulated, 16 and the sum so far a step, with at most 2^-23
    // of their absolute sum lost each, together below 2^-15 of it; forming s G - 1 additions of 2^-24 (1.01: sum_h |q_h| is rounded)
    const float worst = __uint_as_float(s_product) * 3.0517578e-5f + __uint_as_float(s_forming) * (1.01f * 1.1920929e-7f) * G;
    const float bound = worst < 1e34f ? (zero ? 0.f : worst + 1e-35f) : INFINITY;
    const long long list = (static_cast<long long>(row - p.row0) * p.num_kv_heads + g) * p.runs + run;
    const bool any = bound > 0.f && bound < INFINITY;
    if (warp == 0) {
        // (more than 512 are never needed, and where there are fewer than are needed, that is that many pages or fewer a lane, all are listed)
        float f = -INFINITY;
        if (any && page1 - begin > p.cap) f = border_below<kWarps>(kFewThreads, need, [&](int i) { return s_largest[i]; }) - 2.f * bound;
        if (lane == 0) s_floor = f;
    }
    __syncthreads();
    const float floor = any ? s_floor : INFINITY;
    int m = 0;
    for (int j0 = from; j0 < to; j0 += 32) m += __popc(__ballot_sync(0xffffffffu, j0 + lane < to && scores[j0 + lane] >= floor));
    if (lane == 0) s_count[warp] = m;
    __syncthreads();
    int at = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) at += s_count[w];
        all += s_count[w];
    }
    SelectCandidate* const found = p.found + list * 2 * p.cap;
    for (int j0 = from; j0 < to; j0 += 32) {
        const int j = j0 + lane;
        const float y = j < to ? scores[j] : 0.f;
        const bool take = j < to && y >= floor;
        const uint32_t b = __ballot_sync(0xffffffffu, take);
        const int k = at + __popc(b & ((1u << lane) - 1));
        if (take && k < p.cap) found[k] = SelectCandidate{y, j};
        at += __popc(b);
    }
    if (tid == 0) {
        p.bounds[list] = bound;
        p.counts[list * 2] = all;
        p.counts[list * 2 + 1] = 0;
    }
    if (bad) s_bad = 1;
    __syncthreads();
    if (tid == 0) *flag = s_bad ? 2 /* VPP_DEV_BAD_BLOCK */ : 0;
}

__global__ void __launch_bounds__(kSelectThreads + 128, 1) block_filter_kernel(const SelectParams p) {
    extern __shared__ uint8_t smem_raw[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const gen = smem_raw + (base - smem_u32(smem_raw));
    uint8_t* const sB = gen + 2 * kSelectA;
    uint8_t* const sX = sB + 2 * kSelectB;
    const uint32_t bar = base + 2 * kSelectA + 2 * kSelectB;           // [2] scores of a buffer
    volatile int* const s_abort = reinterpret_cast<volatile int*>(sX + 16);
    volatile uint32_t* const s_tmem = reinterpret_cast<volatile uint32_t*>(sX + 20);
    int* const s_badp = reinterpret_cast<int*>(sX + 28);
    uint32_t* const s_square = reinterpret_cast<uint32_t*>(sX + 32);
    float* const s_weight = reinterpret_cast<float*>(sX + 64);         // [256] what a token's bound is made of
    float* const s_floor = s_weight + kSelectItem;                         // [256] lowest score of a candidate
    int32_t* const s_page = reinterpret_cast<int32_t*>(sX + 4096);     // [run_pages] physical page, -1: counts as 0
    int32_t* const cu = reinterpret_cast<int32_t*>(gen);               // [num_reqs + 1], then items before request r [num_reqs + 1]: until the queries come there
    int32_t* const first_item = cu + p.num_reqs + 1;

    if (tid == 0) {
        *s_abort = 0;
        *s_square = 0;
        *s_badp = 0;
        mbar_init(bar, 1);
        mbar_init(bar + 8, 1);
        fence_mbar_init();
    }
    pdl_launch_dependents();
    pdl_wait();
    constexpr int kAll = kSelectThreads + 128;
    const bool ok = scan_lengths<kAll>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu);
    const int item = blockIdx.x;
    if (!ok) {
        if (tid == 0) p.bad[item] = 1 /* VPP_DEV_BAD_LENGTHS */;
        return;
    }
    block_scan<kAll>(p.num_reqs, 0x7fffffffu, first_item, false, [&](int r, bool&) {
        int lo;
        const int n = slab_rows(p, cu, r, lo);
        return n > kSelectFew ? (n + p.item_tokens - 1) / p.item_tokens : 0;      // (the others: block_few_kernel)
    });
    const int run = item % p.runs, tg = item / p.runs, g = tg % p.num_kv_heads, tile = tg / p.num_kv_heads;
    if (tile >= first_item[p.num_reqs]) {
        if (tid == 0) p.bad[item] = 0;
        return;
    }
    const int r = request_of(first_item, p.num_reqs, tile);
    int lo;
    const int rows_r = slab_rows(p, cu, r, lo);
    const int row = lo + (tile - first_item[r]) * p.item_tokens;
    const int n = min(min(p.item_tokens, kSelectItem), lo + rows_r - row);      // (kSelectItem: what the compiler unrolls for)
    const int pos0 = p.prefix_len[r] + (row - cu[r]);
    const int end = select_end(p, (pos0 + n - 1) >> p.block_shift);      // of the item's last token
    // a page run that nobody needs: below the first candidate, past the last, or no token has more pages than it may list
    const int page0 = run * p.run_pages, page1 = min(page0 + p.run_pages, end), begin = max(page0, p.num_first);
    if (page1 <= begin || ((pos0 + n - 1) >> p.block_shift) + 1 <= p.topk) {
        if (tid == 0) p.bad[item] = 0;
        return;
    }
    const int G = p.num_q_heads / p.num_kv_heads, need = p.topk - p.num_first - p.num_last, pages = page1 - page0;
    // of token t of the item: candidates of this run (one past the last), and where its lists are
    auto end_of = [&](int t) {
        const int own = (pos0 + t) >> p.block_shift;
        return own + 1 <= p.topk ? 0 : min(page1, select_end(p, own));
    };
    auto list_of = [&](int t) { return (static_cast<long long>(row - p.row0 + t) * p.num_kv_heads + g) * p.runs + run; };
    if (warp == kSelectThreads / 32) {
        tmem_alloc(smem_u32(const_cast<uint32_t*>(s_tmem)), 512);
        tmem_relinquish();
    }
    {
        const int32_t* const table = p.block_table + static_cast<long long>(r) * p.max_blocks_per_req + page0;
        bool bad = false;
        for (int j = tid; j < pages; j += kAll) {
            const int e = __ldg(table + j);
            const bool fine = e >= 0 && e < p.num_blocks;
            bad |= !fine;
            s_page[j] = fine && page0 + j >= begin ? e : -1;      // (pages that are taken anyway count as 0: what theirs hold must not widen the bound)
        }
        if (bad) *s_badp = 1;
    }
    const int v = tid & 15;
    __syncthreads();                      // (all have read their lengths)
    // ---- the group's queries, summed and split ----
    if (tid < kSelectThreads) {
        const uint8_t* const q0 = p.q + (static_cast<long long>(row) * p.num_q_heads + g * G) * 256 + v * 16;
        for (int t = tid >> 4; t < n; t += kSelectThreads / 16) {
            float s[8] = {}, a[8] = {};
            const uint8_t* const src = q0 + static_cast<long long>(t) * p.num_q_heads * 256;
#pragma unroll 8
            for (int h = 0; h < G; ++h) {
                const uint4 y = ld_once(src + h * 256);
                const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    s[2 * k] += bf16_lo(w[k]);
                    s[2 * k + 1] += bf16_hi(w[k]);
                    a[2 * k] += fabsf(bf16_lo(w[k]));
                    a[2 * k + 1] += fabsf(bf16_hi(w[k]));
                }
            }
            const unsigned half_mask = 0xffffu << (lane & 16);        // (the other half's token may not exist)
            float ss = 0.f, aa = 0.f, sum = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                ss = fmaf(s[k], s[k], ss);
                aa = fmaf(a[k], a[k], aa);
                sum += a[k];
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) {
                sum += __shfl_xor_sync(half_mask, sum, o);
                aa += __shfl_xor_sync(half_mask, aa, o);
                ss += __shfl_xor_sync(half_mask, ss, o);
            }
            uint32_t hi[4], rest[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                hi[k] = pack_bf16x2(s[2 * k], s[2 * k + 1]);
                rest[k] = pack_bf16x2(s[2 * k] - bf16_lo(hi[k]), s[2 * k + 1] - bf16_hi(hi[k]));
            }
            uint8_t* const to = gen + (t >> 7) * kSelectA + (v >> 3) * (kSelectTile * 128) + (t & 127) * 128 + (((v & 7) ^ (t & 7)) << 4);
            *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4*>(to + kSelectA / 2) = make_uint4(rest[0], rest[1], rest[2], rest[3]);
            if (v == 0) s_weight[t] = token_weight(G, sum, aa, ss);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    // no more candidates than fit: no border is needed, one pass over the pages is enough
    const bool filter = page1 - begin > p.cap;
    const int per_pass = (pages + kSelectTile - 1) / kSelectTile, steps = filter ? 2 * per_pass : per_pass;
    auto first_page = [&](int j) { return (j >= per_pass ? j - per_pass : j) * kSelectTile; };      // (counted from page0)

    if (tid >= kSelectThreads) {
        // ============================ MMA issuer ============================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kSelectRegsLow));
        constexpr uint32_t kIdesc = idesc_bf16(kSelectTile, kSelectTile, false, false), kHi = desc_hi_sw128(1024);
        for (int j = 0; j < steps; ++j) {
            __syncthreads();              // step j's operand is in place, and the scores of two steps ago have left tensor memory
            if (tid == kSelectThreads) {
                tc_fence_after();
                const uint32_t b0 = desc_lo_sw128(base + 2 * kSelectA + (j & 1) * kSelectB, 16);
                for (int t = 0; t * kSelectTile < n; ++t) {
                    const uint32_t a0 = desc_lo_sw128(base + t * kSelectA, 16);
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const uint32_t at = (((k >> 2) & 1) * (kSelectTile * 128) + (k & 3) * 32) >> 4;
                        mma_ss_lhh(tmem + (j & 1) * 256 + t * 128, a0 + (1 - (k >> 3)) * (kSelectA / 2 >> 4) + at, kHi, b0 + at, kHi, kIdesc, k > 0);
                    }
                }
                tc_commit(bar + 8 * (j & 1));
            }
            __syncwarp();
            if (filter && j == per_pass) {      // (with the borders: see below)
                __syncthreads();
                __syncthreads();
            }
        }
        __syncthreads();
        __syncthreads();
        if (warp == kSelectThreads / 32) tmem_dealloc(tmem, 512);
        return;
    }
    // ============================ the others: operands, scores ============================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSelectRegsHigh));
    uint32_t square = 0;
    auto bound_of = [&](int t) { return select_bound(s_weight[t], *s_square); };
    auto share_bounds = [&]() {           // the means' part, before a barrier
        const uint32_t b = __reduce_max_sync(0xffffffffu, square);
        if (lane == 0) atomicMax(s_square, b);
    };
    // The thread's four vectors of the means of step j, of rows tid / 16 + 32 i, on the way into the operand's place; zeros where there is no page.
    auto place_of = [&](int j, int i) -> uint32_t {
        const int t = (tid >> 4) + 32 * i;
        return (j & 1) * kSelectB + (v >> 3) * (kSelectTile * 128) + t * 128 + (((v & 7) ^ (t & 7)) << 4);
    };
    const uint8_t* const my_means = p.means + g * 256 + v * 16;
    const long long mean_stride = static_cast<long long>(p.num_kv_heads) * 256;
    auto fetch = [&](int j) {
        if (j < steps) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = first_page(j) + (tid >> 4) + 32 * i;
                const int e = k < pages ? s_page[k] : -1;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(base + 2 * kSelectA + place_of(j, i)), "l"(my_means + max(e, 0) * mean_stride),
                             "r"(e >= 0 ? 16 : 0) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto landed = [&](int j) {            // the thread's own copies of step j are done, and seen by the tensor core after the barrier that follows
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (j < per_pass) {
            // sums of squares of four rows, 16 lanes each: a lane goes on with two of them, then with one
            float sq[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) sq[i] = mean_square(*reinterpret_cast<const uint4*>(sB + place_of(j, i)));
            const bool up = lane & 8, right = lane & 4;
            const float a = (up ? sq[2] : sq[0]) + __shfl_xor_sync(0xffffffffu, up ? sq[0] : sq[2], 8), b = (up ? sq[3] : sq[1]) + __shfl_xor_sync(0xffffffffu, up ? sq[1] : sq[3], 8);
            float c = (right ? b : a) + __shfl_xor_sync(0xffffffffu, right ? a : b, 4);
            c += __shfl_xor_sync(0xffffffffu, c, 2);
            c += __shfl_xor_sync(0xffffffffu, c, 1);
            square = max(square, __float_as_uint(c) & 0x7fffffffu);
        }
        fence_proxy_async_smem();
    };
    // warps 0-3 and 4-7: the first 128 tokens, left and right halves of a step's pages; warps 8-15: the other tokens
    const int my_row = (warp >> 3) * 128 + (warp & 3) * 32 + lane, half = (warp >> 2) & 1;
    const uint32_t tD = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + (warp >> 3) * 128 + half * 64;
    const bool lives = (warp >> 3) * 128 + (warp & 3) * 32 < n;      // (the warp has a token)
    const int stop = my_row < n ? end_of(my_row) : 0;
    const int gp = p.group_pages, row_groups = gp > 0 ? p.run_pages / gp : 0;
    float* const my_maxima = p.maxima + (static_cast<long long>(item) * kSelectItem + my_row) * row_groups;
    float floor = -3.4e38f;      // (below every score that counts and above the -inf of pages that are no candidates)
    SelectCandidate* const list0 = p.found + (list_of(my_row) * 2 + half) * p.cap;
    SelectCandidate* put_at = list0;
    // (predicated: two of three columns have a row that lists them, and a branch around every store took 5100 clk a step of 64 instead of 4400)
    auto put = [&](float score, int page) {
        asm volatile("{\n.reg .pred q;\nsetp.ge.f32 q, %1, %2;\n@q st.global.v2.b32 [%0], {%3, %4};\n@q add.u64 %0, %0, 8;\n}"
                     : "+l"(put_at) : "f"(score), "f"(floor), "r"(__float_as_uint(score)), "r"(page) : "memory");
    };
    int m = 0;                   // those that found no room
    float mx[32];                // gp == 0: of the pages that are column i of a piece
#pragma unroll
    for (int i = 0; i < 32; ++i) mx[i] = -INFINITY;
    fetch(0);
    landed(0);
    __syncthreads();
    fetch(1);
    bool alive = true;
    for (int j = 0; j < steps; ++j) {
        if (j + 1 < steps) {
            landed(j + 1);
            __syncthreads();
        }
        if (alive) alive = mbar_wait(bar + 8 * (j & 1), (j >> 1) & 1, s_abort, 501);
        // (this step's products have read their operand: the one after next goes to its place -- after the borders, which pass through it)
        const bool borders = filter && j == per_pass - 1;
        if (!borders) fetch(j + 2);
        const bool first_pass = filter && j < per_pass;
        tc_fence_after();
        if (alive && lives) {
            const int k0 = page0 + first_page(j) + half * 64;
            uint32_t sc[2][16];                 // 16 pages at a time, k of the first
            auto mask = [&](uint32_t (&s)[16], int k) {      // those that are no candidates: -inf
                if (k < begin || __any_sync(0xffffffffu, k + 16 > stop)) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (k + i < begin || k + i >= stop) s[i] = 0xff800000u;
                }
            };
            if (first_pass && gp == 0) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    tmem_ld16(tD + (j & 1) * 256 + c * 16, sc[0]);
                    tmem_ld16(tD + (j & 1) * 256 + (c + 2) * 16, sc[1]);
                    tc_wait_ld(sc[0]);
                    tc_wait_ld(sc[1]);
                    mask(sc[0], k0 + c * 16);
                    mask(sc[1], k0 + (c + 2) * 16);
#pragma unroll
                    for (int i = 0; i < 16; ++i) mx[c * 16 + i] = fmax3(mx[c * 16 + i], __uint_as_float(sc[0][i]), __uint_as_float(sc[1][i]));
                }
            }
            if (!(first_pass && gp == 0)) tmem_ld16(tD + (j & 1) * 256, sc[0]);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (first_pass && gp == 0) break;
                uint32_t (&s)[16] = sc[c & 1];
                tc_wait_ld(s);
                if (c < 3) tmem_ld16(tD + (j & 1) * 256 + (c + 1) * 16, sc[(c + 1) & 1]);
                const int k = k0 + c * 16;
                if (k >= page1) continue;
                mask(s, k);
                if (first_pass) {
                    if (my_row < n) {
                        float4* const to = reinterpret_cast<float4*>(my_maxima + (k - page0) / gp);
                        auto at = [&](int i) { return __uint_as_float(s[i]); };
                        auto two = [&](int i) { return fmaxf(at(2 * i), at(2 * i + 1)); };
                        auto four = [&](int i) { return fmax3(at(4 * i), at(4 * i + 1), fmaxf(at(4 * i + 2), at(4 * i + 3))); };
                        if (gp == 4) {
                            to[0] = make_float4(four(0), four(1), four(2), four(3));
                        } else if (gp == 2) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) to[i] = make_float4(two(4 * i), two(4 * i + 1), two(4 * i + 2), two(4 * i + 3));
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i) to[i] = make_float4(at(4 * i), at(4 * i + 1), at(4 * i + 2), at(4 * i + 3));
                        }
                    }
                } else if (put_at - list0 + 16 <= p.cap) {      // (room for them all: no check at each)
#pragma unroll
                    for (int i = 0; i < 16; ++i) put(__uint_as_float(s[i]), k + i);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (put_at - list0 < p.cap) put(__uint_as_float(s[i]), k + i);
                        else m += __uint_as_float(s[i]) >= floor;
                    }
                }
                __syncwarp();
            }
        }
        tc_fence_before();
        if (!borders) continue;
        // ---- the borders ----
        share_bounds();
        // the right halves' maxima go to the threads of the left halves: a thread a token with all 64.  The place is that of the operand that is not in use (the
        // step under way uses the other one).
        float* const swap = reinterpret_cast<float*>(sB + (j & 1) * kSelectB);      // [32][256]: 32 KB
        const bool mine = gp == 0 && half == 0;
        if (gp == 0 && !mine) {
#pragma unroll
            for (int i = 0; i < 32; ++i) swap[i * kSelectItem + my_row] = mx[i];
        }
        __syncthreads();
        if (gp == 0) {
            if (mine && my_row < n) {
                const float bound = bound_of(my_row);
                float f = INFINITY;          // (lists without choice, or bounds that say nothing: no candidates)
                if (stop > begin && bound > 0.f && bound < INFINITY) {
                    f = -3.4e38f;
                    if (stop - begin > p.cap) {
                        float mo[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) mo[i] = swap[i * kSelectItem + my_row];
                        // a value that at least `need` of them reach, and not many more: the span of the 64 halved eight times
                        float least = fminf(mx[0], mo[0]), most = fmaxf(mx[0], mo[0]);
#pragma unroll
                        for (int i = 1; i < 32; ++i) {
                            least = fminf(least, fminf(mx[i], mo[i]));
                            most = fmax3(most, mx[i], mo[i]);
                        }
                        least = fmaxf(least, f);          // (groups of no pages)
#pragma unroll 1
                        for (int b = 0; b < 8; ++b) {
                            const float c = 0.5f * least + 0.5f * most;
                            int k[4] = {};
#pragma unroll
                            for (int i = 0; i < 32; ++i) k[i & 3] += (mx[i] >= c) + (mo[i] >= c);
                            if (k[0] + k[1] + k[2] + k[3] >= need) least = c; else most = c;
                        }
                        f = fmaxf(f, least - 2.f * bound);
                    }
                }
                s_floor[my_row] = f;
            }
        } else {
            const int lead_group = (begin - page0) / gp;
            for (int t = warp; t < n; t += kSelectThreads / 32) {
                const int stop_t = end_of(t);
                float f = INFINITY;
                const float bound = bound_of(t);
                if (stop_t > begin && bound > 0.f && bound < INFINITY) {
                    f = -3.4e38f;
                    if (stop_t - begin > p.cap) {
                        const float* const mxs = p.maxima + (static_cast<long long>(item) * kSelectItem + t) * row_groups + lead_group;
                        f = fmaxf(f, border_of((stop_t - page0 + gp - 1) / gp - lead_group, need, [&](int i) { return mxs[i]; }) - 2.f * bound);
                    }
                }
                if (lane == 0) s_floor[t] = f;
            }
        }
        __syncthreads();
        fetch(j + 2);
        if (my_row < n) floor = s_floor[my_row];
    }
    if (!filter) share_bounds();
    if (*s_abort != 0)
        for (int i = 0; i < 64; ++i) __nanosleep(1000);  // let MMAs in flight drain
    __syncthreads();
    if (my_row < n) {
        p.counts[list_of(my_row) * 2 + half] = static_cast<int>(put_at - list0) + m;
        if (half == 0) p.bounds[list_of(my_row)] = bound_of(my_row);
    }
    if (tid == 0) p.bad[item] = *s_abort != 0 ? 3 /* VPP_DEV_TIMEOUT */ : *s_badp ? 2 /* VPP_DEV_BAD_BLOCK */ : 0;
    __syncthreads();                      // (tensor memory goes back)
}

// ---- the border -----------------------------------------------------------------------------------------------------------------

constexpr int kPickThreads = 256;
constexpr int kPickGather = 512;              // entries a warp can gather
constexpr int kPickClose = 128;               // entries near the border that it can settle at once
static_assert(kSelectMaxTopk + kPickClose <= kPickGather, "what is needed fits");
struct PickScratch {
    union {
        struct {
            double exact[kPickClose];         // of the near ones
            float score[kPickGather];
        };
        double all[kPickGather];              // (pick_thorough)
    };
    int32_t page[kPickGather];
    int32_t close[kPickClose], close_page[kPickClose];      // the near ones: entries of page / score, their pages
};
constexpr int kPickSmem = static_cast<int>(sizeof(PickScratch)) * (kPickThreads / 32);

// A row's own inputs, for scores in 64 bits.
struct PickRow {
    const uint8_t* q;            // the group's first q-head
    const int32_t* table;        // the request's pages
    const uint8_t* means;        // of the kv-head, page 0
    long long mean_stride;
    int group, num_blocks;
};

// Scores in 64 bits of n pages -- pages[c], or first + c -- by a warp.  NaN counts as -inf.  (out of line, arguments by value: rare, and
// the common path keeps its registers)
__device__ __noinline__ void exact_scores(PickRow w, const int32_t* pages, int first, int n, double* out) {
    const int lane = threadIdx.x & 31;
    double ask[4] = {};
#pragma unroll 8
    for (int h = 0; h < w.group; ++h) {
        const uint2 x = __ldg(reinterpret_cast<const uint2*>(w.q + h * 256 + lane * 8));
        ask[0] += static_cast<double>(bf16_lo(x.x));
        ask[1] += static_cast<double>(bf16_hi(x.x));
        ask[2] += static_cast<double>(bf16_lo(x.y));
        ask[3] += static_cast<double>(bf16_hi(x.y));
    }
    for (int c = 0; c < n; ++c) {
        const int e = __ldg(w.table + (pages ? pages[c] : first + c));
        double d = -INFINITY;
        if (e >= 0 && e < w.num_blocks) {        // (an entry out of range is reported already)
            const uint2 x = __ldg(reinterpret_cast<const uint2*>(w.means + e * w.mean_stride + lane * 8));
            d = ask[0] * static_cast<double>(bf16_lo(x.x)) + ask[1] * static_cast<double>(bf16_hi(x.x));
            d += ask[2] * static_cast<double>(bf16_lo(x.y)) + ask[3] * static_cast<double>(bf16_hi(x.y));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
            if (!(d == d)) d = -INFINITY;
        }
        if (lane == 0) out[c] = d;
    }
    __syncwarp();
}

// Keeps of the m gathered entries (all that can be among the best, in any order) the `need` best: their pages move to the front of
// s.page, in any order.  delta > 0: bound on the error of a score.  False: more of them are too close to tell than fit.
__device__ __forceinline__ bool pick_settle(PickScratch& s, const PickRow& w, int m, int need, float delta) {
    const int lane = threadIdx.x & 31;
    const uint32_t k0 = lane < m ? order_key(s.score[lane]) : 0, k1 = lane + 32 < m ? order_key(s.score[lane + 32]) : 0;
    // a key that `need` entries reach (or more, where the need-th and the next are equal), then the least of theirs: the need-th best score
    uint32_t border = 0;
    for (int b = 31; b >= 0; --b) {
        const uint32_t c = border | (1u << b);
        int k = (k0 >= c) + (k1 >= c);
        for (int i = lane + 64; i < m; i += 32) k += order_key(s.score[i]) >= c;
        const int all = static_cast<int>(__reduce_add_sync(0xffffffffu, k));
        if (all >= need) border = c;
        if (all == need) break;
    }
    uint32_t least = 0xffffffffu;
    if (k0 >= border && lane < m) least = k0;
    if (k1 >= border && lane + 32 < m) least = min(least, k1);
    for (int i = lane + 64; i < m; i += 32) {
        const uint32_t k = order_key(s.score[i]);
        if (k >= border) least = min(least, k);
    }
    border = __reduce_min_sync(0xffffffffu, least);
    const float v = key_value(border), hi = v + 2.f * delta, lo = v - 2.f * delta;
    // sure ones (above hi: their exact scores are above those of all but need - 1), and those too close to the border to tell
    int sure = 0, near_n = 0;
    for (int i0 = 0; i0 < m; i0 += 32) {
        const int i = i0 + lane;
        const float x = i < m ? s.score[i] : 0.f;
        const bool in = i < m && x > hi, near = i < m && !in && x >= lo;
        sure += __popc(__ballot_sync(0xffffffffu, in));
        const uint32_t b = __ballot_sync(0xffffffffu, near);
        const int at = near_n + __popc(b & ((1u << lane) - 1));
        if (near && at < kPickClose) {
            s.close[at] = i;
            s.close_page[at] = s.page[i];
        }
        near_n += __popc(b);
    }
    const int left = need - sure;         // to be taken of the near ones: 1 .. near_n
    if (left != near_n) {
        if (near_n > kPickClose) return false;
        __syncwarp();
        exact_scores(w, s.close_page, 0, near_n, s.exact);
        // losers among the near ones get a page of -1
        for (int c = lane; c < near_n; c += 32) {
            const double d = s.exact[c];
            const int page = s.close_page[c];
            int before = 0;
            for (int j = 0; j < near_n; ++j) before += s.exact[j] > d || (s.exact[j] == d && s.close_page[j] < page);
            if (before >= left) s.page[s.close[c]] = -1;
        }
    }
    __syncwarp();
    int kept = 0;
    for (int i0 = 0; i0 < m; i0 += 32) {
        const int i = i0 + lane;
        const int page = i < m ? s.page[i] : -1;
        const bool take = i < m && s.score[i] >= lo && page >= 0;
        const uint32_t t = __ballot_sync(0xffffffffu, take);      // (all have read their page)
        if (take) s.page[kept + __popc(t & ((1u << lane) - 1))] = page;
        kept += __popc(t);
        __syncwarp();
    }
    return true;
}

// Leaves of the m gathered entries those that may be among the need best of these and others, and returns how many.  (Runs' lists may be more than fit.)
__device__ __noinline__ int pick_prune(PickScratch& s, int m, int need, float delta) {
    const int lane = threadIdx.x & 31;
    uint32_t border = 0;                 // (a little below the need-th best will do)
    for (int b = 31; b >= 8; --b) {
        const uint32_t c = border | (1u << b);
        int k = 0;
        for (int i = lane; i < m; i += 32) k += order_key(s.score[i]) >= c;
        const int all = static_cast<int>(__reduce_add_sync(0xffffffffu, k));
        if (all >= need) border = c;
        if (all == need) break;
    }
    if (border < 0x00800000u) return m;  // (fewer than need)
    const float lo = key_value(border) - 2.f * delta;
    int kept = 0;
    for (int i0 = 0; i0 < m; i0 += 32) {
        const int i = i0 + lane;
        const float score = i < m ? s.score[i] : 0.f;
        const int page = i < m ? s.page[i] : 0;
        const bool take = i < m && score >= lo;
        const uint32_t t = __ballot_sync(0xffffffffu, take);
        if (take) {
            const int at = kept + __popc(t & ((1u << lane) - 1));
            s.score[at] = score;
            s.page[at] = page;
        }
        kept += __popc(t);
        __syncwarp();
    }
    return kept;
}

// What the common path does not settle -- infinite or NaN scores, more candidates than fit (many pages that are (nearly) the same): all pages' scores in 64
// bits, 128 at a time, each time joined with the best so far.
__device__ __noinline__ void pick_thorough(PickScratch& s, PickRow w, int begin, int end, int need) {
    const int lane = threadIdx.x & 31;
    int best = 0;
    for (int j0 = begin; j0 < end; j0 += kPickClose) {
        const int n = min(kPickClose, end - j0), m = best + n;
        exact_scores(w, nullptr, j0, n, s.all + best);
        for (int c = lane; c < n; c += 32) s.page[best + c] = j0 + c;
        __syncwarp();
        // ranks: better scores, then lower pages (the best so far are lower pages than the new ones, and in order of their pages)
        uint32_t keep = 0;
#pragma unroll 1
        for (int k = 0; 32 * k < m; ++k) {
            const int i = lane + 32 * k;
            if (i >= m) continue;
            const double d = s.all[i];
            int before = 0;
            for (int j = 0; j < m; ++j) before += s.all[j] > d || (s.all[j] == d && j < i);
            if (before < need) keep |= 1u << k;
        }
        __syncwarp();
        best = 0;
#pragma unroll 1
        for (int k = 0; 32 * k < m; ++k) {       // (to places before their own: those of earlier rounds, and of this one, are read)
            const bool mine = (keep >> k) & 1;
            const double d = mine ? s.all[lane + 32 * k] : 0.0;
            const int page = mine ? s.page[lane + 32 * k] : 0;
            const uint32_t t = __ballot_sync(0xffffffffu, mine);
            if (mine) {
                const int at = best + __popc(t & ((1u << lane) - 1));
                s.all[at] = d;
                s.page[at] = page;
            }
            best += __popc(t);
            __syncwarp();
        }
    }
}

// The same for the common case, two ascending lists of at most 32 candidates each, a lane a candidate of either, and the pages go straight to `out`, ascending.
__device__ __forceinline__ void pick_two(PickScratch& s, const PickRow& w, SelectCandidate x, int an, SelectCandidate y, int bn, int need, float delta,
                                         int32_t* out) {
    const int lane = threadIdx.x & 31;
    const uint32_t below = (1u << lane) - 1;
    if (lane >= an) x = SelectCandidate{-INFINITY, INT32_MAX};
    if (lane >= bn) y = SelectCandidate{-INFINITY, INT32_MAX};
    const uint32_t kx = lane < an ? order_key(x.score) : 0, ky = lane < bn ? order_key(y.score) : 0;
    // (from the highest bit in which they differ: candidates are of one size)
    const uint32_t most = __reduce_max_sync(0xffffffffu, max(kx, ky)), least = __reduce_min_sync(0xffffffffu, min(lane < an ? kx : most, lane < bn ? ky : most));
    int bit = 31 - __clz(most ^ least);
    uint32_t border = bit < 0 ? most : most & ~((2u << bit) - 1);
    for (; bit >= 0; --bit) {
        const uint32_t c = border | (1u << bit);
        const int all = __popc(__ballot_sync(0xffffffffu, kx >= c)) + __popc(__ballot_sync(0xffffffffu, ky >= c));
        if (all >= need) border = c;
        if (all == need) break;
    }
    border = __reduce_min_sync(0xffffffffu, min(kx >= border ? kx : 0xffffffffu, ky >= border ? ky : 0xffffffffu));
    const float v = key_value(border), hi = v + 2.f * delta, lo = v - 2.f * delta;
    bool take_x = x.score > hi, take_y = y.score > hi;
    const bool near_x = !take_x && x.score >= lo, near_y = !take_y && y.score >= lo;
    const uint32_t nx = __ballot_sync(0xffffffffu, near_x), ny = __ballot_sync(0xffffffffu, near_y);
    const int left = need - __popc(__ballot_sync(0xffffffffu, take_x)) - __popc(__ballot_sync(0xffffffffu, take_y)), near_n = __popc(nx) + __popc(ny);
    if (left == near_n) {
        take_x |= near_x;
        take_y |= near_y;
    } else {
        const int at_x = __popc(nx & below), at_y = __popc(nx) + __popc(ny & below);
        if (near_x) s.close_page[at_x] = x.page;
        if (near_y) s.close_page[at_y] = y.page;
        __syncwarp();
        exact_scores(w, s.close_page, 0, near_n, s.exact);
        auto wins = [&](int at, int page) {
            const double d = s.exact[at];
            int before = 0;
            for (int j = 0; j < near_n; ++j) before += s.exact[j] > d || (s.exact[j] == d && s.close_page[j] < page);
            return before < left;
        };
        if (near_x) take_x = wins(at_x, x.page);
        if (near_y) take_y = wins(at_y, y.page);
        __syncwarp();
    }
    const uint32_t tx = __ballot_sync(0xffffffffu, take_x), ty = __ballot_sync(0xffffffffu, take_y);
    // how many of the other list lie before a page
    int in_b = 0, in_a = 0;
#pragma unroll
    for (int step = 16; step > 0; step >>= 1) {
        const int pb = __shfl_sync(0xffffffffu, y.page, in_b + step - 1), pa = __shfl_sync(0xffffffffu, x.page, in_a + step - 1);
        if (pb < x.page) in_b += step;
        if (pa < y.page) in_a += step;
    }
    {   // (the last of 32)
        const int pb = __shfl_sync(0xffffffffu, y.page, in_b), pa = __shfl_sync(0xffffffffu, x.page, in_a);
        if (pb < x.page) ++in_b;
        if (pa < y.page) ++in_a;
    }
    auto first = [](int n) { return n >= 32 ? 0xffffffffu : (1u << n) - 1; };
    if (take_x) out[__popc(tx & below) + __popc(ty & first(in_b))] = x.page;
    if (take_y) out[__popc(ty & below) + __popc(tx & first(in_a))] = y.page;
}

// The first work_blocks blocks pick; the block after them, if there is one, writes the status.
__global__ void __launch_bounds__(kPickThreads, 3) block_pick_kernel(const SelectParams p, const int work_blocks) {
    extern __shared__ __align__(16) uint8_t pick_smem[];
    PickScratch* const scratch = reinterpret_cast<PickScratch*>(pick_smem);
    int32_t* const cu = reinterpret_cast<int32_t*>(pick_smem + kPickSmem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_launch_dependents();
    pdl_wait();
    if (static_cast<int>(blockIdx.x) >= work_blocks) {
        int worst = 0, now = scan_lengths<kPickThreads>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu) ? 0 : 1 /* VPP_DEV_BAD_LENGTHS */;
        for (int i = tid; i < p.items; i += kPickThreads) worst = worse_status(worst, p.bad[i]);
        for (int k = 2; k <= 3; ++k)      // (VPP_DEV_BAD_BLOCK, VPP_DEV_TIMEOUT)
            if (__syncthreads_or(worst == k)) now = worse_status(now, k);
        if (tid == 0) *p.status = p.row0 == 0 ? now : worse_status(now, *p.status);
        return;
    }
    if (!scan_lengths<kPickThreads>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu)) return;
    const int G = p.num_q_heads / p.num_kv_heads, need = p.topk - p.num_first - p.num_last;
    PickScratch& s = scratch[warp];
    const int rows = (p.row1 - p.row0) * p.num_kv_heads, step = work_blocks * (kPickThreads / 32);      // (rows of a slab: far below 2^31)
    // What the common case reads of a row -- one run: its bound, two counts, and the first 32 of both lists, whatever the counts -- is requested a row ahead.
    struct Ahead {
        float delta;
        int2 count;
        SelectCandidate x, y;
    };
    auto request = [&](int i) {
        Ahead a{};
        if (p.runs == 1 && i < rows) {
            const SelectCandidate* const from = p.found + 2ll * i * p.cap + lane;
            a.delta = p.bounds[i];
            a.count = *reinterpret_cast<const int2*>(p.counts + 2ll * i);
            a.x = from[0];
            a.y = from[p.cap];
        }
        return a;
    };
    Ahead next = request(blockIdx.x * (kPickThreads / 32) + warp);
    for (int i = blockIdx.x * (kPickThreads / 32) + warp; i < rows; i += step) {
        const Ahead now = next;
        next = request(i + step);
        const int t0 = i / p.num_kv_heads, t = p.row0 + t0, g = i - t0 * p.num_kv_heads;
        const int r = request_of(cu, p.num_reqs, t);
        const int own = (p.prefix_len[r] + (t - cu[r])) >> p.block_shift;
        int32_t* const out = p.indices + (static_cast<long long>(t) * p.num_kv_heads + g) * p.topk;
        if (own + 1 <= p.topk) {
            for (int k = lane; k < p.topk; k += 32) out[k] = k <= own ? k : -1;
            continue;
        }
        const PickRow w{p.q + (static_cast<long long>(t) * p.num_q_heads + g * G) * 256, p.block_table + static_cast<long long>(r) * p.max_blocks_per_req,
                        p.means + g * 256, static_cast<long long>(p.num_kv_heads) * 256, G, p.num_blocks};
        // (own + 1 > topk >= first + last: the two ends do not meet, and there are more candidates than needed)
        for (int k = lane; k < p.topk; k += 32)
            if (k < p.num_first || k >= p.num_first + need) out[k] = k < p.num_first ? k : own + 1 - (p.topk - k);
        if (need == 0) continue;          // (nothing was scored)
        const int end = select_end(p, own), run0 = p.num_first / p.run_pages, runs = (end + p.run_pages - 1) / p.run_pages;
        if (p.runs == 1 && now.delta > 0.f && now.delta < INFINITY && now.count.x <= 32 && now.count.y <= 32 && now.count.x + now.count.y >= need) {
            pick_two(s, w, now.x, now.count.x, now.y, now.count.y, need, now.delta, out + p.num_first);
            __syncwarp();
            continue;
        }
        float delta = 0.f;
        bool odd = false;
        for (int k = run0 + lane; k < runs; k += 32) {
            const float x = p.bounds[static_cast<long long>(i) * p.runs + k];
            odd |= !(x < INFINITY);
            delta = fmaxf(delta, x);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) delta = fmaxf(delta, __shfl_xor_sync(0xffffffffu, delta, o));
        odd = __any_sync(0xffffffffu, odd);
        if (!odd && delta == 0.f) {       // all scores are 0
            for (int k = lane; k < need; k += 32) out[p.num_first + k] = p.num_first + k;
            continue;
        }
        // the runs' candidates, one behind the other
        int m = 0;
        for (int k0 = 2 * run0; k0 < 2 * runs && !odd; k0 += 32) {
            const int k = k0 + lane, c = k < 2 * runs ? p.counts[static_cast<long long>(i) * p.runs * 2 + k] : 0;
            // (a run whose scores are all 0 lists none)
            odd = __any_sync(0xffffffffu, static_cast<uint32_t>(c) > static_cast<uint32_t>(p.cap) || (k < 2 * runs && !(p.bounds[static_cast<long long>(i) * p.runs + (k >> 1)] > 0.f)));
            for (int l0 = 0; l0 < min(32, 2 * runs - k0) && !odd; l0 += 4) {
                int count[4];
                SelectCandidate x[4];
#pragma unroll
                for (int l = 0; l < 4; ++l) {      // (four lists' first 32 under way at a time)
                    count[l] = __shfl_sync(0xffffffffu, c, l0 + l);
                    if (lane < count[l]) x[l] = p.found[(static_cast<long long>(i) * p.runs * 2 + k0 + l0 + l) * p.cap + lane];
                }
#pragma unroll
                for (int l = 0; l < 4; ++l) {
                    if (m + count[l] > kPickGather) {
                        __syncwarp();
                        m = pick_prune(s, m, need, delta);
                        odd |= m + count[l] > kPickGather;
                        if (odd) break;
                    }
                    if (lane < count[l]) {
                        s.score[m + lane] = x[l].score;
                        s.page[m + lane] = x[l].page;
                    }
                    for (int j = lane + 32; j < count[l]; j += 32) {
                        const SelectCandidate y = p.found[(static_cast<long long>(i) * p.runs * 2 + k0 + l0 + l) * p.cap + j];
                        s.score[m + j] = y.score;
                        s.page[m + j] = y.page;
                    }
                    m += count[l];
                }
            }
        }
        __syncwarp();
        odd |= m < need;                  // (a scoring block that gave up lists too few)
        if (odd || !pick_settle(s, w, m, need, delta)) pick_thorough(s, w, p.num_first, end, need);
        __syncwarp();
        // ascending
        for (int k = lane; k < need; k += 32) {
            const int page = s.page[k];
            int before = 0;
            for (int j = 0; j < need; ++j) before += s.page[j] < page;
            out[p.num_first + before] = page;
        }
        __syncwarp();
    }
}

}  // namespace vpp
