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
// Two kernels a slab of tokens (one slab unless their candidates take more than kSelectSlabBytes):
//  * block_filter_kernel: an item is (up to 128 tokens of one request, kv-head, a run of pages).  The group's queries are
//    summed first, in 32 bits, and the sum split in two bf16 (hi + rest: 16 bits of it), so that the tensor cores do 2 / group
//    of the work of all q-heads; scores of 128 tokens x 128 pages are one accumulator.  They are formed twice: the first time the maxima of groups
//    of pages are kept, whose need-th largest bounds a token's border from below; the second time what is not below that by more than the error
//    bound -- a few more pages than needed -- is written down, a thread a token and half of the pages.  Reading q bounds it (134 MB of
//    8192 tokens of 64 heads are 21 us; the products twice 4).  (All scores written down once, 4.6 KB a token and kv-head, and picked
//    from there: 8192 tokens of 64/4 heads with 1152 pages 420 us.)
//    Items of up to kSelectFew tokens -- decode rows -- take the dot products in registers, half a warp a page, and keep the scores in shared
//    memory: there reading the means is all.
//  * block_pick_kernel: a warp a (token, kv-head) ranks the candidates and settles the border.
#pragma once
#include <cstdint>

#include "lengths.cuh"
#include "ptx.cuh"
#include "rope.cuh"

namespace vpp {

constexpr int kSelectThreads = 256;
constexpr int kSelectTile = 128;              // tokens of an item, pages of a step
constexpr int kSelectFew = 4;
constexpr int kSelectSlabBytes = 128 << 20;
constexpr int kSelectMaxTopk = 256;
constexpr int kSelectMaxRun = 4096;           // pages of an item: scores of kSelectFew tokens are kept in shared memory
constexpr int kSelectA = 2 * 2 * kSelectTile * 128;   // two bf16 parts of 128 x 128, two 64-feature slabs each
constexpr int kSelectB = 2 * kSelectTile * 128;
constexpr int kSelectSmem = kSelectA + kSelectB + 1024 /* alignment */ + 2048 /* barrier, borders */;
static_assert(kSelectFew * kSelectMaxRun * 4 <= kSelectA, "scores of few tokens");

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
    int run_pages, runs;          // pages of an item (a multiple of 128), items along a row
    int group_pages;              // pages of a group of which the maximum is kept (4, 2, 1; 0: 64 groups of every 64th page or so, in registers)
    int cap;                      // candidates of half an item's pages, at most
    SelectCandidate* found;       // [row1 - row0, Hkv, runs, 2, cap]
    int32_t* counts;              // [row1 - row0, Hkv, runs, 2] (past cap: more than fit)
    float* bounds;                // [row1 - row0, Hkv, runs]: error bound of the row's scores of a run
    float* maxima;                // [items, 128, run_pages / group_pages] (group_pages > 0)
    int32_t* bad;                 // one word an item of the slab
    int items;
    int32_t* indices;             // [total_q, Hkv, topk]
    int32_t* status;
};

// Candidates of a token whose own page is `own`: pages [num_first, end).
__device__ __forceinline__ int select_end(const SelectParams& p, int own) { return own + 1 - p.num_last; }

// |x| as ordered bits: NaN above infinity above everything finite
__device__ __forceinline__ uint32_t abs_max(uint32_t m, uint4 v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        m = max(m, w[e] & 0x7fffu);
        m = max(m, (w[e] >> 16) & 0x7fffu);
    }
    return m;
}
// |fp32 score - exact score| <= 2^-14 sum_i a_i max|m| + underflow, a_i = sum_h |q_h,i|: the split leaves 2^-17 of the sum, a sum of G
// terms is off by (G - 1) 2^-24 of a_i (G <= 128), accumulating 256 products by 256 * 2^-23 of their absolute sum: 2^-15, together below 2^-14.  Exactly 0
// where all products are; infinite or NaN where anything is, or where products could overflow.
__device__ __forceinline__ float select_bound(float a, uint32_t max_bits) {
    const float m = __uint_as_float(max_bits << 16);
    if (!(a < 1e38f)) return INFINITY;
    if (a == 0.f && max_bits < 0x7f80u) return 0.f;
    if (max_bits == 0 && a < INFINITY) return 0.f;
    return a * m * 6.103515625e-5f + 1e-35f;
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

__global__ void __launch_bounds__(kSelectThreads, 2) block_filter_kernel(const SelectParams p) {
    extern __shared__ uint8_t smem_raw[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const gen = smem_raw + (base - smem_u32(smem_raw));
    uint8_t* const sA = gen;
    uint8_t* const sB = gen + kSelectA;
    uint8_t* const sX = gen + kSelectA + kSelectB;
    const uint32_t bar = base + kSelectA + kSelectB;
    volatile int* const s_abort = reinterpret_cast<volatile int*>(sX + 8);
    volatile uint32_t* const s_tmem = reinterpret_cast<volatile uint32_t*>(sX + 12);
    uint32_t* const s_max = reinterpret_cast<uint32_t*>(sX + 16);
    int* const s_badp = reinterpret_cast<int*>(sX + 20);
    float* const s_a = reinterpret_cast<float*>(sX + 32);              // [128] what a bound is made of
    float* const s_floor = reinterpret_cast<float*>(sX + 32 + 512);    // [128] lowest score of a candidate
    int32_t* const cu = reinterpret_cast<int32_t*>(sX + 2048);         // [num_reqs + 1], then tile counts [num_reqs + 1]
    int32_t* const first_tile = cu + p.num_reqs + 1;

    pdl_launch_dependents();
    pdl_wait();
    const bool ok = scan_lengths<kSelectThreads>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu, kSelectTile, first_tile);
    const int item = blockIdx.x;
    if (!ok) {
        if (tid == 0) p.bad[item] = 1 /* VPP_DEV_BAD_LENGTHS */;
        return;
    }
    // tiles of every request's rows inside the slab
    auto rows_of = [&](int r, int& lo) {
        lo = max(cu[r], p.row0);
        const int n = min(cu[r + 1], p.row1) - lo;
        return n > 0 ? n : 0;
    };
    if (tid == 0) {
        *s_abort = 0;
        *s_max = 0;
        *s_badp = 0;
        mbar_init(bar, 1);
        fence_mbar_init();
    }
    if (p.row0 == 0 && p.row1 == p.total_q)
        __syncthreads();
    else                              // (a part of the tokens: tiles begin anew)
        block_scan<kSelectThreads>(p.num_reqs, 0x7fffffffu, first_tile, false, [&](int r, bool&) {
            int lo;
            return (rows_of(r, lo) + kSelectTile - 1) / kSelectTile;
        });
    const int run = item % p.runs, tg = item / p.runs, g = tg % p.num_kv_heads, tile = tg / p.num_kv_heads;
    if (tile >= first_tile[p.num_reqs]) {
        if (tid == 0) p.bad[item] = 0;
        return;
    }
    const int r = request_of(first_tile, p.num_reqs, tile);
    int lo;
    const int rows_r = rows_of(r, lo);
    const int row = lo + (tile - first_tile[r]) * kSelectTile;
    const int n = min(kSelectTile, lo + rows_r - row);
    const int pos0 = p.prefix_len[r] + (row - cu[r]);
    const int end = select_end(p, (pos0 + n - 1) >> p.block_shift);      // of the tile's last token
    // a page run that nobody needs: below the first candidate, past the last, or no token has more pages than it may list
    const int page0 = run * p.run_pages, page1 = min(page0 + p.run_pages, end), begin = max(page0, p.num_first);
    if (page1 <= begin || ((pos0 + n - 1) >> p.block_shift) + 1 <= p.topk) {
        if (tid == 0) p.bad[item] = 0;
        return;
    }
    const int G = p.num_q_heads / p.num_kv_heads, need = p.topk - p.num_first - p.num_last;
    const int32_t* const table = p.block_table + static_cast<long long>(r) * p.max_blocks_per_req;
    const uint8_t* const q0 = p.q + (static_cast<long long>(row) * p.num_q_heads + g * G) * 256;
    // of token t of the tile: candidates of this run (one past the last), and where its lists are
    auto end_of = [&](int t) {
        const int own = (pos0 + t) >> p.block_shift;
        return own + 1 <= p.topk ? 0 : min(page1, select_end(p, own));
    };
    auto list_of = [&](int t) { return (static_cast<long long>(row - p.row0 + t) * p.num_kv_heads + g) * p.runs + run; };
    const int v = tid & 15;
    bool bad = false;
    uint32_t top = 0;

    if (n <= kSelectFew) {
        // ---- a few tokens: half a warp a page ----
        float* const s_score = reinterpret_cast<float*>(sA);       // [kSelectFew][run_pages]
        float s[kSelectFew][8], a[kSelectFew];
#pragma unroll
        for (int t = 0; t < kSelectFew; ++t) {
            a[t] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s[t][e] = 0.f;
            if (t < n) {
                const uint8_t* src = q0 + static_cast<long long>(t) * p.num_q_heads * 256 + v * 16;
#pragma unroll 8
                for (int h = 0; h < G; ++h) {
                    const uint4 x = ld_once(src + h * 256);
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[t][2 * e] += bf16_lo(w[e]);
                        s[t][2 * e + 1] += bf16_hi(w[e]);
                        a[t] += fabsf(bf16_lo(w[e])) + fabsf(bf16_hi(w[e]));
                    }
                }
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) a[t] += __shfl_xor_sync(0xffffffffu, a[t], o);
        }
        constexpr int kDeep = 8, kStep = kDeep * (kSelectThreads / 16);
        const int half = tid >> 4;
        int e[kDeep];
        auto look = [&](int j0) {
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const int j = j0 + i * (kSelectThreads / 16) + half;
                e[i] = j < page1 ? __ldg(table + j) : 0;
            }
        };
        look(page0);
        for (int j0 = page0; j0 < page1; j0 += kStep) {
            uint4 x[kDeep];
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const int j = j0 + i * (kSelectThreads / 16) + half;
                const bool fine = e[i] >= 0 && e[i] < p.num_blocks;
                bad |= !fine;
                x[i] = make_uint4(0, 0, 0, 0);
                if (j < page1 && j >= begin && fine) x[i] = ld_once(p.means + (static_cast<long long>(e[i]) * p.num_kv_heads + g) * 256 + v * 16);
            }
            look(j0 + kStep);
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const int j = j0 + i * (kSelectThreads / 16) + half;
                top = abs_max(top, x[i]);
                const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                for (int t = 0; t < kSelectFew; ++t) {
                    if (t >= n) break;
                    float d = 0.f;
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        d = fmaf(s[t][2 * f], bf16_lo(w[f]), d);
                        d = fmaf(s[t][2 * f + 1], bf16_hi(w[f]), d);
                    }
#pragma unroll
                    for (int o = 8; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
                    if (v == 0 && j < page1) s_score[t * p.run_pages + j - page0] = d;
                }
            }
        }
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) atomicMax(s_max, top);
        if (bad) *s_badp = 1;
        __syncthreads();
        if (warp < n) {
            float at = a[0];
#pragma unroll
            for (int t = 1; t < kSelectFew; ++t)
                if (warp == t) at = a[t];
            const float bound = select_bound(at, *s_max);
            const int stop = end_of(warp);
            const long long list = list_of(warp);
            const float* const mine = s_score + warp * p.run_pages - page0;
            if (lane == 0) p.bounds[list] = bound;
            int m = 0;
            if (bound > 0.f && bound < INFINITY && stop > begin) {
                const float floor = stop - begin <= p.cap ? -INFINITY : border_of(stop - begin, need, [&](int i) { return mine[begin + i]; }) - 2.f * bound;
                SelectCandidate* const found = p.found + list * 2 * p.cap;
                for (int j0 = begin; j0 < stop; j0 += 32) {
                    const int j = j0 + lane;
                    const float x = j < stop ? mine[j] : 0.f;
                    const bool take = j < stop && x >= floor;
                    const uint32_t b = __ballot_sync(0xffffffffu, take);
                    const int at_m = m + __popc(b & ((1u << lane) - 1));
                    if (take && at_m < p.cap) found[at_m] = SelectCandidate{x, j};
                    m += __popc(b);
                }
            }
            if (lane == 0) {
                p.counts[list * 2] = m;
                p.counts[list * 2 + 1] = 0;
            }
        }
        if (tid == 0) p.bad[item] = *s_badp ? 2 /* VPP_DEV_BAD_BLOCK */ : 0;
        return;
    }

    // ---- many tokens: tensor cores ----
    if (warp == 0) {
        tmem_alloc(smem_u32(const_cast<uint32_t*>(s_tmem)), 128);
        tmem_relinquish();
    }
    uint4 x[8];
    int e[8];
    auto look = [&](int j0) {         // pages of the thread's eight vectors, rows tid / 16 + 16 i of the step
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = j0 + (tid >> 4) + 16 * i;
            e[i] = j < page1 ? __ldg(table + j) : 0;
        }
    };
    auto fetch = [&](int j0) {        // their means
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = j0 + (tid >> 4) + 16 * i;
            const bool fine = e[i] >= 0 && e[i] < p.num_blocks;
            bad |= !fine;
            x[i] = make_uint4(0, 0, 0, 0);        // (pages that are taken anyway count as 0: what theirs hold must not widen the bound)
            if (j < page1 && j >= begin && fine) x[i] = ld_once(p.means + (static_cast<long long>(e[i]) * p.num_kv_heads + g) * 256 + v * 16);
        }
    };
    look(page0);
    for (int t = tid >> 4; t < n; t += kSelectThreads / 16) {
        float s[8] = {}, a = 0.f;
        const uint8_t* src = q0 + static_cast<long long>(t) * p.num_q_heads * 256 + v * 16;
#pragma unroll 8
        for (int h = 0; h < G; ++h) {
            const uint4 y = ld_once(src + h * 256);
            const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                s[2 * k] += bf16_lo(w[k]);
                s[2 * k + 1] += bf16_hi(w[k]);
                a += fabsf(bf16_lo(w[k])) + fabsf(bf16_hi(w[k]));
            }
        }
        const unsigned half_mask = 0xffffu << (lane & 16);        // (the other half's token may not exist)
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) a += __shfl_xor_sync(half_mask, a, o);
        uint32_t hi[4], rest[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            hi[k] = pack_bf16x2(s[2 * k], s[2 * k + 1]);
            rest[k] = pack_bf16x2(s[2 * k] - bf16_lo(hi[k]), s[2 * k + 1] - bf16_hi(hi[k]));
        }
        uint8_t* const to = sA + (v >> 3) * (kSelectTile * 128) + t * 128 + (((v & 7) ^ (t & 7)) << 4);
        *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(to + kSelectA / 2) = make_uint4(rest[0], rest[1], rest[2], rest[3]);
        if (v == 0) s_a[t] = a;
    }
    fetch(page0);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    constexpr uint32_t kIdesc = idesc_bf16(kSelectTile, kSelectTile, false, false), kHi = desc_hi_sw128(1024);
    const int my_row = (warp & 3) * 32 + lane, half = warp >> 2;
    const int stop = my_row < n ? end_of(my_row) : 0;
    const int gp = p.group_pages, row_groups = gp > 0 ? p.run_pages / gp : 0;
    float* const my_maxima = p.maxima + (static_cast<long long>(item) * kSelectTile + my_row) * row_groups;
    // no more candidates than fit: no border is needed
    const bool filter = page1 - begin > p.cap;
    uint32_t phase = 0;
    bool alive = true;
    float floor = -3.4e38f;      // (below every score that counts and above the -inf of pages that are no candidates)
    SelectCandidate* const found = p.found + (list_of(my_row) * 2 + half) * p.cap;
    SelectCandidate* to_next = found;
    int m = 0;                   // those that found no room
    float mx[32];                // gp == 0: of the pages that are column i of a piece
#pragma unroll
    for (int i = 0; i < 32; ++i) mx[i] = -INFINITY;
    for (int pass = filter ? 0 : 1; pass < 2 && alive; ++pass) {
        for (int j0 = page0; j0 < page1; j0 += kSelectTile) {
            const bool more = j0 + kSelectTile < page1;
            if (more || pass == 0) look(more ? j0 + kSelectTile : page0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int t = (tid >> 4) + 16 * i;
                if (pass == 0 || !filter) top = abs_max(top, x[i]);
                *reinterpret_cast<uint4*>(sB + (v >> 3) * (kSelectTile * 128) + t * 128 + (((v & 7) ^ (t & 7)) << 4)) = x[i];
            }
            fence_proxy_async_smem();
            __syncthreads();              // (operands in place; the last step's scores have left tensor memory)
            if (tid == 0) {
                tc_fence_after();
                const uint32_t a0 = desc_lo_sw128(base, 16), b0 = desc_lo_sw128(base + kSelectA, 16);
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const uint32_t at = (((k >> 2) & 1) * (kSelectTile * 128) + (k & 3) * 32) >> 4;
                    mma_ss_lhh(tmem, a0 + (k >> 3) * (kSelectA / 2 >> 4) + at, kHi, b0 + at, kHi, kIdesc, k > 0);
                }
                tc_commit(bar);
            }
            if (more || pass == 0) fetch(more ? j0 + kSelectTile : page0);
            alive = __syncthreads_and(mbar_wait(bar, phase, s_abort, 501));
            if (!alive) break;
            phase ^= 1;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t s[32];
                tmem_ld32(tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + half * 64 + c * 32, s);
                tc_wait_ld(s);
                const int j = j0 + half * 64 + c * 32;      // page of the first column
                if (j >= page1) continue;
                if (j < begin || __any_sync(0xffffffffu, j + 32 > stop)) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (j + i < begin || j + i >= stop) s[i] = 0xff800000u;   // -inf
                }
                if (pass == 0) {
                    if (gp == 0) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) mx[i] = fmaxf(mx[i], __uint_as_float(s[i]));
                    } else if (my_row < n) {
                        float4* const to = reinterpret_cast<float4*>(my_maxima + (j - page0) / gp);
                        auto at = [&](int i) { return __uint_as_float(s[i]); };
                        auto two = [&](int i) { return fmaxf(at(2 * i), at(2 * i + 1)); };
                        auto four = [&](int i) { return fmax3(at(4 * i), at(4 * i + 1), fmaxf(at(4 * i + 2), at(4 * i + 3))); };
                        if (gp == 4) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) to[i] = make_float4(four(4 * i), four(4 * i + 1), four(4 * i + 2), four(4 * i + 3));
                        } else if (gp == 2) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) to[i] = make_float4(two(4 * i), two(4 * i + 1), two(4 * i + 2), two(4 * i + 3));
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; ++i) to[i] = make_float4(at(4 * i), at(4 * i + 1), at(4 * i + 2), at(4 * i + 3));
                        }
                    }
                } else if (to_next - found <= p.cap - 32) {      // (room for them all: no check at each)
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const float y = __uint_as_float(s[i]);
                        if (y >= floor) *to_next++ = SelectCandidate{y, j + i};
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const float y = __uint_as_float(s[i]);
                        if (y >= floor) {
                            if (to_next - found < p.cap) *to_next++ = SelectCandidate{y, j + i};
                            else ++m;
                        }
                    }
                }
                __syncwarp();
            }
            tc_fence_before();
        }
        if (!alive || pass == 1) continue;
        // ---- the borders ----
        const uint32_t warp_top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) atomicMax(s_max, warp_top);
        __syncthreads();
        if (gp == 0) {
            // a thread a token (each twice): its 64 maxima, half of them from the other half's thread through the operand's place
            float* const other = reinterpret_cast<float*>(sB) + my_row;       // [32][128], twice: 32 KB
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (half == 1) other[i * kSelectTile] = mx[i];
            __syncthreads();
            float f = INFINITY;          // (lists without choice, or bounds that say nothing: no candidates)
            if (half == 0) {
                const float bound = my_row < n ? select_bound(s_a[my_row], *s_max) : 0.f;
                if (stop > begin && bound > 0.f && bound < INFINITY) {
                    f = -3.4e38f;
                    if (stop - begin > p.cap) {
                        float mo[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) mo[i] = other[i * kSelectTile];
                        uint32_t t = 0;      // the need-th largest of them, 16 bits of it
#pragma unroll 1
                        for (int b = 31; b >= 16; --b) {
                            const float c = key_value(t | (1u << b));
                            int k = 0;
#pragma unroll
                            for (int i = 0; i < 32; ++i) k += (mx[i] >= c) + (mo[i] >= c);
                            if (k >= need) t |= 1u << b;
                        }
                        f = fmaxf(f, key_value(t) - 2.f * bound);
                    }
                }
                if (my_row < n) s_floor[my_row] = f;
            }
        } else {
            const int lead_group = (begin - page0) / gp;
            for (int t = warp; t < n; t += kSelectThreads / 32) {
                const int stop_t = end_of(t);
                float f = INFINITY;
                const float bound = select_bound(s_a[t], *s_max);
                if (stop_t > begin && bound > 0.f && bound < INFINITY) {
                    f = -3.4e38f;
                    if (stop_t - begin > p.cap) {
                        const float* const mxs = p.maxima + (static_cast<long long>(item) * kSelectTile + t) * row_groups + lead_group;
                        f = fmaxf(f, border_of((stop_t - page0 + gp - 1) / gp - lead_group, need, [&](int i) { return mxs[i]; }) - 2.f * bound);
                    }
                }
                if (lane == 0) s_floor[t] = f;
            }
        }
        __syncthreads();
        if (my_row < n) floor = s_floor[my_row];
    }
    const uint32_t warp_top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) atomicMax(s_max, warp_top);
    if (bad) *s_badp = 1;
    if (*s_abort != 0)
        for (int i = 0; i < 64; ++i) __nanosleep(1000);  // let MMAs in flight drain
    __syncthreads();
    if (my_row < n) {
        p.counts[list_of(my_row) * 2 + half] = static_cast<int>(to_next - found) + m;
        if (half == 0) p.bounds[list_of(my_row)] = select_bound(s_a[my_row], *s_max);
    }
    if (tid == 0) p.bad[item] = *s_abort != 0 ? 3 /* VPP_DEV_TIMEOUT */ : *s_badp ? 2 /* VPP_DEV_BAD_BLOCK */ : 0;
    if (warp == 0) tmem_dealloc(tmem, 128);
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
    int32_t close[kPickClose];                // (entries of page / score)
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

// Scores in 64 bits of n pages -- pages[index[c]], or first + c -- by a warp.  NaN counts as -inf.  (out of line, arguments by value: rare, and
// the common path keeps its registers)
__device__ __noinline__ void exact_scores(PickRow w, const int32_t* pages, const int32_t* index, int first, int n, double* out) {
    const int lane = threadIdx.x & 31;
    double ask[4] = {};
    for (int h = 0; h < w.group; ++h) {
        const uint2 x = *reinterpret_cast<const uint2*>(w.q + h * 256 + lane * 8);
        ask[0] += static_cast<double>(bf16_lo(x.x));
        ask[1] += static_cast<double>(bf16_hi(x.x));
        ask[2] += static_cast<double>(bf16_lo(x.y));
        ask[3] += static_cast<double>(bf16_hi(x.y));
    }
    for (int c = 0; c < n; ++c) {
        const int e = __ldg(w.table + (pages ? pages[index[c]] : first + c));
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
        if (near && at < kPickClose) s.close[at] = i;
        near_n += __popc(b);
    }
    const int left = need - sure;         // to be taken of the near ones: 1 .. near_n
    if (left != near_n) {
        if (near_n > kPickClose) return false;
        __syncwarp();
        exact_scores(w, s.page, s.close, 0, near_n, s.exact);
        // losers among the near ones get a page of -1
        int lost = 0;
        for (int c = lane; c < near_n; c += 32) {
            const double d = s.exact[c];
            const int page = s.page[s.close[c]];
            int before = 0;
            for (int j = 0; j < near_n; ++j) before += s.exact[j] > d || (s.exact[j] == d && s.page[s.close[j]] < page);
            if (before >= left) lost |= 1 << (c >> 5);
        }
        __syncwarp();                     // (all have read the pages)
        for (int c = lane; c < near_n; c += 32)
            if ((lost >> (c >> 5)) & 1) s.page[s.close[c]] = -1;
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

// What the common path does not settle -- infinite or NaN scores, more candidates than fit (many pages that are (nearly) the same): all pages' scores in 64
// bits, 128 at a time, each time joined with the best so far.
__device__ __noinline__ void pick_thorough(PickScratch& s, PickRow w, int begin, int end, int need) {
    const int lane = threadIdx.x & 31;
    int best = 0;
    for (int j0 = begin; j0 < end; j0 += kPickClose) {
        const int n = min(kPickClose, end - j0), m = best + n;
        exact_scores(w, nullptr, nullptr, j0, n, s.all + best);
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

// The first work_blocks blocks pick; the block after them, if there is one, writes the status.
__global__ void __launch_bounds__(kPickThreads, 4) block_pick_kernel(const SelectParams p, const int work_blocks) {
    extern __shared__ __align__(16) uint8_t pick_smem[];
    PickScratch* const scratch = reinterpret_cast<PickScratch*>(pick_smem);
    int32_t* const cu = reinterpret_cast<int32_t*>(pick_smem + kPickSmem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_launch_dependents();
    pdl_wait();
    if (static_cast<int>(blockIdx.x) >= work_blocks) {
        int worst = 0;
        for (int i = tid; i < p.items; i += kPickThreads) {
            const int b = p.bad[i];
            worst = max(worst, b == 1 ? 8 : b == 3 ? 6 : b);       // (lengths before a timeout before a page)
        }
        const bool lengths = __syncthreads_or(worst == 8), late = __syncthreads_or(worst == 6), page = __syncthreads_or(worst == 2);
        if (tid == 0) {
            const int now = lengths ? 1 : late ? 3 : page ? 2 : 0;
            if (p.row0 == 0) *p.status = now;
            else if (now != 0 && *p.status == 0) *p.status = now;
        }
        return;
    }
    if (!scan_lengths<kPickThreads>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu)) return;
    const int G = p.num_q_heads / p.num_kv_heads, need = p.topk - p.num_first - p.num_last;
    PickScratch& s = scratch[warp];
    const int rows = (p.row1 - p.row0) * p.num_kv_heads, step = work_blocks * (kPickThreads / 32);      // (rows of a slab: far below 2^31)
    for (int i = blockIdx.x * (kPickThreads / 32) + warp; i < rows; i += step) {
        const int t0 = i / p.num_kv_heads, t = p.row0 + t0, g = i - t0 * p.num_kv_heads;
        const int r = request_of(cu, p.num_reqs, t);
        const int own = (p.prefix_len[r] + (t - cu[r])) >> p.block_shift;
        int32_t* const out = p.indices + (static_cast<long long>(t) * p.num_kv_heads + g) * p.topk;
        if (own + 1 <= p.topk) {
            for (int k = lane; k < p.topk; k += 32) out[k] = k <= own ? k : -1;
            continue;
        }
        // (own + 1 > topk >= first + last: the two ends do not meet, and there are more candidates than needed)
        const int end = select_end(p, own), run0 = p.num_first / p.run_pages, runs = (end + p.run_pages - 1) / p.run_pages;
        for (int k = lane; k < p.topk; k += 32)
            if (k < p.num_first || k >= p.num_first + need) out[k] = k < p.num_first ? k : own + 1 - (p.topk - k);
        if (need == 0) continue;
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
        const PickRow w{p.q + (static_cast<long long>(t) * p.num_q_heads + g * G) * 256, p.block_table + static_cast<long long>(r) * p.max_blocks_per_req,
                        p.means + g * 256, static_cast<long long>(p.num_kv_heads) * 256, G, p.num_blocks};
        // the runs' candidates, one behind the other
        int m = 0;
        for (int k = 2 * run0; k < 2 * runs && !odd; ++k) {
            const int c = p.counts[static_cast<long long>(i) * p.runs * 2 + k];
            odd = c > p.cap || m + c > kPickGather || !(p.bounds[static_cast<long long>(i) * p.runs + (k >> 1)] > 0.f);      // (a run whose scores are all 0 lists none)
            if (odd) break;
            const SelectCandidate* const from = p.found + (static_cast<long long>(i) * p.runs * 2 + k) * p.cap;
            for (int j = lane; j < c; j += 32) {
                const SelectCandidate x = from[j];
                s.score[m + j] = x.score;
                s.page[m + j] = x.page;
            }
            m += c;
        }
        __syncwarp();
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
