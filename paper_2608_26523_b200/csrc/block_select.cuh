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
// Two kernels a slab of tokens (as many as have scores of kSelectSlabBytes together, so that these stay in the L2):
//  * block_scores_kernel: an item is (up to 128 tokens of one request, kv-head, a run of pages).  The group's queries are
//    summed first, in 32 bits, and the sum split in two bf16 (hi + rest: 16 bits of it), so that the tensor cores do 2 / group
//    of the work of all q-heads; scores of 128 tokens x 128 pages are one accumulator.  Reading q bounds it (134 MB of 8192 tokens of 64 heads are
//    21 us; the products 8 us at the matrix rate).  Items of up to kSelectFew tokens -- decode rows -- take the dot products in
//    registers instead, half a warp a page: there reading the means is all.
//  * block_pick_kernel: a warp a (token, kv-head).  The need-th largest of 128 group maxima bounds the border from below; what
//    is not below it by more than the error bound (a few more than needed) is gathered in index order, ranked, and the
//    border settled.
#pragma once
#include <cstdint>

#include "lengths.cuh"
#include "ptx.cuh"
#include "rope.cuh"

namespace vpp {

constexpr int kSelectThreads = 256;
constexpr int kSelectTile = 128;              // tokens of an item, pages of a step
constexpr int kSelectFew = 4;
constexpr int kSelectSlabBytes = 64 << 20;
constexpr int kSelectMaxTopk = 256;
constexpr int kSelectA = 2 * 2 * kSelectTile * 128;   // two bf16 parts of 128 x 128, two 64-feature slabs each
constexpr int kSelectB = 2 * kSelectTile * 128;
constexpr int kSelectSmem = kSelectA + kSelectB + 1024 /* alignment */ + 1024 /* barrier, bounds */;

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
    int row_pages;                // floats of a row of scores
    float* scores;                // [row1 - row0, Hkv, row_pages]
    float* bounds;                // [row1 - row0, Hkv, runs]: error bound of the row's scores of a run
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

__device__ __forceinline__ void st_v8(float* p, const uint32_t* r) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]),
                 "r"(r[6]), "r"(r[7]) : "memory");
}

__global__ void __launch_bounds__(kSelectThreads) block_scores_kernel(const SelectParams p) {
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
    float* const s_a = reinterpret_cast<float*>(sX + 32);          // [128]
    int32_t* const cu = reinterpret_cast<int32_t*>(sX + 1024);     // [num_reqs + 1], then tile counts [num_reqs + 1]
    int32_t* const first_tile = cu + p.num_reqs + 1;

    pdl_launch_dependents();
    pdl_wait();
    const bool ok = scan_lengths<kSelectThreads>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu);
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
    if (warp == 0) {
        int carry = 0;
        for (int b = 0; b < p.num_reqs; b += 32) {
            const int r = b + lane;
            int lo, n = 0;
            if (r < p.num_reqs) n = (rows_of(r, lo) + kSelectTile - 1) / kSelectTile;
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
    if (tid == 0) {
        *s_abort = 0;
        *s_max = 0;
        *s_badp = 0;
        mbar_init(bar, 1);
        fence_mbar_init();
    }
    __syncthreads();
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
    const int page0 = run * p.run_pages, page1 = min(page0 + p.run_pages, end);
    if (page1 <= max(page0, p.num_first) || ((pos0 + n - 1) >> p.block_shift) + 1 <= p.topk) {
        if (tid == 0) p.bad[item] = 0;
        return;
    }
    const int G = p.num_q_heads / p.num_kv_heads;
    const int32_t* const table = p.block_table + static_cast<long long>(r) * p.max_blocks_per_req;
    const uint8_t* const q0 = p.q + (static_cast<long long>(row) * p.num_q_heads + g * G) * 256;
    const long long score_row0 = static_cast<long long>(row - p.row0) * p.num_kv_heads + g;      // of the tile's first token; tokens are Hkv rows apart
    const int v = tid & 15;
    bool bad = false;
    uint32_t top = 0;

    if (n <= kSelectFew) {
        // ---- a few tokens: half a warp a page ----
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
        constexpr int kDeep = 4;
        const int half = tid >> 4;
        for (int j0 = page0; j0 < page1; j0 += kDeep * (kSelectThreads / 16)) {
            uint4 x[kDeep];
            int e[kDeep];
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const int j = j0 + i * (kSelectThreads / 16) + half;
                e[i] = j < page1 ? __ldg(table + j) : 0;
            }
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const int j = j0 + i * (kSelectThreads / 16) + half;
                const bool fine = e[i] >= 0 && e[i] < p.num_blocks;
                bad |= !fine;
                x[i] = make_uint4(0, 0, 0, 0);
                if (j < page1 && j >= p.num_first && fine) x[i] = ld_once(p.means + (static_cast<long long>(e[i]) * p.num_kv_heads + g) * 256 + v * 16);
            }
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
                    if (v == 0 && j < page1) p.scores[(score_row0 + static_cast<long long>(t) * p.num_kv_heads) * p.row_pages + j] = d;
                }
            }
        }
        atomicMax(s_max, top);
        if (bad) *s_badp = 1;
        __syncthreads();
        if (tid < n) {
            float at = a[0];
#pragma unroll
            for (int t = 1; t < kSelectFew; ++t)
                if (tid == t) at = a[t];
            p.bounds[(score_row0 + static_cast<long long>(tid) * p.num_kv_heads) * p.runs + run] = select_bound(at, *s_max);
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
    auto fetch = [&](int j0) {        // 128 pages' means: the thread's eight vectors, of rows tid / 16 + 16 i
        int e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = j0 + (tid >> 4) + 16 * i;
            e[i] = j < page1 ? __ldg(table + j) : 0;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = j0 + (tid >> 4) + 16 * i;
            const bool fine = e[i] >= 0 && e[i] < p.num_blocks;
            bad |= !fine;
            x[i] = make_uint4(0, 0, 0, 0);        // (pages that are taken anyway count as 0: what theirs hold must not widen the bound)
            if (j < page1 && j >= p.num_first && fine) x[i] = ld_once(p.means + (static_cast<long long>(e[i]) * p.num_kv_heads + g) * 256 + v * 16);
        }
    };
    for (int t = tid >> 4; t < n; t += kSelectThreads / 16) {
        float s[8] = {}, a = 0.f;
        const uint8_t* src = q0 + static_cast<long long>(t) * p.num_q_heads * 256 + v * 16;
#pragma unroll 8
        for (int h = 0; h < G; ++h) {
            const uint4 y = ld_once(src + h * 256);
            const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[2 * e] += bf16_lo(w[e]);
                s[2 * e + 1] += bf16_hi(w[e]);
                a += fabsf(bf16_lo(w[e])) + fabsf(bf16_hi(w[e]));
            }
        }
        const unsigned half_mask = 0xffffu << (lane & 16);        // (the other half's token may not exist)
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) a += __shfl_xor_sync(half_mask, a, o);
        uint32_t hi[4], rest[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            hi[e] = pack_bf16x2(s[2 * e], s[2 * e + 1]);
            rest[e] = pack_bf16x2(s[2 * e] - bf16_lo(hi[e]), s[2 * e + 1] - bf16_hi(hi[e]));
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
    const int my_row = (warp & 3) * 32 + lane, col0 = (warp >> 2) * 64;
    float* const out = p.scores + (score_row0 + static_cast<long long>(my_row) * p.num_kv_heads) * p.row_pages;
    uint32_t phase = 0;
    bool alive = true;
    for (int j0 = page0; j0 < page1; j0 += kSelectTile) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int t = (tid >> 4) + 16 * i;
            top = abs_max(top, x[i]);
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
        if (j0 + kSelectTile < page1) fetch(j0 + kSelectTile);
        alive = mbar_wait(bar, phase, s_abort, 501);
        if (!__syncthreads_and(alive)) break;
        phase ^= 1;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t s[32];
            tmem_ld32(tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + col0 + c * 32, s);
            tc_wait_ld();
            if (my_row < n) {
#pragma unroll
                for (int i = 0; i < 4; ++i) st_v8(out + j0 + col0 + c * 32 + i * 8, s + i * 8);
            }
        }
        tc_fence_before();
    }
    atomicMax(s_max, top);
    if (bad) *s_badp = 1;
    if (*s_abort != 0)
        for (int i = 0; i < 64; ++i) __nanosleep(1000);  // let MMAs in flight drain
    __syncthreads();
    if (tid < n) p.bounds[(score_row0 + static_cast<long long>(tid) * p.num_kv_heads) * p.runs + run] = select_bound(s_a[tid], *s_max);
    if (tid == 0) p.bad[item] = *s_abort != 0 ? 3 /* VPP_DEV_TIMEOUT */ : *s_badp ? 2 /* VPP_DEV_BAD_BLOCK */ : 0;
    if (warp == 0) tmem_dealloc(tmem, 128);
}

// ---- the border -----------------------------------------------------------------------------------------------------------------

constexpr int kPickThreads = 256;
constexpr int kPickGather = 512;              // entries a warp can gather
constexpr int kPickClose = 128;               // entries near the border that it can settle at once
static_assert(kSelectMaxTopk < kPickGather, "what is needed fits");
struct PickScratch {
    double exact[kPickClose];
    float score[kPickGather];
    int32_t page[kPickGather];
    int32_t close[kPickClose];                // (entries of page / score)
};
constexpr int kPickSmem = static_cast<int>(sizeof(PickScratch)) * (kPickThreads / 32);

// Unsigned integers in the order of floats; NaN below everything.
__device__ __forceinline__ uint32_t order_key(float f) {
    if (!(f == f)) return 0;
    const uint32_t u = __float_as_uint(f + 0.f);          // (-0 becomes 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

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

// Keeps of the m gathered entries (ascending pages, all that can be among the best) the `need` best: their pages move to the
// front of s.page, in order.  delta: bound on the error of a score.  False: more of them are too close to tell than fit.
__device__ __forceinline__ bool pick_settle(PickScratch& s, const PickRow& w, int m, int need, float delta) {
    const int lane = threadIdx.x & 31;
    const uint32_t k0 = lane < m ? order_key(s.score[lane]) : 0, k1 = lane + 32 < m ? order_key(s.score[lane + 32]) : 0;
    uint32_t border = 0;      // the need-th best score
    for (int b = 31; b >= 0; --b) {
        const uint32_t c = border | (1u << b);
        int k = (k0 >= c) + (k1 >= c);
        for (int i = lane + 64; i < m; i += 32) k += order_key(s.score[i]) >= c;
        if (static_cast<int>(__reduce_add_sync(0xffffffffu, k)) >= need) border = c;
    }
    const float v = key_value(border), hi = v + 2.f * delta, lo = v - 2.f * delta;
    // sure ones (above hi: their exact scores are above those of all but need - 1), and those too close to the border to tell
    int sure = 0, near_n = 0;
    for (int i0 = 0; i0 < m; i0 += 32) {
        const int i = i0 + lane;
        const float x = i < m ? s.score[i] : 0.f;
        const uint32_t k = order_key(x);
        const bool in = i < m && k > border && x > hi, near = i < m && !in && (k >= border || x >= lo);
        sure += __popc(__ballot_sync(0xffffffffu, in));
        const uint32_t b = __ballot_sync(0xffffffffu, near);
        const int at = near_n + __popc(b & ((1u << lane) - 1));
        if (near && at < kPickClose) s.close[at] = i;
        near_n += __popc(b);
    }
    const int left = need - sure;         // to be taken of the near ones: 1 .. near_n
    const bool all = left == near_n, same = delta == 0.f;        // (same: all scores are exact, so the near ones are equal)
    if (!all && !same) {
        if (near_n > kPickClose) return false;
        __syncwarp();
        exact_scores(w, s.page, s.close, 0, near_n, s.exact);
        // losers among the near ones get a page of -1
        for (int c = lane; c < near_n; c += 32) {
            const double d = s.exact[c];
            int before = 0;
            for (int j = 0; j < near_n; ++j) before += s.exact[j] > d || (s.exact[j] == d && j < c);
            if (before >= left) s.page[s.close[c]] = -1;
        }
    }
    __syncwarp();
    int kept = 0, seen = 0;
    for (int i0 = 0; i0 < m; i0 += 32) {
        const int i = i0 + lane;
        const float x = i < m ? s.score[i] : 0.f;
        const int page = i < m ? s.page[i] : -1;
        const uint32_t k = order_key(x);
        const bool in = i < m && k > border && x > hi, near = i < m && !in && (k >= border || x >= lo);
        const uint32_t b = __ballot_sync(0xffffffffu, near);
        const bool take = in || (near && page >= 0 && (all || !same || seen + __popc(b & ((1u << lane) - 1)) < left));
        seen += __popc(b);
        const uint32_t t = __ballot_sync(0xffffffffu, take);      // (all have read their page)
        if (take) s.page[kept + __popc(t & ((1u << lane) - 1))] = page;
        kept += __popc(t);
        __syncwarp();
    }
    return true;
}

// Entries of the row at or above `floor`, in order.  Returns their number; those past kPickGather are not stored.
__device__ __forceinline__ int pick_gather(PickScratch& s, const float* row, int begin, int end, float floor) {
    const int lane = threadIdx.x & 31;
    int m = 0;
    for (int j0 = begin; j0 < end; j0 += 32) {
        const int j = j0 + lane;
        const float x = j < end ? row[j] : 0.f;
        const bool take = j < end && x >= floor;
        const uint32_t b = __ballot_sync(0xffffffffu, take);
        const int at = m + __popc(b & ((1u << lane) - 1));
        if (take && at < kPickGather) {
            s.score[at] = x;
            s.page[at] = j;
        }
        m += __popc(b);
    }
    __syncwarp();
    return m;
}

// What the common path does not settle: infinite or NaN scores, long lists of many pages, many pages that are (nearly) the same.
__device__ __noinline__ void pick_thorough(PickScratch& s, PickRow w, float* row, int begin, int end, int need, float delta) {
    const int lane = threadIdx.x & 31;
    if (!(delta < INFINITY)) {
        // scores anew: those of 64 bits, rounded
        float big = 0.f;
        for (int j0 = begin; j0 < end; j0 += kPickClose) {
            const int n = min(kPickClose, end - j0);
            exact_scores(w, nullptr, nullptr, j0, n, s.exact);
            for (int c = lane; c < n; c += 32) {
                const float x = static_cast<float>(s.exact[c]);
                row[j0 + c] = x;
                if (fabsf(x) < INFINITY) big = fmaxf(big, fabsf(x));
            }
            __syncwarp();
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
        delta = big * 1.1920929e-7f + 1e-44f;
    }
    uint32_t t = 0;       // the need-th best score
    for (int b = 31; b >= 0; --b) {
        const uint32_t c = t | (1u << b);
        int k = 0;
        for (int j = begin + lane; j < end; j += 32) k += order_key(row[j]) >= c;
        if (static_cast<int>(__reduce_add_sync(0xffffffffu, k)) >= need) t = c;
    }
    const float floor = key_value(t) - 2.f * delta;       // (-inf stays, inf stays)
    const int m = pick_gather(s, row, begin, end, floor);
    if (m <= kPickGather && pick_settle(s, w, m, need, delta)) return;
    // one after the other, in 64 bits
    double last = INFINITY;
    int last_page = -1;
    for (int k = 0; k < need; ++k) {
        double best = -INFINITY;
        int best_page = INT32_MAX;
        for (int j0 = begin; j0 < end; j0 += kPickClose) {
            const int n = min(kPickClose, end - j0);
            exact_scores(w, nullptr, nullptr, j0, n, s.exact);
            for (int c = lane; c < n; c += 32) {
                const double d = s.exact[c];
                const int j = j0 + c;
                if (d > last || (d == last && j <= last_page)) continue;      // taken already
                if (best_page == INT32_MAX || d > best) {
                    best = d;
                    best_page = j;
                }
            }
            __syncwarp();
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const double d = __shfl_xor_sync(0xffffffffu, best, o);
            const int j = __shfl_xor_sync(0xffffffffu, best_page, o);
            if (j != INT32_MAX && (best_page == INT32_MAX || d > best || (d == best && j < best_page))) {
                best = d;
                best_page = j;
            }
        }
        last = best;
        last_page = best_page;
        // kept ascending: those behind it move up by one
        int before = 0;
        for (int i = lane; i < k; i += 32) before += s.page[i] < best_page;
        before = __reduce_add_sync(0xffffffffu, before);
        for (int i0 = k / 32 * 32; i0 >= 0; i0 -= 32) {
            const int i = i0 + lane;
            const bool moves = i < k && i >= before;
            const int page = moves ? s.page[i] : 0;
            __syncwarp();
            if (moves) s.page[i + 1] = page;
            __syncwarp();
        }
        if (lane == 0) s.page[before] = best_page;
        __syncwarp();
    }
}

// The best `need` of the pages [begin, end), end - begin > need > 0, into s.page, ascending.
__device__ __forceinline__ void pick(PickScratch& s, const PickRow& w, float* row, int begin, int end, int need, float delta) {
    if (delta < INFINITY && need <= 128) {       // (no infinite or NaN score)
        const int lane = threadIdx.x & 31;
        // the need-th largest of 128 maxima is not above the need-th largest of all
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        int j = begin + lane;
        for (; j + 96 < end; j += 128) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], row[j + 32 * k]);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (j + 32 * k < end) mx[k] = fmaxf(mx[k], row[j + 32 * k]);
        uint32_t t = 0, key[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) key[k] = order_key(mx[k]);
        for (int b = 31; b >= 10; --b) {         // (a little below will do)
            const uint32_t c = t | (1u << b);
            int k = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) k += key[e] >= c;
            if (static_cast<int>(__reduce_add_sync(0xffffffffu, k)) >= need) t = c;
        }
        const float floor = t < 0x00800000u ? -INFINITY : key_value(t) - 2.f * delta;      // (maxima of nothing: every page)
        const int m = pick_gather(s, row, begin, end, floor);
        if (m <= kPickGather && pick_settle(s, w, m, need, delta)) return;
    }
    pick_thorough(s, w, row, begin, end, need, delta);
}

// The first work_blocks blocks pick; the block after them, if there is one, writes the status.
__global__ void __launch_bounds__(kPickThreads) block_pick_kernel(const SelectParams p, const int work_blocks) {
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
    const int G = p.num_q_heads / p.num_kv_heads;
    const long long rows = static_cast<long long>(p.row1 - p.row0) * p.num_kv_heads, step = static_cast<long long>(work_blocks) * (kPickThreads / 32);
    for (long long i = static_cast<long long>(blockIdx.x) * (kPickThreads / 32) + warp; i < rows; i += step) {
        const int t = p.row0 + static_cast<int>(i / p.num_kv_heads), g = static_cast<int>(i % p.num_kv_heads);
        const int r = request_of(cu, p.num_reqs, t);
        const int own = (p.prefix_len[r] + (t - cu[r])) >> p.block_shift;
        int32_t* const out = p.indices + (static_cast<long long>(t) * p.num_kv_heads + g) * p.topk;
        if (own + 1 <= p.topk) {
            for (int k = lane; k < p.topk; k += 32) out[k] = k <= own ? k : -1;
            continue;
        }
        const int end = select_end(p, own), need = p.topk - p.num_first - p.num_last;      // (own + 1 > topk >= first + last: no overlap)
        if (need > 0) {
            float delta = 0.f;
            bool odd = false;
            const float* b = p.bounds + i * p.runs;
            for (int k = p.num_first / p.run_pages + lane; k * p.run_pages < end; k += 32) {
                const float x = b[k];
                odd |= !(x < INFINITY);
                delta = fmaxf(delta, x);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) delta = fmaxf(delta, __shfl_xor_sync(0xffffffffu, delta, o));
            if (__any_sync(0xffffffffu, odd)) delta = INFINITY;
            const PickRow w{p.q + (static_cast<long long>(t) * p.num_q_heads + g * G) * 256, p.block_table + static_cast<long long>(r) * p.max_blocks_per_req,
                            p.means + g * 256, static_cast<long long>(p.num_kv_heads) * 256, G, p.num_blocks};
            pick(scratch[warp], w, p.scores + i * p.row_pages, p.num_first, end, need, delta);
        }
        __syncwarp();
        for (int k = lane; k < p.topk; k += 32)
            out[k] = k < p.num_first ? k : k < p.num_first + need ? scratch[warp].page[k - p.num_first] : own + 1 - (p.topk - k);
        __syncwarp();
    }
}

}  // namespace vpp
