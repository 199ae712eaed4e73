// Mean keys of the cache pages that a chunk completes: the summaries that page selection (block_select.cuh) scores.
//
// A page of request r is completed by the call whose chunk holds its last position, so each page's mean is formed once, when all
// its keys are in the cache.  One work item is (completed page, kv-head): block_size rows of 256 bytes, read once -- HBM-bound.  16 lanes
// a key, a lane per 16-byte vector, up to kMeansUnroll loads in flight a lane, and the next item's page looked up under them.  Items of up to 64 keys are
// a warp's, longer ones a block's (which adds its eight groups' sums in shared memory).  Sums are in 32 bits, in one fixed order; the mean is rounded once, to bf16.
// A context of 131072 tokens and 8 kv-heads, pages of 64 / 16: 45.5 / 51.8 us, 5.9 / 5.2 TB/s (a block an item: 66 / 217 us); 16384 keys in pages of 128, 8.2 us, 4.1 TB/s (all in a
// captured graph; as calls one after the other the last takes 9.7).
#pragma once
#include <cstdint>

#include "lengths.cuh"
#include "ptx.cuh"
#include "rope.cuh"

namespace vpp {

constexpr int kMeansThreads = 128;
constexpr int kMeansGroups = kMeansThreads / 16;
constexpr int kMeansUnroll = 8;
constexpr int kMeansWarpShift = 6;             // pages of up to 64 keys: a warp each

struct MeansParams {
    const uint8_t* k_cache;
    long long block_stride, token_stride, head_stride;   // bytes
    uint4* means;             // [num_blocks, Hkv, 128] bf16
    const int32_t* block_table;
    const int32_t* prefix_len;
    const int32_t* chunk_len;
    int num_reqs, max_blocks_per_req, block_shift, num_blocks;
    long long capacity;
    int total_q, num_kv_heads;
    int32_t* status;
};

// The first work_blocks blocks form means; the block after them, if there is one, writes the status.
__global__ void __launch_bounds__(kMeansThreads) block_means_kernel(const MeansParams p, const int work_blocks) {
    extern __shared__ int32_t cu[];   // rows before request r, cu[num_reqs] = all; then pages completed before it, the same
    __shared__ float s_sum[kMeansGroups][16][9];     // (a lane's eight features; 9: no bank conflicts)
    int32_t* const done = cu + p.num_reqs + 1;
    const int tid = threadIdx.x;
    pdl_launch_dependents();
    pdl_wait();
    const bool ok = scan_lengths<kMeansThreads>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu);
    const bool checks = static_cast<int>(blockIdx.x) >= work_blocks;
    if (!ok) {
        if (checks && tid == 0) *p.status = 1 /* VPP_DEV_BAD_LENGTHS */;
        return;
    }
    block_scan<kMeansThreads>(p.num_reqs, 0x7fffffffu, done, false, [&](int r, bool&) {
        const int pre = p.prefix_len[r];
        return ((pre + (cu[r + 1] - cu[r])) >> p.block_shift) - (pre >> p.block_shift);
    });
    const long long pages = done[p.num_reqs];
    auto page_of = [&](int i) {        // physical page of the i-th completed one
        const int r = request_of(done, p.num_reqs, i);
        return __ldg(p.block_table + static_cast<long long>(r) * p.max_blocks_per_req + (p.prefix_len[r] >> p.block_shift) + (i - done[r]));
    };
    if (checks) {
        bool bad = false;
        for (long long i = tid; i < pages; i += kMeansThreads) {
            const int e = page_of(static_cast<int>(i));
            bad |= e < 0 || e >= p.num_blocks;
        }
        const int any = __syncthreads_or(bad);
        if (tid == 0) *p.status = any ? 2 /* VPP_DEV_BAD_BLOCK */ : 0;
        return;
    }
    const int group = tid >> 4, v = tid & 15, B = 1 << p.block_shift;
    const bool by_warp = p.block_shift <= kMeansWarpShift;
    const int workers = by_warp ? work_blocks * (kMeansThreads / 32) : work_blocks;
    const int groups = by_warp ? 2 : kMeansGroups, my_group = by_warp ? group & 1 : group;
    const long long tasks = pages * p.num_kv_heads;
    long long task = by_warp ? blockIdx.x * (kMeansThreads / 32) + (tid >> 5) : blockIdx.x;
    int next = task < tasks ? page_of(static_cast<int>(task / p.num_kv_heads)) : -1;
    for (; task < tasks; task += workers) {
        const int h = static_cast<int>(task % p.num_kv_heads), blk = next;
        const bool valid = blk >= 0 && blk < p.num_blocks;
        const uint8_t* const src = p.k_cache + (valid ? blk : 0) * p.block_stride + h * p.head_stride + v * 16;
        float acc[8] = {};
        for (int t0 = my_group; t0 < B; t0 += groups * kMeansUnroll) {
            uint4 x[kMeansUnroll];
#pragma unroll
            for (int j = 0; j < kMeansUnroll; ++j) {
                x[j] = make_uint4(0, 0, 0, 0);
                if (valid && t0 + j * groups < B) x[j] = ld_once(src + (t0 + j * groups) * p.token_stride);
            }
            // (the next page is looked up under these)
            if (t0 == my_group) next = task + workers < tasks ? page_of(static_cast<int>((task + workers) / p.num_kv_heads)) : -1;
#pragma unroll
            for (int j = 0; j < kMeansUnroll; ++j) {
                const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[2 * e] += bf16_lo(w[e]);
                    acc[2 * e + 1] += bf16_hi(w[e]);
                }
            }
        }
        if (by_warp) {
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], 16);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) s_sum[group][v][e] = acc[e];
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
#pragma unroll
                    for (int g = 1; g < kMeansGroups; ++g) acc[e] += s_sum[g][v][e];
                }
            }
            __syncthreads();
        }
        if ((by_warp ? my_group : group) == 0 && valid) {
            const float by = 1.f / static_cast<float>(B);        // (a power of two: exact)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] *= by;
            p.means[(static_cast<long long>(blk) * p.num_kv_heads + h) * 16 + v] =
                make_uint4(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]), pack_bf16x2(acc[4], acc[5]), pack_bf16x2(acc[6], acc[7]));
        }
    }
}

}  // namespace vpp
