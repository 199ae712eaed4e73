// Mean keys of the cache pages that a chunk completes: the summaries that page selection (block_select.cuh) scores.
//
// A page of request r is completed by the call whose chunk holds its last position, so each page's mean is formed once, when all
// its keys are in the cache.  One work item is (completed page, kv-head): block_size rows of 256 bytes, read once -- HBM-bound.  The
// 128 threads of a block are 8 groups of 16 lanes, a lane per 16-byte vector; each group sums every eighth key, with up to
// kMeansUnroll loads in flight a lane, and group 0 adds the eight sums.  Sums are in 32 bits, in one fixed order; the
// mean is rounded once, to bf16.
#pragma once
#include <cstdint>

#include "lengths.cuh"
#include "ptx.cuh"
#include "rope.cuh"

namespace vpp {

constexpr int kMeansThreads = 128;
constexpr int kMeansGroups = kMeansThreads / 16;
constexpr int kMeansUnroll = 8;

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
    for (long long task = blockIdx.x; task < pages * p.num_kv_heads; task += work_blocks) {
        const int i = static_cast<int>(task / p.num_kv_heads), h = static_cast<int>(task - static_cast<long long>(i) * p.num_kv_heads);
        const int blk = page_of(i);
        const bool valid = blk >= 0 && blk < p.num_blocks;
        float acc[8] = {};
        if (valid) {
            const uint8_t* src = p.k_cache + blk * p.block_stride + h * p.head_stride + v * 16;
            for (int t0 = group; t0 < B; t0 += kMeansGroups * kMeansUnroll) {
                uint4 x[kMeansUnroll];
#pragma unroll
                for (int j = 0; j < kMeansUnroll; ++j)
                    if (t0 + j * kMeansGroups < B) x[j] = ld_once(src + (t0 + j * kMeansGroups) * p.token_stride);
#pragma unroll
                for (int j = 0; j < kMeansUnroll; ++j)
                    if (t0 + j * kMeansGroups < B) {
                        const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            acc[2 * e] += bf16_lo(w[e]);
                            acc[2 * e + 1] += bf16_hi(w[e]);
                        }
                    }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s_sum[group][v][e] = acc[e];
        __syncthreads();
        if (group == 0 && valid) {
            float m[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = 0.f;
#pragma unroll
                for (int g = 0; g < kMeansGroups; ++g) s += s_sum[g][v][e];
                m[e] = s / static_cast<float>(B);        // (a power of two: exact)
            }
            p.means[(static_cast<long long>(blk) * p.num_kv_heads + h) * 16 + v] =
                make_uint4(pack_bf16x2(m[0], m[1]), pack_bf16x2(m[2], m[3]), pack_bf16x2(m[4], m[5]), pack_bf16x2(m[6], m[7]));
        }
        __syncthreads();
    }
}

}  // namespace vpp
