// prefix_len / chunk_len of a launch in shared memory, for the kernels that find a packed row's request themselves.
#pragma once
#include <cstdint>

namespace vpp {

constexpr int kLengthsMaxReqs = 8192;   // the scan of chunk_len lives in shared memory (32 KB + 4)

// Exclusive sums of count(i), i = 0 .. n - 1, into out[0 .. n] (shared memory), by a whole block of kThreads; the sums stop at `most`.  Ends
// with a barrier.  Returns whether any thread was `bad`.
template <int kThreads, typename Count>
__device__ __forceinline__ bool block_scan(int n, uint32_t most, int32_t* out, bool bad, Count count) {
    __shared__ uint32_t s_warp[2][kThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t carry = 0;
    for (int base = 0, round = 0; base < n; base += kThreads, round ^= 1) {
        const int i = base + tid;
        const uint32_t c = i < n ? static_cast<uint32_t>(count(i, bad)) : 0u;
        uint32_t x = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x = min(x + y, most);
        }
        if (lane == 31) s_warp[round][warp] = x;
        __syncthreads();
        uint32_t before = carry;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w == warp) before = carry;
            carry = min(carry + s_warp[round][w], most);
        }
        uint32_t left = __shfl_up_sync(0xffffffffu, x, 1);
        if (lane == 0) left = 0;
        if (i < n) out[i] = static_cast<int32_t>(min(before + left, most));
    }
    if (tid == 0) out[n] = static_cast<int32_t>(carry);
    return __syncthreads_or(bad);
}

// Exclusive scan of chunk_len into cu[0 .. num_reqs] (shared memory), by a whole block of kThreads; true if the lengths describe
// the launch: none negative, no request past `capacity` positions, their sum total_q.  (Sums stop at total_q + 1: lengths that would wrap around to
// total_q do not pass.)  With tile_rows > 0 the tiles of so many rows that every request has are scanned into first_tile as well, under the same barriers.
template <int kThreads>
__device__ __forceinline__ bool scan_lengths(const int32_t* prefix_len, const int32_t* chunk_len, int num_reqs, long long capacity,
                                             int total_q, int32_t* cu, int tile_rows = 0, int32_t* first_tile = nullptr) {
    __shared__ uint2 s_warp[2][kThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t most = static_cast<uint32_t>(total_q) + 1u;      // (tiles are no more than rows)
    uint2 carry = make_uint2(0, 0);
    bool bad = false;
    auto add = [&](uint2 a, uint2 b) { return make_uint2(min(a.x + b.x, most), min(a.y + b.y, most)); };
    for (int base = 0, round = 0; base < num_reqs; base += kThreads, round ^= 1) {
        const int r = base + tid;
        uint2 x = make_uint2(0, 0);
        if (r < num_reqs) {
            const int c = chunk_len[r], pre = prefix_len[r];
            if (c >= 0 && c <= total_q && pre >= 0 && static_cast<long long>(pre) + c <= capacity) {
                x.x = static_cast<uint32_t>(c);
                if (tile_rows > 0) x.y = (x.x + tile_rows - 1) / tile_rows;
            } else {
                bad = true;
            }
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint2 y = make_uint2(__shfl_up_sync(0xffffffffu, x.x, o), __shfl_up_sync(0xffffffffu, x.y, o));
            if (lane >= o) x = add(x, y);
        }
        if (lane == 31) s_warp[round][warp] = x;
        uint2 left = make_uint2(__shfl_up_sync(0xffffffffu, x.x, 1), __shfl_up_sync(0xffffffffu, x.y, 1));
        if (lane == 0) left = make_uint2(0, 0);
        __syncthreads();
        uint2 before = carry;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w == warp) before = carry;
            carry = add(carry, s_warp[round][w]);
        }
        before = add(before, left);
        if (r < num_reqs) {
            cu[r] = static_cast<int32_t>(before.x);
            if (tile_rows > 0) first_tile[r] = static_cast<int32_t>(before.y);
        }
    }
    if (tid == 0) {
        cu[num_reqs] = static_cast<int32_t>(carry.x);
        if (tile_rows > 0) first_tile[num_reqs] = static_cast<int32_t>(carry.y);
    }
    const bool any = __syncthreads_or(bad);
    return !any && cu[num_reqs] == total_q;
}

// Request of row g (0 <= g < total_q): the last r with cu[r] <= g.
__device__ __forceinline__ int request_of(const int32_t* cu, int num_reqs, int g) {
    int lo = 0, hi = num_reqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cu[mid] <= g) lo = mid; else hi = mid - 1;
    }
    return lo;
}

}  // namespace vpp
