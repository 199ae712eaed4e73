// prefix_len / chunk_len of a launch in shared memory, for the kernels that find a packed row's request themselves.
#pragma once
#include <cstdint>

namespace vpp {

constexpr int kLengthsMaxReqs = 8192;   // the scan of chunk_len lives in shared memory (32 KB + 4)

// Exclusive scan of chunk_len into cu[0 .. num_reqs] (shared memory), by a whole block of kThreads; true if the lengths describe
// the launch: none negative, no request past `capacity` positions, their sum total_q.  (The sums are formed in 64 bits: lengths that
// wrap around to total_q must not pass.)
template <int kThreads>
__device__ __forceinline__ bool scan_lengths(const int32_t* prefix_len, const int32_t* chunk_len, int num_reqs, long long capacity,
                                             int total_q, int32_t* cu) {
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & 31;
    if (tid == 0) s_bad = 0;
    __syncthreads();
    bool bad = false;
    for (int r = tid; r < num_reqs; r += kThreads) {   // (all loads at once, then the scan from shared memory)
        int c = chunk_len[r];
        const int pre = prefix_len[r];
        if (c < 0 || c > total_q || pre < 0 || static_cast<long long>(pre) + c > capacity) {
            bad = true;
            c = 0;
        }
        cu[r] = c;
    }
    if (bad) s_bad = 1;
    __syncthreads();
    if (tid < 32) {
        long long carry = 0;
        for (int base = 0; base < num_reqs; base += 32) {
            const int r = base + lane;
            const int c = r < num_reqs ? cu[r] : 0;
            long long x = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            if (r < num_reqs) cu[r] = static_cast<int32_t>(carry + x - c);
            carry += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) {
            cu[num_reqs] = static_cast<int32_t>(carry);
            if (carry != total_q) s_bad = 1;
        }
    }
    __syncthreads();
    return !s_bad;
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
