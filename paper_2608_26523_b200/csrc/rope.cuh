// Rotary positions, by themselves and on the way into the paged cache.
//
// Feature pairs (a, b) of a row at position pos are turned by the angle pos * inv_freq[i]:
//     a' = a cos - b sin,   b' = b cos + a sin        (times `amplitude`)
// with pairs (i, i + rot_dim / 2) of the rotated part ("half") or (2 i, 2 i + 1) ("interleaved"); features outside it are copied.
// inv_freq is the caller's table, so every scaling of it for long contexts is the same code.
//
// Every byte is read once and written once, so HBM bounds it.  A warp takes one piece of a token at a time: up to kRopePiece units of
// its rows, a unit being two 16-byte vectors of one head that hold each other's partners ("half": vectors u and u + rot_dim / 16).
// Its loads are issued first; while they are in flight the warp looks up the token's request, position and page and works out the
// token's cosines and sines, once for all heads of the piece (two angles a lane at 128 rotated features), in 512 bytes of
// shared memory of its own.
//
// Angles: pos * inv_freq is formed in 64 bits and reduced to half a turn there (32 bits are off by 0.03 rad at a position of a million), the
// cosine and sine of what is left, which is below one turn, in 32 bits.  Rotated features are rounded once, to bf16; the products
// are in 32 bits.
#pragma once
#include <cstdint>

#include "lengths.cuh"
#include "ptx.cuh"

namespace vpp {

constexpr int kRopeThreads = 256;
constexpr int kRopeUnroll = 4;
constexpr int kRopePiece = 32 * kRopeUnroll;   // units of 32 bytes a warp moves at a time
constexpr int kRopeMaxPairs = 128;             // pairs of features (rot_dim / 2)

// Rows of one kind: heads x head_dim features a token, both sides described by strides in bytes.
struct RopeRows {
    const uint8_t* src;
    long long src_token, src_head;
    uint8_t* dst;                 // dense-by-stride destination; the cache for keys and values
    long long dst_block, dst_token, dst_head;   // (dst_block: cache only)
    int units;                    // heads * units_per_head
    int per_head;                 // units of a head: head_dim / 16
};

struct RopeParams {
    RopeRows q, k, v;             // units = 0: none of that kind
    const float* inv_freq;
    int pairs;                    // rot_dim / 2
    int first_vec;                // rot_offset / 8
    float amplitude;
    const int32_t* block_table;
    const int32_t* prefix_len;
    const int32_t* chunk_len;
    int num_reqs, max_blocks_per_req, block_shift, num_blocks;
    long long capacity;           // positions a request can hold
    int total_q;
    int32_t* status;
};

// (not the read-only path: a rotation in place writes what this kernel reads)
__device__ __forceinline__ uint4 ld_once(const uint8_t* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Two vectors that hold each other's partners: eight pairs, cs[0..7] = (cos, sin) of theirs.
__device__ __forceinline__ void turn_half(uint4& a, uint4& b, const float2* cs) {
    uint32_t* x = &a.x;
    uint32_t* y = &b.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 t = *reinterpret_cast<const float4*>(cs + 2 * i);
        const float a0 = bf16_lo(x[i]), a1 = bf16_hi(x[i]), b0 = bf16_lo(y[i]), b1 = bf16_hi(y[i]);
        x[i] = pack_bf16x2(a0 * t.x - b0 * t.y, a1 * t.z - b1 * t.w);
        y[i] = pack_bf16x2(b0 * t.x + a0 * t.y, b1 * t.z + a1 * t.w);
    }
}
// A vector of four pairs.
__device__ __forceinline__ void turn_interleaved(uint4& a, const float2* cs) {
    uint32_t* x = &a.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = cs[i];
        const float a0 = bf16_lo(x[i]), b0 = bf16_hi(x[i]);
        x[i] = pack_bf16x2(a0 * t.x - b0 * t.y, b0 * t.x + a0 * t.y);
    }
}

// The two vectors of unit u of a head, and whether they are rotated: the first pairs / 8 units hold the rotated vectors
// (first_vec + u and that plus pairs / 8), the others the rest in order, half a rest apart.
__device__ __forceinline__ bool rope_unit(int u, int per_head, int first_vec, int rot_units, int& va, int& vb) {
    if (u < rot_units) {
        va = first_vec + u;
        vb = va + rot_units;
        return true;
    }
    const int rest = per_head - rot_units;
    va = u - rot_units;
    vb = va + rest;
    if (va >= first_vec) va += 2 * rot_units;
    if (vb >= first_vec) vb += 2 * rot_units;
    return false;
}

// The first work_blocks blocks rotate; the block after them, if there is one, writes the status.
template <bool kInterleaved>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeParams p, const int work_blocks) {
    extern __shared__ int32_t cu[];   // cu[r] = rows before request r; cu[num_reqs] = total
    __shared__ __align__(16) float2 s_cs[kRopeThreads / 32][kRopeMaxPairs];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_launch_dependents();
    pdl_wait();                       // rows, lengths and table may come from the kernel launched just before
    const bool ok = scan_lengths<kRopeThreads>(p.prefix_len, p.chunk_len, p.num_reqs, p.capacity, p.total_q, cu);
    if (static_cast<int>(blockIdx.x) >= work_blocks) {
        // pages of each request's first and last row and of every block_size-th row of the launch: every page is among theirs
        bool bad = false;
        if (ok && p.block_table != nullptr) {
            auto outside = [&](int r, int pos) {
                const int e = __ldg(p.block_table + static_cast<long long>(r) * p.max_blocks_per_req + (pos >> p.block_shift));
                return e < 0 || e >= p.num_blocks;
            };
            for (int r = threadIdx.x; r < p.num_reqs; r += kRopeThreads) {
                const int n = cu[r + 1] - cu[r];
                if (n > 0) bad |= outside(r, p.prefix_len[r]) | outside(r, p.prefix_len[r] + n - 1);
            }
            for (long long g = static_cast<long long>(threadIdx.x) << p.block_shift; g < p.total_q; g += static_cast<long long>(kRopeThreads) << p.block_shift) {
                const int r = request_of(cu, p.num_reqs, static_cast<int>(g));
                bad |= outside(r, p.prefix_len[r] + (static_cast<int>(g) - cu[r]));
            }
        }
        const int any = __syncthreads_or(bad);
        if (threadIdx.x == 0) *p.status = !ok ? 1 /* VPP_DEV_BAD_LENGTHS */ : any ? 2 /* VPP_DEV_BAD_BLOCK */ : 0;
        return;
    }
    if (!ok) return;                  // lengths that do not describe this launch: write nothing
    const int units = p.q.units + p.k.units + p.v.units;
    const int pieces = (units + kRopePiece - 1) / kRopePiece;
    const long long tasks = static_cast<long long>(p.total_q) * pieces, stride = static_cast<long long>(work_blocks) * (kRopeThreads / 32);
    const int rot_units = p.pairs >> 3;
    float2* const cs = s_cs[warp];
    for (long long task = static_cast<long long>(blockIdx.x) * (kRopeThreads / 32) + warp; task < tasks; task += stride) {
        const int row = static_cast<int>(task / pieces);
        const int u0 = static_cast<int>(task - static_cast<long long>(row) * pieces) * kRopePiece + lane;
        // where a unit's vectors are: kind, head, the two vectors
        auto place = [&](int u, int& kind, int& head, int& va, int& vb) -> bool {
            kind = u < p.q.units ? 0 : u < p.q.units + p.k.units ? 1 : 2;
            const RopeRows& w = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
            const int x = u - (kind == 0 ? 0 : kind == 1 ? p.q.units : p.q.units + p.k.units);
            head = x / w.per_head;
            const int in = x - head * w.per_head;
            if (kind == 2) {
                va = in;
                vb = in + w.per_head;
                return false;
            }
            return rope_unit(in, w.per_head, p.first_vec, rot_units, va, vb);
        };
        uint4 a[kRopeUnroll], b[kRopeUnroll];
#pragma unroll
        for (int i = 0; i < kRopeUnroll; ++i) {
            const int u = u0 + 32 * i;
            if (u >= units) continue;
            int kind, head, va, vb;
            place(u, kind, head, va, vb);
            const RopeRows& w = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
            const uint8_t* from = w.src + row * w.src_token + head * w.src_head;
            a[i] = ld_once(from + va * 16);
            b[i] = ld_once(from + vb * 16);
        }
        const int r = request_of(cu, p.num_reqs, row);
        const int pos = p.prefix_len[r] + (row - cu[r]);
        long long blk = 0;
        int slot = 0;
        if (p.k.units + p.v.units > 0) {
            if (p.block_table == nullptr) {
                blk = r;
                slot = pos;
            } else {
                blk = p.block_table[static_cast<long long>(r) * p.max_blocks_per_req + (pos >> p.block_shift)];
                slot = pos & ((1 << p.block_shift) - 1);
                if (blk < 0 || blk >= p.num_blocks) blk = -1;      // the row's page is not valid: its keys and values are skipped
            }
        }
        __syncwarp();                 // (the last piece's readers of cs are done)
        for (int i = lane; i < p.pairs; i += 32) {
            const double turns = static_cast<double>(pos) * static_cast<double>(__ldg(p.inv_freq + i)) * 0.15915494309189533577;   // 1 / (2 pi)
            float sn, c;
            sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &sn, &c);
            cs[i] = make_float2(c * p.amplitude, sn * p.amplitude);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kRopeUnroll; ++i) {
            const int u = u0 + 32 * i;
            if (u >= units) continue;
            int kind, head, va, vb;
            if (place(u, kind, head, va, vb)) {
                if (kInterleaved) {
                    turn_interleaved(a[i], cs + (va - p.first_vec) * 4);
                    turn_interleaved(b[i], cs + (vb - p.first_vec) * 4);
                } else {
                    turn_half(a[i], b[i], cs + (va - p.first_vec) * 8);
                }
            }
            const RopeRows& w = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
            if (kind != 0 && blk < 0) continue;
            uint8_t* to = w.dst + head * w.dst_head + (kind == 0 ? row * w.dst_token : blk * w.dst_block + slot * w.dst_token);
            *reinterpret_cast<uint4*>(to + va * 16) = a[i];
            *reinterpret_cast<uint4*>(to + vb * 16) = b[i];
        }
    }
}

}  // namespace vpp
