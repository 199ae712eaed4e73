// Rotary positions, by themselves and on the way into the paged cache.
//
// Feature pairs (a, b) of a row at position pos are turned by the angle pos * inv_freq[i]:
//     a' = a cos - b sin,   b' = b cos + a sin        (times `amplitude`)
// with pairs (i, i + rot_dim / 2) of the rotated part ("half") or (2 i, 2 i + 1) ("interleaved"); features outside it are copied.
// inv_freq is the caller's table, so every scaling of it for long contexts is the same code.
//
// Every byte is read once and written once, so HBM bounds it, as long as few instructions go with a byte.  A warp takes a piece of one token's rows of one
// kind (queries, keys or values) at a time, kRopeUnroll units a lane, a unit being two 16-byte vectors of one head that hold each other's
// partners ("half": vectors u and u + rot_dim / 16).  Its loads are issued first; while they are in flight the warp looks up the token's
// request, position and page and works out the token's cosines and sines, once for all heads of the piece (two angles a lane at 128 rotated
// features), in 512 bytes of shared memory of its own.  16384 tokens of 64/8 heads: 112 us in a captured graph, 6.0 TB/s, 92 % of the copy rate (as calls one after the other 121, 85 %); 8192 tokens of
// 128 x 64 features into wider rows 46.3 us, 89 % (48.6).  Tried: pieces that mix the kinds, with a division for each unit (1160 instructions a piece, 69 % of the issue
// slots: 119 and 52 us); pieces of two and four rounds with one set of angles (146 and 129 us, 46.3 both); 32 warps an SM instead of 24 (114 and 51 us).
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
    uint32_t inverse;             // ceil(2^32 / per_head), 0 for 1: x / per_head is the high word of x * inverse as long as x * per_head < 2^32
    int pieces;                   // of a token
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
    const int q_pieces = p.q.pieces, k_pieces = p.k.pieces, pieces = q_pieces + k_pieces + p.v.pieces;
    const long long tasks = static_cast<long long>(p.total_q) * pieces, stride = static_cast<long long>(work_blocks) * (kRopeThreads / 32);
    const int rot_units = p.pairs >> 3, first_vec = p.first_vec;
    float2* const cs = s_cs[warp];
    for (long long task = static_cast<long long>(blockIdx.x) * (kRopeThreads / 32) + warp; task < tasks; task += stride) {
        const int row = static_cast<int>(task / pieces);
        const int piece = static_cast<int>(task - static_cast<long long>(row) * pieces);
        const int kind = piece < q_pieces ? 0 : piece < q_pieces + k_pieces ? 1 : 2;
        const RopeRows& w = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
        const int u_begin = (piece - (kind == 0 ? 0 : kind == 1 ? q_pieces : q_pieces + k_pieces)) * kRopePiece;
        const int u_end = w.units, per_head = w.per_head, turned = kind == 2 ? 0 : rot_units, rest = per_head - turned;
        const uint32_t inverse = w.inverse;
        const long long src_head = w.src_head, dst_head = w.dst_head;
        const uint8_t* const src = w.src + row * w.src_token;
        uint8_t* dst = w.dst;
        // a unit's head and first vector, and how far the second one is: the first `turned` units of a head hold the rotated vectors, the others the rest
        // in order, half a rest apart
        auto place = [&](int u, int& head, int& va, int& vb) -> bool {
            head = inverse ? __umulhi(static_cast<uint32_t>(u), inverse) : u;
            const int in = u - head * per_head;
            const bool turn = in < turned;
            va = turn ? first_vec + in : in - turned;
            vb = va + (turn ? turned : rest);
            if (!turn) {
                if (va >= first_vec) va += 2 * turned;
                if (vb >= first_vec) vb += 2 * turned;
            }
            return turn;
        };
        uint4 a[kRopeUnroll], b[kRopeUnroll];
#pragma unroll
        for (int i = 0; i < kRopeUnroll; ++i) {
            const int u = u_begin + lane + 32 * i;
            if (u >= u_end) continue;
            int head, va, vb;
            place(u, head, va, vb);
            const uint8_t* const from = src + head * src_head;
            a[i] = ld_once(from + va * 16);
            b[i] = ld_once(from + vb * 16);
        }
        const int r = request_of(cu, p.num_reqs, row);
        const int pos = p.prefix_len[r] + (row - cu[r]);
        bool write = true;
        if (kind == 0) {
            dst += row * w.dst_token;
        } else {
            long long blk = r;
            int slot = pos;
            if (p.block_table != nullptr) {
                blk = p.block_table[static_cast<long long>(r) * p.max_blocks_per_req + (pos >> p.block_shift)];
                slot = pos & ((1 << p.block_shift) - 1);
                write = blk >= 0 && blk < p.num_blocks;      // (the row's page is not valid: its keys and values are skipped)
            }
            dst += blk * w.dst_block + slot * w.dst_token;
        }
        if (kind != 2) {
            __syncwarp();                 // (the last piece's readers of cs are done)
            for (int i = lane; i < p.pairs; i += 32) {
                const double turns = static_cast<double>(pos) * static_cast<double>(__ldg(p.inv_freq + i)) * 0.15915494309189533577;   // 1 / (2 pi)
                float sn, c;
                sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &sn, &c);
                cs[i] = make_float2(c * p.amplitude, sn * p.amplitude);
            }
            __syncwarp();
        }
        if (!write) continue;
#pragma unroll
        for (int i = 0; i < kRopeUnroll; ++i) {
            const int u = u_begin + lane + 32 * i;
            if (u >= u_end) continue;
            int head, va, vb;
            if (place(u, head, va, vb)) {
                if (kInterleaved) {
                    turn_interleaved(a[i], cs + (va - first_vec) * 4);
                    turn_interleaved(b[i], cs + (vb - first_vec) * 4);
                } else {
                    turn_half(a[i], b[i], cs + (va - first_vec) * 8);
                }
            }
            uint8_t* const to = dst + head * dst_head;
            *reinterpret_cast<uint4*>(to + va * 16) = a[i];
            *reinterpret_cast<uint4*>(to + vb * 16) = b[i];
        }
    }
}

}  // namespace vpp
