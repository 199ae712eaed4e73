// Host side of the rotary and block-sparse entry points of include/vpp.h: argument checks and launches.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/vpp.h"
#include "attn_blk.cuh"
#include "block_means.cuh"
#include "block_select.cuh"
#include "common.cuh"
#include "host.h"
#include "lengths.cuh"
#include "rope.cuh"

using namespace vpp::host;

namespace {

// The dynamic shared memory that launches of a kernel may have: the most that any call's has, not this call's, for it holds for the launches of other host
// threads too.
constexpr int kLengthsMaxBytes = 4 * (vpp::kLengthsMaxReqs + 1);
template <typename Kernel>
cudaError_t allow_smem(Kernel kernel, int most) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
}

bool mis16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

vpp_status check_rope(const vpp_rope_spec& r, int head_dim, int heads) {
    // (also: units of a row times units of a head stay below 2^32, see RopeRows::inverse)
    if (head_dim > 1024 || heads > 65536) return fail(VPP_ERR_UNSUPPORTED, "head dims up to 1024 and up to 65536 heads");
    if (!r.inv_freq) return fail(VPP_ERR_INVALID_ARG, "inv_freq is null");
    if (r.layout != VPP_ROPE_HALF && r.layout != VPP_ROPE_INTERLEAVED) return fail(VPP_ERR_INVALID_ARG, "layout must be VPP_ROPE_HALF or VPP_ROPE_INTERLEAVED");
    if (!std::isfinite(r.amplitude)) return fail(VPP_ERR_INVALID_ARG, "amplitude must be finite");
    if (r.rot_dim <= 0 || r.rot_dim % 16 || r.rot_dim > 2 * vpp::kRopeMaxPairs)
        return fail(VPP_ERR_UNSUPPORTED, "rot_dim must be a multiple of 16 in 16..%d", 2 * vpp::kRopeMaxPairs);
    if (r.rot_offset < 0 || r.rot_offset % 8) return fail(VPP_ERR_UNSUPPORTED, "rot_offset must be a non-negative multiple of 8");
    if (r.rot_offset > head_dim - r.rot_dim) return fail(VPP_ERR_INVALID_ARG, "rot_offset + rot_dim exceeds the head dim (%d)", head_dim);
    return VPP_OK;
}

bool good_stride(int64_t s) { return s >= 0 && s % 8 == 0; }

// One launch of the rotation; p's rows, lengths and table are filled in.
vpp_status launch_rope(vpp::RopeParams& p, const vpp_rope_spec& r, cudaStream_t stream) {
    p.inv_freq = r.inv_freq;
    p.pairs = r.rot_dim / 2;
    p.first_vec = r.rot_offset / 8;
    p.amplitude = r.amplitude;
    const int warps = vpp::kRopeThreads / 32;
    vpp::RopeRows* const kinds[3] = {&p.q, &p.k, &p.v};
    long long pieces = 0;
    for (vpp::RopeRows* w : kinds) pieces += w->pieces = (w->units + vpp::kRopePiece - 1) / vpp::kRopePiece;
    const long long tasks = pieces * p.total_q;
    long long blocks = (tasks + warps - 1) / warps;
    const long long cap = 16ll * sm_count_or_default();
    if (blocks > cap) blocks = cap;
    const int work_blocks = static_cast<int>(blocks);
    auto kern = r.layout == VPP_ROPE_INTERLEAVED ? vpp::rope_kernel<true> : vpp::rope_kernel<false>;
    const cudaError_t ce = launch(kern, static_cast<unsigned>(work_blocks + (p.status ? 1 : 0)), vpp::kRopeThreads,
                                  sizeof(int32_t) * (static_cast<size_t>(p.num_reqs) + 1), stream, p, work_blocks);
    if (ce != cudaSuccess) return fail(VPP_ERR_CUDA, "rotation launch: %s", cudaGetErrorString(ce));
    return VPP_OK;
}

vpp::RopeRows rows_of(const void* src, int64_t src_token, int64_t src_head, void* dst, int64_t dst_block, int64_t dst_token, int64_t dst_head, int heads, int dim) {
    vpp::RopeRows w{};
    w.src = static_cast<const uint8_t*>(src);
    w.src_token = src_token * 2;
    w.src_head = src_head * 2;
    w.dst = static_cast<uint8_t*>(dst);
    w.dst_block = dst_block * 2;
    w.dst_token = dst_token * 2;
    w.dst_head = dst_head * 2;
    w.per_head = dim / 16;
    w.units = heads * w.per_head;
    w.inverse = static_cast<uint32_t>((0x100000000ull + w.per_head - 1) / w.per_head);      // (2^32 itself becomes 0)
    return w;
}

// Positions a request's pages can hold, as far as positions are counted (0: bad arguments).
long long paged_capacity(int max_blocks_per_req, int block_size) {
    const long long n = static_cast<long long>(max_blocks_per_req) * block_size;
    return n < INT32_MAX ? n : INT32_MAX;
}

vpp_status check_paged(const int32_t* block_table, int block_size, int max_blocks_per_req, int num_blocks) {
    if (!block_table) return fail(VPP_ERR_UNSUPPORTED, "a block table is required: pages are the blocks");
    if (!is_pow2(block_size)) return fail(VPP_ERR_UNSUPPORTED, "block_size must be a power of two");
    if (max_blocks_per_req <= 0 || num_blocks <= 0) return fail(VPP_ERR_INVALID_ARG, "max_blocks_per_req and num_blocks must be > 0");
    return VPP_OK;
}

// ---- page selection: slabs of tokens, and where their scores are ----
struct SelectPlan {
    int slab;                   // tokens of a slab
    int run_pages, runs;        // pages of an item, items along a row
    int group_pages, cap;
    int item_tokens;            // most tokens of an item
    int many_items, few_items;  // most items of a slab: of up to 256 tokens; of one
    size_t found, counts, bounds, maxima, bad, total;
};

vpp_status select_plan(const vpp_block_select_args* a, SelectPlan* s) {
    if (!a) return fail(VPP_ERR_INVALID_ARG, "args is null");
    if (a->num_reqs < 0 || a->total_q < 0 || a->max_seq_len < 0) return fail(VPP_ERR_INVALID_ARG, "num_reqs, total_q and max_seq_len must be >= 0");
    if (a->num_q_heads <= 0 || a->num_kv_heads <= 0 || a->num_q_heads % a->num_kv_heads != 0)
        return fail(VPP_ERR_INVALID_ARG, "num_q_heads (%d) must be a positive multiple of num_kv_heads (%d)", a->num_q_heads, a->num_kv_heads);
    if (a->head_dim != 128 || a->num_q_heads / a->num_kv_heads > 128)
        return fail(VPP_ERR_UNSUPPORTED, "head_dim must be 128 and groups of q-heads at most 128");
    if (a->num_reqs > vpp::kLengthsMaxReqs) return fail(VPP_ERR_UNSUPPORTED, "at most %d requests", vpp::kLengthsMaxReqs);
    if (!is_pow2(a->block_size)) return fail(VPP_ERR_UNSUPPORTED, "block_size must be a power of two");
    if (a->topk < 1 || a->topk > vpp::kSelectMaxTopk) return fail(VPP_ERR_UNSUPPORTED, "topk must be in 1..%d", vpp::kSelectMaxTopk);
    if (a->num_first < 0 || a->num_last < 1 || a->num_first > a->topk || a->num_last > a->topk - a->num_first)
        return fail(VPP_ERR_INVALID_ARG, "need num_first >= 0, num_last >= 1 and num_first + num_last <= topk");
    const long long T = a->total_q > 0 ? a->total_q : 1, H = a->num_kv_heads, N = vpp::kSelectTile;
    const long long sms = sm_count_or_default(), steps = (a->max_seq_len / a->block_size + N) / N;       // of 128 pages along a row
    auto tiles_of = [&](long long rows, long long item) {
        const long long tiles = (rows + a->num_reqs * (item - 1)) / item;      // (every request rounds up)
        return tiles < rows ? tiles : rows;                                    // (every tile has a token)
    };
    long long I = vpp::kSelectItem;
    const int need = a->topk - a->num_first - a->num_last;
    if (need == 0) {          // no page is scored: lists by position alone
        *s = SelectPlan{};
        s->slab = static_cast<int>(T * H <= 1 << 30 ? T : (1 << 30) / H);
        s->run_pages = vpp::kSelectTile;
        s->total = 256;
        return VPP_OK;
    }
    // A border that is the need-th largest of the maxima of groups lets through about need (1 + need * group / (2 * pages)) pages.  Rows of few pages
    // list them all, others have pages enough for twice as many groups as are needed.
    // (Up to 32 are needed: 64 groups, kept in registers.)
    s->group_pages = need <= 32 ? 0 : need <= 64 ? 4 : need <= 128 ? 2 : 1;
    s->cap = need <= 128 ? 128 : 256;
    // Launches of no more tokens than requests, or of a few tokens: decode rows alone, an item a token.
    const bool few_only = T <= a->num_reqs || T <= vpp::kSelectFew;
    long long few = few_only ? T : a->num_reqs > 1 ? static_cast<long long>(a->num_reqs) * vpp::kSelectFew : 0;
    // Runs of pages, each of which lists its own best: one where the items fill half of the SMs, else as many as fill them all, of 1024 pages or more (decode rows: those
    // are read in 5 us) or 256.
    const long long work = (few_only ? few : tiles_of(T, I)) * H;
    long long runs = work > 0 ? sms / work : 1;
    const long long shortest = few_only ? 8 : 2;
    if (runs > steps / shortest) runs = steps / shortest;
    // (each lists what is needed and a few more, and block_pick_kernel gathers 512 at a time)
    const long long gathered = 2 * 512 / (3 * (need > 0 ? need : 1));
    if (runs > gathered) runs = gathered;
    const long long least = (steps * N + vpp::kSelectMaxRun - 1) / vpp::kSelectMaxRun;
    if (runs < least) runs = least;
    if (runs < 1) runs = 1;
    // Tokens of an item: 256, or fewer where there are SMs for twice as many items all the same (few pages: 3150 tokens of 8/1 heads, 150 pages 60 -> 34 us.  Instead of
    // runs it does not pay: 506 tokens of 32/8 heads, 1539 pages 52 -> 83).
    while (I > 32 && tiles_of(T, I / 2) * H * runs <= sms) I /= 2;
    s->item_tokens = static_cast<int>(I);
    s->run_pages = static_cast<int>((steps + runs - 1) / runs * N);
    s->runs = static_cast<int>((steps * N + s->run_pages - 1) / s->run_pages);
    const long long list = s->runs * (2ll * s->cap * static_cast<long long>(sizeof(vpp::SelectCandidate)) + 12);     // bytes of a row
    const long long item = s->group_pages > 0 ? vpp::kSelectItem * (s->run_pages / s->group_pages) * 4 : 0;                        // of an item
    long long slab = vpp::kSelectSlabBytes / (H * (list + item * s->runs / I));
    slab = slab / I * I;                              // (whole items of a long chunk)
    if (slab < I) slab = I;
    if (slab > T) slab = T;
    s->slab = static_cast<int>(slab);
    // (a request by itself has few rows only in a last slab that is a rest of so many)
    if (few == 0 && T % slab >= 1 && T % slab <= vpp::kSelectFew) few = vpp::kSelectFew;
    const long long many = (few_only ? 0 : tiles_of(slab, I)) * H * s->runs, few_items = (few_only ? slab : few) * H * s->runs;
    if (many + few_items > INT32_MAX) return fail(VPP_ERR_UNSUPPORTED, "too many requests times heads");
    s->many_items = static_cast<int>(many);
    s->few_items = static_cast<int>(few_items);
    const size_t rows = static_cast<size_t>(slab) * H * s->runs;
    if (rows > UINT32_MAX / (2 * s->cap * sizeof(vpp::SelectCandidate)))            // (4 GiB: nobody has so many pages)
        return fail(VPP_ERR_UNSUPPORTED, "too many kv-heads times pages of max_seq_len");
    s->found = 0;
    s->counts = align_up(rows * 2 * s->cap * sizeof(vpp::SelectCandidate), 256);
    s->bounds = align_up(s->counts + rows * 2 * sizeof(int32_t), 256);
    s->maxima = align_up(s->bounds + rows * sizeof(float), 256);
    s->bad = align_up(s->maxima + static_cast<size_t>(many) * item, 256);
    s->total = align_up(s->bad + static_cast<size_t>(many + few_items) * sizeof(int32_t), 256);
    return VPP_OK;
}

// ---- attention over listed pages: tiles, parts and where the lists are ----
struct BlockPlan {
    int group, tile_tokens, words, max_tiles, max_pages, splits;
    size_t items, pages, masks, o_parts, lse_parts, total;
};
constexpr int kBlockMaxTopk = 1024;

vpp_status block_plan(const vpp_chunk_attn_args* a, int32_t topk, BlockPlan* b) {
    if (!a) return fail(VPP_ERR_INVALID_ARG, "args is null");
    if (a->num_reqs < 0 || a->total_q < 0 || a->max_seq_len < 0) return fail(VPP_ERR_INVALID_ARG, "num_reqs, total_q and max_seq_len must be >= 0");
    if (a->num_q_heads <= 0 || a->num_kv_heads <= 0 || a->num_q_heads % a->num_kv_heads != 0)
        return fail(VPP_ERR_INVALID_ARG, "num_q_heads (%d) must be a positive multiple of num_kv_heads (%d)", a->num_q_heads, a->num_kv_heads);
    if (!(a->softmax_scale > 0.f) || !std::isfinite(a->softmax_scale)) return fail(VPP_ERR_INVALID_ARG, "softmax_scale must be positive and finite");
    if (a->num_kv_splits < 0 || a->num_kv_splits > 64) return fail(VPP_ERR_INVALID_ARG, "num_kv_splits must be in [0, 64]");
    b->group = a->num_q_heads / a->num_kv_heads;
    if (a->head_dim_qk != 128 || a->head_dim_v != 128 || b->group > 128)
        return fail(VPP_ERR_UNSUPPORTED, "head dims must be (128, 128) and groups of q-heads at most 128");
    if (!is_pow2(a->block_size) || a->block_size < 16 || a->block_size > 128) return fail(VPP_ERR_UNSUPPORTED, "block_size must be 16, 32, 64 or 128");
    if (topk < 1 || topk > kBlockMaxTopk) return fail(VPP_ERR_UNSUPPORTED, "topk must be in 1..%d", kBlockMaxTopk);
    if (a->num_reqs > vpp::kLengthsMaxReqs) return fail(VPP_ERR_UNSUPPORTED, "at most %d requests", vpp::kLengthsMaxReqs);
    b->tile_tokens = 128 / b->group;
    b->words = (b->tile_tokens + 31) / 32;
    const long long T = a->total_q, H = a->num_kv_heads;
    long long tiles = (T + b->tile_tokens - 1) / b->tile_tokens + a->num_reqs;
    if (tiles > T) tiles = T;                                  // (every tile has a token)
    const long long context = (static_cast<long long>(a->max_seq_len) + a->block_size - 1) / a->block_size;
    long long pages = static_cast<long long>(b->tile_tokens) * topk;
    if (pages > context) pages = context;
    if (pages < 1) pages = 1;
    b->max_tiles = static_cast<int>(tiles);
    b->max_pages = static_cast<int>(pages);
    // Parts of the unions: where there are fewer tiles than SMs.
    const int per_step = 128 / a->block_size;
    const long long listed = T <= a->num_reqs && topk < pages ? topk : pages;      // (decode rows: a tile has one list)
    const long long steps = (listed + per_step - 1) / per_step, work = tiles * H, sms = sm_count_or_default();
    long long s = a->num_kv_splits;
    if (s == 0) {
        s = work > 0 ? sms / work : 1;
        if (s > steps / 2) s = steps / 2;
        if (s > 16) s = 16;
    }
    if (s > steps) s = steps;
    if (s < 1) s = 1;
    b->splits = static_cast<int>(s);
    if (tiles * H * s > INT32_MAX) return fail(VPP_ERR_UNSUPPORTED, "too many tokens times heads");
    const size_t lists = static_cast<size_t>(tiles * H) * pages;
    b->items = align_up(sizeof(vpp::WorkHeader), 256);
    b->pages = align_up(b->items + sizeof(vpp::BlkItem) * static_cast<size_t>(tiles * H), 256);
    b->masks = align_up(b->pages + sizeof(int32_t) * lists, 256);
    b->o_parts = b->lse_parts = b->total = align_up(b->masks + sizeof(uint2) * lists * b->words, 256);
    if (s > 1) {
        const size_t rows = static_cast<size_t>(s) * T * a->num_q_heads;
        b->lse_parts = align_up(b->o_parts + rows * 128 * sizeof(float), 256);
        b->total = align_up(b->lse_parts + rows * sizeof(float), 256);
    }
    return VPP_OK;
}

}  // namespace

extern "C" {

vpp_status vpp_rope(const vpp_rope_args* a, vpp_stream_t stream_) {
    g_err[0] = 0;
    if (!a) return fail(VPP_ERR_INVALID_ARG, "args is null");
    if (a->num_reqs < 0 || a->total_q < 0 || a->num_heads <= 0 || a->head_dim <= 0)
        return fail(VPP_ERR_INVALID_ARG, "num_reqs, total_q >= 0 and num_heads, head_dim > 0 required");
    if (a->head_dim % 16) return fail(VPP_ERR_UNSUPPORTED, "head_dim must be a multiple of 16");
    if (static_cast<int64_t>(a->num_heads) * a->head_dim > INT32_MAX) return fail(VPP_ERR_UNSUPPORTED, "num_heads * head_dim exceeds 2^31 - 1");
    if (a->num_reqs > vpp::kLengthsMaxReqs) return fail(VPP_ERR_UNSUPPORTED, "at most %d requests", vpp::kLengthsMaxReqs);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (a->total_q == 0 || a->num_reqs == 0) return zero_status(a->status, stream);
    const vpp_status st = check_rope(a->rope, a->head_dim, a->num_heads);
    if (st != VPP_OK) return st;
    if (!a->x || !a->out || !a->prefix_len || !a->chunk_len) return fail(VPP_ERR_INVALID_ARG, "x, out, prefix_len and chunk_len must be non-null");
    if (mis16(a->x) || mis16(a->out)) return fail(VPP_ERR_INVALID_ARG, "x and out must be 16-byte aligned");
    if (!good_stride(a->x_token_stride) || !good_stride(a->x_head_stride) || !good_stride(a->out_token_stride) || !good_stride(a->out_head_stride))
        return fail(VPP_ERR_INVALID_ARG, "strides must be non-negative multiples of 8 elements");
    vpp::RopeParams p{};
    p.q = rows_of(a->x, a->x_token_stride, a->x_head_stride, a->out, 0, a->out_token_stride, a->out_head_stride, a->num_heads, a->head_dim);
    p.prefix_len = a->prefix_len;
    p.chunk_len = a->chunk_len;
    p.num_reqs = a->num_reqs;
    p.capacity = INT32_MAX;
    p.total_q = a->total_q;
    p.status = a->status;
    p.k.per_head = p.v.per_head = 1;
    return launch_rope(p, a->rope, stream);
}

vpp_status vpp_kv_append_rope(const vpp_kv_append_rope_args* args, vpp_stream_t stream_) {
    g_err[0] = 0;
    if (!args) return fail(VPP_ERR_INVALID_ARG, "args is null");
    const vpp_kv_append_args* a = &args->append;
    if (a->num_reqs < 0 || a->total_q < 0 || a->num_kv_heads <= 0 || a->head_dim_qk <= 0 || a->head_dim_v <= 0)
        return fail(VPP_ERR_INVALID_ARG, "num_reqs, total_q >= 0 and num_kv_heads, head dims > 0 required");
    if (a->head_dim_qk % 16 || a->head_dim_v % 16) return fail(VPP_ERR_UNSUPPORTED, "head dims must be multiples of 16");
    if ((args->q == nullptr) != (args->q_out == nullptr)) return fail(VPP_ERR_INVALID_ARG, "q and q_out go together");
    if (args->q && args->num_q_heads <= 0) return fail(VPP_ERR_INVALID_ARG, "num_q_heads must be > 0 with q");
    const int64_t heads = static_cast<int64_t>(args->q ? args->num_q_heads : 0) + a->num_kv_heads;
    if (heads * a->head_dim_qk + static_cast<int64_t>(a->num_kv_heads) * a->head_dim_v > INT32_MAX)
        return fail(VPP_ERR_UNSUPPORTED, "a token's heads exceed 2^31 - 1 features");
    if (a->num_reqs > vpp::kLengthsMaxReqs) return fail(VPP_ERR_UNSUPPORTED, "at most %d requests", vpp::kLengthsMaxReqs);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (a->total_q == 0 || a->num_reqs == 0) return zero_status(a->status, stream);
    vpp_status st = check_rope(args->rope, a->head_dim_qk > a->head_dim_v ? a->head_dim_qk : a->head_dim_v, args->q && args->num_q_heads > a->num_kv_heads ? args->num_q_heads : a->num_kv_heads);
    if (st == VPP_OK && args->rope.rot_offset > a->head_dim_qk - args->rope.rot_dim)
        st = fail(VPP_ERR_INVALID_ARG, "rot_offset + rot_dim exceeds the keys' head dim (%d)", a->head_dim_qk);
    if (st != VPP_OK) return st;
    if (!a->k_new || !a->k_cache || !a->prefix_len || !a->chunk_len)
        return fail(VPP_ERR_INVALID_ARG, "k_new, k_cache, prefix_len and chunk_len must be non-null");
    if (a->v_new && !a->v_cache) return fail(VPP_ERR_INVALID_ARG, "v_new given without v_cache");
    vpp::RopeParams p{};
    p.capacity = a->max_seq_len;
    if (a->block_table) {
        st = check_paged(a->block_table, a->block_size, a->max_blocks_per_req, a->num_blocks);
        if (st != VPP_OK) return st;
        p.block_shift = ilog2(a->block_size);
        p.capacity = paged_capacity(a->max_blocks_per_req, a->block_size);
    } else if (a->max_seq_len <= 0) {
        return fail(VPP_ERR_INVALID_ARG, "max_seq_len must be > 0 for a contiguous cache");
    }
    bool good = good_stride(a->k_block_stride) && good_stride(a->k_token_stride) && good_stride(a->k_head_stride) &&
                good_stride(args->k_new_token_stride) && good_stride(args->k_new_head_stride);
    bool mis = mis16(a->k_new) || mis16(a->k_cache);
    if (a->v_new) {
        good = good && good_stride(a->v_block_stride) && good_stride(a->v_token_stride) && good_stride(a->v_head_stride) &&
               good_stride(args->v_new_token_stride) && good_stride(args->v_new_head_stride);
        mis = mis || mis16(a->v_new) || mis16(a->v_cache);
    }
    if (args->q) {
        good = good && good_stride(args->q_token_stride) && good_stride(args->q_head_stride) && good_stride(args->q_out_token_stride) &&
               good_stride(args->q_out_head_stride);
        mis = mis || mis16(args->q) || mis16(args->q_out);
    }
    if (!good) return fail(VPP_ERR_INVALID_ARG, "strides must be non-negative multiples of 8 elements");
    if (mis) return fail(VPP_ERR_INVALID_ARG, "k_new, v_new, q, q_out and the caches must be 16-byte aligned");
    p.q.per_head = p.v.per_head = 1;
    if (args->q)
        p.q = rows_of(args->q, args->q_token_stride, args->q_head_stride, args->q_out, 0, args->q_out_token_stride, args->q_out_head_stride,
                      args->num_q_heads, a->head_dim_qk);
    p.k = rows_of(a->k_new, args->k_new_token_stride, args->k_new_head_stride, a->k_cache, a->k_block_stride, a->k_token_stride, a->k_head_stride,
                  a->num_kv_heads, a->head_dim_qk);
    if (a->v_new)
        p.v = rows_of(a->v_new, args->v_new_token_stride, args->v_new_head_stride, a->v_cache, a->v_block_stride, a->v_token_stride, a->v_head_stride,
                      a->num_kv_heads, a->head_dim_v);
    p.block_table = a->block_table;
    p.prefix_len = a->prefix_len;
    p.chunk_len = a->chunk_len;
    p.num_reqs = a->num_reqs;
    p.max_blocks_per_req = a->max_blocks_per_req;
    p.num_blocks = a->num_blocks;
    p.total_q = a->total_q;
    p.status = a->status;
    return launch_rope(p, args->rope, stream);
}

vpp_status vpp_block_means(const vpp_block_means_args* a, vpp_stream_t stream_) {
    g_err[0] = 0;
    if (!a) return fail(VPP_ERR_INVALID_ARG, "args is null");
    if (a->num_reqs < 0 || a->total_q < 0 || a->num_kv_heads <= 0) return fail(VPP_ERR_INVALID_ARG, "num_reqs, total_q >= 0 and num_kv_heads > 0 required");
    if (a->head_dim != 128) return fail(VPP_ERR_UNSUPPORTED, "head_dim must be 128");
    if (a->num_reqs > vpp::kLengthsMaxReqs) return fail(VPP_ERR_UNSUPPORTED, "at most %d requests", vpp::kLengthsMaxReqs);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (a->total_q == 0 || a->num_reqs == 0) return zero_status(a->status, stream);
    const vpp_status st = check_paged(a->block_table, a->block_size, a->max_blocks_per_req, a->num_blocks);
    if (st != VPP_OK) return st;
    if (!a->k_cache || !a->k_means || !a->prefix_len || !a->chunk_len)
        return fail(VPP_ERR_INVALID_ARG, "k_cache, k_means, prefix_len and chunk_len must be non-null");
    if (mis16(a->k_cache) || mis16(a->k_means)) return fail(VPP_ERR_INVALID_ARG, "k_cache and k_means must be 16-byte aligned");
    if (!good_stride(a->k_block_stride) || !good_stride(a->k_token_stride) || !good_stride(a->k_head_stride))
        return fail(VPP_ERR_INVALID_ARG, "strides must be non-negative multiples of 8 elements");
    vpp::MeansParams p{};
    p.k_cache = static_cast<const uint8_t*>(a->k_cache);
    p.block_stride = a->k_block_stride * 2;
    p.token_stride = a->k_token_stride * 2;
    p.head_stride = a->k_head_stride * 2;
    p.means = static_cast<uint4*>(a->k_means);
    p.block_table = a->block_table;
    p.prefix_len = a->prefix_len;
    p.chunk_len = a->chunk_len;
    p.num_reqs = a->num_reqs;
    p.max_blocks_per_req = a->max_blocks_per_req;
    p.block_shift = ilog2(a->block_size);
    p.num_blocks = a->num_blocks;
    p.capacity = paged_capacity(a->max_blocks_per_req, a->block_size);
    p.total_q = a->total_q;
    p.num_kv_heads = a->num_kv_heads;
    p.status = a->status;
    // a request completes at most one page more than its chunk fills
    long long pages = static_cast<long long>(a->total_q) / a->block_size + a->num_reqs;
    if (pages > a->total_q) pages = a->total_q;
    const bool by_warp = a->block_size <= 1 << vpp::kMeansWarpShift;
    long long blocks = by_warp ? (pages * a->num_kv_heads + vpp::kMeansThreads / 32 - 1) / (vpp::kMeansThreads / 32) : pages * a->num_kv_heads;
    // (every block scans the lengths, and most of a decode step's find no page that is complete: 256 rows of 8 heads 4.3 us, with 16 blocks an SM 7.3)
    const long long cap = 4ll * sm_count_or_default();
    if (blocks > cap) blocks = cap;
    const int work_blocks = static_cast<int>(blocks);
    cudaError_t ce = cudaSuccess;
    if (a->num_reqs > 4096) ce = allow_smem(vpp::block_means_kernel, 2 * kLengthsMaxBytes);
    if (ce == cudaSuccess) ce = launch(vpp::block_means_kernel, static_cast<unsigned>(work_blocks + (a->status ? 1 : 0)), vpp::kMeansThreads,
                                  2 * sizeof(int32_t) * (static_cast<size_t>(a->num_reqs) + 1), stream, p, work_blocks);
    if (ce != cudaSuccess) return fail(VPP_ERR_CUDA, "page means launch: %s", cudaGetErrorString(ce));
    return VPP_OK;
}

size_t vpp_block_select_workspace_size(const vpp_block_select_args* a) {
    g_err[0] = 0;
    SelectPlan s{};
    return select_plan(a, &s) == VPP_OK ? s.total : 0;
}

vpp_status vpp_block_select(const vpp_block_select_args* a, vpp_stream_t stream_) {
    g_err[0] = 0;
    SelectPlan s{};
    vpp_status st = select_plan(a, &s);
    if (st != VPP_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (a->total_q == 0 || a->num_reqs == 0) return zero_status(a->status, stream);
    st = check_paged(a->block_table, a->block_size, a->max_blocks_per_req, a->num_blocks);
    if (st != VPP_OK) return st;
    if (!a->q || !a->k_means || !a->prefix_len || !a->chunk_len || !a->indices)
        return fail(VPP_ERR_INVALID_ARG, "q, k_means, prefix_len, chunk_len and indices must be non-null");
    if (mis16(a->q) || mis16(a->k_means)) return fail(VPP_ERR_INVALID_ARG, "q and k_means must be 16-byte aligned");
    if (!a->workspace || a->workspace_bytes < s.total) return fail(VPP_ERR_WORKSPACE, "workspace: need %zu bytes, got %zu", s.total, a->workspace_bytes);
    if (reinterpret_cast<uintptr_t>(a->workspace) & 255u) return fail(VPP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    uint8_t* ws = static_cast<uint8_t*>(a->workspace);
    vpp::SelectParams p{};
    p.q = static_cast<const uint8_t*>(a->q);
    p.means = static_cast<const uint8_t*>(a->k_means);
    p.block_table = a->block_table;
    p.prefix_len = a->prefix_len;
    p.chunk_len = a->chunk_len;
    p.num_reqs = a->num_reqs;
    p.max_blocks_per_req = a->max_blocks_per_req;
    p.block_shift = ilog2(a->block_size);
    p.num_blocks = a->num_blocks;
    // the runs go as far as max_seq_len has pages, and the table as max_blocks_per_req
    p.capacity = paged_capacity(a->max_blocks_per_req, a->block_size);
    if (p.capacity > a->max_seq_len) p.capacity = a->max_seq_len;
    p.total_q = a->total_q;
    p.num_q_heads = a->num_q_heads;
    p.num_kv_heads = a->num_kv_heads;
    p.topk = a->topk;
    p.num_first = a->num_first;
    p.num_last = a->num_last;
    p.run_pages = s.run_pages;
    p.runs = s.runs;
    p.group_pages = s.group_pages;
    p.item_tokens = s.item_tokens;
    p.cap = s.cap;
    p.found = reinterpret_cast<vpp::SelectCandidate*>(ws + s.found);
    p.counts = reinterpret_cast<int32_t*>(ws + s.counts);
    p.bounds = reinterpret_cast<float*>(ws + s.bounds);
    p.maxima = reinterpret_cast<float*>(ws + s.maxima);
    p.bad = reinterpret_cast<int32_t*>(ws + s.bad);
    p.many_items = s.many_items;
    p.items = s.many_items + s.few_items;
    p.indices = a->indices;
    p.status = a->status;
    const size_t lens = sizeof(int32_t) * (static_cast<size_t>(a->num_reqs) + 1);
    const size_t smem_many = vpp::kSelectSmem + 4 * static_cast<size_t>(s.run_pages), smem_pick = vpp::kPickSmem + lens;
    const size_t smem_few = 4 * static_cast<size_t>(s.run_pages) + lens;
    cudaError_t ce = cudaSuccess;
    if (s.many_items > 0) ce = allow_smem(vpp::block_filter_kernel, vpp::kSelectSmem + 4 * vpp::kSelectMaxRun);
    if (ce == cudaSuccess && s.few_items > 0) ce = allow_smem(vpp::block_few_kernel, 4 * vpp::kSelectMaxRun + kLengthsMaxBytes);
    if (ce == cudaSuccess) ce = allow_smem(vpp::block_pick_kernel, vpp::kPickSmem + kLengthsMaxBytes);
    if (ce != cudaSuccess) return fail(VPP_ERR_CUDA, "page selection attributes: %s", cudaGetErrorString(ce));
    for (int64_t row0 = 0; row0 < a->total_q; row0 += s.slab) {
        p.row0 = static_cast<int32_t>(row0);
        p.row1 = static_cast<int32_t>(row0 + s.slab < a->total_q ? row0 + s.slab : a->total_q);
        if (s.many_items > 0) ce = launch(vpp::block_filter_kernel, static_cast<unsigned>(s.many_items), vpp::kSelectThreads + 128, smem_many, stream, p);
        if (ce == cudaSuccess && s.few_items > 0)
            ce = launch(vpp::block_few_kernel, static_cast<unsigned>(s.few_items), vpp::kFewThreads, smem_few, stream, p, s.many_items == 0 ? 1 : 0);
        if (ce != cudaSuccess) return fail(VPP_ERR_CUDA, "page scores launch: %s", cudaGetErrorString(ce));
        const long long rows = static_cast<long long>(p.row1 - p.row0) * a->num_kv_heads, warps = vpp::kPickThreads / 32;
        long long blocks = (rows + warps - 1) / warps;
        const long long cap = 3ll * sm_count_or_default();          // (those that fit at a time; 8: 3 us more of 8192 tokens, the last wave half empty)
        if (blocks > cap) blocks = cap;
        const int work_blocks = static_cast<int>(blocks);
        ce = launch(vpp::block_pick_kernel, static_cast<unsigned>(work_blocks + (a->status ? 1 : 0)), vpp::kPickThreads, smem_pick, stream, p, work_blocks);
        if (ce != cudaSuccess) return fail(VPP_ERR_CUDA, "page selection launch: %s", cudaGetErrorString(ce));
    }
    return VPP_OK;
}

size_t vpp_block_attn_workspace_size(const vpp_chunk_attn_args* a, int32_t topk) {
    g_err[0] = 0;
    BlockPlan b{};
    return block_plan(a, topk, &b) == VPP_OK ? b.total : 0;
}

vpp_status vpp_block_attn_fwd(const vpp_chunk_attn_args* a, const int32_t* block_indices, int32_t topk, vpp_stream_t stream_) {
    g_err[0] = 0;
    BlockPlan b{};
    vpp_status st = block_plan(a, topk, &b);
    if (st != VPP_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    g_launches = 0;
    if (a->total_q == 0 || a->num_reqs == 0) return zero_status(a->status, stream);
    st = check_paged(a->block_table, a->block_size, a->max_blocks_per_req, a->num_blocks);
    if (st != VPP_OK) return st;
    if (!a->q || !a->out || !a->k_cache || !a->v_cache || !block_indices || !a->prefix_len || !a->chunk_len)
        return fail(VPP_ERR_INVALID_ARG, "q, k_cache, v_cache, out, block_indices, prefix_len and chunk_len must be non-null");
    if (mis16(a->q) || mis16(a->out) || mis16(a->k_cache) || mis16(a->v_cache))
        return fail(VPP_ERR_INVALID_ARG, "q, out, k_cache and v_cache must be 16-byte aligned");
    const int64_t strides[6] = {a->k_block_stride, a->k_token_stride, a->k_head_stride, a->v_block_stride, a->v_token_stride, a->v_head_stride};
    for (int i = 0; i < 6; ++i)
        if (strides[i] <= 0 || strides[i] % 8 != 0) return fail(VPP_ERR_INVALID_ARG, "cache strides must be positive multiples of 8 elements");
    if (!a->workspace || a->workspace_bytes < b.total) return fail(VPP_ERR_WORKSPACE, "workspace: need %zu bytes, got %zu", b.total, a->workspace_bytes);
    if (reinterpret_cast<uintptr_t>(a->workspace) & 255u) return fail(VPP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    uint8_t* ws = static_cast<uint8_t*>(a->workspace);

    CUtensorMap tm_q, tm_q1, tm_k, tm_v, tm_kx, tm_vx;
    vpp::BlkParams p{};
    {
        const uint64_t dq[3] = {128, static_cast<uint64_t>(a->num_q_heads), static_cast<uint64_t>(a->total_q)};
        const uint64_t sq[2] = {256, 256ull * a->num_q_heads};
        const uint32_t bq[3] = {64, static_cast<uint32_t>(b.group), static_cast<uint32_t>(b.tile_tokens)}, b1[3] = {64, static_cast<uint32_t>(b.group), 1};
        if (!make_tmap(&tm_q, a->q, 3, dq, sq, bq) || !make_tmap(&tm_q1, a->q, 3, dq, sq, b1)) return fail(VPP_ERR_CUDA, "cuTensorMapEncodeTiled(q) failed");
        int32_t k_from = INT32_MAX, v_from = INT32_MAX;        // (0: the other map cannot express the strides)
        if (!make_kv_maps(a->k_cache, a->k_block_stride, a->k_token_stride, a->k_head_stride, a->block_size, a->num_blocks, a->num_kv_heads, a->block_size,
                          &tm_k, &tm_kx, &p.k_block_units, &p.k_head_units, &p.k_end, &k_from) ||
            !make_kv_maps(a->v_cache, a->v_block_stride, a->v_token_stride, a->v_head_stride, a->block_size, a->num_blocks, a->num_kv_heads, a->block_size,
                          &tm_v, &tm_vx, &p.v_block_units, &p.v_head_units, &p.v_end, &v_from))
            return fail(VPP_ERR_CUDA, "cuTensorMapEncodeTiled(k/v) failed");
        p.k_exact = k_from == 0;
        p.v_exact = v_from == 0;
    }
    vpp::BlkListParams lp{};
    lp.indices = block_indices;
    lp.block_table = a->block_table;
    lp.prefix_len = a->prefix_len;
    lp.chunk_len = a->chunk_len;
    lp.num_reqs = a->num_reqs;
    lp.max_blocks_per_req = a->max_blocks_per_req;
    lp.block_shift = ilog2(a->block_size);
    lp.num_blocks = a->num_blocks;
    lp.capacity = paged_capacity(a->max_blocks_per_req, a->block_size);
    if (lp.capacity > a->max_seq_len) lp.capacity = a->max_seq_len;
    lp.total_q = a->total_q;
    lp.num_kv_heads = a->num_kv_heads;
    lp.topk = topk;
    lp.tile_tokens = b.tile_tokens;
    lp.words = b.words;
    lp.max_tiles = b.max_tiles;
    lp.max_pages = b.max_pages;
    lp.header = reinterpret_cast<vpp::WorkHeader*>(ws);
    lp.items = reinterpret_cast<vpp::BlkItem*>(ws + b.items);
    lp.pages = reinterpret_cast<int32_t*>(ws + b.pages);
    lp.masks = reinterpret_cast<uint2*>(ws + b.masks);
    lp.status = a->status;
    const int context = (a->max_seq_len + a->block_size - 1) / a->block_size, most = vpp::kBlkWindow / b.words;
    lp.window = context < 1 ? 1 : context < most ? context : most;
    const size_t lens = sizeof(int32_t) * (2 * (static_cast<size_t>(a->num_reqs) + 1) + static_cast<size_t>(lp.window) * (b.words + 1));
    // (a window's masks and pages: most where a page's mask is one word)
    cudaError_t ce = allow_smem(vpp::block_lists_kernel, 2 * kLengthsMaxBytes + 2 * 4 * vpp::kBlkWindow);
    if (ce == cudaSuccess) ce = allow_smem(vpp::attn_blk_kernel, vpp::kBlkSmem);
    if (ce != cudaSuccess) return fail(VPP_ERR_CUDA, "block-sparse attention attributes: %s", cudaGetErrorString(ce));
    const unsigned tiles = static_cast<unsigned>(b.max_tiles) * a->num_kv_heads;
    ce = launch(vpp::block_lists_kernel, tiles, vpp::kBlkListThreads, lens, stream, lp);
    if (ce != cudaSuccess) return fail(VPP_ERR_CUDA, "page lists launch: %s", cudaGetErrorString(ce));
    ++g_launches;

    p.header_ro = p.header = lp.header;
    p.items = lp.items;
    p.pages = lp.pages;
    p.masks = lp.masks;
    p.max_tiles = b.max_tiles;
    p.max_pages = b.max_pages;
    p.words = b.words;
    p.block_shift = lp.block_shift;
    p.num_blocks = a->num_blocks;
    p.num_q_heads = a->num_q_heads;
    p.num_kv_heads = a->num_kv_heads;
    p.group = b.group;
    p.total_q = a->total_q;
    p.tile_tokens = b.tile_tokens;
    p.splits = b.splits;
    p.box_rows = a->block_size;
    p.scale_log2e = a->softmax_scale * 1.4426950408889634f;
    p.out = static_cast<uint8_t*>(a->out);
    p.lse = a->lse;
    p.o_parts = reinterpret_cast<float*>(ws + b.o_parts);
    p.lse_parts = reinterpret_cast<float*>(ws + b.lse_parts);
    p.status = a->status;
    const long long work = static_cast<long long>(tiles) * b.splits, sms = sm_count_or_default();
    ce = launch(vpp::attn_blk_kernel, static_cast<unsigned>(work < sms ? work : sms), vpp::kWsThreads, vpp::kBlkSmem, stream, tm_q, tm_q1,
                p.k_exact ? tm_kx : tm_k, p.v_exact ? tm_vx : tm_v, p);
    if (ce != cudaSuccess) return fail(VPP_ERR_CUDA, "block-sparse attention launch: %s", cudaGetErrorString(ce));
    ++g_launches;
    if (b.splits > 1) {
        ce = launch_merge(p.o_parts, p.lse_parts, b.splits, a->total_q, a->num_q_heads, 128, lp.header, a->out, a->lse, stream);
        if (ce != cudaSuccess) return fail(VPP_ERR_CUDA, "merge launch: %s", cudaGetErrorString(ce));
        ++g_launches;
    }
    return VPP_OK;
}

}  // extern "C"
