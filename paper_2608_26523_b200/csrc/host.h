// What the entry points of api.cu and block_sparse.cu share on the host: errors, launches, tensor maps, the merge of partial results.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/vpp.h"

namespace vpp {
struct WorkHeader;
namespace host {

extern thread_local char g_err[512];      // vpp_last_error
extern thread_local int32_t g_launches;   // vpp_last_launch_count

vpp_status fail(vpp_status s, const char* fmt, ...);
vpp_status zero_status(int32_t* status, cudaStream_t stream);
int sm_count_or_default();

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool is_pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
inline int ilog2(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

// bf16 tensor, innermost dimension contiguous, 128-byte swizzle, zero fill out of bounds (encoded maps are cached).
bool make_tmap(CUtensorMap* m, const void* base, int rank, const uint64_t* dims, const uint64_t* strides_bytes, const uint32_t* box);
bool make_kv_maps(const void* base, int64_t block_stride, int64_t token_stride, int64_t head_stride, int B, int n_blocks, int heads, int box_rows,
                  CUtensorMap* tm, CUtensorMap* tm_exact, int32_t* block_units, int32_t* head_units, int32_t* end, int32_t* exact_from);

// Every row's `splits` partial results joined (merge.cuh); nothing where the header has an error.
cudaError_t launch_merge(const float* o_parts, const float* lse_parts, int splits, int total_q, int num_q_heads, int head_dim_v,
                         const WorkHeader* header, void* out, float* lse, cudaStream_t stream);

// Launch with programmatic stream serialization: the kernel may start (and set itself up) while its predecessor in the
// stream still runs, and waits for it (griddepcontrol.wait) before it touches memory.
template <typename... Params, typename... Args>
cudaError_t launch(void (*kernel)(Params...), unsigned blocks, unsigned threads, size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

}  // namespace host
}  // namespace vpp
