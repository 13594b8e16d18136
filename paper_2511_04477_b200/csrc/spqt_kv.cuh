// What the kernels over the 8-bit cache share: argument checks, the layout of their workspace, access to the table.
// Included after spqt_common.cuh and spqt_gemv_device.cuh.
#pragma once

#include <algorithm>

namespace spqt {

constexpr int kCacheRefused = 3;        // status word: a length, a count or a block number outside its range
constexpr int kMaxStreams = 16384, kMaxTableWidth = 16384;

inline bool kv_dim_supported(int d) { return d == 64 || d == 96 || d == 128 || d == 256; }

inline spqt_status check_cache(const spqt_kv_cache* c)
{
    if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail || !c->table || !c->length)
        return SPQT_ERR_INVALID_ARG;
    if (c->batch <= 0 || c->kv_heads <= 0 || c->blocks <= 0 || c->table_width <= 0) return SPQT_ERR_INVALID_ARG;
    if (c->format != SPQT_KV_INT8 && c->format != SPQT_KV_E4M3) return SPQT_ERR_UNSUPPORTED;
    const int bt = c->block_tokens;
    if (!kv_dim_supported(c->head_dim) || (bt != 16 && bt != 32 && bt != 64 && bt != 128)) return SPQT_ERR_UNSUPPORTED;
    if ((long long)c->batch * c->kv_heads > kMaxStreams || c->table_width > kMaxTableWidth) return SPQT_ERR_UNSUPPORTED;
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_tail, 16) || !aligned(c->v_tail, 16) || !aligned(c->weight, 16) ||
        !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4) || !aligned(c->table, 4) || !aligned(c->length, 4))
        return SPQT_ERR_ALIGNMENT;
    return SPQT_OK;
}

// Workspace of the cache's calls: the header with the status word, which all of them need; the attention's counts of parts, zero
// between calls; behind them what a call leaves for its own CTAs and its second kernel.
constexpr size_t kKvHeader = kSlotsOffset, kKvScratch = kKvHeader + (size_t)kMaxStreams * 4;
inline size_t kv_lengths_bytes(const spqt_kv_cache& c) { return ((size_t)c.batch * c.kv_heads * 4 + 255) / 256 * 256; }

inline spqt_status check_kv_workspace(const void* workspace, size_t bytes, size_t need)
{
    if (!workspace) return SPQT_ERR_INVALID_ARG;
    if (!aligned(workspace, 16)) return SPQT_ERR_ALIGNMENT;
    return bytes < need ? SPQT_ERR_WORKSPACE : SPQT_OK;
}

// Rows of `row` values that are written, along some strides (of extents above one): whether each stride, in the order of their size,
// has room for all that the smaller ones reach, so that no two rows share a place.
struct RowStride {
    long long stride;
    int extent;
};
template <int N>
inline bool rows_apart(long long row, RowStride (&s)[N])
{
    std::sort(s, s + N, [](const RowStride& a, const RowStride& b) { return a.stride < b.stride; });
    __int128 reach = row;
    for (const RowStride& d : s) {
        if (d.extent <= 1) continue;
        if (d.stride < reach) return false;
        reach += (__int128)d.stride * (d.extent - 1);
    }
    return true;
}

__device__ __forceinline__ void refuse(int* status) { *status = kCacheRefused; }   // (all writers write the same)

// The length of a stream, 0 where it is none that the table's row can hold.
__device__ __forceinline__ int length_or_none(int n, const spqt_kv_cache& c, int* status)
{
    if (n >= 0 && n <= c.table_width * c.block_tokens) return n;
    refuse(status);
    return 0;
}

// One launch that may begin while the previous kernel of the stream drains.
template <class... P, class... A>
cudaError_t launch_overlapping(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = g_no_pdl ? 0 : 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
    if (err == cudaSuccess) count_launch();
    return err;
}

inline spqt_status launched(cudaError_t err)
{
    if (err == cudaSuccess) return SPQT_OK;
    (void)cudaGetLastError();
    return SPQT_ERR_CUDA;
}

}  // namespace spqt
