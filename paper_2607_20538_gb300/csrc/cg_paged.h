// cg_paged.h -- internal interface between the paged-cache entry points and their kernels.
#pragma once

#include <atomic>

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/codecgauge_paged.h"
#include "cg_launch.h"

namespace cg {

// Paged attention of one layer (cg_paged_attention's arguments, with log2(page)).
struct PagedArgs {
    const uint16_t* q;
    const uint16_t* pool;
    const int32_t* table;
    const int32_t* seq_lens;
    const int32_t* cu_new;
    uint16_t* out;
    float* lse;
    int32_t* status;
    int dtype, n_pages, page, page_log2, H, d, n_req, max_pages;
    int n_tok, n_rep, max_new, window, sinks;
    float scale;
    int64_t q_tok, q_head, o_tok, o_head;
    uint64_t wait_ns;
    // A tree of drafted tokens (cg_tree_attention): the new tokens that a row sees are the bits of its
    // mask, masks[n_tok][words]; masks null: those up to its own. positions: only with a window.
    const uint32_t* masks;
    const int32_t* positions;
    int words;
    uint32_t rep_mul;     // x / n_rep = x * rep_mul >> rep_shift for 0 <= x < 2^31
    int rep_shift;
};

// Checks of cg_paged_attention's parameters; fills what of `a` they say.
int paged_attn_check(const cg_pages* p, const cg_paged_attn* h, PagedArgs* a);
// Checks of the pointers, and the launch (masks and positions are set in `a`, or null).
int paged_attn_run(PagedArgs& a, const void* q, const void* pool, const int32_t* block_table, const int32_t* seq_lens,
                   const int32_t* cu_new, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream);

// Workspace of the paged attention: bytes, and the launch (workspace of that size).
size_t paged_attn_workspace(const PagedArgs& a);
cudaError_t launch_paged_attn(const PagedArgs& a, void* workspace, cudaStream_t st);

// A kernel's dynamic shared memory limit, raised once per device.
struct SmemOptIn {
    std::atomic<uint64_t> done{0};
    cudaError_t set(const void* kernel, int bytes) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
        if (bit && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
        return e;
    }
};

// Tensor map of the pool with boxes of box_rows tokens x 64 channels.
bool paged_pool_map(CUtensorMap* map, const PagedArgs& a, uint32_t box_rows);

// Requests of at least min_rows query rows on the tcgen05 tiles.
size_t paged_chunk_workspace(int d);
// after_rows: the last launch on the stream is this call's paged_rows_kernel.
cudaError_t launch_paged_chunk(const PagedArgs& a, int min_rows, bool after_rows, void* workspace, cudaStream_t st);

}  // namespace cg
