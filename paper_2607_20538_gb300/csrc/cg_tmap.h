// cg_tmap.h -- host-side creation of TMA tensor maps (cuTensorMapEncodeTiled through the
// runtime's driver entry point, so the library links only against cudart).
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <mutex>

namespace cg {

template <class F>
inline F driver_fn(const char* name) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q{};
    const bool found = cudaGetDriverEntryPointByVersion(name, &p, 12000, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess;
    return found ? reinterpret_cast<F>(p) : nullptr;
}

// The tensor map encoder, or null. It is a driver call and wants a current context, which a host thread gets
// with its first runtime call that needs one: a thread whose first call is this library's has none yet, and
// gets its device's here. A context that is current stays so.
inline PFN_cuTensorMapEncodeTiled_v12000 tmap_encode_fn() {
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    static PFN_cuCtxGetCurrent_v4000 current = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        fn = driver_fn<PFN_cuTensorMapEncodeTiled_v12000>("cuTensorMapEncodeTiled");
        current = driver_fn<PFN_cuCtxGetCurrent_v4000>("cuCtxGetCurrent");
    });
    CUcontext ctx = nullptr;
    int dev = 0;
    if (current && current(&ctx) == CUDA_SUCCESS && !ctx && cudaGetDevice(&dev) == cudaSuccess) cudaSetDevice(dev);
    return fn;
}

// 2-D bf16 tensor [rows][cols] (row pitch `pitch_bytes`), loaded in boxes of
// box_rows x 64 columns (128 B) with the 128-byte swizzle; out-of-range rows read as 0.
inline bool make_tmap_bf16_sw128(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols,
                                 uint64_t pitch_bytes, uint32_t box_rows) {
    auto fn = tmap_encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {pitch_bytes};
    cuuint32_t box[2] = {64, box_rows};
    cuuint32_t estr[2] = {1, 1};
    CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS;
}

}  // namespace cg
