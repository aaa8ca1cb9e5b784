// Host helpers of the entry points beside the soft top-k's own: sizes, error returns, dispatch by type, tensor maps, the device's SMs.
#pragma once
#include <cuda.h>

#include "host.h"

namespace lapsum {

inline size_t align_up(size_t x, size_t a = 256) { return (x + a - 1) / a * a; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

#define CU_OK(x)                                      \
    do {                                              \
        const cudaError_t e__ = (x);                  \
        if (e__ != cudaSuccess) return cuda_fail(e__); \
    } while (0)
#define RUN(x)                    \
    do {                          \
        const int rc__ = (x);     \
        if (rc__ != 0) return rc__; \
    } while (0)
#define BY_TYPE(fn, dtype, ...)                                  \
    ((dtype) == LAPSUM_IO_F32   ? fn<float>(__VA_ARGS__)          \
     : (dtype) == LAPSUM_IO_F16 ? fn<__half>(__VA_ARGS__)         \
                                : fn<__nv_bfloat16>(__VA_ARGS__))

using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);
inline EncodeFn encode_fn()
{
    static const EncodeFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}

// dims from the innermost; strides in elements for dimensions 1..; 128-byte swizzle; reads beyond the tensor give zeros
inline int tensor_map(CUtensorMap *map, int dtype, const void *base, int rank, const int64_t *dims, const int64_t *strides, const int *box)
{
    const EncodeFn fn = encode_fn();
    if (!fn) return cuda_fail(cudaErrorNotSupported);
    cuuint64_t d[3], s[2];
    cuuint32_t b[3], one[3] = {1, 1, 1};
    for (int i = 0; i < rank; ++i) d[i] = (cuuint64_t)dims[i], b[i] = (cuuint32_t)box[i];
    for (int i = 0; i + 1 < rank; ++i) s[i] = (cuuint64_t)strides[i] * 2;
    const CUresult r = fn(map, dtype == LAPSUM_IO_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank,
                          const_cast<void *>(base), d, s, b, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? LAPSUM_OK : cuda_fail(cudaErrorInvalidValue);
}
inline int map_2d(CUtensorMap *m, int dtype, const void *base, int64_t cols, int64_t rows, int64_t stride, int box_rows)
{
    const int64_t d[2] = {cols, rows}, s[1] = {stride};
    const int b[2] = {64, box_rows};
    return tensor_map(m, dtype, base, 2, d, s, b);
}
inline int sm_count(int *n)
{
    static thread_local int dev_known = -1, sms = 0;
    int dev = 0;
    CU_OK(cudaGetDevice(&dev));
    if (dev != dev_known) {
        CU_OK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        dev_known = dev;
    }
    *n = sms;
    return LAPSUM_OK;
}

}  // namespace lapsum
