// Host side of the tensor-core products: tensor maps, the failure word, the number of SMs.
#include <mutex>

#include <cudaTypedefs.h>

#include "tile_product.cuh"

namespace cast {
namespace product {

namespace {

PFN_cuTensorMapEncodeTiled_v12000 encode_entry()
{
    static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    }();
    return fn;
}

}  // namespace

int make_map(CUtensorMap* map, const void* base, int elem_bytes, uint64_t inner, uint64_t rows, uint64_t batch, uint64_t ld,
             uint64_t batch_stride, uint32_t box_inner, uint32_t box_rows, bool swizzle)
{
    const auto encode = encode_entry();
    if (!encode) return cuda_failed(cudaErrorNotSupported);
    // the two outer strides only matter where there is more than one row or matrix, but must be valid all the same
    const cuuint64_t dims[3] = {inner, rows, batch};
    const cuuint64_t strides[2] = {ld * (uint64_t)elem_bytes, (batch > 1 ? batch_stride : ld) * (uint64_t)elem_bytes};
    const cuuint32_t box[3] = {box_inner, box_rows, 1};
    const cuuint32_t steps[3] = {1, 1, 1};
    const CUtensorMapDataType type = elem_bytes == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
    const CUresult r = encode(map, type, 3, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? CAST_OK : cuda_failed(cudaErrorInvalidValue);
}

namespace {

// Allocated at the first use and kept until the process ends: kernels may still be reading its address.
int the_word(unsigned long long** word)
{
    static std::mutex lock;
    static unsigned long long* w = nullptr;
    std::lock_guard<std::mutex> hold(lock);
    if (!w) {
        void* p = nullptr;
        CAST_CUDA_TRY(cudaHostAlloc(&p, sizeof(unsigned long long), cudaHostAllocPortable | cudaHostAllocMapped));
        w = static_cast<unsigned long long*>(p);
        *w = 0ull;
    }
    *word = w;
    return CAST_OK;
}

}  // namespace

int fail_word(unsigned long long** word)
{
    const int rc = the_word(word);
    if (rc != CAST_OK) return rc;
    return *static_cast<volatile unsigned long long*>(*word) == 0ull ? CAST_OK : CAST_ERR_STAGING;
}

int sm_count(int* n)
{
    static std::atomic<int> known[64];      // calls may come from several threads
    int dev;
    CAST_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 64 && (*n = known[dev].load(std::memory_order_relaxed)) > 0) return CAST_OK;
    CAST_CUDA_TRY(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev));
    if (dev < 64) known[dev].store(*n, std::memory_order_relaxed);
    return CAST_OK;
}

}  // namespace product
}  // namespace cast

extern "C" int cast_product_failures(unsigned long long* count_out, int action)
{
    if (action < 0 || action > 2) return CAST_ERR_HYPER;
    unsigned long long* w;
    const int rc = cast::product::the_word(&w);
    if (rc != CAST_OK) return rc;
    volatile unsigned long long* v = w;
    if (count_out) *count_out = *v;
    if (action == 1) *v = *v + 1;
    else if (action == 2) *v = 0;
    return CAST_OK;
}
