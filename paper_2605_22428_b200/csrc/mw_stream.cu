// Host side of the engine in mw_stream.cuh: tensor maps, shared memory.
#include "mw_stream.cuh"

namespace mw_stream {

// The driver's encoder, fetched at run time so that the library needs no link against the driver.
static PFN_cuTensorMapEncodeTiled_v12000 encoder()
{
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return (PFN_cuTensorMapEncodeTiled_v12000)p;
    }();
    return fn;
}

bool encode_map(CUtensorMap *map, const void *base, int rank, const uint64_t *dims, const uint64_t *strides, const uint32_t *box)
{
    const PFN_cuTensorMapEncodeTiled_v12000 fn = encoder();
    if (!fn) return false;
    cuuint64_t d[5], s[4];
    cuuint32_t b[5], e[5];
    for (int i = 0; i < rank; ++i) { d[i] = dims[i]; b[i] = box[i]; e[i] = 1; if (i + 1 < rank) s[i] = strides[i]; }
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void *>(base), d, s, b, e, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

void split_memory(Common *c, size_t bytes, size_t ring)
{
    const size_t room = bytes - 1024 - sizeof(Shared), slot = (size_t)kWeightBytes * c->steps;   // 1024: alignment
    size_t slots = (room - ring) / slot;
    if (slots > (size_t)kSlots) slots = kSlots;
    c->slots = (int)slots;
    c->ring_bytes = (uint32_t)((room - slots * slot) & ~(size_t)1023);
}

}  // namespace mw_stream
