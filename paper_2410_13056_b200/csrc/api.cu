// Host-only helpers of the C ABI, and the tensor maps.
#include "common.cuh"
#include "tc5.cuh"

namespace cmpq {

bool make_byte_map(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<Encode>(f);
    }();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace cmpq

using namespace cmpq;

extern "C" size_t cmpq_workspace_bytes(cmpq_op op, int64_t d_in, int64_t d_out) {
    if (d_in < 1 || d_in > CMPQ_MAX_D_IN) return 0;
    switch (op) {
        case CMPQ_OP_COLLECT_STATS: return stats_ws_bytes(d_in);
        case CMPQ_OP_ALLOCATE_BITS: return alloc_ws_bytes(d_in);
        case CMPQ_OP_EXTRACT_OUTLIERS:
            if (d_out < 1 || d_out > CMPQ_MAX_D_OUT) return 0;
            return outliers_ws_bytes(d_in, d_out);
        case CMPQ_OP_QUANTIZE_LAYER:
            if (d_out < 1 || d_out > CMPQ_MAX_D_OUT) return 0;
            return quantize_ws_bytes(d_in, d_out);
        case CMPQ_OP_PACK:
            if (d_out < 1 || d_out > CMPQ_MAX_D_OUT) return 0;
            return pack_ws_bytes(d_in, d_out);
        case CMPQ_OP_PROTECT_AND_QUANTIZE:
            if (d_out < 1 || d_out > CMPQ_MAX_D_OUT) return 0;
            return protect_quantize_ws_bytes(d_in, d_out);
        case CMPQ_OP_OUTLIERS_BY_COLUMN:
            if (d_out < 1 || d_out > CMPQ_MAX_D_OUT) return 0;
            return by_column_ws_bytes(d_out);
        case CMPQ_OP_MATVEC:
            if (d_out < 1 || d_out > CMPQ_MAX_D_OUT) return 0;
            return matvec_ws_bytes(d_in, d_out);
        case CMPQ_OP_QUANTIZE_LAYER_PACKED:
            if (d_out < 1 || d_out > CMPQ_MAX_D_OUT) return 0;
            return quantize_packed_ws_bytes(d_in, d_out);
        case CMPQ_OP_PROTECT_QUANTIZE_PACK:
            if (d_out < 1 || d_out > CMPQ_MAX_D_OUT) return 0;
            return protect_quantize_pack_ws_bytes(d_in, d_out);
    }
    return 0;
}

extern "C" const char* cmpq_status_string(cmpq_status s) {
    switch (s) {
        case CMPQ_OK: return "ok";
        case CMPQ_ERR_INVALID_ARG: return "invalid argument";
        case CMPQ_ERR_UNSUPPORTED: return "unsupported argument combination";
        case CMPQ_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case CMPQ_ERR_CUDA: return "CUDA runtime error";
        case CMPQ_ERR_INTERNAL: return "internal error";
        case CMPQ_ERR_NONFINITE: return "an input held a NaN or an infinity";
    }
    return "unknown status";
}
