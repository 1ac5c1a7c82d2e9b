// The single-token attention of paged_decode.cuh over pools of int8 codes.
#include "paged_decode.cuh"

namespace vt {

cudaError_t launch_paged_decode_int8(const PagedAttnArgs& a, int dtype, int dh, cudaStream_t st) {
    return dtype == VT_F16 ? decode_src<PoolMx<__half, VT_MX_INT8>>(a, dh, st) : decode_src<PoolMx<__nv_bfloat16, VT_MX_INT8>>(a, dh, st);
}
cudaError_t init_paged_decode_int8() {
    const cudaError_t e = init_src<PoolMx<__half, VT_MX_INT8>>();
    return e != cudaSuccess ? e : init_src<PoolMx<__nv_bfloat16, VT_MX_INT8>>();
}

}  // namespace vt
