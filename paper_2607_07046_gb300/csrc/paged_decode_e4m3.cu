// The single-token attention of paged_decode.cuh over pools of e4m3 codes.
#include "paged_decode.cuh"

namespace vt {

cudaError_t launch_paged_decode_e4m3(const PagedAttnArgs& a, int dtype, int dh, cudaStream_t st) {
    return dtype == VT_F16 ? decode_src<PoolMx<__half, VT_MX_E4M3>>(a, dh, st) : decode_src<PoolMx<__nv_bfloat16, VT_MX_E4M3>>(a, dh, st);
}
cudaError_t init_paged_decode_e4m3() {
    const cudaError_t e = init_src<PoolMx<__half, VT_MX_E4M3>>();
    return e != cudaSuccess ? e : init_src<PoolMx<__nv_bfloat16, VT_MX_E4M3>>();
}

}  // namespace vt
