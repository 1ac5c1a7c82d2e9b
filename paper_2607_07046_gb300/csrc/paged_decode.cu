// The single-token attention of paged_decode.cuh over pools of 16 bits.
#include "paged_decode.cuh"

namespace vt {

int64_t paged_decode_line(const PagedAttnArgs& a, int cols) { return paged_decode_line_of<PdGeom<PoolPlain<__half>, 128, 1>>(a, cols); }

cudaError_t launch_paged_decode(const PagedAttnArgs& a, int dtype, int dh, cudaStream_t st) {
    return dtype == VT_F16 ? decode_src<PoolPlain<__half>>(a, dh, st) : decode_src<PoolPlain<__nv_bfloat16>>(a, dh, st);
}
cudaError_t init_paged_decode() {
    const cudaError_t e = init_src<PoolPlain<__half>>();
    return e != cudaSuccess ? e : init_src<PoolPlain<__nv_bfloat16>>();
}

}  // namespace vt
