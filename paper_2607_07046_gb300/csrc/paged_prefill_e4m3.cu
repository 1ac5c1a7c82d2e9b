// The tiles' kernel of paged_prefill.cu over pools of e4m3 codes.
#define VT_POOL_CODES
#include "paged_prefill.cu"

namespace vt {

template <class T>
using Pool = PoolMx<T, VT_MX_E4M3>;
VT_PAGED_TILES(Pool, _e4m3)

}  // namespace vt
