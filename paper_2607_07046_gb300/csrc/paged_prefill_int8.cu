// The tiles' kernel of paged_prefill.cu over pools of int8 codes.
#define VT_POOL_CODES
#include "paged_prefill.cu"

namespace vt {

template <class T>
using Pool = PoolMx<T, VT_MX_INT8>;
VT_PAGED_TILES(Pool, _int8)

}  // namespace vt
