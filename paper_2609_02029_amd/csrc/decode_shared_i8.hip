// decode_shared_i8.hip -- decode attention over shared pages of int8 caches (all
// head dims).
#include "decode_shared.h"

namespace hwkv {
template hipError_t launch_decode_shared_fmt<HWKV_KV_I8>(int, const SharedArgs &, hipStream_t);
}  // namespace hwkv
