// decode_shared_f16.hip -- decode attention over shared pages of binary16 caches (all
// head dims).
#include "decode_shared.h"

namespace hwkv {
template hipError_t launch_decode_shared_fmt<HWKV_KV_F16>(int, const SharedArgs &, hipStream_t);
}  // namespace hwkv
