// decode_shared_fp8.hip -- decode attention over shared pages of fp8-E4M3 caches (all
// head dims).
#include "decode_shared.h"

namespace hwkv {
template hipError_t launch_decode_shared_fmt<HWKV_KV_FP8_E4M3>(int, const SharedArgs &, hipStream_t);
}  // namespace hwkv
