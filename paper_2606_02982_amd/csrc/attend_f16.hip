#include "attend.h"

namespace ds {

hipError_t decode_attend_f16(const DecodeArgs &a, hipStream_t s) { return attend<F16, false>(a, s); }

}  // namespace ds
