#include "attend.h"

namespace ds {

hipError_t decode_attend_f16_e4m3(const DecodeArgs &a, hipStream_t s) { return attend<F16, true>(a, s); }

}  // namespace ds
