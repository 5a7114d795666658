#include "attend.h"

namespace ds {

hipError_t decode_attend_bf16(const DecodeArgs &a, hipStream_t s) { return attend<Bf16, false>(a, s); }

}  // namespace ds
