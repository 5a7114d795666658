#include "attend.h"

namespace ds {

hipError_t decode_attend_bf16_e4m3(const DecodeArgs &a, hipStream_t s) { return attend<Bf16, true>(a, s); }

}  // namespace ds
