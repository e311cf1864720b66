// Expert activations in float32, for results that are rounded once at the end
// (the bf16 FFN's cheaper forms, whose error hides under its hidden rows'
// rounding, are its own).
#pragma once

#include "luffy_common.h"

namespace luffy {

template <int ACT>
__device__ __forceinline__ float act_f32(float z) {
  if constexpr (ACT == LUFFY_ACT_GELU) {
    return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
  } else {
    return z / (1.0f + expf(-z));
  }
}

}  // namespace luffy
