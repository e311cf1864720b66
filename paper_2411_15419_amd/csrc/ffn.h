// The FFN's weight-gradient product, for other gradients of the same form (defined in
// ffn.hip).
#pragma once

#include "luffy_common.h"

namespace luffy {

// out[p] = P_p^T Q_p, [parts, M, N] float32, over the rows rows[p] .. rows[p + 1] - 1
// of P [*, M] and Q [*, N] (bf16, row-major).  M and N multiples of 64, at most 64
// parts, a part's rows of either matrix below 4 GiB - 64 KiB.
void row_product_enqueue(const char* name, const uint16_t* P, const uint16_t* Q, const int32_t* rows, int parts, int M,
                         int N, float* out, hipStream_t s);

}  // namespace luffy
