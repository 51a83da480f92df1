// Launcher of dropout.hip.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "philox.h"

namespace ckpt {

// y [rows, cols] = [res +] dropout(x); xf: x fp32 (else bf16), yf: y and res.
void dropout(hipStream_t s, int64_t rows, int64_t cols, bool xf, const void *x, int64_t ldx, const void *res,
             int64_t ldr, bool yf, void *y, int64_t ldy, const DropArgs &drop);

}  // namespace ckpt
