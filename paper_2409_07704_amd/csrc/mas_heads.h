// Tensors of heads, [B, T, H, D], as the attention and the norm-and-rotation
// kernels take them.
#pragma once

#include <stdint.h>

namespace mas {

enum ElemType { kF32 = 0, kF16 = 1, kBF16 = 2 };

// Element strides of an item, a token and a head; channels are contiguous.
struct HeadView {
  char* data;
  int64_t sb, st, sh;
};

}  // namespace mas
