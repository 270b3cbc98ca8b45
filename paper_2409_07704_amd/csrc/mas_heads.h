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

// Outputs of more bytes than this are stored around the caches: what is used next
// would find only its end there.  Writing 168 MB of queries and keys took 8 of 219 us
// less of a training pass, 350 MB of the loss's gradients 9 of 147 us less.
constexpr double kPastBytes = 64 << 20;

}  // namespace mas
