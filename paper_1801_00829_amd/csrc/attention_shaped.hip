// Attention with capped scores, a bias by distance or a prefix, forward.
#include "attention_forward.h"

namespace fuse {
namespace forward {
#define FUSE_SHAPES(T) FUSE_FORWARD(, T, 1) FUSE_FORWARD(, T, 3) FUSE_FORWARD(, T, 5) FUSE_FORWARD(, T, 7)
FUSE_SHAPES(__bf16)
FUSE_SHAPES(_Float16)
}  // namespace forward
}  // namespace fuse
