// Attention with capped scores, a bias by distance or a prefix, gradients.
#include "attention_backward.h"

namespace fuse {
namespace backward {
FUSE_BACKWARD(, _Float16, 1) FUSE_BACKWARD(, _Float16, 3) FUSE_BACKWARD(, _Float16, 5) FUSE_BACKWARD(, _Float16, 7)
}  // namespace backward
}  // namespace fuse
