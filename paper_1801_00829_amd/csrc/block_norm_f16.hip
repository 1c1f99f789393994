// The norms' kernels of one type.
#include "block_norm.h"

namespace fuse {
FUSE_NORM_TYPE(, _Float16)
}  // namespace fuse
