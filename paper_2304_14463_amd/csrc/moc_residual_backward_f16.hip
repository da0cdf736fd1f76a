// The residual connection's gradients, the norm's and the block's in float16.
#include "moc_residual_backward.h"

ResidualShape moc_residual_backward_f16(int stream, int block, int mode, bool own, int64_t cols) { return backward_shape_of<MOC_F16>(stream, block, mode, own, cols); }
