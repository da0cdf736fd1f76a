// The residual connection's gradients, the norm's and the block's in float32.
#include "moc_residual_backward.h"

ResidualShape moc_residual_backward_f32(int stream, int block, int mode, bool own, int64_t cols) { return backward_shape_of<MOC_F32>(stream, block, mode, own, cols); }
