// What a network's step uses of layer norm (layer_norm.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "layer_norm_args.h"

namespace ngsgd {

// fp32 rows, weight and bias; N > 0, and all arguments are the network's own.
int layernorm_forward_f32(const LayerNormForward& a, hipStream_t s);
// dy may be the sum of n_slabs partial products; dx may be the first of them.  (`groups` is filled in.)
int layernorm_backward_f32(LayerNormBackward a, hipStream_t s);
size_t layernorm_part_floats(int64_t max_rows, int D);

}  // namespace ngsgd
