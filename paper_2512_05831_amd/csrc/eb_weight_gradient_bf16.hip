// Weight gradients: the kernels for output gradients in bfloat16.
#include "eb_weight_gradient.h"

namespace eb_gradient {

Choice choice_bf16(int32_t x_type, bool exact, bool direct, bool narrow) { return choice_of<Bf16>(x_type, exact, direct, narrow); }

} // namespace eb_gradient
