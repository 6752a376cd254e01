// Weight gradients: the kernels for output gradients in fp16.
#include "eb_weight_gradient.h"

namespace eb_gradient {

Choice choice_f16(int32_t x_type, bool exact, bool direct, bool narrow) { return choice_of<_Float16>(x_type, exact, direct, narrow); }

} // namespace eb_gradient
