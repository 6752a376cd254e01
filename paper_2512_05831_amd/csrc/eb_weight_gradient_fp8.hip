// Weight gradients: the kernels for output gradients in 8 bits.
#include "eb_weight_gradient.h"

namespace eb_gradient {

Choice choice_fp8(int32_t x_type, bool exact, bool direct, bool narrow) { return choice_of<Fp8>(x_type, exact, direct, narrow); }

} // namespace eb_gradient
