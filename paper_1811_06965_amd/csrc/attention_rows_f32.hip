// attention_rows_f32.hip -- attention_rows_kernels.hpp for f32.
#include "attention_rows_kernels.hpp"

namespace gp {
template gp_status attend_forward_as<float>(const AttendArgs&, hipStream_t);
template gp_status attend_backward_as<float>(const AttendArgs&, bool, const Shape&, const Shape&, hipStream_t);
} // namespace gp
