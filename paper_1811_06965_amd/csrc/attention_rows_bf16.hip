// attention_rows_bf16.hip -- attention_rows_kernels.hpp for bf16.
#include "attention_rows_kernels.hpp"

namespace gp {
template gp_status attend_forward_as<bf16>(const AttendArgs&, hipStream_t);
template gp_status attend_backward_as<bf16>(const AttendArgs&, bool, const Shape&, const Shape&, hipStream_t);
} // namespace gp
