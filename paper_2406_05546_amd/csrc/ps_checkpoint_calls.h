// Encoding and decoding of whole matrices (ps_checkpoint.hip), for the calls of ps_linear.hip.
#pragma once
#include "ps_linear.h"

namespace ps {

ps_status check_checkpoint(const char* call, const char* name, const ps_checkpoint* c, int64_t rows, int64_t cols);
// Rows in no group are left as they are.
void launch_checkpoint_encode(int dtype, const Groups& groups, int64_t rows, int64_t cols, const ps_matrix& x, const ps_checkpoint& to, hipStream_t s);
// Rows of cols_to >= cols elements, zeros behind.
void launch_checkpoint_decode(int dtype, int64_t rows, int64_t cols, const ps_checkpoint& from, int activation, const ps_matrix& x, int64_t cols_to, hipStream_t s);

}  // namespace ps
