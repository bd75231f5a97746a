// Shared by the operators on tokens (include/ps_tokens.h): checks of their arguments.
#pragma once
#include "../../include/ps_tokens.h"

namespace ps {

ps_status check_tokens(const char* call, const ps_tokens* tokens, int64_t rows, bool needed);
ps_status check_rows(const char* call, const char* name, int dtype, const ps_matrix* m, int64_t rows, int64_t cols, int64_t matrices);
ps_status tokens_launched(const char* call);

}  // namespace ps
