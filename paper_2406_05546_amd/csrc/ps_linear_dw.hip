// The products of ps_linear.h for one kind of operands.
#include "ps_linear.h"

void ps::launch_linear_dw(const Product& p, int dtype, bool direct, int tile, hipStream_t s)
{
    start_linear_typed<false, false, RAGGED_K>(p, dtype, direct, tile, s);
}
