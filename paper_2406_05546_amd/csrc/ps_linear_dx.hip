// The products of ps_linear.h for one kind of operands.
#include "ps_linear.h"

void ps::launch_linear_dx(const Product& p, int dtype, bool direct, int tile, hipStream_t s)
{
    start_linear_typed<true, false, RAGGED_R>(p, dtype, direct, tile, s);
}
