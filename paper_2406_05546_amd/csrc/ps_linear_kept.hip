// The products of ps_linear.h for a forward pass that keeps its pre-activations in 8 bits.
#include "ps_linear.h"

void ps::launch_linear_forward_kept(const Product& p, int dtype, bool direct, int tile, hipStream_t s)
{
    start_linear_typed<true, true, RAGGED_R, true>(p, dtype, direct, tile, s);
}
