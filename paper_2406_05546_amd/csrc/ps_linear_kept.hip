// The products of ps_linear.h for a forward pass that keeps its pre-activations in 8 bits.  Bound by the products; the encoding adds to the tiles' last
// steps and takes from their stores (bf16, 8192 rows 2048 -> 8192 with GELU: 270-288 us, 256-276 with the pre-activations in bf16).
#include "ps_linear.h"

void ps::launch_linear_forward_kept(const Product& p, int dtype, bool direct, int tile, hipStream_t s)
{
    start_linear_typed<true, true, RAGGED_R, true>(p, dtype, direct, tile, s);
}
