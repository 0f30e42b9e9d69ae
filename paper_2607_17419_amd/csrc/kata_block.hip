// kata_block.hip -- the operators of a mixer's layer in 8 bits: residual norm, quantiser, product
// of e4m3 operands with block scales, and the gated linear recurrence.  Host checks:
// kata_block_api.hpp.
#include "kata_addnorm.hpp"
#include "kata_f8_gemm.hpp"
#include "kata_recur.hpp"
