// Backward rows of the norms around a block, residual stream in fp32 (norm_block_bwd.hpp).
#include "norm_block_bwd.hpp"

int kge_norm::rows_bwd32(const BwdArgs &a, bool b16, hipStream_t st) { return launch_bwd<false>(a, b16, st); }
