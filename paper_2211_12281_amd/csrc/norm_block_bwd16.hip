// Backward rows of the norms around a block, residual stream in bf16 (norm_block_bwd.hpp).
#include "norm_block_bwd.hpp"

int kge_norm::rows_bwd16(const BwdArgs &a, bool b16, hipStream_t st) { return launch_bwd<true>(a, b16, st); }
