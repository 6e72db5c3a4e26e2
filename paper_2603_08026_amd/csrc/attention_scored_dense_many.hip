// Attention with masked and reshaped scores in bf16: over [B, L] caches, many rows (a file of its own: they compile side by side).
#include "attention_scored_kernels.h"

namespace dy {
void launch_scored_dense_many(const ScoredAttn &a, hipStream_t s) { launch_by_shape<Form::MANY, false>(a, s); }
}  // namespace dy
