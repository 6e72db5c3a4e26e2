// Attention with masked and reshaped scores in bf16: over pages, few rows (a file of its own: they compile side by side).
#include "attention_scored_kernels.h"

namespace dy {
void launch_scored_pages_few(const ScoredAttn &a, hipStream_t s) { launch_by_shape<Form::FEW, true>(a, s); }
}  // namespace dy
