// Attention backward for fp32 operands (attention_backward.hpp).
#include "attention_backward.hpp"

namespace slimfit {
void attention_backward_f32(const Attention &a, const Gradients &g, hipStream_t st) { attention_backward_of<float>(a, g, st); }
}  // namespace slimfit
