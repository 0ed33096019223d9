// Attention backward for bf16 operands (attention_backward.hpp).
#include "attention_backward.hpp"

namespace slimfit {
void attention_backward_bf16(const Attention &a, const Gradients &g, hipStream_t st) { attention_backward_of<uint16_t>(a, g, st); }
}  // namespace slimfit
