// Attention forward for fp32 operands (attention_forward.hpp).
#include "attention_forward.hpp"

namespace slimfit {
void attention_forward_f32(const Attention &a, void *out, float *stats, hipStream_t st) { attention_forward_of<float>(a, out, stats, st); }
}  // namespace slimfit
