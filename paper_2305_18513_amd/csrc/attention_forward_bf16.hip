// Attention forward for bf16 operands (attention_forward.hpp).
#include "attention_forward.hpp"

namespace slimfit {
void attention_forward_bf16(const Attention &a, void *out, float *stats, hipStream_t st) { attention_forward_of<uint16_t>(a, out, stats, st); }
}  // namespace slimfit
