// Attention forward for bf16 operands (attention_forward.hpp).
#include "attention_forward.hpp"

namespace slimfit {
void attention_forward_bf16(const Attention &a, void *out, float *stats, float *parts, int splits, hipStream_t st)
{
    attention_forward_of<uint16_t>(a, out, stats, parts, splits, st);
}
}  // namespace slimfit
