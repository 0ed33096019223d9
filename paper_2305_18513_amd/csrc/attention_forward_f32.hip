// Attention forward for fp32 operands (attention_forward.hpp).
#include "attention_forward.hpp"

namespace slimfit {
void attention_forward_f32(const Attention &a, void *out, float *stats, float *parts, int splits, hipStream_t st)
{
    attention_forward_of<float>(a, out, stats, parts, splits, st);
}
}  // namespace slimfit
