// Launches of the windowed attention's kernels in float32 arithmetic (attention_float.cu), for attention.cu.
#pragma once

#include <type_traits>

#include "attention_rows.cuh"
#include "host.cuh"

namespace brace {

constexpr int kFloatRows = 64;   // of a CTA

cudaError_t attn_forward_float(int type, const AttnArgs& a, cudaStream_t st);
cudaError_t attn_grad_float(int type, const AttnArgs& a, cudaStream_t st);

}  // namespace brace
