// Attention of bf16 values.
#include "attention_kernel.hpp"

namespace pqt {
template void launch_attention<Bf16>(const AttentionArgs&, int, bool, hipStream_t);
}  // namespace pqt
