// Attention of f32 values.
#include "attention_kernel.hpp"

namespace pqt {
template void launch_attention<float>(const AttentionArgs&, int, bool, hipStream_t);
}  // namespace pqt
