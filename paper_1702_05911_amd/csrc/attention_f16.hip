// Attention of f16 values.
#include "attention_kernel.hpp"

namespace pqt {
template void launch_attention<Half>(const AttentionArgs&, int, bool, hipStream_t);
}  // namespace pqt
