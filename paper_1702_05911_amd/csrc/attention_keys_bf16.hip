// The gradients of keys and values, bf16 values.
#include "attention_keys.hpp"

namespace pqt {
template void launch_attention_keys<Bf16>(const AttentionArgs&, int, int, bool, hipStream_t);
}  // namespace pqt
