// The gradients of keys and values, f32 values.
#include "attention_keys.hpp"

namespace pqt {
template void launch_attention_keys<float>(const AttentionArgs&, int, int, bool, hipStream_t);
}  // namespace pqt
