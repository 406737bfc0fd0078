// The gradients of keys and values, f16 values.
#include "attention_keys.hpp"

namespace pqt {
template void launch_attention_keys<Half>(const AttentionArgs&, int, int, bool, hipStream_t);
}  // namespace pqt
