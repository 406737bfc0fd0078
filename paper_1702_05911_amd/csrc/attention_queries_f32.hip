// The gradients of queries and bias, f32 values.
#include "attention_queries.hpp"

namespace pqt {
template void launch_attention_queries<float>(const AttentionArgs&, int, bool, hipStream_t);
}  // namespace pqt
