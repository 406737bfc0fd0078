// The gradients of queries and bias, f16 values.
#include "attention_queries.hpp"

namespace pqt {
template void launch_attention_queries<Half>(const AttentionArgs&, int, bool, hipStream_t);
}  // namespace pqt
