// The gradients of queries and bias, bf16 values.
#include "attention_queries.hpp"

namespace pqt {
template void launch_attention_queries<Bf16>(const AttentionArgs&, int, bool, hipStream_t);
}  // namespace pqt
