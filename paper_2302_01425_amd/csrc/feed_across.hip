// The kernels of feed_across.hpp.
#include "feed_across.hpp"

namespace topk {

template <>
int launch_feed_across<float>(const FeedArgs& g, Work work, bool narrow, hipStream_t stream) {
  return across_work<float>(g, work, narrow, stream);
}
template <>
int launch_feed_across<bf16>(const FeedArgs& g, Work work, bool narrow, hipStream_t stream) {
  return across_work<bf16>(g, work, narrow, stream);
}
template <>
int launch_feed_across<f16>(const FeedArgs& g, Work work, bool narrow, hipStream_t stream) {
  return across_work<f16>(g, work, narrow, stream);
}

}  // namespace topk
