// The kernels of feed_thin.hpp.
#include "feed_thin.hpp"

namespace topk {

template <>
int launch_feed_thin<float>(const FeedArgs& g, Work work, bool narrow, hipStream_t stream) {
  return thin_work<float>(g, work, narrow, stream);
}
template <>
int launch_feed_thin<bf16>(const FeedArgs& g, Work work, bool narrow, hipStream_t stream) {
  return thin_work<bf16>(g, work, narrow, stream);
}
template <>
int launch_feed_thin<f16>(const FeedArgs& g, Work work, bool narrow, hipStream_t stream) {
  return thin_work<f16>(g, work, narrow, stream);
}
template <>
int launch_feed_thin<int8_t>(const FeedArgs& g, Work work, bool narrow, hipStream_t stream) {
  return thin_work<int8_t>(g, work, narrow, stream);
}

}  // namespace topk
