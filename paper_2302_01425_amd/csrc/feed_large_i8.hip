// The kernels of feed_large.hpp for one type of operands.
#include "feed_large.hpp"

namespace topk {

template <>
int launch_feed_large<int8_t>(const FeedArgs& g, bool k_contiguous, Work work, hipStream_t stream) {
  return large_work<int8_t>(g, k_contiguous, work, stream);
}

}  // namespace topk
