// The kernels of feed_large.hpp for one type of operands.
#include "feed_large.hpp"

namespace topk {

template <>
int launch_feed_large<f16>(const FeedArgs& g, bool k_contiguous, Work work, hipStream_t stream) {
  return large_work<f16>(g, k_contiguous, work, stream);
}

}  // namespace topk
