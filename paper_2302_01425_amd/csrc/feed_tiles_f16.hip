// The kernels of feed_tiles.hpp for one type of operands.
#include "feed_tiles.hpp"

namespace topk {

template <>
int launch_feed_tiles<f16>(const FeedArgs& g, bool k_contiguous, Work work, TileKind kind, hipStream_t stream) {
  return feed_work<f16>(g, k_contiguous, work, kind, stream);
}

}  // namespace topk
