// Places of the chosen (token, choice) pairs in expert order, from the list of chosen experts alone: a counting sort of the
// pairs by expert that keeps their order.
//   load[e] = pairs that chose e, kept[e] = min(load[e], capacity), offset = exclusive sums of kept (offset[n]: all places),
//   slot[p] = offset[e] + rank of p among the pairs of e, or -1 (no expert, or rank >= capacity);  source[slot[p]] = p.
// The pairs are cut into chunks of consecutive ones, a workgroup each.  First launch: counts of every chunk.  Second: every
// workgroup adds up the counts of the chunks before its own and places its pairs, wavefront after wavefront, equal experts
// inside a wavefront ranked by ballots over the bits of the expert.  No atomics decide an order, nothing waits for another
// workgroup.  One chunk: the second launch alone.
//
// Bound by the launches and by the chain load - count - sums - place inside them, not by bytes: 64 x 2 pairs, 64 experts 3.0 us;
// 32768 x 8 pairs, 128 experts 3.0 + 8.0 us (3.3 MB, 0.7 us at the rate of a copy).
#include "common.hpp"
#include "experts.hpp"

namespace topk {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int64_t kChunk = 2048;       // pairs per workgroup, at least
constexpr int kTurns = int(kChunk) / kThreads;      // pairs of a lane that stay in registers
constexpr int kOwn = kExpertsMax / kThreads;        // experts per thread

__device__ __forceinline__ int expert_of(const MapArgs& a, int64_t p, int64_t end) {
  if (p >= end) return -1;
  const int e = a.idx[p];
  return e >= 0 && e < a.n ? e : -1;
}

__global__ __launch_bounds__(kThreads) void map_count_kernel(MapArgs a, int64_t chunk, int width) {
  __shared__ int32_t count[kExpertsMax + 4];
  for (int e = threadIdx.x; e < width; e += kThreads) count[e] = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * chunk, end = min(begin + chunk, a.pairs);
  for (int64_t p = begin + threadIdx.x; p < end; p += kThreads) {
    const int e = expert_of(a, p, end);
    if (e >= 0) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < width; e += kThreads) a.scratch[int64_t(blockIdx.x) * width + e] = count[e];
}

// width: counts of a chunk in the scratch, n up to a multiple of four
__global__ __launch_bounds__(kThreads) void map_place_kernel(MapArgs a, int64_t chunk, int width, int bits) {
  __shared__ int32_t next[kWaves][kExpertsMax];      // next place of an expert's pairs in a wavefront's part
  __shared__ int32_t load[kExpertsMax + 4], before[kExpertsMax + 4];
  __shared__ int32_t limit[kExpertsMax];             // end of an expert's places
  __shared__ int32_t wave_total[kWaves];
  __shared__ int32_t all;
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid & (kWave - 1);
  const int64_t begin = blockIdx.x * chunk, end = min(begin + chunk, a.pairs);
  const int64_t part = (chunk + kWaves - 1) / kWaves;
  const int64_t wbegin = min(begin + wave * part, end), wend = min(wbegin + part, end);

  int kept_e[kTurns];                                // experts of the first turns
#pragma unroll
  for (int q = 0; q < kTurns; ++q) kept_e[q] = expert_of(a, wbegin + q * kWave + lane, wend);
  for (int e = tid; e < width; e += kThreads) {
    load[e] = before[e] = 0;
    if (e < a.n)
      for (int w = 0; w < kWaves; ++w) next[w][e] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kTurns; ++q)
    if (kept_e[q] >= 0) atomicAdd(&next[wave][kept_e[q]], 1);
  for (int64_t p = wbegin + kTurns * kWave + lane; p < wend; p += kWave) {
    const int e = expert_of(a, p, wend);
    if (e >= 0) atomicAdd(&next[wave][e], 1);
  }
  // counts of the chunks before this one, and of all: whole rows of counts by 16-byte reads, four experts per thread
  if (gridDim.x > 1) {
    const int quads = width / 4, q = tid % quads, b0 = tid / quads, step = kThreads / quads;
    if (b0 < step) {
      int32_t sum[4] = {0, 0, 0, 0}, mine[4] = {0, 0, 0, 0};
#pragma unroll 8
      for (int b = b0; b < int(gridDim.x); b += step) {
        const int4 c = *reinterpret_cast<const int4*>(a.scratch + int64_t(b) * width + 4 * q);
        const bool earlier = b < int(blockIdx.x);
        sum[0] += c.x, sum[1] += c.y, sum[2] += c.z, sum[3] += c.w;
        mine[0] += earlier ? c.x : 0, mine[1] += earlier ? c.y : 0, mine[2] += earlier ? c.z : 0, mine[3] += earlier ? c.w : 0;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        atomicAdd(&load[4 * q + i], sum[i]);
        atomicAdd(&before[4 * q + i], mine[i]);
      }
    }
  }
  __syncthreads();

  // every thread has kOwn consecutive experts
  int32_t kept[kOwn], mine = 0;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int e = tid * kOwn + i;
    kept[i] = 0;
    if (e < a.n) {
      if (gridDim.x == 1) {
        int32_t c = 0;
        for (int w = 0; w < kWaves; ++w) c += next[w][e];
        load[e] = c;
      }
      kept[i] = int32_t(min(int64_t(load[e]), a.capacity));
    }
    mine += kept[i];
  }
  int32_t scan = mine;
  for (int off = 1; off < kWave; off <<= 1) {
    const int32_t v = __shfl_up(scan, off, kWave);
    if (lane >= off) scan += v;
  }
  if (lane == kWave - 1) wave_total[wave] = scan;
  __syncthreads();
  int32_t start = scan - mine;
  for (int w = 0; w < wave; ++w) start += wave_total[w];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int e = tid * kOwn + i;
    if (e < a.n) {
      limit[e] = start + kept[i];
      int32_t at = start + before[e];                // (beyond the limit where the expert is full)
      for (int w = 0; w < kWaves; ++w) {
        const int32_t c = next[w][e];
        next[w][e] = at;
        at += c;
      }
      if (blockIdx.x == 0) {
        a.offset[e] = start;
        a.load[e] = load[e];
      }
      if (e == a.n - 1) {
        all = start + kept[i];
        if (blockIdx.x == 0) a.offset[a.n] = all;
      }
    }
    start += kept[i];
  }
  __syncthreads();

  const auto place_pairs = [&](int64_t p, int e) {
    unsigned long long same = __ballot(e >= 0);
    for (int b = 0; b < bits; ++b) {
      const unsigned long long set = __ballot((e >> b) & 1);
      same &= (e >> b) & 1 ? set : ~set;
    }
    int32_t place = -1;
    if (e >= 0) {
      const int rank = __popcll(same & ((1ull << lane) - 1ull));
      const int32_t at = __hip_atomic_load(&next[wave][e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) + rank;
      if (at < limit[e]) place = at;
      // the last of the equal ones moves the counter on, after all have read it (LDS accesses of a wavefront are in order)
      if ((same >> lane) == 1ull)
        __hip_atomic_store(&next[wave][e], at + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    if (p < wend) a.slot[p] = place;
    if (place >= 0) a.source[place] = int32_t(p);
  };
#pragma unroll
  for (int q = 0; q < kTurns; ++q)
    if (wbegin + q * kWave < wend) place_pairs(wbegin + q * kWave + lane, kept_e[q]);
  for (int64_t p0 = wbegin + kTurns * kWave; p0 < wend; p0 += kWave) place_pairs(p0 + lane, expert_of(a, p0 + lane, wend));
  // places that nothing takes
  for (int64_t p = max(begin, int64_t(all)) + tid; p < end; p += kThreads) a.source[p] = -1;
}

}  // namespace

int64_t map_chunks(int64_t pairs, int n) {
  // every workgroup reads the counts of all chunks: at most 2^15 of them
  const int64_t most = max(int64_t(1), min(int64_t(256), int64_t(32768) / n));
  return max(int64_t(1), min(most, (pairs + kChunk - 1) / kChunk));
}

int launch_expert_map(const MapArgs& a, hipStream_t stream) {
  const int64_t chunks = map_chunks(a.pairs, a.n);
  const int64_t chunk = max(int64_t(1), (a.pairs + chunks - 1) / chunks);
  const int width = map_width(a.n);
  int bits = 0;
  while ((1 << bits) < a.n) ++bits;
  if (chunks > 1) hipLaunchKernelGGL(map_count_kernel, dim3(unsigned(chunks)), dim3(kThreads), 0, stream, a, chunk, width);
  hipLaunchKernelGGL(map_place_kernel, dim3(unsigned(chunks)), dim3(kThreads), 0, stream, a, chunk, width, bits);
  return 0;
}

}  // namespace topk
