// Places of the chosen (token, choice) pairs in expert order, from the list of chosen experts alone: a counting sort of the
// pairs by expert that keeps their order.
//   load[e] = pairs that chose e, kept[e] = min(load[e], capacity), offset = exclusive sums of kept (offset[n]: all places),
//   slot[p] = offset[e] + rank of p among the pairs of e, or -1 (no expert, or rank >= capacity);  source[slot[p]] = p.
// The pairs are cut into chunks of consecutive ones, a workgroup each.  First launch: counts of every chunk.  Second: every
// workgroup adds up the counts of the chunks before its own and places its pairs, wavefront after wavefront, equal experts
// inside a wavefront ranked by ballots over the bits of the expert.  No atomics decide an order, nothing waits for another
// workgroup.  One chunk: the second launch alone.
#include "common.hpp"
#include "experts.hpp"

namespace topk {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int64_t kChunk = 2048;       // pairs per workgroup, at least
constexpr int kOwn = kExpertsMax / kThreads;   // experts per thread

__device__ __forceinline__ int expert_of(const MapArgs& a, int64_t p, int64_t end) {
  if (p >= end) return -1;
  const int e = a.idx[p];
  return e >= 0 && e < a.n ? e : -1;
}

__global__ __launch_bounds__(kThreads) void map_count_kernel(MapArgs a, int64_t chunk) {
  __shared__ int32_t count[kExpertsMax];
  for (int e = threadIdx.x; e < a.n; e += kThreads) count[e] = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * chunk, end = min(begin + chunk, a.pairs);
  for (int64_t p = begin + threadIdx.x; p < end; p += kThreads) {
    const int e = expert_of(a, p, end);
    if (e >= 0) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.n; e += kThreads) a.scratch[int64_t(blockIdx.x) * a.n + e] = count[e];
}

__global__ __launch_bounds__(kThreads) void map_place_kernel(MapArgs a, int64_t chunk, int bits) {
  __shared__ int32_t next[kWaves][kExpertsMax];      // next place of an expert's pairs in a wavefront's part
  __shared__ int32_t offset[kExpertsMax + 1];
  __shared__ int32_t limit[kExpertsMax];             // end of an expert's places
  __shared__ int32_t wave_total[kWaves];
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid & (kWave - 1);
  const int64_t begin = blockIdx.x * chunk, end = min(begin + chunk, a.pairs);
  const int64_t part = (chunk + kWaves - 1) / kWaves;
  const int64_t wbegin = min(begin + wave * part, end), wend = min(wbegin + part, end);

  for (int i = tid; i < kWaves * a.n; i += kThreads) next[i / a.n][i % a.n] = 0;
  __syncthreads();
  for (int64_t p = wbegin + lane; p < wend; p += kWave) {
    const int e = expert_of(a, p, wend);
    if (e >= 0) atomicAdd(&next[wave][e], 1);
  }
  __syncthreads();

  // counts of the chunks before this one and of all; every thread has kOwn consecutive experts
  int32_t before[kOwn], load[kOwn], kept[kOwn], mine = 0;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int e = tid * kOwn + i;
    before[i] = load[i] = kept[i] = 0;
    if (e < a.n) {
      if (gridDim.x == 1) {
        for (int w = 0; w < kWaves; ++w) load[i] += next[w][e];
      } else {
        for (unsigned b = 0; b < gridDim.x; ++b) {
          const int32_t c = a.scratch[int64_t(b) * a.n + e];
          load[i] += c;
          if (b < blockIdx.x) before[i] += c;
        }
      }
      kept[i] = int32_t(min(int64_t(load[i]), a.capacity));
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
      offset[e] = start;
      limit[e] = start + kept[i];
      int32_t at = start + before[i];                // (beyond the limit where the expert is full)
      for (int w = 0; w < kWaves; ++w) {
        const int32_t c = next[w][e];
        next[w][e] = at;
        at += c;
      }
      if (e == a.n - 1) offset[a.n] = start + kept[i];
    }
    start += kept[i];
    if (blockIdx.x == 0 && e < a.n) a.load[e] = load[i];
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int e = tid; e <= a.n; e += kThreads) a.offset[e] = offset[e];

  for (int64_t p0 = wbegin; p0 < wend; p0 += kWave) {
    const int64_t p = p0 + lane;
    const int e = expert_of(a, p, wend);
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
  }
  // places that nothing takes
  for (int64_t p = max(begin, int64_t(offset[a.n])) + tid; p < end; p += kThreads) a.source[p] = -1;
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
  int bits = 0;
  while ((1 << bits) < a.n) ++bits;
  if (chunks > 1) hipLaunchKernelGGL(map_count_kernel, dim3(unsigned(chunks)), dim3(kThreads), 0, stream, a, chunk);
  hipLaunchKernelGGL(map_place_kernel, dim3(unsigned(chunks)), dim3(kThreads), 0, stream, a, chunk, bits);
  return 0;
}

}  // namespace topk
