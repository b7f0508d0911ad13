// Eviction from the 4-bit cache: per (sample, KV head) the newest rows and the
// ones of largest accumulated attention weight, moved in order to a new cache.
//
// The weights are ranked by a 32-bit key that orders them as the reals do (NaN
// above all, -0 with +0). The smallest key kept is found byte by byte from the
// top (a histogram of the keys that share the bytes found so far); the rows above
// it, and the lowest positions of those equal to it, are then numbered in order.
#include "cache4.hpp"
#include "launch.hpp"

namespace litevlm {
namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / kWave;
constexpr int kMoveThreads = 256, kMoveRows = 64;

struct EvictParams {
  const uint8_t* cache;
  const float* weight;
  const int32_t* lengths;
  uint8_t* cache_out;
  float* weight_out;
  int32_t* lengths_out;
  int32_t* kept;
  int Hkv, cap, cap_out, max_len, budget, recent;
};

__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 + 0 = +0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelThreads) void cache4_select_kernel(EvictParams p) {
  const int b = blockIdx.y, g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n = min(max(p.lengths[b], 0), p.max_len);
  const int64_t head = (int64_t)b * p.Hkv + g;
  int32_t* kept = p.kept + head * p.budget;
  if (g == 0 && tid == 0) p.lengths_out[b] = min(n, p.budget);
  if (n <= p.budget) {
    for (int i = tid; i < n; i += kSelThreads) kept[i] = i;
    return;
  }
  const int old = n - p.recent, want = p.budget - p.recent;
  const float* wt = p.weight + head * p.cap;
  for (int i = tid; i < p.recent; i += kSelThreads) kept[want + i] = old + i;
  if (want == 0) return;

  __shared__ uint32_t hist[256];
  __shared__ uint32_t s_prefix, s_left;
  __shared__ uint32_t s_wave[2][kSelWaves];
  uint32_t prefix = 0, left = want;  // keys with the prefix: `left` of the largest are wanted
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < old; i += kSelThreads) {
      const uint32_t k = order_key(wt[i]);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      uint32_t seen = 0;
      int d = 255;
      while (seen + hist[d] < left) seen += hist[d--];  // old >= want: it ends by 0
      s_prefix = prefix | ((uint32_t)d << shift);
      s_left = left - seen;
    }
    __syncthreads();
    prefix = s_prefix;
    left = s_left;
  }
  // prefix is the smallest key kept, `left` of its rows
  uint32_t done = 0, ties = 0;
  for (int i0 = 0; i0 < old; i0 += kSelThreads) {
    const int i = i0 + tid;
    const uint32_t k = i < old ? order_key(wt[i]) : 0u;
    const bool tie = i < old && k == prefix;
    const uint64_t tmask = __ballot(tie);
    if (lane == 0) s_wave[0][w] = __popcll(tmask);
    __syncthreads();
    uint32_t t = ties, tall = 0;
    for (int x = 0; x < kSelWaves; ++x) {
      if (x < w) t += s_wave[0][x];
      tall += s_wave[0][x];
    }
    const uint64_t below = (1ull << lane) - 1;
    const bool take = i < old && (k > prefix || (tie && t + __popcll(tmask & below) < left));
    const uint64_t mask = __ballot(take);
    if (lane == 0) s_wave[1][w] = __popcll(mask);
    __syncthreads();
    uint32_t at = done, all = 0;
    for (int x = 0; x < kSelWaves; ++x) {
      if (x < w) at += s_wave[1][x];
      all += s_wave[1][x];
    }
    if (take) kept[at + __popcll(mask & below)] = i;
    done += all;
    ties += tall;
    __syncthreads();
  }
}

template <int D>
__global__ __launch_bounds__(kMoveThreads) void cache4_move_kernel(EvictParams p) {
  constexpr int VPR = D / 32;  // 16-byte pieces of a row of codes
  constexpr int NB = D / kCacheBlock;
  const int b = blockIdx.z, g = blockIdx.y, tid = threadIdx.x;
  const int L = min(min(max(p.lengths[b], 0), p.max_len), p.budget);
  const int i0 = blockIdx.x * kMoveRows;
  if (i0 >= L) return;
  const int64_t head = (int64_t)b * p.Hkv + g;
  const CacheHead<D> src(p.cache, head, p.cap), dst(p.cache_out, head, p.cap_out);
  const int32_t* kept = p.kept + head * p.budget;
  const int rows = min(kMoveRows, L - i0);
  for (int x = tid; x < rows * VPR; x += kMoveThreads) {
    const int i = i0 + x / VPR, piece = x % VPR;
    const int64_t from = kept[i];
    reinterpret_cast<uint4*>(dst.kc)[(int64_t)i * VPR + piece] = reinterpret_cast<const uint4*>(src.kc)[from * VPR + piece];
    reinterpret_cast<uint4*>(dst.vc)[(int64_t)i * VPR + piece] = reinterpret_cast<const uint4*>(src.vc)[from * VPR + piece];
  }
  for (int x = tid; x < rows * NB; x += kMoveThreads) {
    const int i = i0 + x % rows, blk = x / rows;
    const int64_t from = kept[i];
    dst.ks[(int64_t)blk * p.cap_out + i] = src.ks[(int64_t)blk * p.cap + from];
    dst.vs[(int64_t)blk * p.cap_out + i] = src.vs[(int64_t)blk * p.cap + from];
  }
  if (tid < rows) p.weight_out[head * p.cap_out + i0 + tid] = p.weight[head * p.cap + kept[i0 + tid]];
}

}  // namespace

hipError_t launch_cache4_evict(const Cache4EvictArgs& a, hipStream_t stream) {
  const EvictParams p{static_cast<const uint8_t*>(a.cache),
                      a.weight,
                      a.lengths,
                      static_cast<uint8_t*>(a.cache_out),
                      a.weight_out,
                      a.lengths_out,
                      a.kept_index,
                      a.Hkv,
                      a.cap,
                      a.cap_out,
                      a.max_len,
                      a.budget,
                      a.recent};
  hipLaunchKernelGGL(cache4_select_kernel, dim3(a.Hkv, a.B), dim3(kSelThreads), 0, stream, p);
  const int most = std::min(a.budget, a.max_len);
  if (most > 0) {
    const dim3 grid((most + kMoveRows - 1) / kMoveRows, a.Hkv, a.B);
    if (a.D == 128) hipLaunchKernelGGL(cache4_move_kernel<128>, grid, dim3(kMoveThreads), 0, stream, p);
    else hipLaunchKernelGGL(cache4_move_kernel<64>, grid, dim3(kMoveThreads), 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace litevlm
