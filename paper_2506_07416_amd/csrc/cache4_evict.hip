// Eviction from the 4-bit cache: per (sample, KV head) the newest rows and the
// ones of largest accumulated attention weight, moved in order to a new cache.
//
// The weights are ranked by a 32-bit key that orders them as the reals do (NaN
// above all, -0 with +0). One workgroup a head finds the smallest key kept, 11, 11
// and 10 bits at a time: a histogram of the keys that share the bits found so far,
// summed from the top. The rows above it, and the lowest positions of those equal
// to it, are then numbered in order. Each thread holds consecutive keys, so an
// order over threads is one over positions.
#include "cache4.hpp"
#include "launch.hpp"

namespace litevlm {
namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / kWave;
constexpr int kBins = 2048;  // two a thread
// Rows up to which the selecting workgroup moves them too, in one launch (8 heads,
// on the GPU alone: 256 rows 7.7 us and 8.8 with two launches, 512 rows 8.1 and 8.2,
// 1024 rows 10.4 and 8.4; 256 heads: 512 rows 13.0 and 15.3, 2048 rows 36.9 and 36.0).
constexpr int kFusedRows = 512;
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

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_add(uint32_t x) {
  return x + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
}

// Exclusive sum of x over the workgroup's threads in order; s_wave is free again
// after the next barrier.
__device__ __forceinline__ uint32_t scan(uint32_t x, uint32_t* s_wave, uint32_t& all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t y = x;
  y = dpp_add<0x111, 0xF>(y);  // row_shr 1, 2, 4, 8
  y = dpp_add<0x112, 0xF>(y);
  y = dpp_add<0x114, 0xF>(y);
  y = dpp_add<0x118, 0xF>(y);
  y = dpp_add<0x142, 0xA>(y);  // row_bcast 15, 31
  y = dpp_add<0x143, 0xC>(y);
  if (lane == kWave - 1) s_wave[w] = y;
  __syncthreads();
  uint32_t before = 0;
  all = 0;
#pragma unroll
  for (int k = 0; k < kSelWaves; ++k) {
    const uint32_t z = s_wave[k];
    before += k < w ? z : 0u;
    all += z;
  }
  return before + y - x;
}

// Numbers the rows that one head keeps, by the whole workgroup. KPT keys a thread
// and tile; one tile stays in registers.
template <int KPT>
__device__ __forceinline__ void select_rows(const EvictParams& p, int64_t head, int n) {
  constexpr int kTileKeys = kSelThreads * KPT;
  const int tid = threadIdx.x;
  int32_t* kept = p.kept + head * p.budget;
  if (n <= p.budget) {
    for (int i = tid; i < n; i += kSelThreads) kept[i] = i;
    return;
  }
  const int old = n - p.recent, want = p.budget - p.recent;
  const float* wt = p.weight + head * p.cap;
  for (int i = tid; i < p.recent; i += kSelThreads) kept[want + i] = old + i;
  if (want == 0) return;

  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t s_digit, s_left, s_whole;
  __shared__ uint32_t s_wave[2][kSelWaves];
  const int tiles = (old + kTileKeys - 1) / kTileKeys;
  uint32_t key[KPT];
  const auto load = [&](int tile) __attribute__((always_inline)) {
    const int i0 = tile * kTileKeys + tid * KPT;
    float x[KPT];
    if (i0 + KPT <= old && (reinterpret_cast<uintptr_t>(wt) & 15) == 0) {
#pragma unroll
      for (int j = 0; j < KPT; j += 4) {
        const float4 v = *reinterpret_cast<const float4*>(wt + i0 + j);
        x[j] = v.x, x[j + 1] = v.y, x[j + 2] = v.z, x[j + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < KPT; ++j) x[j] = i0 + j < old ? wt[i0 + j] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < KPT; ++j) key[j] = order_key(x[j]);
  };

  uint32_t prefix = 0, left = want;  // of the keys with these bits, `left` of the largest are wanted
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    hist[tid] = 0;
    hist[tid + kSelThreads] = 0;
    __syncthreads();
    for (int tile = 0; tile < tiles; ++tile) {
      if (pass == 0 || tiles > 1) load(tile);
      const int i0 = tile * kTileKeys + tid * KPT;
#pragma unroll
      for (int j = 0; j < KPT; ++j) {
        const bool in = i0 + j < old && (pass == 0 || key[j] >> (shift + bits) == prefix >> (shift + bits));
        const uint32_t d = (key[j] >> shift) & ((1u << bits) - 1);
        // a wave whose keys fall into one bin (zeros of rows never looked at) adds
        // them at once: additions to one address take their turns
        const uint64_t mask = __ballot(in);
        if (mask == 0) continue;
        const uint32_t lead = (uint32_t)__builtin_amdgcn_readlane((int)d, __ffsll((unsigned long long)mask) - 1);
        if (__ballot(in && d != lead) == 0) {
          if ((tid & 63) == 0) atomicAdd(&hist[lead], (uint32_t)__popcll(mask));
        } else if (in) {
          atomicAdd(&hist[d], 1u);
        }
      }
    }
    __syncthreads();
    // thread t: bins 2047 - 2t and 2046 - 2t, so that the sum runs from the top
    const int hi = kBins - 1 - 2 * tid;
    const uint32_t h0 = hist[hi], h1 = hist[hi - 1];
    uint32_t all;
    const uint32_t above = scan(h0 + h1, s_wave[0], all);
    if (above < left && left <= above + h0 + h1) {
      const bool first = left <= above + h0;
      s_digit = first ? hi : hi - 1;
      s_left = left - (first ? above : above + h0);
      s_whole = s_left == (first ? h0 : h1);
    }
    __syncthreads();
    prefix |= s_digit << shift;
    left = s_left;
    if (s_whole) {  // every key with these bits is kept: no more of them are needed
      prefix -= 1;  // no weight's key is 0
      left = 0;
      break;
    }
  }
  // keys above prefix are kept, and `left` of those equal to it
  uint32_t done = 0, ties = 0;  // kept, and equal to it, in the tiles before
  for (int tile = 0; tile < tiles; ++tile) {
    if (tiles > 1) load(tile);
    const int i0 = tile * kTileKeys + tid * KPT;
    uint32_t more = 0, same = 0;
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
      more += i0 + j < old && key[j] > prefix;
      same += i0 + j < old && key[j] == prefix;
    }
    uint32_t all_more, all_same;
    uint32_t t = ties + scan(same, s_wave[0], all_same);
    uint32_t at = done + scan(more, s_wave[1], all_more) + min(t, left);  // ties before this thread that are kept
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
      if (i0 + j >= old) continue;
      const bool tie = key[j] == prefix;
      if (key[j] > prefix || (tie && t < left)) kept[at++] = i0 + j;
      t += tie;
    }
    done += all_more;
    ties += all_same;
    __syncthreads();
  }
}

// Moves rows i0 .. i0 + rows - 1 of a head's kept ones, with their scales and weights.
template <int D, int THREADS>
__device__ __forceinline__ void move_rows(const EvictParams& p, int64_t head, int i0, int rows) {
  constexpr int VPR = D / 32;  // 16-byte pieces of a row of codes
  constexpr int NB = D / kCacheBlock;
  const int tid = threadIdx.x;
  const CacheHead<D> src(p.cache, head, p.cap), dst(p.cache_out, head, p.cap_out);
  const int32_t* kept = p.kept + head * p.budget;
  for (int x = tid; x < rows * VPR; x += THREADS) {
    const int i = i0 + x / VPR, piece = x % VPR;
    const int64_t from = kept[i];
    reinterpret_cast<uint4*>(dst.kc)[(int64_t)i * VPR + piece] = reinterpret_cast<const uint4*>(src.kc)[from * VPR + piece];
    reinterpret_cast<uint4*>(dst.vc)[(int64_t)i * VPR + piece] = reinterpret_cast<const uint4*>(src.vc)[from * VPR + piece];
  }
  for (int x = tid; x < rows * NB; x += THREADS) {
    const int i = i0 + x % rows, blk = x / rows;
    const int64_t from = kept[i];
    dst.ks[(int64_t)blk * p.cap_out + i] = src.ks[(int64_t)blk * p.cap + from];
    dst.vs[(int64_t)blk * p.cap_out + i] = src.vs[(int64_t)blk * p.cap + from];
  }
  for (int i = i0 + tid; i < i0 + rows; i += THREADS) p.weight_out[head * p.cap_out + i] = p.weight[head * p.cap + kept[i]];
}

template <int D>
__global__ __launch_bounds__(kMoveThreads) void cache4_move_kernel(EvictParams p) {
  const int b = blockIdx.z, g = blockIdx.y;
  const int L = min(min(max(p.lengths[b], 0), p.max_len), p.budget);
  const int i0 = blockIdx.x * kMoveRows;
  if (i0 >= L) return;
  move_rows<D, kMoveThreads>(p, (int64_t)b * p.Hkv + g, i0, min(kMoveRows, L - i0));
}

// One workgroup a head: the rows it keeps and, for D > 0, their move.
template <int KPT, int D>
__global__ __launch_bounds__(kSelThreads) void cache4_select_kernel(EvictParams p) {
  const int b = blockIdx.y, g = blockIdx.x;
  const int n = min(max(p.lengths[b], 0), p.max_len);
  const int64_t head = (int64_t)b * p.Hkv + g;
  if (g == 0 && threadIdx.x == 0) p.lengths_out[b] = min(n, p.budget);
  select_rows<KPT>(p, head, n);
  if constexpr (D > 0) {
    __syncthreads();  // the workgroup's own stores to kept are seen behind it
    move_rows<D, kSelThreads>(p, head, 0, min(n, p.budget));
  }
}

template <int D>
void launch_select(const EvictParams& p, int B, hipStream_t stream) {
  const dim3 grid(p.Hkv, B);
  if (p.max_len <= 4 * kSelThreads)
    hipLaunchKernelGGL((cache4_select_kernel<4, D>), grid, dim3(kSelThreads), 0, stream, p);
  else
    hipLaunchKernelGGL((cache4_select_kernel<16, D>), grid, dim3(kSelThreads), 0, stream, p);
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
  const int most = std::min(a.budget, a.max_len);
  if (most <= kFusedRows) {
    if (a.D == 128) launch_select<128>(p, a.B, stream);
    else launch_select<64>(p, a.B, stream);
    return hipGetLastError();
  }
  launch_select<0>(p, a.B, stream);
  const dim3 grid((most + kMoveRows - 1) / kMoveRows, a.Hkv, a.B);
  if (a.D == 128) hipLaunchKernelGGL(cache4_move_kernel<128>, grid, dim3(kMoveThreads), 0, stream, p);
  else hipLaunchKernelGGL(cache4_move_kernel<64>, grid, dim3(kMoveThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace litevlm
