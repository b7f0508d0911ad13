// Rows of keys and values into the 4-bit cache and back.
//
// A block of 32 elements x with a = max|x| gets the least E with a <= 7 * 2^E and
// the codes RNE_E2M1(x * 2^-E). Both are exact: with a = f * 2^t, 1 <= f < 2, E is
// t - 2 for f <= 1.75 and t - 1 beyond, read off a's bits, and the scaling is by
// a power of two. 7 rather than E2M1's largest value 6: what lies between is
// rounded down by at most 1, half of the step below, so no element is further
// from its code than at the top of the range anyway.
//
// Both directions move D elements and D/2 + D/32 bytes a row with a few
// conversions each: bound by memory.
#include "cache4.hpp"
#include "launch.hpp"

namespace litevlm {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 32;  // rows of a workgroup (1M rows read back: 32 116 us, 64 122 us)

// Eight elements of a row as they lie in memory, and the bits of their fp32 values.
template <bool BF16>
struct Eight {
  i32x4 w[BF16 ? 1 : 2];
  // read once and never again: past the caches (20.7K rows of 8 heads 30 -> 20 us)
  __device__ __forceinline__ void load(const void* base, int64_t elem) {
    const i32x4* p = reinterpret_cast<const i32x4*>(static_cast<const uint8_t*>(base) + elem * (BF16 ? 2 : 4));
    w[0] = __builtin_nontemporal_load(p);
    if constexpr (!BF16) w[1] = __builtin_nontemporal_load(p + 1);
  }
  __device__ __forceinline__ void bits(uint32_t* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        x[2 * i] = (uint32_t)w[0][i] << 16;
        x[2 * i + 1] = (uint32_t)w[0][i] & 0xFFFF0000u;
      } else {
        x[i] = (uint32_t)w[0][i];
        x[4 + i] = (uint32_t)w[1][i];
      }
    }
  }
};

__device__ __forceinline__ uint32_t umax_dpp_quad(uint32_t m) {
  const uint32_t a = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, false);  // lane ^ 1
  m = max(m, a);
  const uint32_t b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, false);  // lane ^ 2
  return max(m, b);
}

// Codes (8, as one word) and scale byte of the block that the lane shares with
// the other three of its quad.
__device__ __forceinline__ uint32_t encode8(const uint32_t* x, uint32_t& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, x[i] & 0x7FFFFFFFu);  // NaN > infinity > numbers
  top = umax_dpp_quad(top);
  // t - 2 + 127 with t + 127 the exponent field; the sum carries into it for f > 1.75
  const int e = (int)((top + 0x1FFFFFu) >> 23) - 2;
  const bool bad = top >= 0x7F800000u;
  const int ec = min(max(e, 2), 252);
  byte = bad ? 255u : (uint32_t)ec;
  const float scale = __uint_as_float((uint32_t)ec << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[0]), __uint_as_float(x[1]), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[2]), __uint_as_float(x[3]), scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[4]), __uint_as_float(x[5]), scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x[6]), __uint_as_float(x[7]), scale, 3);
  return bad ? 0u : w;
}

struct RowsParams {
  const void* k_in;
  const void* v_in;
  void* k_out;
  void* v_out;
  uint8_t* cache;
  float* weight;
  const int32_t* cu;
  const int32_t* start;
  int Hkv, cap, max_rows;
};

// One workgroup: 32 rows of one head, K and V; lane t of D/8 holds elements
// [8t, 8t + 8) of a row, so the four lanes of a block are a quad. The scales are
// gathered in LDS, since those of consecutive rows lie side by side in the cache.
template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void cache4_append_kernel(RowsParams p) {
  constexpr int LPR = D / 8, RPI = kThreads / LPR, NB = D / kCacheBlock;
  __shared__ uint8_t s_scale[2][NB][kTile];
  const int b = blockIdx.z, g = blockIdx.y, tid = threadIdx.x;
  const int lo = p.cu[b], n = min(p.cu[b + 1] - lo, p.max_rows);
  const int i0 = blockIdx.x * kTile;
  if (i0 >= n) return;
  const int64_t pos0 = (int64_t)p.start[b] + i0;
  const CacheHead<D> c(p.cache, (int64_t)b * p.Hkv + g, p.cap);
  const int t = tid % LPR;
  // the rows of kAhead passes are requested before the first is encoded (behind the
  // last row, that row again)
  constexpr int kPasses = kTile / RPI, kAhead = BF16 ? (kPasses < 4 ? kPasses : 4) : (kPasses < 2 ? kPasses : 2);
#pragma unroll
  for (int it0 = 0; it0 < kPasses; it0 += kAhead) {
    if (i0 + it0 * RPI >= n) break;
    Eight<BF16> k[kAhead], v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int row = min(i0 + (it0 + i) * RPI + tid / LPR, n - 1);
      const int64_t elem = ((int64_t)(lo + row) * p.Hkv + g) * D + t * 8;
      k[i].load(p.k_in, elem);
      v[i].load(p.v_in, elem);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int r = (it0 + i) * RPI + tid / LPR;
      const int64_t pos = pos0 + r;
      uint32_t x[8], kb, vb;
      k[i].bits(x);
      const uint32_t kw = encode8(x, kb);
      v[i].bits(x);
      const uint32_t vw = encode8(x, vb);
      if ((t & 3) == 0) {
        s_scale[0][t >> 2][r] = (uint8_t)kb;
        s_scale[1][t >> 2][r] = (uint8_t)vb;
      }
      if (i0 + r < n && pos >= 0 && pos < p.cap) {
        reinterpret_cast<uint32_t*>(c.kc + pos * CacheHead<D>::kRow)[t] = kw;
        reinterpret_cast<uint32_t*>(c.vc + pos * CacheHead<D>::kRow)[t] = vw;
      }
    }
  }
  __syncthreads();
  const int r = tid % kTile;
  const int64_t pos = pos0 + r;
  if (i0 + r >= n || pos < 0 || pos >= p.cap) return;
  for (int q = tid / kTile; q < 2 * NB; q += kThreads / kTile) {
    const int blk = q % NB;
    uint8_t* dst = (q < NB ? c.ks : c.vs) + (int64_t)blk * p.cap + pos;
    *dst = s_scale[q / NB][blk][r];
  }
  if (p.weight && tid < kTile) p.weight[((int64_t)b * p.Hkv + g) * p.cap + pos] = 0.f;
}

// Past the caches, for the sake of what lies in them: the rows of an eviction that
// is read back, 16 samples of 8192 rows, move in 62 instead of 78 us, and are read
// in 122 instead of 128.
template <bool BF16>
__device__ __forceinline__ void store8(void* base, int64_t elem, uint32_t w, float scale) {
  if constexpr (BF16) {
    __builtin_nontemporal_store(__builtin_bit_cast(i32x4, decode8(w, scale)), reinterpret_cast<i32x4*>(static_cast<uint16_t*>(base) + elem));
  } else {
    f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(base) + elem);
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
    const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
    const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    __builtin_nontemporal_store(f32x4{a[0], a[1], b[0], b[1]}, o);
    __builtin_nontemporal_store(f32x4{c[0], c[1], d[0], d[1]}, o + 1);
  }
}

template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void cache4_read_kernel(RowsParams p) {
  constexpr int LPR = D / 8, RPI = kThreads / LPR;
  const int b = blockIdx.z, g = blockIdx.y, tid = threadIdx.x;
  const int lo = p.cu[b], n = min(p.cu[b + 1] - lo, p.max_rows);
  const int i0 = blockIdx.x * kTile;
  if (i0 >= n) return;
  const CacheHead<D> c(p.cache, (int64_t)b * p.Hkv + g, p.cap);
  const int t = tid % LPR;
#pragma unroll
  for (int it = 0; it < kTile / RPI; ++it) {
    const int r = it * RPI + tid / LPR;
    if (i0 + r >= n) continue;
    const int64_t pos = (int64_t)p.start[b] + i0 + r;
    uint32_t kw = 0, vw = 0, kb = 0, vb = 0;
    if (pos >= 0 && pos < p.cap) {
      kw = reinterpret_cast<const uint32_t*>(c.kc + pos * CacheHead<D>::kRow)[t];
      vw = reinterpret_cast<const uint32_t*>(c.vc + pos * CacheHead<D>::kRow)[t];
      kb = c.ks[(int64_t)(t >> 2) * p.cap + pos];
      vb = c.vs[(int64_t)(t >> 2) * p.cap + pos];
    }
    const int64_t elem = ((int64_t)(lo + i0 + r) * p.Hkv + g) * D + t * 8;
    store8<BF16>(p.k_out, elem, kw, e8m0_scale(kb));
    store8<BF16>(p.v_out, elem, vw, e8m0_scale(vb));
  }
}

}  // namespace

hipError_t launch_cache4_append(const Cache4RowsArgs& a, hipStream_t stream) {
  if (a.max_rows == 0) return hipSuccess;
  const RowsParams p{a.k_in, a.v_in, nullptr, nullptr, static_cast<uint8_t*>(a.cache), a.weight,
                     a.cu,   a.start, a.Hkv,  a.cap,   a.max_rows};
  const dim3 grid((a.max_rows + kTile - 1) / kTile, a.Hkv, a.B);
  const bool bf16 = a.dtype == LITEVLM_BF16;
  if (a.D == 128) {
    if (bf16) hipLaunchKernelGGL((cache4_append_kernel<128, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((cache4_append_kernel<128, false>), grid, dim3(kThreads), 0, stream, p);
  } else {
    if (bf16) hipLaunchKernelGGL((cache4_append_kernel<64, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((cache4_append_kernel<64, false>), grid, dim3(kThreads), 0, stream, p);
  }
  return hipGetLastError();
}

hipError_t launch_cache4_read(const Cache4RowsArgs& a, hipStream_t stream) {
  if (a.max_rows == 0) return hipSuccess;
  const RowsParams p{nullptr, nullptr, a.k_out, a.v_out, static_cast<uint8_t*>(a.cache), nullptr,
                     a.cu,    a.start, a.Hkv,   a.cap,   a.max_rows};
  const dim3 grid((a.max_rows + kTile - 1) / kTile, a.Hkv, a.B);
  const bool bf16 = a.dtype == LITEVLM_BF16;
  if (a.D == 128) {
    if (bf16) hipLaunchKernelGGL((cache4_read_kernel<128, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((cache4_read_kernel<128, false>), grid, dim3(kThreads), 0, stream, p);
  } else {
    if (bf16) hipLaunchKernelGGL((cache4_read_kernel<64, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((cache4_read_kernel<64, false>), grid, dim3(kThreads), 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace litevlm
