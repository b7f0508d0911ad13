// Attention of each sample's newest tokens over its rows of the 4-bit cache.
//
// o_r = sum_j softmax_j(s * q_r . K_j) V_j in one pass over the keys with the
// running maximum m and sum l of each row r (a row is one query of one head; the
// G = Hq/Hkv heads that read a KV head share its rows of keys). The codes are
// decoded to bf16, which holds every E2M1 value times a power of two, so the
// products run on the bf16 matrix instructions without loss; an fp32 operand goes
// through them as three bf16 terms, which hold its 24 bits.
//
// 16x16x32 products, lane = (lg = lane / 16, c = lane % 16):
//   S^T = K Q^T   A: key c of a 16-key tile, the 32 contraction slots of step t are
//                 the elements lg*D/4 + 8t.. of the row, so a lane reads D/8
//                 consecutive bytes of one key, with one scale;
//                 B: row c at the same elements.
//                 The result has row c, keys 4*lg + i.
//   O^T = V^T P^T B: row c, keys 4*lg + i of two 16-key tiles: the results of the
//                 first product as they stand, no exchange between lanes.
//                 A: for tile t element c*D/16 + t of those keys.
//                 The result has row c, elements (4*lg + i)*D/16 + t: D/4
//                 consecutive elements a lane, all of one block.
#include "cache4.hpp"
#include "launch.hpp"

namespace litevlm {
namespace {

struct AttnParams {
  const void* q;
  void* o;
  const uint8_t* cache;
  const int32_t* cu;
  const int32_t* lengths;
  const float* weight_in;
  float* weight_out;
  float2* stat;  // [B][Hkv][G * weight_rows]: (maximum, 1 / sum) of the rows that add weight
  int Hq, Hkv, G, cap, max_q, max_len, weight_rows;
  float scale_log2;
};

// x as TERMS bf16 values whose sum is x (3 terms: exactly, by cutting 8 bits at a time).
template <int TERMS>
__device__ __forceinline__ void split_terms(float x, __bf16* t) {
  if constexpr (TERMS == 1) {
    t[0] = (__bf16)x;
  } else {
    const float a = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
    const float r = x - a;
    const float b = __uint_as_float(__float_as_uint(r) & 0xFFFF0000u);
    t[0] = (__bf16)a;
    t[1] = (__bf16)b;
    t[2] = (__bf16)(r - b);
  }
}

template <int D, int TERMS>
struct Attn {
  static constexpr int kSteps = D / 32;  // first product: steps of a key tile
  static constexpr int kTiles = D / 16;  // second product: tiles of the output
  static constexpr bool kF32 = TERMS == 3;

  struct Rows {  // the queries of 16 rows, as the lane's operands
    bf16x8 q[kSteps][TERMS];
  };

  static __device__ __forceinline__ void load_rows(const AttnParams& p, int64_t row, bool live, int lg, Rows& f) {
#pragma unroll
    for (int t = 0; t < kSteps; ++t) {
      const int64_t e = row * D + lg * (D / 4) + 8 * t;
      if constexpr (kF32) {
        float x[8];
        const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(p.q) + e);
        const float4 z = make_float4(0.f, 0.f, 0.f, 0.f), a = live ? src[0] : z, b = live ? src[1] : z;
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          __bf16 s[3];
          split_terms<3>(x[i], s);
#pragma unroll
          for (int k = 0; k < 3; ++k) f.q[t][k][i] = s[k];
        }
      } else {
        const i32x4 z = {0, 0, 0, 0};
        const i32x4 w = live ? *reinterpret_cast<const i32x4*>(static_cast<const uint16_t*>(p.q) + e) : z;
        f.q[t][0] = __builtin_bit_cast(bf16x8, w);
      }
    }
  }

  // Logits (without the scale) of the 16 rows against the 16 keys at k0.
  static __device__ __forceinline__ f32x4 logits(const CacheHead<D>& c, int cap, int k0, int lg, int col,
                                                 const Rows& f) {
    const int key = k0 + col;
    const float scale = e8m0_scale(c.ks[(int64_t)(lg * D / 128) * cap + key]);
    const uint32_t* src = reinterpret_cast<const uint32_t*>(c.kc + (int64_t)key * (D / 2) + lg * (D / 8));
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < kSteps; ++t) {
      const bf16x8 k = decode8(src[t], scale);
#pragma unroll
      for (int n = TERMS - 1; n >= 0; --n) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, f.q[t][n], s, 0, 0, 0);
    }
    return s;
  }
};

// One wave: 16 rows of one (sample, KV head), every key.
template <int D, int TERMS>
__global__ __launch_bounds__(64) void cache4_attn_kernel(AttnParams p) {
  using A = Attn<D, TERMS>;
  constexpr int ET = D / 16;  // elements of a key that a lane decodes for the second product
  const int b = blockIdx.z, g = blockIdx.y, lane = threadIdx.x, lg = lane >> 4, col = lane & 15;
  const int lo = p.cu[b], m = min(p.cu[b + 1] - lo, p.max_q);
  const int rows = m * p.G;
  const int r = blockIdx.x * 16 + col;
  if (blockIdx.x * 16 >= rows) return;
  const int n = min(max(p.lengths[b], 0), p.max_len);
  const bool live = r < rows;
  const int qi = r / p.G;
  const int64_t qrow = (int64_t)(lo + qi) * p.Hq + g * p.G + r % p.G;
  const int seen = live ? max(n - m + qi + 1, 0) : 0;  // keys that the row sees
  const int last = max(n - m + min(blockIdx.x * 16 + 15, rows - 1) / p.G + 1, 0);  // the most of any row
  const CacheHead<D> c(p.cache, (int64_t)b * p.Hkv + g, p.cap);
  typename A::Rows f;
  A::load_rows(p, qrow, live, lg, f);

  f32x4 acc[A::kTiles];
#pragma unroll
  for (int t = 0; t < A::kTiles; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float mx = -INFINITY, sum = 0.f;
  for (int k0 = 0; k0 < last; k0 += 32) {
    float x[8];
    float top = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 s = A::logits(c, p.cap, k0 + 16 * h, lg, col, f);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[4 * h + i] = k0 + 16 * h + 4 * lg + i < seen ? s[i] * p.scale_log2 : -INFINITY;
        top = fmaxf(top, x[4 * h + i]);
      }
    }
    top = fmaxf(mx, max_xor32(max_xor16(top)));
    // a row without a finite logit so far keeps 0 as its reference: exp2(-inf) = 0
    const float ref = top == -INFINITY ? 0.f : top;
    const float alpha = __builtin_amdgcn_exp2f(mx - ref);
    mx = top;
    sum *= alpha;
    bf16x8 pf[TERMS];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool see = k0 + 16 * (i >> 2) + 4 * lg + (i & 3) < seen;
      const float e = see ? __builtin_amdgcn_exp2f(x[i] - ref) : 0.f;
      sum += e;
      __bf16 s[TERMS];
      split_terms<TERMS>(e, s);
#pragma unroll
      for (int k = 0; k < TERMS; ++k) pf[k][i] = s[k];
    }
#pragma unroll
    for (int t = 0; t < A::kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[t][i] *= alpha;

    // V: elements col*ET.. of the lane's eight keys, then keys side by side
    bf16x8 vt[ET];
    bool nan_here = false;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const int key = k0 + 16 * (kk >> 2) + 4 * lg + (kk & 3);
      uint32_t byte = c.vs[(int64_t)(col * ET / kCacheBlock) * p.cap + key];
      // rows behind the length hold anything, and a NaN block may be hidden from
      // some of the rows: both are left out here
      nan_here |= byte == 255u && key < n;
      if (key >= n || byte == 255u) byte = 0;
      const uint8_t* src = c.vc + (int64_t)key * (D / 2) + col * (ET / 2);
      const uint32_t w = ET == 8 ? *reinterpret_cast<const uint32_t*>(src) : *reinterpret_cast<const uint16_t*>(src);
      const bf16x8 v = decode8(w, e8m0_scale(byte));
#pragma unroll
      for (int t = 0; t < ET; ++t) vt[t][kk] = v[t];
    }
#pragma unroll
    for (int t = 0; t < ET; ++t)
#pragma unroll
      for (int k = TERMS - 1; k >= 0; --k)
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[t], pf[k], acc[t], 0, 0, 0);
    if (__any(nan_here)) {  // NaN blocks reach the rows that see them
      bool bad = false;
      for (int kk = 0; kk < 32; ++kk)
        bad |= k0 + kk < seen && c.vs[(int64_t)(lg * D / 128) * p.cap + k0 + kk] == 255u;
      if (bad) {
#pragma unroll
        for (int t = 0; t < A::kTiles; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[t][i] = __builtin_nanf("");
      }
    }
  }
  sum = sum_xor32(sum_xor16(sum));
  if (!live) return;
  const float inv = seen > 0 ? 1.f / sum : 0.f;  // all logits -inf: 0 * inf, a NaN
  if (lg == 0 && qi < p.weight_rows)
    p.stat[((int64_t)b * p.Hkv + g) * p.weight_rows * p.G + r] = make_float2(mx == -INFINITY ? 0.f : mx, inv);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int t = 0; t < ET; ++t) {
      const int64_t e = qrow * D + (4 * lg + i) * ET + t;
      const float y = acc[t][i] * inv;
      if constexpr (TERMS == 3) static_cast<float*>(p.o)[e] = y;
      else static_cast<__bf16*>(p.o)[e] = (__bf16)y;
    }
  }
}

// One wave: the weight of 16 keys, the logits taken again.
template <int D, int TERMS>
__global__ __launch_bounds__(64) void cache4_weight_kernel(AttnParams p) {
  using A = Attn<D, TERMS>;
  const int b = blockIdx.z, g = blockIdx.y, lane = threadIdx.x, lg = lane >> 4, col = lane & 15;
  const int n = min(max(p.lengths[b], 0), p.max_len);
  const int k0 = blockIdx.x * 16;
  if (k0 >= n) return;
  const int lo = p.cu[b], m = min(p.cu[b + 1] - lo, p.max_q);
  const int rows = min(m, p.weight_rows) * p.G;
  const int64_t head = (int64_t)b * p.Hkv + g;
  const CacheHead<D> c(p.cache, head, p.cap);
  float w[4] = {0.f, 0.f, 0.f, 0.f};
  for (int r0 = 0; r0 < rows; r0 += 16) {
    const int r = r0 + col, qi = r / p.G;
    const bool live = r < rows;
    const int seen = live ? n - m + qi + 1 : 0;
    typename A::Rows f;
    A::load_rows(p, (int64_t)(lo + qi) * p.Hq + g * p.G + r % p.G, live, lg, f);
    const float2 st = live ? p.stat[head * p.weight_rows * p.G + r] : make_float2(0.f, 0.f);
    const f32x4 s = A::logits(c, p.cap, k0, lg, col, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float e = __builtin_amdgcn_exp2f(s[i] * p.scale_log2 - st.x) * st.y;
      w[i] += k0 + 4 * lg + i < seen ? e : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float y = row16_sum(w[i]);
    const int key = k0 + 4 * lg + i;
    if (col == 0 && key < n) {
      const int64_t at = head * p.cap + key;
      p.weight_out[at] = (p.weight_in ? p.weight_in[at] : 0.f) + y;
    }
  }
}

template <int D, int TERMS>
void launch(const AttnParams& p, int B, hipStream_t stream) {
  if (p.max_q > 0)
    hipLaunchKernelGGL((cache4_attn_kernel<D, TERMS>), dim3(((int64_t)p.max_q * p.G + 15) / 16, p.Hkv, B), dim3(64),
                       0, stream, p);
  if (p.weight_rows > 0 && p.max_len > 0)
    hipLaunchKernelGGL((cache4_weight_kernel<D, TERMS>), dim3((p.max_len + 15) / 16, p.Hkv, B), dim3(64), 0, stream,
                       p);
}

}  // namespace

Cache4AttnLayout cache4_attn_layout(int dtype, int B, int Hq, int Hkv, int D, int max_q, int max_len,
                                    int weight_rows) {
  Cache4AttnLayout lay;
  lay.total = std::max<size_t>(256, (size_t)B * Hq * weight_rows * sizeof(float2));
  return lay;
}

hipError_t launch_cache4_attn(const Cache4AttnArgs& a, hipStream_t stream) {
  const AttnParams p{a.q,
                     a.o,
                     static_cast<const uint8_t*>(a.cache),
                     a.cu_q,
                     a.lengths,
                     a.weight_in,
                     a.weight_out,
                     static_cast<float2*>(a.workspace),
                     a.Hq,
                     a.Hkv,
                     a.Hq / a.Hkv,
                     a.cap,
                     a.max_q,
                     a.max_len,
                     a.weight_rows,
                     a.scale_log2};
  const bool bf16 = a.dtype == LITEVLM_BF16;
  if (a.D == 128) {
    if (bf16) launch<128, 1>(p, a.B, stream);
    else launch<128, 3>(p, a.B, stream);
  } else {
    if (bf16) launch<64, 1>(p, a.B, stream);
    else launch<64, 3>(p, a.B, stream);
  }
  return hipGetLastError();
}

}  // namespace litevlm
