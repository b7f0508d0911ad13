// Attention of each sample's newest tokens over its rows of the 4-bit cache.
//
// o_r = sum_j softmax_j(s * q_r . K_j) V_j in one pass over the keys with the
// running maximum m and sum l of each row r (a row is one query of one head; the
// G = Hq/Hkv heads that read a KV head share its rows of keys). The codes are
// decoded to bf16, which holds every E2M1 value times a power of two, so the
// products run on the bf16 matrix instructions without loss; an fp32 operand goes
// through them as three bf16 terms, which hold its 24 bits.
//
// For bf16 queries a probability is one bf16 term. It is off by at most 2^-8 of
// itself, as the result's own rounding is, and the errors of many keys average: root
// mean square of the outputs' errors 3.09e-4 for one query of 3200 rows, 4.47e-4 for
// drafts of batch 8, 3.87e-4 for 256 queries over 6528 rows, where probabilities of
// two terms (16 bits) leave the result's rounding alone, 3.06e-4, 3.64e-4 and 3.06e-4,
// and take 8.0, 17.9 and 53.3 us where one term takes 7.9, 16.7 and 43.3. A caller who
// wants them whole passes the same queries in fp32 (81 us).
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

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kKeys = 32;              // keys of a wave's step
constexpr int kStep = kWaves * kKeys;  // keys of a workgroup's step
constexpr int kFewSplits = 4;          // splits of a row that one thread joins
constexpr int kKept = 8;               // rows of a KV head whose logits are kept
constexpr int kWhole = 512;            // keys up to which one workgroup takes them all
constexpr float kSlack = 8.f;          // the running reference may lag the maximum by this (log2)

struct AttnParams {
  const void* q;
  void* o;
  const uint8_t* cache;
  const int32_t* cu;
  const int32_t* lengths;
  const float* weight_in;
  float* weight_out;
  float* part_o;    // [B][Hkv][rows][nsplit][D]  unnormalised outputs of the splits
  float2* part_ml;  // [B][Hkv][rows][nsplit]     their (reference, sum)
  float2* stat;     // [B][Hkv][weight rows]      (reference, 1 / sum) of the rows that add weight
  float* logit;     // [B][Hkv][weight rows][lpad] their logits (log2), where they are kept
  int Hq, Hkv, G, cap, max_q, max_len, weight_rows;
  int rows;    // max_q * G: rows of a KV head
  int wrows;   // weight_rows * G
  int blocks;  // row blocks
  int nsplit, split_len, lpad;
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

// The rows of one sample that a workgroup or wave deals with.
struct Sample {
  int lo, m, rows, n;
  __device__ __forceinline__ Sample(const AttnParams& p, int b) {
    lo = p.cu[b];
    m = min(p.cu[b + 1] - lo, p.max_q);
    rows = m * p.G;
    n = min(max(p.lengths[b], 0), p.max_len);
  }
  // Keys that row r sees, and the row of q and o that it is.
  __device__ __forceinline__ int seen(const AttnParams& p, int r) const { return max(n - m + r / p.G + 1, 0); }
  __device__ __forceinline__ int64_t qrow(const AttnParams& p, int g, int r) const {
    return (int64_t)(lo + r / p.G) * p.Hq + g * p.G + r % p.G;
  }
};

template <int D, int TERMS>
struct Attn {
  static constexpr int kSteps = D / 32;  // first product: steps of a key tile
  static constexpr int kTiles = D / 16;  // second product: tiles of the output, elements of a key per lane
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

  // The lane's share of 16 keys: D/8 bytes of key col and their scale.
  struct Key {
    uint32_t w[kSteps];
    uint32_t scale;
  };
  template <bool ONCE>
  static __device__ __forceinline__ void load_key(const CacheHead<D>& c, int cap, int k0, int lg, int col, Key& k) {
    const uint8_t* src = c.kc + ((uint32_t)(k0 + col) * (D / 2) + lg * (D / 8));
    typedef uint32_t words __attribute__((ext_vector_type(kSteps)));
    const words* row = reinterpret_cast<const words*>(src);
    const words x = ONCE ? __builtin_nontemporal_load(row) : *row;
#pragma unroll
    for (int t = 0; t < kSteps; ++t) k.w[t] = x[t];
    k.scale = c.ks[(uint32_t)(lg * D / 128) * (uint32_t)cap + k0 + col];
  }
  // Logits (without the scale) of 16 * MT rows against those keys.
  template <int MT>
  static __device__ __forceinline__ void logits(const Key& k, const Rows* f, f32x4* s) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) s[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < kSteps; ++t) {
      const bf16x8 x = decode8(k.w[t], e8m0_scale(k.scale));
#pragma unroll
      for (int n = TERMS - 1; n >= 0; --n)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, f[mt].q[t][n], s[mt], 0, 0, 0);
    }
  }

  // The lane's share of 32 values: elements col*D/16.. of keys 16h + 4lg + i, and
  // the scales of the four keys of each h in one word.
  struct Value {
    uint32_t w[8];
    uint32_t scale[2];
  };
  static __device__ __forceinline__ void load_value(const CacheHead<D>& c, int cap, int k0, int lg, int col, Value& v) {
    const uint32_t row = (uint32_t)(k0 + 4 * lg) * (D / 2) + col * (kTiles / 2);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const uint8_t* src = c.vc + (row + (16 * (kk >> 2) + (kk & 3)) * (D / 2));
      v.w[kk] = D == 128 ? *reinterpret_cast<const uint32_t*>(src) : *reinterpret_cast<const uint16_t*>(src);
    }
    const uint8_t* sc = c.vs + ((uint32_t)(col * kTiles / kCacheBlock) * (uint32_t)cap + k0 + 4 * lg);
    v.scale[0] = *reinterpret_cast<const uint32_t*>(sc);
    v.scale[1] = *reinterpret_cast<const uint32_t*>(sc + 16);
  }
  // O^T += V^T P^T. Two elements of a key come from one byte; pairs of elements of
  // a key become pairs of keys of an element.
  template <int MT>
  static __device__ __forceinline__ void add_values(const Value& v, const bf16x8 (*pf)[TERMS], f32x4 (*acc)[kTiles]) {
    float scale[8];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const uint32_t w = v.scale[kk >> 2];
      const int by = 23 - 8 * (kk & 3);  // the key's byte to the exponent's place
      scale[kk] = __uint_as_float((by >= 0 ? w << by : w >> -by) & 0x7F800000u);
    }
#pragma unroll
    for (int j = 0; j < kTiles / 2; ++j) {
      uint32_t d[8];
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) d[kk] = decode2(v.w[kk], scale[kk], j);
      i32x4 even, odd;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        even[i] = (int)__builtin_amdgcn_perm(d[2 * i + 1], d[2 * i], 0x05040100u);
        odd[i] = (int)__builtin_amdgcn_perm(d[2 * i + 1], d[2 * i], 0x07060302u);
      }
#pragma unroll
      for (int k = TERMS - 1; k >= 0; --k)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          acc[mt][2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), pf[mt][k],
                                                                   acc[mt][2 * j], 0, 0, 0);
          acc[mt][2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), pf[mt][k],
                                                                       acc[mt][2 * j + 1], 0, 0, 0);
        }
    }
  }
};

// What becomes of the logits of the rows that add weight.
enum Keep {
  kForget,    // no weights, or the logits are taken again
  kWorkspace, // kept for the joining kernel
  kLds        // all keys are this workgroup's: kept in LDS, it adds the weights itself
};

// One workgroup: 16 * MT rows of one (sample, KV head) and the keys of one split,
// of which wave w takes steps of 32 keys w, w + 4, ... Each wave keeps its own
// reference, sum and output; they are joined at the end. The reference of a row
// follows its maximum only when a logit exceeds it by kSlack: until then the
// probabilities are at most 2^kSlack, and neither an exchange between lanes nor a
// rescaling of the output is needed.
template <int D, int TERMS, int MT, Keep KEEP, bool ONCE>
__global__ __launch_bounds__(kThreads, TERMS == 1 && MT == 1 ? (KEEP == kLds ? 3 : 4) : 2) void cache4_attn_kernel(AttnParams p) {
  using A = Attn<D, TERMS>;
  constexpr int LD = D + 4;  // row of the joining buffer: 16 rows start in different banks
  __shared__ float s_o[kWaves][16 * LD];
  __shared__ float2 s_ml[kWaves][16];
  const int tid = threadIdx.x, lane = tid & 63, lg = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = blockIdx.x % p.Hkv, rb = blockIdx.x / p.Hkv % p.blocks, split = blockIdx.x / (p.Hkv * p.blocks);
  const int b = blockIdx.y;
  const Sample sm(p, b);
  const int r0 = rb * 16 * MT;
  const int64_t head = (int64_t)b * p.Hkv + g;
  constexpr int kLogitRow = kWhole + 4;
  __shared__ float s_logit[KEEP == kLds ? kKept * kLogitRow : 1];
  __shared__ float2 s_stat[kKept];
  // the weights from s_logit and s_stat, as the joining kernel takes them
  const auto add_weights = [&](int rows) __attribute__((always_inline)) {
    for (int k = tid; k < sm.n; k += kThreads) {
      float w = 0.f;
      for (int r = 0; r < rows; ++r)
        w += k < sm.seen(p, r) ? __builtin_amdgcn_exp2f(s_logit[r * kLogitRow + k] - s_stat[r].x) * s_stat[r].y : 0.f;
      const int64_t at = head * p.cap + k;
      p.weight_out[at] = (p.weight_in ? p.weight_in[at] : 0.f) + w;
    }
  };
  if (r0 >= sm.rows) {
    if (KEEP == kLds) add_weights(0);  // no queries: the weights pass through
    return;
  }
  const int most = sm.seen(p, min(r0 + 16 * MT, sm.rows) - 1);  // keys that the block's last row sees
  const int begin = split * p.split_len, end = min(begin + p.split_len, most);
  if (begin >= end && split > 0) return;
  const int all = sm.seen(p, r0);  // keys that every row of the block sees
  const CacheHead<D> c(p.cache, head, p.cap);

  typename A::Rows f[MT];
  int seen[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = r0 + 16 * mt + col;
    const bool live = r < sm.rows;
    seen[mt] = live ? sm.seen(p, r) : 0;
    A::load_rows(p, live ? sm.qrow(p, g, r) : 0, live, lg, f[mt]);
  }
  f32x4 acc[MT][A::kTiles];
  float ref[MT], sum[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    ref[mt] = -INFINITY;
    sum[mt] = 0.f;
#pragma unroll
    for (int t = 0; t < A::kTiles; ++t) acc[mt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  uint32_t bad = 0;  // row tiles whose lane's outputs are NaN
  typename A::Key kn[2];
  typename A::Value vn;
  int k0 = begin + wave * kKeys;
  if (k0 < end) {
    A::template load_key<ONCE>(c, p.cap, k0, lg, col, kn[0]);
    A::template load_key<ONCE>(c, p.cap, k0 + 16, lg, col, kn[1]);
    A::load_value(c, p.cap, k0, lg, col, vn);
  }
  for (; k0 < end; k0 += kStep) {
    const typename A::Key kc[2] = {kn[0], kn[1]};
    typename A::Value vc = vn;
    if (k0 + kStep < end) {
      A::template load_key<ONCE>(c, p.cap, k0 + kStep, lg, col, kn[0]);
      A::template load_key<ONCE>(c, p.cap, k0 + kStep + 16, lg, col, kn[1]);
      A::load_value(c, p.cap, k0 + kStep, lg, col, vn);
    }
    f32x4 s[2][MT];
    A::template logits<MT>(kc[0], f, s[0]);
    A::template logits<MT>(kc[1], f, s[1]);
    if (KEEP == kLds && col < p.wrows && col < kKept) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<f32x4*>(&s_logit[col * kLogitRow + k0 + 16 * h + 4 * lg]) = s[h][0] * p.scale_log2;
    }
    if (KEEP == kWorkspace) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if (r0 + 16 * mt + col >= p.wrows) continue;
        float* dst = p.logit + (head * p.wrows + r0 + 16 * mt + col) * p.lpad + k0 + 4 * lg;
#pragma unroll
        for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4*>(dst + 16 * h) = s[h][mt] * p.scale_log2;
      }
    }
    if (k0 + kKeys > all) {  // some row does not see some key
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (k0 + 16 * (i >> 2) + 4 * lg + (i & 3) >= seen[mt]) s[i >> 2][mt][i & 3] = -INFINITY;
      // rows behind the length hold anything, and a NaN block may be hidden from
      // some of the rows: both are left out of the product
      bool nan_here = false;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) {
        const int key = k0 + 16 * (kk >> 2) + 4 * lg + (kk & 3);
        const uint32_t ones = 255u << (8 * (kk & 3));
        const bool nan = (vc.scale[kk >> 2] & ones) == ones;
        nan_here |= nan && key < sm.n;
        if (nan || key >= sm.n) vc.scale[kk >> 2] &= ~ones;
      }
      if (__any(nan_here)) {  // but reach the rows that see them
        const uint8_t* sc = c.vs + ((uint32_t)(lg * D / 128) * (uint32_t)p.cap + k0);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll 1
          for (int kk = 0; kk < kKeys; ++kk)
            if (k0 + kk < seen[mt] && sc[kk] == 255u) bad |= 1u << mt;
      }
    }
    bf16x8 pf[MT][TERMS];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s[i >> 2][mt][i & 3];
      // three at a time; a NaN stays one, compares false below, and spoils the sum
      const auto max3 = [](float a, float b, float c) __attribute__((always_inline)) {
        return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
      };
      float top = __builtin_elementwise_maximum(max3(max3(x[0], x[1], x[2]), x[3], x[4]), max3(x[5], x[6], x[7]));
      top *= p.scale_log2;
      if (__any(top > ref[mt] + kSlack)) {
        top = fmaxf(ref[mt], max_xor32(max_xor16(top)));
        // a row without a finite logit so far keeps 0 as its reference: exp2(-inf) = 0
        const float alpha = __builtin_amdgcn_exp2f(ref[mt] - (top == -INFINITY ? 0.f : top));
        ref[mt] = top;
        sum[mt] *= alpha;
#pragma unroll
        for (int t = 0; t < A::kTiles; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[mt][t][i] *= alpha;
      }
      const float base = ref[mt] == -INFINITY ? 0.f : ref[mt];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = __builtin_amdgcn_exp2f(fmaf(x[i], p.scale_log2, -base));
        sum[mt] += e;
        __bf16 z[TERMS];
        split_terms<TERMS>(e, z);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) pf[mt][k][i] = z[k];
      }
    }
    A::template add_values<MT>(vc, pf, acc);
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int t = 0; t < A::kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[mt][t][i] = bad >> mt & 1 ? __builtin_nanf("") : acc[mt][t][i];

  // The waves' parts, 16 rows at a time.
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const float l = sum_xor32(sum_xor16(sum[mt]));
    if (mt > 0) __syncthreads();
    if (lg == 0) s_ml[wave][col] = make_float2(ref[mt], l);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < A::kTiles; t += 4)
        *reinterpret_cast<float4*>(&s_o[wave][col * LD + (4 * lg + i) * A::kTiles + t]) =
            make_float4(acc[mt][t][i], acc[mt][t + 1][i], acc[mt][t + 2][i], acc[mt][t + 3][i]);
    __syncthreads();
    constexpr int TPR = kThreads / 16, EPT = D / TPR;  // threads of a row, elements of a thread
    const int row = tid / TPR, e0 = tid % TPR * EPT, r = r0 + 16 * mt + row;
    if (r >= sm.rows) continue;  // the barriers are outside
    float top = -INFINITY, w[kWaves], all_l = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) top = fmaxf(top, s_ml[k][row].x);
    const float base = top == -INFINITY ? 0.f : top;
    float y[EPT];
#pragma unroll
    for (int e = 0; e < EPT; ++e) y[e] = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      w[k] = __builtin_amdgcn_exp2f(s_ml[k][row].x - base);
      all_l = fmaf(w[k], s_ml[k][row].y, all_l);
#pragma unroll
      for (int e = 0; e < EPT; ++e) y[e] = fmaf(w[k], s_o[k][row * LD + e0 + e], y[e]);
    }
    if (p.nsplit == 1) {
      const bool some = sm.seen(p, r) > 0;
      const float inv = some ? 1.f / all_l : 0.f;  // every logit -inf: 0 * inf, a NaN
      const int64_t at = sm.qrow(p, g, r) * D + e0;
#pragma unroll
      for (int e = 0; e < EPT; ++e) {
        const float z = some ? y[e] * inv : 0.f;
        if constexpr (A::kF32) static_cast<float*>(p.o)[at + e] = z;
        else static_cast<__bf16*>(p.o)[at + e] = (__bf16)z;
      }
      if (e0 == 0 && r < p.wrows) {
        if (KEEP == kLds) s_stat[r] = make_float2(base, inv);
        else if (KEEP == kWorkspace) p.part_ml[head * p.rows + r] = make_float2(top, all_l);
        else p.stat[head * p.wrows + r] = make_float2(base, inv);
      }
    } else {
      const int64_t at = (head * p.rows + r) * p.nsplit + split;
#pragma unroll
      for (int e = 0; e < EPT; ++e) p.part_o[at * D + e0 + e] = y[e];
      if (e0 == 0) p.part_ml[at] = make_float2(top, all_l);
    }
  }
  if (KEEP == kLds) {
    __syncthreads();
    add_weights(min(sm.rows, p.wrows));
  }
}

// Splits of row r that hold a key of its block (at least one: it writes the row).
template <int MT>
__device__ __forceinline__ int live_splits(const AttnParams& p, const Sample& sm, int r) {
  const int r0 = r / (16 * MT) * 16 * MT;
  const int most = sm.seen(p, min(r0 + 16 * MT, sm.rows) - 1);
  return max((most + p.split_len - 1) / p.split_len, 1);
}

// (reference, 1 / sum) of a row over its ns splits, by one wave; the same in every lane.
__device__ __forceinline__ float2 join_stat(const float2* ml, int ns, bool some) {
  const int lane = threadIdx.x & 63;
  float2 x = lane < ns ? ml[lane] : make_float2(-INFINITY, 0.f);
  float top = x.x;
  for (int s = lane + kWave; s < ns; s += kWave) top = fmaxf(top, ml[s].x);
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) top = wave_max_xor(top, k);
  const float base = top == -INFINITY ? 0.f : top;
  float l = __builtin_amdgcn_exp2f(x.x - base) * x.y;
  for (int s = lane + kWave; s < ns; s += kWave) l = fmaf(__builtin_amdgcn_exp2f(ml[s].x - base), ml[s].y, l);
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) l += __shfl_xor(l, k, kWave);
  return make_float2(base, some ? 1.f / l : 0.f);
}

// Four elements of an output row.
template <int TERMS>
__device__ __forceinline__ void store4(void* o, int64_t at, const f32x4& y) {
  if constexpr (TERMS == 3) {
    *reinterpret_cast<f32x4*>(static_cast<float*>(o) + at) = y;
  } else {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(o) + at) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
  }
}

// Two kinds of workgroup. The first `joins` of a KV head (where the keys were
// split) join the splits of rows, a thread 16 bytes of them. Up to kFewSplits splits:
// SLOTS rows a workgroup, a slot of threads each. More: one row, slot k sums splits
// k, k + SLOTS, ..., then the slots are summed in order. The other workgroups (where
// the logits were kept) take the weight of 1024 keys each.
template <int D, int TERMS, int MT>
__global__ __launch_bounds__(kThreads) void cache4_join_kernel(AttnParams p, int joins) {
  constexpr int V4 = D / 4, SLOTS = kThreads / V4, R = kFewSplits;
  const int g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const Sample sm(p, b);
  const int64_t head = (int64_t)b * p.Hkv + g;
  if ((int)blockIdx.x < joins) {
    __shared__ f32x4 s_part[SLOTS][V4];
    const bool few = p.nsplit <= kFewSplits;
    const int slot = tid / V4, c = tid % V4;
    const int r = few ? blockIdx.x * SLOTS + slot : blockIdx.x;
    if (r >= sm.rows) return;  // uniform where there is a barrier below
    const int ns = live_splits<MT>(p, sm, r);
    const bool some = sm.seen(p, r) > 0;
    const int64_t at = (head * p.rows + r) * p.nsplit;
    const float2* ml = p.part_ml + at;
    const f32x4* po = reinterpret_cast<const f32x4*>(p.part_o + at * D);
    const int s0 = few ? 0 : slot, step = few ? 1 : SLOTS;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    // the first of the thread's splits are requested before the sum is known
    f32x4 x[R];
    float2 m[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int s = min(s0 + i * step, ns - 1);
      x[i] = po[s * V4 + c];
      m[i] = ml[s];
    }
    float2 st;
    if (few) {
      float top = m[0].x, l = 0.f;
#pragma unroll
      for (int i = 1; i < R; ++i) top = fmaxf(top, m[i].x);  // repeats of the last split change no maximum
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (i < ns) l = fmaf(__builtin_amdgcn_exp2f(m[i].x - base), m[i].y, l);
      st = make_float2(base, some ? 1.f / l : 0.f);
    } else {
      st = join_stat(ml, ns, some);
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (s0 + i * step < ns) y += __builtin_amdgcn_exp2f(m[i].x - st.x) * x[i];
    if (!few) {
#pragma unroll 4
      for (int s = slot + R * SLOTS; s < ns; s += SLOTS) y += __builtin_amdgcn_exp2f(ml[s].x - st.x) * po[(int64_t)s * V4 + c];
      s_part[slot][c] = y;
      __syncthreads();
      if (slot > 0) return;
#pragma unroll
      for (int k = 1; k < SLOTS; ++k) y += s_part[k][c];
    }
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    store4<TERMS>(p.o, sm.qrow(p, g, r) * D + c * 4, some ? y * st.y : zero);
    if (c == 0 && r < p.wrows) p.stat[head * p.wrows + r] = st;
    return;
  }
  __shared__ float2 s_stat[kKept];
  const int k0 = (((int)blockIdx.x - joins) * kThreads + tid) * 4;
  if (k0 - tid * 4 >= sm.n) return;
  const int rows = min(sm.rows, p.wrows);
  const int64_t at = head * p.cap + k0;
  const bool live = k0 < sm.n;
  const auto vec = [&](const float* q) { return k0 + 4 <= sm.n && (reinterpret_cast<uintptr_t>(q) & 15) == 0; };
  f32x4 w = {0.f, 0.f, 0.f, 0.f}, x[kKept];
  // requested before the statistics; rows that do not see the keys may not have
  // written them: their numbers are not used
#pragma unroll
  for (int r = 0; r < kKept; ++r)
    if (live && r < rows) x[r] = *reinterpret_cast<const f32x4*>(p.logit + (head * p.wrows + r) * p.lpad + k0);
  if (live && p.weight_in) {
    if (vec(p.weight_in)) {
      w = *reinterpret_cast<const f32x4*>(p.weight_in + at);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k0 + i < sm.n) w[i] = p.weight_in[at + i];
    }
  }
  for (int r = tid >> 6; r < rows; r += kWaves) {
    const float2 st = join_stat(p.part_ml + (head * p.rows + r) * p.nsplit, live_splits<MT>(p, sm, r), sm.seen(p, r) > 0);
    if ((tid & 63) == 0) s_stat[r] = st;
  }
  __syncthreads();
  if (!live) return;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int r = 0; r < kKept; ++r) {
    if (r >= rows) break;
    const int seen = sm.seen(p, r);
    const float2 st = s_stat[r];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += k0 + i < seen ? __builtin_amdgcn_exp2f(x[r][i] - st.x) * st.y : 0.f;
  }
  if (vec(p.weight_out)) {
    *reinterpret_cast<f32x4*>(p.weight_out + at) = w + s;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (k0 + i < sm.n) p.weight_out[at + i] = w[i] + s[i];
  }
}

// The same, the logits taken again: a wave has 64 keys, decoded once, and goes
// through the rows 16 at a time, the next ones on their way (36 rows, 8 samples of
// 3200 rows: 16 keys a wave 15.8 us, 64 keys 12.1 us; 64 rows, 4 of 16300: 56 and
// 31 us).
constexpr int kAgainKeys = 64;
template <int D, int TERMS>
__global__ __launch_bounds__(kThreads) void cache4_weight_again_kernel(AttnParams p) {
  using A = Attn<D, TERMS>;
  constexpr int KT = kAgainKeys / 16;
  const int b = blockIdx.z, g = blockIdx.y, lane = threadIdx.x & 63, lg = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Sample sm(p, b);
  const int k0 = (blockIdx.x * kWaves + wave) * kAgainKeys;
  if (k0 >= sm.n) return;
  const int rows = min(sm.rows, p.wrows);
  const int64_t head = (int64_t)b * p.Hkv + g;
  const CacheHead<D> c(p.cache, head, p.cap);
  typename A::Key kn[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t)  // cap is a multiple of 32: the tiles behind it are not there
    A::template load_key<false>(c, p.cap, min(k0 + 16 * t, p.cap - 16), lg, col, kn[t]);
  bf16x8 kf[KT][A::kSteps];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int i = 0; i < A::kSteps; ++i) kf[t][i] = decode8(kn[t].w[i], e8m0_scale(kn[t].scale));
  float w[KT][4];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) w[t][i] = 0.f;

  typename A::Rows next;
  float2 st_next = make_float2(0.f, 0.f);
  const auto request = [&](int r0) __attribute__((always_inline)) {
    const int r = r0 + col;
    const bool live = r < rows;
    A::load_rows(p, live ? sm.qrow(p, g, r) : 0, live, lg, next);
    st_next = live ? p.stat[head * p.wrows + r] : make_float2(0.f, 0.f);
  };
  if (rows > 0) request(0);
  for (int r0 = 0; r0 < rows; r0 += 16) {
    const typename A::Rows f = next;
    const float2 st = st_next;
    if (r0 + 16 < rows) request(r0 + 16);
    const int r = r0 + col;
    const int seen = r < rows ? sm.seen(p, r) : 0;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < A::kSteps; ++i)
#pragma unroll
        for (int n = TERMS - 1; n >= 0; --n) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][i], f.q[i][n], s, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[i], p.scale_log2, -st.x)) * st.y;
        w[t][i] += k0 + 16 * t + 4 * lg + i < seen ? e : 0.f;
      }
    }
  }
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y = row16_sum(w[t][i]);
      const int key = k0 + 16 * t + 4 * lg + i;
      if (col == 0 && key < sm.n) {
        const int64_t at = head * p.cap + key;
        p.weight_out[at] = (p.weight_in ? p.weight_in[at] : 0.f) + y;
      }
    }
}

// Row tiles of a workgroup. Two decode a key once for 32 rows; four would hold 128
// registers of outputs and leave one wave a SIMD (256 queries of 4 heads over 6528
// rows: 2 tiles 46-48 us, 4 tiles 61 us, 1 tile 57 us). While the steps of 16 rows and
// 128 keys do not fill the chip, one tile in twice the workgroups is through sooner
// (5 queries of 4 heads, on the GPU alone: 1500 rows 7.8 us and 9.0 with two tiles;
// 1600 such steps 12.2 and 11.8 us, 3200 17.3 and 13.9), unless two save a launch.
int row_tiles(int64_t rows, int64_t heads, int max_len) {
  if (rows <= 16) return 1;
  if (rows <= 32 && max_len <= kWhole) return 2;
  return heads * ((rows + 15) / 16) * ((max_len + kStep - 1) / kStep) <= 1536 ? 1 : 2;
}

// Keeping the logits of a row costs 8 bytes a key (written and read), taking them
// again D/2 + D/32 bytes a key for all of them, and a launch (8 samples of 3200 rows,
// the whole call: 4 rows 16.1 us kept, 24.1 again; 8 rows 18.7 and 23.8; 12 rows
// 30.1 and 23.9; 4 samples of 16300 rows: 8 rows 28.4 and 43.6, 12 rows 53 and 42).
bool keep_logits(int64_t wrows) { return wrows <= kKept; }

template <int D, int TERMS, int MT>
void launch_mt(const AttnParams& p, int B, const Cache4AttnLayout& lay, hipStream_t stream) {
  const bool keep = lay.keep;
  const dim3 grid(p.Hkv * p.blocks * p.nsplit, B);
  // keys of more caches than the last-level cache holds half of, each read by one
  // workgroup, pass it by (493 MB of 32 samples: 119 -> 113 us with the join; at
  // 3.7 MB, which stay in it, 4.6 -> 5.0 us), unless they are read again for the
  // weights (4 queries, the whole call, past it and through it: 139 MB 82.2 and
  // 80.1 us, 246 MB 136.8 and 134.2, 493 MB 261.7 and 264.2, there with 8 queries
  // 282.7 and 281.5)
  const bool once = (keep || p.wrows == 0) && p.blocks == 1 &&
                    CacheHead<D>::bytes(p.max_len) * p.Hkv * B > ((int64_t)128 << 20);
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, p); };
  if (lay.whole) {
    run(cache4_attn_kernel<D, TERMS, MT, kLds, false>);
    return;
  }
  if (keep) {
    if (once) run(cache4_attn_kernel<D, TERMS, MT, kWorkspace, true>);
    else run(cache4_attn_kernel<D, TERMS, MT, kWorkspace, false>);
  } else {
    if (once) run(cache4_attn_kernel<D, TERMS, MT, kForget, true>);
    else run(cache4_attn_kernel<D, TERMS, MT, kForget, false>);
  }
  const int slots = kThreads / (D / 4);
  const int joins = p.nsplit == 1 ? 0 : p.nsplit <= kFewSplits ? (p.rows + slots - 1) / slots : p.rows;
  const int chunks = keep ? (p.max_len + 4 * kThreads - 1) / (4 * kThreads) : 0;
  if (joins + chunks > 0)
    hipLaunchKernelGGL((cache4_join_kernel<D, TERMS, MT>), dim3(joins + chunks, p.Hkv, B), dim3(kThreads), 0, stream, p,
                       joins);
  if (p.wrows > 0 && !keep)
    hipLaunchKernelGGL((cache4_weight_again_kernel<D, TERMS>),
                       dim3((p.max_len + kWaves * kAgainKeys - 1) / (kWaves * kAgainKeys), p.Hkv, B), dim3(kThreads), 0,
                       stream, p);
}

template <int D>
void launch_d(const AttnParams& p, int dtype, int B, const Cache4AttnLayout& lay, hipStream_t stream) {
  if (dtype == LITEVLM_F32) {
    if (lay.tiles == 1) launch_mt<D, 3, 1>(p, B, lay, stream);
    else launch_mt<D, 3, 2>(p, B, lay, stream);
  } else {
    if (lay.tiles == 1) launch_mt<D, 1, 1>(p, B, lay, stream);
    else launch_mt<D, 1, 2>(p, B, lay, stream);
  }
}

}  // namespace

Cache4AttnLayout cache4_attn_layout(int dtype, int B, int Hq, int Hkv, int D, int max_q, int max_len,
                                    int weight_rows) {
  Cache4AttnLayout lay;
  const int G = Hq / Hkv;
  const int64_t rows = (int64_t)max_q * G, wrows = (int64_t)weight_rows * G, heads = (int64_t)B * Hkv;
  lay.tiles = row_tiles(rows, heads, max_len);
  const int per = 16 * lay.tiles;
  lay.blocks = (int)((rows + per - 1) / per);
  // Splits of whole steps of 128 keys. With one row tile memory is the bound: two
  // workgroups a CU, and splits of at most 512 keys, so that the CUs finish together
  // (32 samples of 10-16K rows: 512 keys 101 us, 1024 106 us, 2048 112 us, 4096 117
  // us). With two the issue of instructions is, and a split's start and end cost more
  // than its keys: one workgroup a CU at D = 128 (8 samples of 3200 rows, 5 queries:
  // 256 workgroups 13.2 us, 512 14.3, 1664 19.5; 256 queries over 6528 rows with the
  // join: 48.5, 49.7, 51.8 us at 256, 512, 768), two at D = 64, whose waves take half
  // the registers (43.0, 36.8, 36.4 us).
  const int64_t groups = std::max<int64_t>(heads * lay.blocks, 1);
  const int64_t steps = std::max((max_len + kStep - 1) / kStep, 1);
  const int64_t aim = per == 16 || D == 64 ? 512 : 256;  // workgroups
  int64_t want = (aim + groups - 1) / groups;
  // at most 16384 workgroups: a part takes 4 * D bytes a row of the workspace
  if (per == 16) want = std::max(want, std::min<int64_t>((steps + 3) / 4, (16384 + groups - 1) / groups));
  want = std::min(want, steps);
  // few keys: one workgroup a head, which adds the weights too, and one launch (8
  // heads, 1 query, in a graph: 128 keys 4.4 us, 7.2 with a join; 512 keys 6.9 and 7.3)
  if (max_len <= kWhole && lay.blocks == 1) want = 1;
  const int64_t each = (steps + want - 1) / want;
  lay.split_len = (int)(each * kStep);
  lay.nsplit = (int)((steps + each - 1) / each);
  lay.lpad = (max_len + kKeys - 1) / kKeys * kKeys;
  const bool weights = weight_rows > 0 && max_len > 0;
  lay.keep = weights && keep_logits(wrows);
  lay.whole = lay.keep && lay.nsplit == 1 && lay.blocks == 1 && max_len <= kWhole;
  const auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const bool logits = lay.keep && !lay.whole;
  const size_t parts = (size_t)heads * rows * lay.nsplit;
  lay.part_o_off = 0;
  lay.part_ml_off = up(lay.nsplit > 1 ? parts * D * sizeof(float) : 0);
  lay.stat_off = lay.part_ml_off + up(lay.nsplit > 1 || logits ? parts * sizeof(float2) : 0);
  lay.logit_off = lay.stat_off + up(weights && !lay.whole ? (size_t)heads * wrows * sizeof(float2) : 0);
  lay.total = lay.logit_off + up(logits ? (size_t)heads * wrows * lay.lpad * sizeof(float) : 0);
  return lay;
}

hipError_t launch_cache4_attn(const Cache4AttnArgs& a, hipStream_t stream) {
  if (a.max_q == 0) return hipSuccess;
  const Cache4AttnLayout lay =
      cache4_attn_layout(a.dtype, a.B, a.Hq, a.Hkv, a.D, a.max_q, a.max_len, a.weight_rows);
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  AttnParams p;
  p.q = a.q;
  p.o = a.o;
  p.cache = static_cast<const uint8_t*>(a.cache);
  p.cu = a.cu_q;
  p.lengths = a.lengths;
  p.weight_in = a.weight_in;
  p.weight_out = a.weight_out;
  p.part_o = reinterpret_cast<float*>(ws + lay.part_o_off);
  p.part_ml = reinterpret_cast<float2*>(ws + lay.part_ml_off);
  p.stat = reinterpret_cast<float2*>(ws + lay.stat_off);
  p.logit = reinterpret_cast<float*>(ws + lay.logit_off);
  p.Hq = a.Hq;
  p.Hkv = a.Hkv;
  p.G = a.Hq / a.Hkv;
  p.cap = a.cap;
  p.max_q = a.max_q;
  p.max_len = a.max_len;
  p.weight_rows = a.weight_rows;
  p.rows = a.max_q * p.G;
  p.wrows = a.max_len > 0 ? a.weight_rows * p.G : 0;
  p.blocks = lay.blocks;
  p.nsplit = lay.nsplit;
  p.split_len = lay.split_len;
  p.lpad = lay.lpad;
  p.scale_log2 = a.scale_log2;
  if (a.D == 128) launch_d<128>(p, a.dtype, a.B, lay, stream);
  else launch_d<64>(p, a.dtype, a.B, lay, stream);
  return hipGetLastError();
}

}  // namespace litevlm
