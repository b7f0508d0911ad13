// Verification of drafted tokens against the target's probabilities.
//
// Draft i is accepted while u_i * q_i(x_i) < p_i(x_i): 24-bit numbers, so the
// product is exact in 64 bits and the decision does not depend on rounding. The
// token behind the accepted ones is drawn by inverting the cumulative sum of
// w = max(p - q, 0) (or p) over the vocabulary, again in 64 bits, where sums of
// fp32 probabilities are exact down to 2^-29 of the total.
//
// What is read is one row of p and one of q: the first kernel sums chunks of them
// (every workgroup takes the acceptance decision, a few numbers, itself), the
// second finds the chunk that holds the r-th part of the sum and the token in it.
// A small vocabulary is one workgroup's.
#include "common.hpp"
#include "launch.hpp"

namespace litevlm {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave, kPer = 8;
constexpr int kChunk = kThreads * kPer;  // vocabulary entries of a workgroup

struct Accepted {
  int a, n;  // accepted drafts, drafts
  int x;     // the refused one's token, -1 if there is none
};

struct VerifyParams {
  const int32_t* draft;
  const int32_t* n_draft;
  const void* target;
  const void* proposal;
  const float* u;
  const float* r;
  const int32_t* lengths;
  int32_t* tokens;
  int32_t* n_accepted;
  int32_t* lengths_out;
  double2* part;  // [B][chunks]: sums of max(p - q, 0) and of p
  Accepted* acc;  // [B]
  int m, V, chunks;
};

template <bool BF16>
__device__ __forceinline__ float prob(const void* base, int64_t i) {
  if constexpr (BF16) return bf16_bits_to_f32(static_cast<const uint16_t*>(base)[i]);
  else return static_cast<const float*>(base)[i];
}

__device__ __forceinline__ double usable(double x) { return x > 0.0 && x < (double)INFINITY ? x : 0.0; }

// The accepted drafts of sample b; every lane of the wave has the result.
template <bool BF16>
__device__ __forceinline__ Accepted accepted(const VerifyParams& p, int b) {
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)b * p.m + min(lane, p.m - 1);
  const int x = p.draft[at];
  const double u = (double)p.u[at];
  const int n = p.n_draft ? min(max(p.n_draft[b], 0), p.m) : p.m;
  bool good = false;
  if (lane < p.m && x >= 0 && x < p.V) {
    const double px = prob<BF16>(p.target, (at + b) * p.V + x);
    const double qx = p.proposal ? prob<BF16>(p.proposal, at * p.V + x) : 1.0;
    good = u * qx < px;
  }
  good = good && lane < n;
  const uint64_t refused = __ballot(!good);
  const int a = min(refused ? (int)__ffsll((unsigned long long)refused) - 1 : 64, n);
  return {a, n, a < n ? __shfl(x, a, kWave) : -1};
}

typedef uint32_t words2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(4)));

// Eight entries of two rows from entry v on, 0 from V on. Rows start at any element:
// the hardware takes vectors at their elements' alignment.
template <bool BF16>
__device__ __forceinline__ void load_probs(const void* pb, int64_t prow, const void* qb, int64_t qrow, int v, int V,
                                           float* x, float* y) {
  if (v + kPer <= V) {
    if constexpr (BF16) {
      const words2 w = *reinterpret_cast<const words2*>(static_cast<const uint16_t*>(pb) + prow + v);
      const words2 z = *reinterpret_cast<const words2*>(static_cast<const uint16_t*>(qb) + qrow + v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        y[2 * i] = __uint_as_float(z[i] << 16);
        y[2 * i + 1] = __uint_as_float(z[i] & 0xFFFF0000u);
      }
    } else {
      const words4* wp = reinterpret_cast<const words4*>(static_cast<const float*>(pb) + prow + v);
      const words4* zp = reinterpret_cast<const words4*>(static_cast<const float*>(qb) + qrow + v);
      const words4 w[2] = {wp[0], wp[1]}, z[2] = {zp[0], zp[1]};
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        x[i] = __uint_as_float(w[i >> 2][i & 3]);
        y[i] = __uint_as_float(z[i >> 2][i & 3]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      x[i] = v + i < V ? prob<BF16>(pb, prow + v + i) : 0.f;
      y[i] = v + i < V ? prob<BF16>(qb, qrow + v + i) : 0.f;
    }
  }
}

// Weights of eight entries: d from the difference (or, all accepted, from p), t from
// p. Both rows are requested together; without q it is p's again, not used.
template <bool BF16>
__device__ __forceinline__ void weights(const VerifyParams& p, int b, const Accepted& ac, int v, double* d, double* t) {
  const bool rest = ac.a < ac.n, both = rest && p.proposal;
  const int64_t trow = ((int64_t)b * (p.m + 1) + ac.a) * p.V, qrow = ((int64_t)b * p.m + ac.a) * p.V;
  float pv[kPer], qv[kPer];
  load_probs<BF16>(p.target, trow, both ? p.proposal : p.target, both ? qrow : trow, v, p.V, pv, qv);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const float q = both ? qv[i] : rest && v + i == ac.x ? 1.f : 0.f;
    d[i] = usable((double)pv[i] - (double)q);
    t[i] = usable((double)pv[i]);
  }
}

// x of the lane that CTRL names, 0 where there is none or ROWS leaves the row out.
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp64(double x) {
  const long long u = __double_as_longlong(x);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)u, CTRL, ROWS, 0xF, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xF, false);
  return __longlong_as_double(((long long)hi << 32) | (uint32_t)lo);
}

__device__ __forceinline__ double readlane64(double x, int lane) {
  const long long u = __double_as_longlong(x);
  const int lo = __builtin_amdgcn_readlane((int)u, lane), hi = __builtin_amdgcn_readlane((int)(u >> 32), lane);
  return __longlong_as_double(((long long)hi << 32) | (uint32_t)lo);
}

// Inclusive sum over the wave's lanes in order: within rows of 16 lanes, then the
// row before (last lane of rows 0 and 2 to rows 1 and 3), then the half before.
__device__ __forceinline__ double wave_scan(double x) {
  x += dpp64<0x111, 0xF>(x);  // row_shr 1
  x += dpp64<0x112, 0xF>(x);
  x += dpp64<0x114, 0xF>(x);
  x += dpp64<0x118, 0xF>(x);
  x += dpp64<0x142, 0xA>(x);  // row_bcast 15
  x += dpp64<0x143, 0xC>(x);  // row_bcast 31
  return x;
}

// Inclusive sums of x and y over the workgroup's threads in order, and their totals.
__device__ __forceinline__ void scan2(double2& x, double2* s_wave, double2& all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  x.x = wave_scan(x.x);
  x.y = wave_scan(x.y);
  __syncthreads();
  if (lane == kWave - 1) s_wave[w] = x;
  __syncthreads();
  double2 before = make_double2(0.0, 0.0);
  all = before;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    const double2 z = s_wave[k];
    if (k < w) {
      before.x += z.x;
      before.y += z.y;
    }
    all.x += z.x;
    all.y += z.y;
  }
  x.x += before.x;
  x.y += before.y;
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void verify_sum_kernel(VerifyParams p) {
  __shared__ double2 s_wave[kWaves];
  const int b = blockIdx.y, c = blockIdx.x;
  const Accepted ac = accepted<BF16>(p, b);
  double d[kPer], t[kPer];
  weights<BF16>(p, b, ac, c * kChunk + threadIdx.x * kPer, d, t);
  double2 s = make_double2(0.0, 0.0), all;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    s.x += d[i];
    s.y += t[i];
  }
  scan2(s, s_wave, all);
  if (threadIdx.x == 0) {
    p.part[(int64_t)b * p.chunks + c] = all;
    if (c == 0) p.acc[b] = ac;
  }
}

// The first thread's `first` that is not `none` and the last thread's `last` that is
// not -1, over the workgroup (both ascend with the thread).
__device__ __forceinline__ int2 find(int first, int last, int none, int2* s_found) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint64_t fm = __ballot(first != none), lm = __ballot(last >= 0);
  const int f = fm ? __builtin_amdgcn_readlane(first, __ffsll((unsigned long long)fm) - 1) : none;
  const int l = lm ? __builtin_amdgcn_readlane(last, 63 - __clzll((long long)lm)) : -1;
  if (lane == 0) s_found[w] = make_int2(f, l);
  __syncthreads();
  int2 all = s_found[0];
#pragma unroll
  for (int k = 1; k < kWaves; ++k) {
    const int2 z = s_found[k];
    if (all.x == none) all.x = z.x;
    if (z.y >= 0) all.y = z.y;
  }
  return all;
}

// One workgroup a sample: the chunk, then the entry, whose cumulative sum passes
// the goal. Each thread has `per` consecutive chunks, then 8 consecutive entries;
// the sums are those of the first kernel to the bit.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void verify_draw_kernel(VerifyParams p) {
  __shared__ double2 s_wave[kWaves];
  __shared__ int2 s_found[2][kWaves];
  __shared__ double s_before;
  const int b = blockIdx.x, tid = threadIdx.x;
  const Accepted ac = p.acc[b];
  const double2* part = p.part + (int64_t)b * p.chunks;
  const double r = (double)p.r[b];
  const int drafted = tid < p.m ? p.draft[(int64_t)b * p.m + tid] : -1;
  const int length = p.lengths ? p.lengths[b] : 0;
  if (tid == 0) s_before = 0.0;
  const int per = (p.chunks + kThreads - 1) / kThreads;
  double2 s = make_double2(0.0, 0.0), all;
  for (int i = 0; i < per; ++i) {
    const int c = tid * per + i;
    if (c < p.chunks) {
      s.x += part[c].x;
      s.y += part[c].y;
    }
  }
  const double2 own = s;
  scan2(s, s_wave, all);
  const bool diff = all.x > 0.0;  // else p itself
  const double total = diff ? all.x : all.y, goal = r * total;
  // chunks of this thread whose end passes the goal, and the last that holds anything
  double run = diff ? s.x - own.x : s.y - own.y;
  int first = p.chunks, last = -1;
  double before = 0.0;
  for (int i = 0; i < per; ++i) {
    const int c = tid * per + i;
    double2 z = own;
    if (per > 1) z = c < p.chunks ? part[c] : make_double2(0.0, 0.0);
    const double w = diff ? z.x : z.y;
    if (w > 0.0) {
      last = c;
      if (first == p.chunks && run + w > goal) {
        first = c;
        before = run;
      }
    }
    run += w;
  }
  int2 found = find(first, last, p.chunks, s_found[0]);
  const bool beyond = found.x >= p.chunks;  // no chunk: the last weight there is
  const int chunk = beyond ? found.y : found.x;
  if (!beyond && first == chunk) s_before = before;  // read behind the next barriers
  int token = -1;
  if (chunk >= 0) {  // uniform
    const int v0 = chunk * kChunk + tid * kPer;
    double d[kPer], t[kPer];
    weights<BF16>(p, b, ac, v0, d, t);
    double2 z = make_double2(0.0, 0.0);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (!diff) d[i] = t[i];
      z.x += d[i];
    }
    const double mine = z.x;
    scan2(z, s_wave, all);
    run = s_before + (z.x - mine);
    first = p.V;
    last = -1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      run += d[i];
      if (d[i] > 0.0) {
        last = v0 + i;
        if (first == p.V && run > goal) first = v0 + i;
      }
    }
    found = find(beyond ? p.V : first, last, p.V, s_found[1]);
    token = found.x < p.V ? found.x : found.y;
  }
  if (tid <= p.m) p.tokens[(int64_t)b * (p.m + 1) + tid] = tid < ac.a ? drafted : tid == ac.a ? token : -1;
  if (tid == 0) {
    p.n_accepted[b] = ac.a;
    if (p.lengths) p.lengths_out[b] = length - (ac.n - ac.a);
  }
}

// A whole sample: up to four tiles of 8192 entries, eight a thread. The first wave
// finds the part (a tile's 512 entries of one wave) that passes the goal, the wave
// that has it looks at it again.
constexpr int kOneThreads = 1024, kOneWaves = kOneThreads / kWave, kOneTile = kOneThreads * kPer;
constexpr int kOneTiles = kWave / kOneWaves;
template <bool BF16>
__global__ __launch_bounds__(kOneThreads) void verify_one_kernel(VerifyParams p) {
  __shared__ double2 s_part[kWave];
  __shared__ double s_before, s_goal;
  __shared__ int s_at, s_token;
  __shared__ bool s_diff, s_beyond;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const Accepted ac = accepted<BF16>(p, b);
  const double r = (double)p.r[b];
  const int drafted = tid < p.m ? p.draft[(int64_t)b * p.m + tid] : -1;
  const int length = p.lengths ? p.lengths[b] : 0;
  const int tiles = (p.V + kOneTile - 1) / kOneTile;
  double2 sums[kOneTiles];
#pragma unroll
  for (int k = 0; k < kOneTiles; ++k) {
    sums[k] = make_double2(0.0, 0.0);
    if (k >= tiles) continue;  // uniform
    double d[kPer], t[kPer];
    weights<BF16>(p, b, ac, k * kOneTile + tid * kPer, d, t);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      sums[k].x += d[i];
      sums[k].y += t[i];
    }
  }
#pragma unroll
  for (int k = 0; k < kOneTiles; ++k) {
    const double2 s = make_double2(wave_scan(sums[k].x), wave_scan(sums[k].y));
    if (lane == kWave - 1) s_part[k * kOneWaves + w] = s;
  }
  __syncthreads();
  if (w == 0) {
    const double2 own = s_part[lane];
    double2 s = make_double2(wave_scan(own.x), wave_scan(own.y));
    const double dall = readlane64(s.x, kWave - 1), tall = readlane64(s.y, kWave - 1);
    const bool diff = dall > 0.0;  // else p itself
    const double goal = r * (diff ? dall : tall), end = diff ? s.x : s.y, part = diff ? own.x : own.y;
    const uint64_t passes = __ballot(part > 0.0 && end > goal), any = __ballot(part > 0.0);
    const int at = passes ? __ffsll((unsigned long long)passes) - 1 : any ? 63 - __clzll((long long)any) : -1;
    const double before = readlane64(end, max(at - 1, 0));
    if (lane == 0) {
      s_at = at;
      s_before = at > 0 ? before : 0.0;
      s_goal = goal;
      s_diff = diff;
      s_beyond = passes == 0;  // no part: the last weight there is
      s_token = -1;
    }
  }
  __syncthreads();
  const int at = s_at;
  if (at >= 0 && w == at % kOneWaves) {
    const int v0 = at / kOneWaves * kOneTile + tid * kPer;
    double d[kPer], t[kPer], s = 0.0;
    weights<BF16>(p, b, ac, v0, d, t);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (!s_diff) d[i] = t[i];
      s += d[i];
    }
    double run = s_before + dpp64<0x138, 0xF>(wave_scan(s));  // of the lanes in front
    int first = p.V, last = -1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      run += d[i];
      if (d[i] > 0.0) {
        last = v0 + i;
        if (first == p.V && run > s_goal) first = v0 + i;
      }
    }
    const uint64_t fm = s_beyond ? 0 : __ballot(first != p.V), lm = __ballot(last >= 0);
    const int token = fm   ? __builtin_amdgcn_readlane(first, __ffsll((unsigned long long)fm) - 1)
                      : lm ? __builtin_amdgcn_readlane(last, 63 - __clzll((long long)lm))
                           : -1;
    if (lane == 0) s_token = token;
  }
  __syncthreads();
  if (tid <= p.m) p.tokens[(int64_t)b * (p.m + 1) + tid] = tid < ac.a ? drafted : tid == ac.a ? s_token : -1;
  if (tid == 0) {
    p.n_accepted[b] = ac.a;
    if (p.lengths) p.lengths_out[b] = length - (ac.n - ac.a);
  }
}

template <bool BF16>
void launch(const VerifyParams& p, int B, bool one, hipStream_t stream) {
  // One launch up to the 64 parts that one wave scans, 32768 entries. The time of a
  // program that launches call by call decides: 9.3-9.8 us a call for 8000 to 32000
  // entries, 13.8-14.2 with two launches and the workspace that they need, at batches
  // of 1, 16 and 64 alike. In a graph the two are within 1.5 us: 8000 entries 5.6-6.1
  // and 6.7-7.4 us, 16000 6.4-7.0 and 6.7-8.0, 24000 7.4-8.7 and 6.8-8.8, 32000
  // 8.3-9.8 and 6.9-9.5 (batch 1-64).
  if (one) {
    hipLaunchKernelGGL(verify_one_kernel<BF16>, dim3(B), dim3(kOneThreads), 0, stream, p);
  } else {
    hipLaunchKernelGGL(verify_sum_kernel<BF16>, dim3(p.chunks, B), dim3(kThreads), 0, stream, p);
    hipLaunchKernelGGL(verify_draw_kernel<BF16>, dim3(B), dim3(kThreads), 0, stream, p);
  }
}

}  // namespace

VerifyLayout verify_layout(int B, int V) {
  VerifyLayout lay;
  lay.chunks = (V + kChunk - 1) / kChunk;
  lay.acc_off = (size_t)B * lay.chunks * sizeof(double2);
  lay.one = V <= kOneTiles * kOneTile;
  lay.total = lay.one ? 0 : lay.acc_off + (size_t)B * sizeof(Accepted);
  return lay;
}

hipError_t launch_verify_draft(const VerifyArgs& a, hipStream_t stream) {
  const VerifyLayout lay = verify_layout(a.B, a.V);
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  VerifyParams p;
  p.draft = a.draft;
  p.n_draft = a.n_draft;
  p.target = a.target;
  p.proposal = a.proposal;
  p.u = a.u;
  p.r = a.r;
  p.lengths = a.lengths;
  p.tokens = a.tokens;
  p.n_accepted = a.n_accepted;
  p.lengths_out = a.lengths_out;
  p.part = reinterpret_cast<double2*>(ws);
  p.acc = reinterpret_cast<Accepted*>(ws + lay.acc_off);
  p.m = a.max_draft;
  p.V = a.V;
  p.chunks = lay.chunks;
  if (a.dtype == LITEVLM_BF16) launch<true>(p, a.B, lay.one, stream);
  else launch<false>(p, a.B, lay.one, stream);
  return hipGetLastError();
}

}  // namespace litevlm
