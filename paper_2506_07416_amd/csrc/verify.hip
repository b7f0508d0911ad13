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
#include "common.hpp"
#include "launch.hpp"

namespace litevlm {
namespace {

constexpr int kThreads = 256, kPer = 16;
constexpr int kChunk = kThreads * kPer;

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
  int m, V, chunks;
};

template <bool BF16>
__device__ __forceinline__ float prob(const void* base, int64_t i) {
  if constexpr (BF16) return bf16_bits_to_f32(static_cast<const uint16_t*>(base)[i]);
  else return static_cast<const float*>(base)[i];
}

__device__ __forceinline__ double usable(double x) { return x > 0.0 && x < (double)INFINITY ? x : 0.0; }

struct Accepted {
  int a, n;  // accepted drafts, drafts
};

// The accepted drafts of sample b; every lane of the wave has the result.
template <bool BF16>
__device__ __forceinline__ Accepted accepted(const VerifyParams& p, int b) {
  const int lane = threadIdx.x & 63;
  const int n = p.n_draft ? min(max(p.n_draft[b], 0), p.m) : p.m;
  bool good = false;
  if (lane < n) {
    const int x = p.draft[(int64_t)b * p.m + lane];
    if (x >= 0 && x < p.V) {
      const double px = prob<BF16>(p.target, ((int64_t)b * (p.m + 1) + lane) * p.V + x);
      const double qx = p.proposal ? prob<BF16>(p.proposal, ((int64_t)b * p.m + lane) * p.V + x) : 1.0;
      good = (double)p.u[(int64_t)b * p.m + lane] * qx < px;
    }
  }
  const uint64_t refused = __ballot(!good);
  return {min(refused ? (int)__ffsll((unsigned long long)refused) - 1 : 64, n), n};
}

// The weights of vocabulary entry v: (difference, target).
template <bool BF16>
struct Row {
  const VerifyParams& p;
  int64_t t, q;
  bool rest;
  int x;
  __device__ __forceinline__ Row(const VerifyParams& p_, int b, const Accepted& ac) : p(p_) {
    rest = ac.a < ac.n;
    t = ((int64_t)b * (p.m + 1) + ac.a) * p.V;
    q = ((int64_t)b * p.m + ac.a) * p.V;
    x = rest ? p.draft[(int64_t)b * p.m + ac.a] : -1;
  }
  __device__ __forceinline__ double2 at(int v) const {
    const double pv = prob<BF16>(p.target, t + v);
    double d = pv;
    if (rest) d = pv - (p.proposal ? (double)prob<BF16>(p.proposal, q + v) : v == x ? 1.0 : 0.0);
    return make_double2(usable(d), usable(pv));
  }
};

__device__ __forceinline__ double shfl_up64(double x, int by) {
  const long long u = __double_as_longlong(x);
  const int lo = __shfl_up((int)u, by, kWave), hi = __shfl_up((int)(u >> 32), by, kWave);
  return __longlong_as_double(((long long)hi << 32) | (uint32_t)lo);
}

// Inclusive sum over the workgroup's threads in order; total in `all`.
__device__ __forceinline__ double scan(double x, double* s_wave, double& all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) {
    const double y = shfl_up64(x, k);
    if (lane >= k) x += y;
  }
  __syncthreads();
  if (lane == kWave - 1) s_wave[w] = x;
  __syncthreads();
  double before = 0.0;
  all = 0.0;
  for (int k = 0; k < kThreads / kWave; ++k) {
    if (k < w) before += s_wave[k];
    all += s_wave[k];
  }
  return x + before;
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void verify_sum_kernel(VerifyParams p) {
  __shared__ double s_wave[kThreads / kWave];
  const int b = blockIdx.y, c = blockIdx.x;
  const Row<BF16> row(p, b, accepted<BF16>(p, b));
  const int v0 = c * kChunk + threadIdx.x * kPer;
  double d = 0.0, t = 0.0;
  for (int i = 0; i < kPer; ++i) {
    if (v0 + i < p.V) {
      const double2 w = row.at(v0 + i);
      d += w.x;
      t += w.y;
    }
  }
  double dall, tall;
  scan(d, s_wave, dall);
  scan(t, s_wave, tall);
  if (threadIdx.x == 0) p.part[(int64_t)b * p.chunks + c] = make_double2(dall, tall);
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void verify_draw_kernel(VerifyParams p) {
  __shared__ double s_wave[kThreads / kWave];
  __shared__ int s_chunk, s_last, s_token, s_token_last;
  __shared__ double s_before;
  const int b = blockIdx.x, tid = threadIdx.x;
  const Accepted ac = accepted<BF16>(p, b);
  const Row<BF16> row(p, b, ac);
  const double2* part = p.part + (int64_t)b * p.chunks;
  // totals
  double d = 0.0, t = 0.0, dall, tall;
  for (int c = tid; c < p.chunks; c += kThreads) {
    d += part[c].x;
    t += part[c].y;
  }
  scan(d, s_wave, dall);
  scan(t, s_wave, tall);
  const bool diff = dall > 0.0;
  const double goal = (double)p.r[b] * (diff ? dall : tall);
  if (tid == 0) {
    s_chunk = p.chunks;
    s_last = -1;
    s_token = p.V;
    s_token_last = -1;
  }
  __syncthreads();
  // the first chunk whose end lies beyond the goal, and the last that holds anything
  double base = 0.0;
  for (int c0 = 0; c0 < p.chunks; c0 += kThreads) {
    const int c = c0 + tid;
    const double x = c < p.chunks ? (diff ? part[c].x : part[c].y) : 0.0;
    double all;
    const double end = base + scan(x, s_wave, all);
    if (x > 0.0) {
      atomicMax(&s_last, c);
      if (end > goal) atomicMin(&s_chunk, c);
    }
    base += all;
  }
  __syncthreads();
  const bool beyond = s_chunk >= p.chunks;  // no chunk: the last weight there is
  const int chunk = beyond ? s_last : s_chunk;
  int token = -1;
  if (chunk >= 0) {  // uniform
    base = 0.0;
    for (int c0 = 0; c0 <= chunk; c0 += kThreads) {
      const int c = c0 + tid;
      const double x = c < chunk ? (diff ? part[c].x : part[c].y) : 0.0;
      double all;
      const double end = base + scan(x, s_wave, all);
      if (c == chunk) s_before = end;
      base += all;
    }
    __syncthreads();
    const int v0 = chunk * kChunk + tid * kPer;
    double w[kPer], own = 0.0, all;
    for (int i = 0; i < kPer; ++i) {
      w[i] = 0.0;
      if (v0 + i < p.V) {
        const double2 z = row.at(v0 + i);
        w[i] = diff ? z.x : z.y;
      }
      own += w[i];
    }
    double run = s_before + (scan(own, s_wave, all) - own);
    for (int i = 0; i < kPer; ++i) {
      run += w[i];
      if (w[i] > 0.0) {
        atomicMax(&s_token_last, v0 + i);
        if (!beyond && run > goal) atomicMin(&s_token, v0 + i);
      }
    }
    __syncthreads();
    token = s_token < p.V ? s_token : s_token_last;
  }
  if (tid <= p.m)
    p.tokens[(int64_t)b * (p.m + 1) + tid] = tid < ac.a ? p.draft[(int64_t)b * p.m + tid] : tid == ac.a ? token : -1;
  if (tid == 0) {
    p.n_accepted[b] = ac.a;
    if (p.lengths) p.lengths_out[b] = p.lengths[b] - (ac.n - ac.a);
  }
}

}  // namespace

VerifyLayout verify_layout(int B, int V) {
  VerifyLayout lay;
  lay.chunks = (V + kChunk - 1) / kChunk;
  lay.total = (size_t)B * lay.chunks * sizeof(double2);
  return lay;
}

hipError_t launch_verify_draft(const VerifyArgs& a, hipStream_t stream) {
  const VerifyLayout lay = verify_layout(a.B, a.V);
  const VerifyParams p{a.draft, a.n_draft,    a.target,      a.proposal,
                       a.u,     a.r,          a.lengths,     a.tokens,
                       a.n_accepted, a.lengths_out, static_cast<double2*>(a.workspace), a.max_draft,
                       a.V,     lay.chunks};
  const dim3 grid(lay.chunks, a.B);
  if (a.dtype == LITEVLM_BF16) {
    hipLaunchKernelGGL(verify_sum_kernel<true>, grid, dim3(kThreads), 0, stream, p);
    hipLaunchKernelGGL(verify_draw_kernel<true>, dim3(a.B), dim3(kThreads), 0, stream, p);
  } else {
    hipLaunchKernelGGL(verify_sum_kernel<false>, grid, dim3(kThreads), 0, stream, p);
    hipLaunchKernelGGL(verify_draw_kernel<false>, dim3(a.B), dim3(kThreads), 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace litevlm
