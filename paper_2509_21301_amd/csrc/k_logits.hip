// Log probabilities from rows of logits: of given tokens, the entropy of the distribution, and the most
// likely tokens.  With m the row's maximum, S = sum e^(x - m) and T = sum e^(x - m) (x - m):
//   log p_t = x_t - m - log S,   entropy = log S - T / S,
// sums in fp32 over parts of the row whose lanes keep a maximum of their own, so every e^(x - m) is at
// most 1 and T / S loses nothing to cancellation.  The logits are read once; bound by HBM for a batch
// of vocabulary rows, by launches and latency for one.
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"

namespace nova {

constexpr int LP_EPL = 32;                 // logits of a lane at a time
constexpr int LP_CHUNK = 64 * LP_EPL;      // of a wave
constexpr int LP_MAX_PARTS = 1024;
constexpr int LP_MAX_TOP = 32;

// An unsigned number that orders as the values do: -0 equals 0, NaN is above infinity; 0 is no value's.
NOVA_DEV uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  if (x != x) return 0xFFFFFFFFu;
  return (u >> 31) ? ~u : u | 0x80000000u;
}
NOVA_DEV float key_value(uint32_t k) { return __uint_as_float((k >> 31) ? k & 0x7FFFFFFFu : ~k); }
// Larger first, equal values by the lower id.
NOVA_DEV unsigned long long rank_key(uint32_t key, int id) { return ((unsigned long long)key << 32) | (0xFFFFFFFFu - (uint32_t)id); }

template <typename T> NOVA_DEV void load_logits(const T* row, int i0, int vocab, float* x) {
  constexpr int N = 16 / sizeof(T);        // i0: the lane's first logit, N of them
  if (i0 + N <= vocab && ((uintptr_t)(row + i0) & 15) == 0) {
    const uint4 w = *reinterpret_cast<const uint4*>(row + i0);
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < N; ++e)
      x[e] = sizeof(T) == 4 ? __uint_as_float(a[e]) : __uint_as_float((e & 1) ? a[e / 2] & 0xFFFF0000u : a[e / 2] << 16);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = i0 + e < vocab ? to_f<T>(row[i0 + e]) : -INFINITY;
  }
}

// m, S, T of two sets of logits together.
struct LogSum { float m, s, t; };
NOVA_DEV LogSum log_sum_join(const LogSum& a, float m) {
  // a's sums taken to the maximum m >= a.m
  if (a.m == m || a.s == 0.f) return LogSum{m, a.s, a.t};
  const float d = a.m - m, f = __expf(d);
  return LogSum{m, f * a.s, f > 0.f ? f * (a.t + d * a.s) : 0.f * a.t};
}
NOVA_DEV LogSum log_sum_wave(const LogSum& a) {
  const float m = wave_max(a.m);
  const LogSum j = log_sum_join(a, m);
  return LogSum{m, wave_sum(j.s), wave_sum(j.t)};
}

// The k largest keys of a wave's values, sorted, to out[0 .. k) (0 where there are fewer).  x: the lane's
// values, idx(j): the id of its j-th (-1: none).  The k-th largest of the lanes' maxima bounds the k-th
// largest value from below and is found by bisection with ballots; the values that reach it (k or a few
// more) are packed into LDS and ranked by counting.  With too many equal ones, k rounds of a wave maximum.
template <typename F>
NOVA_DEV void wave_top(const uint32_t (&key)[LP_EPL], F idx, int k, unsigned long long* sm, unsigned long long* out) {
  const int lane = threadIdx.x & 63;
  uint32_t best = 0;
#pragma unroll
  for (int j = 0; j < LP_EPL; ++j) best = max(best, key[j]);
  uint32_t tau = 0;                        // largest number that at least k lanes' maxima reach
#pragma unroll 1
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t trial = tau | (1u << bit);
    const int c = __popcll(__ballot(best >= trial));
    if (c >= k) tau = trial;
    if (c == k) break;
  }
  tau = max(tau, 1u);
  int n = 0;
#pragma unroll
  for (int j = 0; j < LP_EPL; ++j) n += __popcll(__ballot(key[j] >= tau));
  if (n <= 64) {
    int at = 0;
#pragma unroll
    for (int j = 0; j < LP_EPL; ++j) {
      const unsigned long long m = __ballot(key[j] >= tau);
      if (key[j] >= tau) sm[at + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0))] = rank_key(key[j], idx(j));
      at += __popcll(m);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const unsigned long long mine = lane < n ? sm[lane] : 0;
    int rank = 0;
    for (int i = 0; i < n; ++i) rank += sm[i] > mine;
    if (lane < n && rank < k) out[rank] = mine;
    if (lane >= n && lane < k) out[lane] = 0;
    return;
  }
  unsigned long long last = ~0ull;
#pragma unroll 1
  for (int r = 0; r < k; ++r) {
    unsigned long long top = 0;
#pragma unroll
    for (int j = 0; j < LP_EPL; ++j) {
      const unsigned long long c = key[j] ? rank_key(key[j], idx(j)) : 0;
      if (c < last && c > top) top = c;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      const unsigned long long c = __shfl_xor(top, o, 64);
      top = c > top ? c : top;
    }
    if (lane == 0) out[r] = top;
    if (top) last = top;                   // 0: every value is taken, and the rest of the list is 0
    else last = 0;
  }
}

// Wave (part of a row): chunks of 2048 logits, 32 per lane in registers; one chunk with n_top > 0.
template <typename T>
__global__ void __launch_bounds__(256) logprobs_part_kernel(LogprobArgs p, int parts, int chunks) {
  constexpr int N = 16 / sizeof(T);
  __shared__ unsigned long long sm[4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long unit = (long)blockIdx.x * 4 + wave;
  if (unit >= (long)p.rows * parts) return;
  const int r = (int)(unit / parts), part = (int)(unit % parts);
  const T* row = reinterpret_cast<const T*>(p.logits) + r * p.stride;
  LogSum a{-INFINITY, 0.f, 0.f};
  for (int c = 0; c < chunks; ++c) {
    const long c0 = ((long)part * chunks + c) * LP_CHUNK;
    if (c0 >= p.vocab) break;
    float x[LP_EPL];
#pragma unroll
    for (int j = 0; j < LP_EPL; j += N) load_logits(row, (int)min(c0 + j * 64 + lane * N, (long)p.vocab), p.vocab, x + j);
    float m = a.m;
#pragma unroll
    for (int j = 0; j < LP_EPL; ++j) m = fmaxf(m, x[j]);
    a = log_sum_join(a, m);
    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int j = 0; j < LP_EPL; ++j) {
      const float d = x[j] - mu, e = __expf(d);
      a.s += e;
      a.t += e == 0.f ? 0.f : e * d;
    }
    if (p.n_top > 0) {
      uint32_t key[LP_EPL];
      auto idx = [&](int j) { return (int)(c0 + (j / N) * N * 64 + lane * N + j % N); };
#pragma unroll
      for (int j = 0; j < LP_EPL; ++j) key[j] = idx(j) < p.vocab ? order_key(x[j]) : 0;
      wave_top(key, idx, p.n_top, sm[wave], p.part_top + unit * p.n_top);
    }
  }
  a = log_sum_wave(a);
  if (lane == 0) reinterpret_cast<float4*>(p.part_sum)[unit] = make_float4(a.m, a.s, a.t, 0.f);
}

// Workgroup (row): the parts' sums joined, the given tokens' log probabilities, and the parts' sorted lists
// merged: the k-th largest of their first entries bounds the k-th of all from below, so at most k lists
// have entries that reach it; those are ranked by counting.
template <typename T>
__global__ void __launch_bounds__(256) logprobs_row_kernel(LogprobArgs p, int parts) {
  __shared__ unsigned long long head[LP_MAX_PARTS], cand[LP_MAX_TOP * LP_MAX_TOP];
  __shared__ float sm_m[4], sm_s[4], sm_t[4];
  __shared__ unsigned long long tau;
  __shared__ int n_cand;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = p.n_top;
  const unsigned long long* lists = p.part_top + (long)r * parts * k;
  if (tid == 0) { tau = 1; n_cand = 0; }
  LogSum a{-INFINITY, 0.f, 0.f};
  for (int i = tid; i < parts; i += 256) {
    const float4 v = reinterpret_cast<const float4*>(p.part_sum)[(long)r * parts + i];
    const LogSum b{v.x, v.y, v.z};
    const float m = fmaxf(a.m, b.m);
    const LogSum x = log_sum_join(a, m), y = log_sum_join(b, m);
    a = LogSum{m, x.s + y.s, x.t + y.t};
    if (k > 0) head[i] = lists[(long)i * k];
  }
  a = log_sum_wave(a);
  if (lane == 0) { sm_m[wave] = a.m; sm_s[wave] = a.s; sm_t[wave] = a.t; }
  __syncthreads();
  const float m = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
  LogSum z{m, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const LogSum j = log_sum_join(LogSum{sm_m[w], sm_s[w], sm_t[w]}, m);
    z.s += j.s;
    z.t += j.t;
  }
  // nothing but -infinity: no distribution
  const float log_s = z.s == 0.f ? __uint_as_float(0x7FC00000u) : logf(z.s);
  if (tid == 0 && p.entropy) p.entropy[r] = log_s - z.t / z.s;
  const T* row = reinterpret_cast<const T*>(p.logits) + r * p.stride;
  for (int i = tid; i < p.n_given; i += 256) {
    const int id = p.given[(long)r * p.n_given + i];
    p.given_lp[(long)r * p.n_given + i] = (unsigned)id < (unsigned)p.vocab ? to_f<T>(row[id]) - m - log_s : -INFINITY;
  }
  if (k == 0) return;
  if (parts >= k) {
    for (int i = tid; i < parts; i += 256) {
      const unsigned long long h = head[i];
      int rank = 0;
      for (int j = 0; j < parts; ++j) rank += head[j] > h;
      if (rank == k - 1 && h > 0) tau = h;
    }
  }
  __syncthreads();
  for (int i = tid; i < parts; i += 256) {
    if (head[i] < tau) continue;
    for (int j = 0; j < k; ++j) {
      const unsigned long long c = lists[(long)i * k + j];
      if (c < tau) break;
      cand[atomicAdd(&n_cand, 1)] = c;
    }
  }
  __syncthreads();
  const int n = n_cand;
  for (int i = tid; i < n; i += 256) {
    const unsigned long long c = cand[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += cand[j] > c;
    if (rank < k) {
      p.top_lp[(long)r * k + rank] = key_value((uint32_t)(c >> 32)) - m - log_s;
      p.top_ids[(long)r * k + rank] = (int)(0xFFFFFFFFu - (uint32_t)c);
    }
  }
}

struct LogprobPlan { int parts, chunks; };
static LogprobPlan logprob_plan(int rows, int vocab, int n_top) {
  LogprobPlan t;
  const int chunks = (vocab + LP_CHUNK - 1) / LP_CHUNK;
  t.chunks = 1;
  if (n_top == 0) {                       // waves for the whole GPU, 16 on a compute unit
    const long waves = (long)rows * chunks;
    t.chunks = (int)std::min<long>(chunks, std::max<long>(1, waves / 4096));
  }
  t.parts = (chunks + t.chunks - 1) / t.chunks;
  return t;
}

bool logprobs_fits(int vocab, int n_top) { return n_top <= LP_MAX_TOP && vocab <= LP_MAX_PARTS * LP_CHUNK; }

void logprobs_part_sizes(int rows, int vocab, int n_top, size_t* sum_floats, size_t* top_keys) {
  const LogprobPlan t = logprob_plan(rows, vocab, n_top);
  *sum_floats = (size_t)rows * t.parts * 4;
  *top_keys = (size_t)rows * t.parts * n_top;
}

template <typename T> static hipError_t logprobs_launch(const LogprobArgs& p, hipStream_t s) {
  const LogprobPlan t = logprob_plan(p.rows, p.vocab, p.n_top);
  const long waves = (long)p.rows * t.parts;
  hipLaunchKernelGGL((logprobs_part_kernel<T>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, p, t.parts, t.chunks);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((logprobs_row_kernel<T>), dim3(p.rows), dim3(256), 0, s, p, t.parts);
  return hipGetLastError();
}

hipError_t logprobs(const LogprobArgs& p, hipStream_t s) {
  if (p.rows <= 0) return hipSuccess;
  if (p.vocab <= 0 || !logprobs_fits(p.vocab, p.n_top)) return hipErrorInvalidValue;
  return p.f32 ? logprobs_launch<float>(p, s) : logprobs_launch<bf16_t>(p, s);
}

}  // namespace nova
