// Log probabilities from rows of logits: of given tokens, the entropy of the distribution, and the most
// likely tokens.  With m the row's maximum, S = sum e^(x - m) and T = sum e^(x - m) (x - m):
//   log p_t = x_t - m - log S,   entropy = log S - T / S.
// One pass: every lane keeps a maximum, S and T of its own (fp32; every e^(x - m) is at most 1 and T / S
// loses nothing to cancellation), joined at the end.  For the most likely tokens the pass keeps the
// maximum of every 16 consecutive logits: the n_top largest logits (equal ones by the lower id) lie in
// the n_top groups of largest maximum (equal ones by the lower group), whatever ties there are, because
// each better group holds a better logit.  So a selection among vocab / 16 numbers and n_top groups
// read again give them exactly.  A short row is one workgroup and one launch; a long one is cut into
// parts that a second kernel joins.  Bound by HBM for many rows, by launches and latency for one.
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"

namespace nova {

constexpr int LP_EPL = 16;                 // logits of a lane at a time
constexpr int LP_CHUNK = 64 * LP_EPL;      // of a wave
constexpr int LP_GROUP = 16;               // consecutive logits with one maximum
constexpr int LP_ONE = 8;                  // chunks of a row that one workgroup takes
constexpr int LP_MAX_PARTS = 512;
constexpr int LP_MAX_TOP = 32;
constexpr int LP_CAND = 2048;              // candidates that are ranked by counting

// An unsigned number that orders as the values do: -0 equals 0, NaN is above infinity; 0 is no value's.
NOVA_DEV uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  if (x != x) return 0xFFFFFFFFu;
  return (u >> 31) ? ~u : u | 0x80000000u;
}
NOVA_DEV float key_value(uint32_t k) { return __uint_as_float((k >> 31) ? k & 0x7FFFFFFFu : ~k); }
// Larger first, equal values by the lower id; 0: none.
NOVA_DEV unsigned long long rank_key(uint32_t key, int id) { return ((unsigned long long)key << 32) | (0xFFFFFFFFu - (uint32_t)id); }

// A lane's logits of a chunk as loaded: 16 bytes at a time, N = 16 / sizeof(T) logits from first + 64 N j + N lane
// on (an address that is a multiple of 16).  Those outside the row are -infinity.
template <typename T> struct RawLogits { u32x4 w[LP_EPL * sizeof(T) / 16]; };
template <typename T> NOVA_DEV void load_logits(const T* row, long first, int vocab, RawLogits<T>& x) {
  constexpr int N = 16 / sizeof(T);
  const int lane = threadIdx.x & 63;
  if (first >= 0 && first + LP_CHUNK <= vocab) {                  // the same for every lane
#pragma unroll
    for (int j = 0; j < LP_EPL / N; ++j) x.w[j] = reinterpret_cast<const u32x4*>(row + first)[64 * j + lane];
    return;
  }
#pragma unroll
  for (int j = 0; j < LP_EPL / N; ++j) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint32_t v = 0;
#pragma unroll
      for (int h = 0; h < (sizeof(T) == 2 ? 2 : 1); ++h) {
        const long i = first + 64 * N * j + N * lane + (sizeof(T) == 2 ? 2 * d + h : d);
        const bool in = i >= 0 && i < vocab;
        if constexpr (sizeof(T) == 4) v = in ? __float_as_uint(row[i]) : 0xFF800000u;
        else v |= (in ? (uint32_t)row[i] : 0xFF80u) << (16 * h);
      }
      x.w[j][d] = v;
    }
  }
}
template <typename T> NOVA_DEV float logit_of(const RawLogits<T>& x, int j) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(x.w[j / 4][j % 4]);
  const uint32_t w = x.w[j / 8][j % 8 / 2];
  return __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
}

// m, S, T of a set of logits.
struct LogSum { float m, s, t; };
// a's sums taken to a maximum m >= a.m.
NOVA_DEV LogSum log_sum_at(const LogSum& a, float m) {
  if (a.m == m || a.s == 0.f) return LogSum{m, a.s, a.t};
  const float d = a.m - m, f = __expf(d);
  return LogSum{m, f * a.s, f > 0.f ? f * (a.t + d * a.s) : 0.f * a.t};
}
NOVA_DEV LogSum log_sum_join(const LogSum& a, const LogSum& b) {
  const float m = fmaxf(a.m, b.m);
  const LogSum x = log_sum_at(a, m), y = log_sum_at(b, m);
  return LogSum{m, x.s + y.s, x.t + y.t};
}
NOVA_DEV LogSum log_sum_wave(const LogSum& a) {
  const float m = wave_max(a.m);
  const LogSum j = log_sum_at(a, m);
  return LogSum{m, wave_sum(j.s), wave_sum(j.t)};
}

// The logit of the thread's first given token, requested before the sums are known.
template <typename T> NOVA_DEV float given_logit(const LogprobArgs& p, int r, int i) {
  const int id = i < p.n_given ? p.given[(long)r * p.n_given + i] : -1;
  return (unsigned)id < (unsigned)p.vocab ? to_f<T>(reinterpret_cast<const T*>(p.logits)[r * p.stride + id]) : -INFINITY;
}
// What a row's sums say; `x`: given_logit() of the thread's first.  Called by every thread of a workgroup.
template <typename T>
NOVA_DEV float row_sums(const LogprobArgs& p, int r, const LogSum& a, float x) {
  // nothing but -infinity: no distribution
  const float log_s = a.s == 0.f ? __uint_as_float(0x7FC00000u) : logf(a.s);
  if (threadIdx.x == 0 && p.entropy) p.entropy[r] = log_s - a.t / a.s;
  for (int i = threadIdx.x; i < p.n_given; i += blockDim.x) {
    if (i >= (int)blockDim.x) x = given_logit<T>(p, r, i);
    const int id = p.given[(long)r * p.n_given + i];
    p.given_lp[(long)r * p.n_given + i] = (unsigned)id < (unsigned)p.vocab ? x - a.m - log_s : -INFINITY;
  }
  return log_s;
}

// The larger of two values, NaN where either is (one instruction for three on gfx950).
NOVA_DEV float nan_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// LDS of the selection.
template <int W> struct TopShared {
  unsigned long long cand[LP_CAND];
  int group[LP_CAND], rank[LP_CAND];
  float set[W][64];
  int count[W], n, m;
};

// The n_top most likely tokens of a row whose groups have the maxima gmax[0 .. groups) (NaN if one is in it);
// group g is logits 16 g - lead ...  Every thread of a workgroup of W waves.
//  1. The groups are dealt to 64 sets (one per lane number).  The k-th largest of the sets' maxima bounds
//     the k-th logit of the row from below, and few groups reach it: some 64 ln(64 / (64 - k)).
//  2. Their logits that reach it are ranked by counting the larger ones.
//  3. Where more reach it (a row that is masked but for a few tokens), those above it are taken, and if they are
//     fewer than k, the first ones that equal it.
//  4. Where even those above it are too many (the best ones side by side), and where the row holds a NaN, the k-th
//     group is bisected exactly, on its maximum and its number, and the logits of the best k groups that are not
//     below its maximum are ranked: at most 16 k.
// A thread takes V groups at a time; the first AHEAD times V are requested before anything waits.
template <typename T, int W, int V, int AHEAD>
struct RowTop {
  static constexpr int THREADS = 64 * W, STRIDE = THREADS * V;
  const LogprobArgs& p;
  const float* gmax;
  int r, groups, lead;
  float first[AHEAD][V];

  NOVA_DEV void take(int g, float (&m)[V]) const {               // groups is a multiple of 64
    if (g < groups) {
      if constexpr (V == 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(gmax + g);
#pragma unroll
        for (int q = 0; q < 4; ++q) m[q] = v[q];
      } else {
        m[0] = gmax[g];
      }
    } else {
#pragma unroll
      for (int q = 0; q < V; ++q) m[q] = -INFINITY;
    }
  }
  NOVA_DEV void request() {
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) take(e * STRIDE + V * (int)threadIdx.x, first[e]);
  }
  // f(maximum, group) of the thread's groups, for the passes that are rare
  template <typename F> NOVA_DEV void each(F f) {
#pragma unroll 1
    for (int g = V * (int)threadIdx.x; g < groups; g += STRIDE) {
      float m[V];
      take(g, m);
#pragma unroll
      for (int q = 0; q < V; ++q) f(m[q], g + q);
    }
  }
  // The logits of the n groups in sm.group that are not below `least`, into sm.cand (those that fit): how many.
  NOVA_DEV int logits_of(int n, uint32_t least, TopShared<W>& sm) {
    const int tid = threadIdx.x;
    const T* row = reinterpret_cast<const T*>(p.logits) + r * p.stride;
    for (int i0 = 0; i0 < n * LP_GROUP; i0 += 4 * THREADS) {
      float x[4];
      int id[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {                               // requested together
        const int i = i0 + u * THREADS + tid;
        id[u] = i < n * LP_GROUP ? sm.group[i / LP_GROUP] * LP_GROUP - lead + i % LP_GROUP : -1;
        if (id[u] >= p.vocab) id[u] = -1;
        x[u] = id[u] >= 0 ? to_f<T>(row[id[u]]) : 0.f;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t key = order_key(x[u]);
        if (id[u] < 0 || key < least) continue;
        const int to = atomicAdd(&sm.m, 1);
        if (to < LP_CAND) {
          sm.cand[to] = rank_key(key, id[u]);
          sm.rank[to] = 0;
        }
      }
    }
    __syncthreads();
    return sm.m;
  }

  // The first groups with the maximum `value` (k - have of them at least), into sm.group from `have` up to k.
  NOVA_DEV void first_equal(float value, int have, int k, TopShared<W>& sm) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll 1
    for (int g0 = 0; g0 < groups && have < k; g0 += STRIDE) {
      float m[V];
      take(g0 + V * tid, m);
      int mine = 0, upto;
#pragma unroll
      for (int q = 0; q < V; ++q) mine += g0 + V * tid + q < groups && m[q] == value;
      upto = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(upto, o, 64);
        if (lane >= o) upto += up;
      }
      if (lane == 63) sm.count[wave] = upto;
      __syncthreads();
      int at = have + upto - mine;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        at += w < wave ? sm.count[w] : 0;
        have += sm.count[w];
      }
#pragma unroll
      for (int q = 0; q < V; ++q) {
        if (!(g0 + V * tid + q < groups && m[q] == value)) continue;
        if (at < k) sm.group[at] = g0 + V * tid + q;
        ++at;
      }
      __syncthreads();
    }
  }

  NOVA_DEV void operator()(const LogSum& a, float log_s, TopShared<W>& sm) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = p.n_top;
    float best = -INFINITY;
#pragma unroll
    for (int e = 0; e < AHEAD; ++e)
#pragma unroll
      for (int q = 0; q < V; ++q) best = nan_max(best, first[e][q]);
    if (groups > AHEAD * STRIDE) each([&](float m, int) { best = nan_max(best, m); });
    sm.set[wave][lane] = best;
    if (tid == 0) sm.n = sm.m = 0;
    __syncthreads();
    best = sm.set[0][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) best = nan_max(best, sm.set[w][lane]);
    const bool nan = __any(best != best);
    int above = 0;                                                // sets with a larger maximum
#pragma unroll
    for (int l = 0; l < 64; ++l) above += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(best), l)) > best;
    const float tau = -wave_max(above < k ? -best : -INFINITY);
    int n = LP_CAND + 1;
    // the groups whose maximum is above `least`, or with `equal` not below it: how many
    auto reach = [&](float least, bool equal) {
      auto put = [&](float m, int g) {
        if (!(m > least || (equal && m == least))) return;
        const int to = atomicAdd(&sm.n, 1);
        if (to < LP_CAND) sm.group[to] = g;
      };
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
#pragma unroll
        for (int q = 0; q < V; ++q)
          if (e * STRIDE + V * tid + q < groups) put(first[e][q], e * STRIDE + V * tid + q);
      if (groups > AHEAD * STRIDE)
        each([&](float m, int g) {
          if (g >= AHEAD * STRIDE) put(m, g);
        });
      __syncthreads();
      return sm.n;
    };
    if (!nan) {
      n = reach(tau, true);
      if (n <= 64 + k) {
        n = logits_of(n, order_key(tau), sm);
      } else {
        __syncthreads();
        if (tid == 0) sm.n = 0;
        __syncthreads();
        n = reach(tau, false);
        if (n < k) {
          first_equal(tau, n, k, sm);
          n = logits_of(k, order_key(tau), sm);
        } else if (n <= LP_CAND) {
          n = logits_of(n, order_key(tau) + 1, sm);
        }
      }
    }
    if (n > LP_CAND) {
      // the largest bound that k groups reach (there are 64 at least): exactly k, since keys differ
      unsigned long long bound = 1;
#pragma unroll 1
      for (int bit = 63; bit >= 0; --bit) {
        const unsigned long long trial = bound | (1ull << bit);
        int c = 0;
        each([&](float m, int g) { c += rank_key(order_key(m), g) >= trial; });
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) c += __shfl_xor(c, o, 64);
        __syncthreads();
        if (lane == 0) sm.count[wave] = c;
        __syncthreads();
        c = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) c += sm.count[w];
        if (c >= k) bound = trial;
      }
      if (tid == 0) sm.n = sm.m = 0;
      __syncthreads();
      each([&](float m, int g) {
        if (rank_key(order_key(m), g) >= bound) sm.group[atomicAdd(&sm.n, 1)] = g;
      });
      __syncthreads();
      n = logits_of(k, (uint32_t)(bound >> 32), sm);
    }
    // a candidate's rank is the number of larger ones; `split` threads share a candidate
    const int span = (n + 63) & ~63, split = max(1, THREADS / span), per = (n + split - 1) / split;
    for (int t = tid; t < span * split; t += THREADS) {
      const int i = t % span, j0 = t / span * per, j1 = min(j0 + per, n);
      const unsigned long long c = i < n ? sm.cand[i] : ~0ull;
      int x = 0;
#pragma unroll 8
      for (int j = j0; j < j1; ++j) x += sm.cand[j] > c;
      if (i < n && x) atomicAdd(&sm.rank[i], x);
    }
    __syncthreads();
    for (int i = tid; i < n; i += THREADS) {
      const int at = sm.rank[i];
      if (at >= k) continue;
      p.top_lp[(long)r * k + at] = key_value((uint32_t)(sm.cand[i] >> 32)) - a.m - log_s;
      p.top_ids[(long)r * k + at] = (int)(0xFFFFFFFFu - (uint32_t)sm.cand[i]);
    }
  }
};

// Workgroup (part of a row), its waves taking chunks of 1024 logits in turn, the next one's loads in
// flight.  ONE: the part is the whole row, and the workgroup finishes it (4096 logits: 5.7 us, a chain of loads,
// reductions and barriers).  Bound by HBM for many rows: 601 of 152064 in bf16 38.5 us, 4.8 TB/s; 32 of 152064
// in fp32 7.1 us, of which 3.9 are their bytes at a large copy's rate and the rest launch, ramp and drain.
template <typename T, bool ONE>
__global__ void __launch_bounds__(256) logprobs_part_kernel(LogprobArgs p, int parts, int chunks, int groups) {
  constexpr int N = 16 / sizeof(T), LPG = LP_GROUP / N;           // a load's logits, lanes that share a group
  __shared__ LogSum sm[4];
  __shared__ __align__(16) float sm_max[ONE ? LP_ONE * 64 : 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = ONE ? blockIdx.x : blockIdx.x / parts, part = ONE ? 0 : blockIdx.x % parts;
  const T* row = reinterpret_cast<const T*>(p.logits) + r * p.stride;
  const int lead = (int)(((uintptr_t)row & 15) / sizeof(T));      // chunks start at the aligned address at or before the row
  const int total = (p.vocab + lead + LP_CHUNK - 1) / LP_CHUNK;
  const int c0 = part * chunks, c1 = min(c0 + chunks, total);
  const float gx = ONE ? given_logit<T>(p, r, tid) : 0.f;
  // A lane's sums S and T relative to its maximum m, T in powers of 2.
  constexpr float LOG2E = 1.44269504f;
  float m = -INFINITY, s = 0.f, t = 0.f;
  auto load = [&](int c, RawLogits<T>& x) { load_logits(row, (long)c * LP_CHUNK - lead, p.vocab, x); };
  auto take = [&](int c, const RawLogits<T>& raw) {
    float x[LP_EPL], top[LP_EPL / N], m_new = m;
#pragma unroll
    for (int j = 0; j < LP_EPL; ++j) x[j] = logit_of(raw, j);
#pragma unroll
    for (int j = 0; j < LP_EPL / N; ++j) {
      top[j] = x[j * N];
#pragma unroll
      for (int e = 1; e < N; ++e) top[j] = nan_max(top[j], x[j * N + e]);
      m_new = fmaxf(m_new, top[j]);
    }
    if (p.n_top > 0) {                                            // lane LPG q + j writes group q of the j-th loads
      float mine = 0.f;
#pragma unroll
      for (int j = 0; j < LP_EPL / N; ++j) {
        float g = nan_max(top[j], __shfl_xor(top[j], 1, 64));
        if (LPG == 4) g = nan_max(g, __shfl_xor(g, 2, 64));
        if (lane % LPG == j) mine = g;
      }
      const int g = c * (LP_CHUNK / LP_GROUP) + lane % LPG * (64 / LPG) + lane / LPG;
      if constexpr (ONE) sm_max[g] = mine;
      else p.part_max[(long)r * groups + g] = mine;
    }
    if (m_new > m) {
      const float d = (m - m_new) * LOG2E, f = s == 0.f ? 0.f : __builtin_amdgcn_exp2f(d);
      t = f > 0.f ? f * (t + d * s) : 0.f * t;
      s *= f;
      m = m_new;
    }
    const float mu = m == -INFINITY ? 0.f : m;                    // nothing but -infinity yet: every e is 0
    if (__all(fabsf(mu) < 65536.f)) {
      // one fused multiply and an exponential each: relative to the rounded m log2e, and then to m itself
      const float base = mu * LOG2E, off = fmaf(mu, LOG2E, -base), back = __builtin_amdgcn_exp2f(-off);
      float sc = 0.f, tc = 0.f;
#pragma unroll
      for (int j = 0; j < LP_EPL; ++j) {
        const float d = fmaf(x[j], LOG2E, -base), e = __builtin_amdgcn_exp2f(d);
        sc += e;
        tc = fmaf(e, fmaxf(d, -200.f), tc);                       // e is 0 there: -infinity adds 0
      }
      s += sc * back;
      t += (tc - off * sc) * back;
    } else {                                                      // where m log2e is no longer exact enough, or infinite
#pragma unroll 4
      for (int j = 0; j < LP_EPL; ++j) {
        const float d = (x[j] - mu) * LOG2E, e = __builtin_amdgcn_exp2f(d);
        s += e;
        t = fmaf(e, fmaxf(d, -200.f), t);
      }
    }
  };
  RawLogits<T> x, y;
  int c = c0 + wave;
  if (c < c1) load(c, x);
  for (; c < c1; c += 8) {                                        // two buffers in turn
    if (c + 4 < c1) load(c + 4, y);
    take(c, x);
    if (c + 4 >= c1) break;
    if (c + 8 < c1) load(c + 8, x);
    take(c + 4, y);
  }
  LogSum a{m, s, t * 0.693147181f};
  a = log_sum_wave(a);
  if (lane == 0) sm[wave] = a;
  __syncthreads();
  a = sm[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) a = log_sum_join(a, sm[w]);
  if constexpr (ONE) {
    __shared__ TopShared<4> ts;
    const float log_s = row_sums<T>(p, r, a, gx);
    if (p.n_top > 0) {
      RowTop<T, 4, 1, (LP_ONE * 64 + 255) / 256> top{p, sm_max, r, total * (LP_CHUNK / LP_GROUP), lead, {}};
      top.request();
      top(a, log_s, ts);
    }
  } else if (tid == 0) {
    reinterpret_cast<float4*>(p.part_sum)[blockIdx.x] = make_float4(a.m, a.s, a.t, 0.f);
  }
}

// Workgroup (row): the parts' sums joined, the most likely tokens from the groups' maxima.  Bound by latency:
// 32 rows of 152064 with 20 tokens 6.7 us (9504 maxima, a bound, 20 groups, a rank), 601 rows without tokens 4.8 us.
template <typename T, bool TOP>
__global__ void __launch_bounds__(TOP ? 512 : 64) logprobs_join_kernel(LogprobArgs p, int parts, int groups) {
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const T* row = reinterpret_cast<const T*>(p.logits) + r * p.stride;
  const int lead = (int)(((uintptr_t)row & 15) / sizeof(T)), total = (p.vocab + lead + LP_CHUNK - 1) / LP_CHUNK;
  const float gx = given_logit<T>(p, r, tid);
  float4 v = make_float4(-INFINITY, 0.f, 0.f, 0.f);
  if (lane < parts) v = reinterpret_cast<const float4*>(p.part_sum)[(long)r * parts + lane];
  RowTop<T, 8, 4, TOP ? 6 : 1> top{p, p.part_max + (long)r * groups, r, total * (LP_CHUNK / LP_GROUP), lead, {}};
  if constexpr (TOP) top.request();
  LogSum a{v.x, v.y, v.z};                                        // every wave the same: no barrier
  for (int i = lane + 64; i < parts; i += 64) {
    v = reinterpret_cast<const float4*>(p.part_sum)[(long)r * parts + i];
    a = log_sum_join(a, LogSum{v.x, v.y, v.z});
  }
  a = log_sum_wave(a);
  const float log_s = row_sums<T>(p, r, a, gx);
  if constexpr (TOP) {
    __shared__ TopShared<8> ts;
    top(a, log_s, ts);
  }
}

// Parts of a row and the chunks of each.  A row of up to LP_ONE chunks is one workgroup.  Above, parts until
// there are 32 waves for each of 256 compute units, at least one chunk a wave (601 rows of 152064 bf16
// logits, when a wave took 44.0 us with 32: 62 us with 8, 45.5 with 16, 43.6 with 64, and a longer join).
struct LogprobPlan { int parts, chunks, groups; };
static LogprobPlan logprob_plan(int rows, int vocab) {
  const int total = (vocab + 7 + LP_CHUNK - 1) / LP_CHUNK;       // an unaligned row starts up to 7 logits early
  LogprobPlan t{1, total, total * (LP_CHUNK / LP_GROUP)};
  if (total <= LP_ONE) return t;
  const long per = std::max<long>(1, (long)rows * total / 8192);
  t.chunks = (int)std::min<long>(total, per * 4);
  t.chunks = std::max(t.chunks, (total + LP_MAX_PARTS - 1) / LP_MAX_PARTS);
  t.parts = (total + t.chunks - 1) / t.chunks;
  return t;
}
static bool logprob_one(int vocab) { return (vocab + 7 + LP_CHUNK - 1) / LP_CHUNK <= LP_ONE; }

bool logprobs_fits(int vocab, int n_top) { return n_top <= LP_MAX_TOP && vocab <= 1 << 21; }

void logprobs_part_sizes(int rows, int vocab, int n_top, size_t* sum_floats, size_t* max_floats) {
  const LogprobPlan t = logprob_plan(rows, vocab);
  const bool one = logprob_one(vocab);
  *sum_floats = one ? 0 : (size_t)rows * t.parts * 4;
  *max_floats = one || n_top == 0 ? 0 : (size_t)rows * t.groups;
}

template <typename T> static hipError_t logprobs_launch(const LogprobArgs& p, hipStream_t s) {
  const LogprobPlan t = logprob_plan(p.rows, p.vocab);
  if (logprob_one(p.vocab)) {
    hipLaunchKernelGGL((logprobs_part_kernel<T, true>), dim3(p.rows), dim3(256), 0, s, p, 1, t.chunks, t.groups);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((logprobs_part_kernel<T, false>), dim3((unsigned)((long)p.rows * t.parts)), dim3(256), 0, s, p, t.parts, t.chunks, t.groups);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.n_top > 0) hipLaunchKernelGGL((logprobs_join_kernel<T, true>), dim3(p.rows), dim3(512), 0, s, p, t.parts, t.groups);
  else hipLaunchKernelGGL((logprobs_join_kernel<T, false>), dim3(p.rows), dim3(64), 0, s, p, t.parts, t.groups);
  return hipGetLastError();
}

hipError_t logprobs(const LogprobArgs& p, hipStream_t s) {
  if (p.rows <= 0) return hipSuccess;
  if (p.vocab <= 0 || !logprobs_fits(p.vocab, p.n_top)) return hipErrorInvalidValue;
  return p.f32 ? logprobs_launch<float>(p, s) : logprobs_launch<bf16_t>(p, s);
}

}  // namespace nova
