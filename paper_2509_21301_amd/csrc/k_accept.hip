// Which drafted tokens the target's probabilities keep, and the token that is drawn behind them, from given numbers.
// With z = l / T, p = e^(z - max z) / sum: a row's probabilities at its sequence's temperature T.
//  * With the draft's probabilities q (a chain): row j's token x is kept while u_j q_j(x) < p_(j-1)(x); behind the
//    first that is not, the token is drawn from max(p - q, 0), behind the last row from p (speculative sampling: what
//    comes out is distributed as the target's own tokens).
//  * Without (a tree or a chain of tokens): every row draws its token from p, and the walk goes on in the row that
//    brought it.
// A draw is the first token whose running sum exceeds u times the total.  The running sums reach over the whole
// vocabulary and are compared with a number that may lie next to any of them, so weights and sums are in 64 bits (an
// fp32 sum would move about one draw in a thousand at 152064 logits).
// Two launches: the first reads every logit once (maximum, sums and largest id of chunks of 8192), the second decides and
// draws, reading again only parts of the rows where something is drawn, and with a draft the two rows behind which a
// token was not kept.
#include <algorithm>

#include "paged.hpp"

namespace nova {

constexpr int AC_CHUNK = 8192;             // logits of a workgroup
constexpr int AC_THREADS = 256;
constexpr int AC_PER = AC_CHUNK / AC_THREADS;
constexpr int AC_PART = AC_CHUNK / AC_PARTS;
constexpr int AC_MAX_CHUNKS = (1 << 21) / AC_CHUNK;   // of the largest vocabulary

// A value of another lane by a data-parallel move: 0 where there is no such lane (or its row is left out of ROWS).
template <int CTRL, int ROWS> NOVA_DEV double dpp64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
NOVA_DEV double lane_of(double v, int l) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, l), hi = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), l);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Inclusive running sum over a wave, and its sum; both in a fixed order, so that every call gives the same draws.
// (Within the 16 lanes of a row by shifts of 1, 2, 4 and 8, then row ends to the rows behind them.)
NOVA_DEV double wave_scan64(double v) {
  v += dpp64<0x111, 0xf>(v);
  v += dpp64<0x112, 0xf>(v);
  v += dpp64<0x114, 0xf>(v);
  v += dpp64<0x118, 0xf>(v);
  v += dpp64<0x142, 0xa>(v);
  v += dpp64<0x143, 0xc>(v);
  return v;
}
NOVA_DEV double wave_sum64(double v) { return lane_of(wave_scan64(v), 63); }

// The sequence of a row in *b (batch: none) and its rows; a wave looks at 64 row starts at a time.
NOVA_DEV SeqRows seq_of_row(const BatchRows& p, int r, int* b) {
  *b = p.batch;
  if (!p.row_start) {
    *b = r / p.max_rows;
    return seq_rows(p, *b);
  }
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < p.batch; base += 64) {
    const int i = min(base + lane, p.batch - 1), from = p.row_start[i], to = p.row_start[i + 1];
    const unsigned long long m = __ballot(to > r);
    if (!m) continue;
    const int l = __ffsll(m) - 1;
    *b = min(base + l, p.batch - 1);
    SeqRows s;
    s.r0 = min(max(__builtin_amdgcn_readlane(from, l), 0), p.rows);
    s.n = min(min(max(__builtin_amdgcn_readlane(to, l), s.r0), p.rows) - s.r0, p.max_rows);
    s.ctx = 0;
    return s;
  }
  return SeqRows{0, 0, 0};
}

// A sequence's temperature T: inv = log2(e) / T, 0 for T = 0 (the largest logit takes all), negative where T gives no
// distribution; least: the difference of logits below which every weight is 0.
struct Heat { double inv, least; };
NOVA_DEV Heat heat_of(const AcceptArgs& p, int b) {
  const float t = p.temperature ? p.temperature[b] : 1.f;
  if (t == 0.f) return Heat{0.0, 0.0};
  if (!(t > 0.f && t < INFINITY)) return Heat{-1.0, 0.0};
  return Heat{1.4426950408889634 / (double)t, -762.4618986159398 * (double)t};     // 2^-1100 and below
}

// 2^z for z <= 0 in 64 bits (0 below 2^-1074 and for -infinity): z = k + j / 256 + f with |f| <= 2^-9, the table's
// 2^(j/256), and the Taylor series of 2^f to f^4 (its rest is below 4e-17): 16 instructions, where a series without a
// table takes 30, and there is one to be formed for every logit: the first pass over 384 rows of 152064 took 96 us with
// the longer one, 62 us with this one in its first form (17 instructions, 16 logits a thread).
struct Exp2Table { double t[256]; };       // in LDS
NOVA_DEV void fill_table(Exp2Table& tab) { // by the workgroup's threads; a barrier has to follow
  for (int j = threadIdx.x; j < 256; j += blockDim.x) {
    const double r = (j - 128) * (0.6931471805599453 / 256);
    double y = 1.0 / 6227020800.0;         // Taylor series of e^r to r^13, |r| <= ln 2 / 2: its rest is below 5e-18
    constexpr double C[13] = {1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040, 1.0 / 40320, 1.0 / 362880,
                              1.0 / 3628800, 1.0 / 39916800, 1.0 / 479001600};
#pragma unroll
    for (int n = 12; n >= 0; --n) y = fma(y, r, C[n]);
    tab.t[j] = j ? y * 1.4142135623730951 : 1.0;   // the largest logit's weight is 1 exactly
  }
}
// 2^(d inv), d <= 0 and d inv at least -1100.
NOVA_DEV double exp2_times(const Exp2Table& tab, double d, double inv) {
  constexpr double MAGIC = 0x1.8p44;       // a sum with it ends at the 8th binary place
  const double t = fma(d, inv, MAGIC), f = fma(d, inv, -(t - MAGIC));
  const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, t);
  double y = fma(f, 9.6181291076284772e-3, 5.5504108664821580e-2);
  y = fma(y, f, 2.4022650695910072e-1);
  y = fma(y, f, 6.9314718055994531e-1);
  const double b = tab.t[n & 255];
  return ldexp(fma(b, y * f, b), n >> 8);
}
NOVA_DEV double exp2_neg(const Exp2Table& tab, double z) { return exp2_times(tab, fmax(z, -1100.0), 1.0); }

// Weights of logits relative to a maximum m at log2(e) / T = inv: the difference first (it is exact, where a product with a
// small temperature's inverse would not cancel at the maximum).
struct Weigh {
  double m;
  Heat h;
  NOVA_DEV Weigh(float m, const Heat& h) : m(m), h(h) {}
  NOVA_DEV double operator()(const Exp2Table& tab, float x) const { return exp2_times(tab, fmax((double)x - m, h.least), h.inv); }
};
constexpr double LN2 = 0.6931471805599453;

// A logit of a row, from memory in its type.
template <typename T> NOVA_DEV float logit(const T* row, int i) { return to_f<T>(row[i]); }

// The larger of two values, NaN where either is.
NOVA_DEV float nan_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <int CTRL, int ROWS> NOVA_DEV float dpp_max(float v) {
  return nan_max(v, __int_as_float(__builtin_amdgcn_update_dpp((int)0xFF800000u, __float_as_int(v), CTRL, ROWS, 0xf, false)));
}
NOVA_DEV float wave_nan_max(float v) {
  v = dpp_max<0x111, 0xf>(v);
  v = dpp_max<0x112, 0xf>(v);
  v = dpp_max<0x114, 0xf>(v);
  v = dpp_max<0x118, 0xf>(v);
  v = dpp_max<0x142, 0xa>(v);
  v = dpp_max<0x143, 0xc>(v);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// A thread's logits of a chunk, of which every wave has a part: 16 bytes at a time where the row allows it (x[i]: number
// place_of(i) of the chunk); -infinity behind the vocabulary.
template <typename T> NOVA_DEV int place_of(int i) {
  constexpr int N = 16 / sizeof(T);
  return (threadIdx.x >> 6) * AC_PART + (i / N * 64 + (threadIdx.x & 63)) * N + i % N;
}
template <typename T> NOVA_DEV void load_chunk(const T* row, int c0, int vocab, float* x) {
  constexpr int N = 16 / sizeof(T);
  if (((uintptr_t)row & 15) == 0 && c0 + AC_CHUNK <= vocab) {
    u32x4 w[AC_PER / N];
#pragma unroll
    for (int i = 0; i < AC_PER / N; ++i) w[i] = *reinterpret_cast<const u32x4*>(row + c0 + place_of<T>(i * N));
#pragma unroll
    for (int i = 0; i < AC_PER; ++i) {
      if constexpr (N == 4) x[i] = __uint_as_float(w[i / 4][i % 4]);
      else x[i] = __uint_as_float(i & 1 ? w[i / 8][i % 8 / 2] & 0xFFFF0000u : w[i / 8][i % 8 / 2] << 16);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < AC_PER; ++i) {
    const int at = c0 + place_of<T>(i);
    x[i] = at < vocab ? logit(row, at) : -INFINITY;
  }
}

// ------------------------------------------------------------------ first pass
// Workgroup: a chunk of one row.  Rows 0 .. rows - 1 are the target's, the next `rows` the draft's.  384 rows of 152064
// logits (32 sequences of 5 to 8 rows with their draft's): 48 to 50 us, 4.7 TB/s of 5.1 that a large copy reaches; in bf16
// 44 us, bound by the vector instructions (in fp32 they issue in 71% of the cycles).
template <typename TL, typename TD>
__global__ void __launch_bounds__(256) accept_stats_kernel(AcceptArgs p) {
  // what the second kernel counts, and the outputs of sequences without rows
  for (long b = (long)blockIdx.x * 256 + threadIdx.x; b < p.r.batch; b += (long)gridDim.x * 256) {
    p.counters[b] = 0u;
    if (seq_rows(p.r, (int)b).n > 0) continue;
    p.n_keep[b] = 0;
    for (int i = 0; i < p.r.max_rows; ++i) {
      p.path[b * p.r.max_rows + i] = p.tokens[b * p.r.max_rows + i] = -1;
      p.lp[b * p.r.max_rows + i] = 0.f;
    }
  }
  const int item = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
  if (item >= p.items) return;
  const bool draft = item >= p.r.rows;
  const int r = draft ? item - p.r.rows : item;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c0 = chunk * AC_CHUNK;
  float x[AC_PER];
  if (!draft) load_chunk((const TL*)p.logits + (long)r * p.row, c0, p.vocab, x);
  int b;
  const SeqRows sr = seq_of_row(p.r, r, &b);
  if (b >= p.r.batch || r < sr.r0 + (draft ? 1 : 0) || r >= sr.r0 + sr.n) return;   // a sequence's first row was drawn by nobody
  if (draft) load_chunk((const TD*)p.draft + (long)r * p.draft_row, c0, p.vocab, x);
  __shared__ Exp2Table tab;
  __shared__ float sm_m[4];
  __shared__ int sm_arg[4];
  const Heat h = heat_of(p, b);
  fill_table(tab);                         // while the logits are on their way
  float m = x[0];
#pragma unroll
  for (int i = 1; i < AC_PER; ++i) m = nan_max(m, x[i]);
  m = wave_nan_max(m);
  if (lane == 0) sm_m[wave] = m;
  __syncthreads();
  m = nan_max(nan_max(sm_m[0], sm_m[1]), nan_max(sm_m[2], sm_m[3]));
  double sum = 0.0;
  if (h.inv > 0.0 && m > -INFINITY && m < INFINITY) {
    const Weigh weight(m, h);
#pragma unroll
    for (int i = 0; i < AC_PER; ++i) sum += weight(tab, x[i]);
  }
  sum = wave_sum64(sum);
  int arg = 0x7FFFFFFF;
  if (h.inv == 0.0) {                        // greedy: the first of the largest
#pragma unroll
    for (int i = 0; i < AC_PER; ++i)
      if (x[i] == m) arg = min(arg, c0 + (draft ? place_of<TD>(i) : place_of<TL>(i)));
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) arg = min(arg, __shfl_xor(arg, o, 64));
  }
  const long at = (long)item * p.chunks + chunk;
  if (lane == 0) {
    p.part_sum[at * AC_PARTS + wave] = sum;
    sm_arg[wave] = arg;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    p.part_max[at] = m < INFINITY ? m : __uint_as_float(0x7FC00000u);   // NaN or +infinity: no distribution
    p.part_arg[at] = min(min(sm_arg[0], sm_arg[1]), min(sm_arg[2], sm_arg[3]));
  }
}

// ------------------------------------------------------------------ a row's chunks joined
// m: the row's maximum (NaN: no distribution), s: its sum relative to it, arg: the first of the largest logits.
struct RowStats { float m; int arg; double s; };
NOVA_DEV bool has_dist(const RowStats& a, const Heat& h) { return a.m > -INFINITY && h.inv >= 0.0; }   // NaN compares false

// A lane's chunks of a row: a request for all that is known of them (of more than 64 chunks those before are joined).
struct LaneParts { float m; int arg; double s; };
NOVA_DEV LaneParts lane_parts(const AcceptArgs& p, const Exp2Table& tab, int item, const Heat& h) {
  const long at = (long)item * p.chunks;
  LaneParts a{-INFINITY, 0x7FFFFFFF, 0.0};
  for (int c = threadIdx.x & 63; c < p.chunks; c += 64) {
    const double* sums = p.part_sum + (at + c) * AC_PARTS;
    const LaneParts n{p.part_max[at + c], p.part_arg[at + c], ((sums[0] + sums[1]) + sums[2]) + sums[3]};
    if (c < 64) {
      a = n;
      continue;
    }
    const float m = nan_max(a.m, n.m);
    const double of_a = a.m > -INFINITY ? a.s * exp2_neg(tab, ((double)a.m - (double)m) * h.inv) : 0.0;
    const double of_n = n.m > -INFINITY ? n.s * exp2_neg(tab, ((double)n.m - (double)m) * h.inv) : 0.0;
    a.arg = n.m > a.m ? n.arg : a.arg;
    a.m = m, a.s = of_a + of_n;
  }
  return a;
}
// By one wave; every lane returns the same.
NOVA_DEV RowStats join_parts(const Exp2Table& tab, const LaneParts& l, const Heat& h) {
  RowStats a{wave_nan_max(l.m), 0x7FFFFFFF, 0.0};
  if (!(a.m > -INFINITY)) return a;
  if (h.inv == 0.0) {
    a.arg = l.m == a.m ? l.arg : 0x7FFFFFFF;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) a.arg = min(a.arg, __shfl_xor(a.arg, o, 64));
  } else if (h.inv > 0.0) {
    a.s = wave_sum64(l.m > -INFINITY ? l.s * exp2_neg(tab, ((double)l.m - (double)a.m) * h.inv) : 0.0);
  }
  return a;
}

// A number in [0, 1) (1 and above: the largest below; NaN and below 0: 0).
NOVA_DEV double uniform(float u) { return u > 0.f ? (double)fminf(u, 0x1.fffffep-1f) : 0.0; }

// The first place of 0 .. n - 1 whose running sum exceeds `target` (none, by rounding: the last with a positive value),
// and the running sum before it.  value(i) is asked for in order; by one wave, every lane returns the same.
template <typename F> NOVA_DEV int first_above(int n, double target, double* before, F&& value) {
  const int lane = threadIdx.x & 63;
  double run = 0.0, run_last = 0.0;
  int last = 0;
  for (int i0 = 0; i0 < n; i0 += 64) {
    const double v = i0 + lane < n ? value(i0 + lane) : 0.0;
    const double incl = run + wave_scan64(v);
    const unsigned long long over = __ballot(incl > target && v > 0.0), some = __ballot(v > 0.0);
    if (over) {
      const int l = __ffsll(over) - 1;
      *before = lane_of(incl - v, l);
      return i0 + l;
    }
    if (some) {
      const int l = 63 - __clzll(some);
      last = i0 + l;
      run_last = lane_of(incl - v, l);
    }
    run = lane_of(incl, 63);
  }
  *before = run_last;
  return last;
}

// The token of SIZE logits from c0 on whose running sum of weight(i) exceeds `target` (-1: none has a weight); by the whole
// workgroup of THREADS.  First the thread's range of consecutive logits, then the logit in it, one a lane.
template <int SIZE, int THREADS, typename F> NOVA_DEV int draw_in_part(int c0, int vocab, double target, F&& weight) {
  constexpr int PER = SIZE / THREADS;
  __shared__ double sm_sum[THREADS];
  const int first = c0 + threadIdx.x * PER;
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const double w = weight(min(first + i, vocab - 1));      // the loads together
    sum += first + i < vocab ? w : 0.0;
  }
  __syncthreads();
  sm_sum[threadIdx.x] = sum;
  __syncthreads();
  double before = 0.0;
  const int t = first_above(THREADS, target, &before, [&](int i) { return sm_sum[i]; });
  if (!(sm_sum[t] > 0.0)) return -1;
  const int from = c0 + t * PER;
  double none;
  return from + first_above(min(PER, vocab - from), target - before, &none, [&](int i) { return weight(from + i); });
}

// A token drawn from a target row by its number u; by the whole workgroup.  -1: the row has no distribution.
template <int THREADS, typename TL> NOVA_DEV int draw_row(const AcceptArgs& p, const Exp2Table& tab, int r, const RowStats& a, const Heat& h, float u) {
  if (!has_dist(a, h)) return -1;
  if (h.inv == 0.0) return a.arg;
  const TL* row = (const TL*)p.logits + (long)r * p.row;
  const long at = (long)r * p.chunks;
  double before = 0.0;
  const double target = uniform(u) * a.s;
  const Weigh weight(a.m, h);
  auto scale = [&](float m) { return m > -INFINITY ? weight(tab, m) : 0.0; };
  // the parts' sums side by side in LDS, requested together
  __shared__ double sm_parts[AC_MAX_CHUNKS * AC_PARTS];
  for (int i = threadIdx.x; i < p.chunks * AC_PARTS; i += THREADS) sm_parts[i] = p.part_sum[at * AC_PARTS + i] * scale(p.part_max[at + i / AC_PARTS]);
  __syncthreads();
  // A part's sum, which was formed relative to its chunk's maximum, may be positive where each of its weights underflows
  // (met by numbers of 0 only): then the draw goes on behind it.  The part of the largest logit has a weight of 1.
  while (true) {
    const int c = first_above(p.chunks * AC_PARTS, target, &before, [&](int i) { return sm_parts[i]; });
    const int token = draw_in_part<AC_PART, THREADS>(c * AC_PART, p.vocab, target - before, [&](int i) { return weight(tab, logit(row, i)); });
    if (token >= 0) return token;
    __syncthreads();
    if (threadIdx.x == 0) sm_parts[c] = 0.0;
    __syncthreads();
  }
}

// log p of a token of a row.
template <typename TL> NOVA_DEV float log_p(const AcceptArgs& p, int r, const RowStats& a, const Heat& h, int token) {
  if (token < 0) return __uint_as_float(0x7FC00000u);
  if (h.inv == 0.0) return 0.f;
  return (float)(((double)logit((const TL*)p.logits + (long)r * p.row, token) - (double)a.m) * h.inv * LN2 - log(a.s));
}

// The workgroups of a sequence that have come this far, this one included; what each stored before (with
// device-scope stores) is at the coherent level then.
NOVA_DEV unsigned arrive(unsigned* counter) {
  __shared__ unsigned sm_n;
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (threadIdx.x == 0) sm_n = 1u + __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  return sm_n;
}
template <typename T> NOVA_DEV void put(T* at, T v) { __hip_atomic_store(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T> NOVA_DEV T get(const T* at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// ------------------------------------------------------------------ second pass without the draft's probabilities
// Workgroup: a row, which draws its token; the last of a sequence walks from its first row on.  Bound by latency, a chain of
// eight dependent loads: 7 us for five rows of 4096 logits and for 208 of 152064.
template <typename TL>
__global__ void __launch_bounds__(256) accept_follow_kernel(AcceptArgs p) {
  __shared__ Exp2Table tab;
  fill_table(tab);
  const int r = blockIdx.x;
  int b;
  const SeqRows sr = seq_of_row(p.r, r, &b);
  if (b >= p.r.batch || r < sr.r0 || r >= sr.r0 + sr.n) return;
  const float u = p.u[r];
  const Heat h = heat_of(p, b);
  __syncthreads();
  const RowStats a = join_parts(tab, lane_parts(p, tab, r, h), h);
  const int token = draw_row<AC_THREADS, TL>(p, tab, r, a, h, u);
  if (threadIdx.x == 0) {
    put(p.row_token + r, token);
    put(p.row_lp + r, log_p<TL>(p, r, a, h, token));
  }
  if (arrive(p.counters + b) != (unsigned)sr.n) return;
  if (threadIdx.x >= 64) return;
  // lane j: row j of the sequence (at most 64), the row that it hangs under (-1: none) and its token
  const int j = threadIdx.x;
  const bool live = j < sr.n;
  int parent = j - 1;
  if (p.mask) {
    const unsigned long long up = live ? p.mask[sr.r0 + j] & ((1ull << j) - 1) : 0;
    parent = up ? 63 - __clzll(up) : -1;
  }
  const int id = live ? p.ids[sr.r0 + j] : -1;
  const int drawn = live ? get(p.row_token + sr.r0 + j) : -1;
  const float lp = live ? get(p.row_lp + sr.r0 + j) : 0.f;
  int path = -1, n = 0, at = 0;            // lane i: the i-th kept row
  while (true) {
    if (j == n) path = at;
    ++n;
    const int t = __shfl(drawn, at, 64);
    const unsigned long long kids = __ballot(live && j > at && parent == at && id == t && t >= 0);
    if (!kids) break;
    at = __ffsll(kids) - 1;
  }
  const int from = path < 0 ? 0 : path;
  const int tok = __shfl(drawn, from, 64);
  const float tlp = __shfl(lp, from, 64);
  if (j == 0) p.n_keep[b] = n;
  if (j < p.r.max_rows) {
    const long o = (long)b * p.r.max_rows + j;
    p.path[o] = path;
    p.tokens[o] = path < 0 ? -1 : tok;
    p.lp[o] = path < 0 ? 0.f : tlp;
  }
}

// ------------------------------------------------------------------ second pass with the draft's probabilities
// Workgroup: a chunk of a sequence.  Each finds the first row that is not kept (a wave tests a row, eight at a time); where the token is
// drawn from what the target has more than the draft, it sums that over its chunk, and the last to arrive draws.  Else
// the first chunk's workgroup draws from the target's row.  Bound by latency: 11 us for one sequence, 18 us for 32 of 152064
// logits, 4 of which are the weights of two rows a sequence.
constexpr int AC_TEST = 512, AC_WAVES = AC_TEST / 64;
static_assert(AC_PARTS == AC_THREADS / 64 && AC_SHARES == AC_WAVES);
template <typename TL, typename TD>
__global__ void __launch_bounds__(AC_TEST) accept_draft_kernel(AcceptArgs p) {
  const int b = blockIdx.y, chunk = blockIdx.x;
  const SeqRows sr = seq_rows(p.r, b);
  if (sr.n <= 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const Heat h = heat_of(p, b);
  __shared__ double sm_z[64], sm_s[64];    // of a kept row's token: its logit relative to the maximum, and the row's sum
  __shared__ int sm_kept[AC_WAVES], sm_rest[AC_WAVES];   // of a wave's row: its token is kept; else what remains of p is drawn from
  __shared__ RowStats sm_p[AC_WAVES], sm_q[AC_WAVES];
  __shared__ Exp2Table tab;
  fill_table(tab);
  __syncthreads();
  int at = 0;                              // the last kept row
  bool rest = false;
  RowStats tp{}, tq{};                     // of it, and of the draft's row behind it
  for (int j0 = 1;; j0 += AC_WAVES) {
    // wave w: row j0 + w against its draft, the target's row before it
    const int j = j0 + wave;
    if (j <= sr.n) {
      // everything that is known of the two rows at once
      const int r = sr.r0 + j - 1, next = j < sr.n ? r + 1 : r, x = p.ids[next];
      const bool test = j < sr.n, in = (unsigned)x < (unsigned)p.vocab;
      const float u = p.u[next], lx = logit((const TL*)p.logits + (long)r * p.row, in ? x : 0),
                  dx = test ? logit((const TD*)p.draft + (long)next * p.draft_row, in ? x : 0) : 0.f;
      const LaneParts lp_ = lane_parts(p, tab, r, h), lq = test ? lane_parts(p, tab, p.r.rows + next, h) : LaneParts{-INFINITY, 0, 0.0};
      const RowStats a = join_parts(tab, lp_, h), q = join_parts(tab, lq, h);
      bool kept = false, some = false;
      double zp = 0.0;
      if (test && has_dist(a, h)) {
        if (h.inv == 0.0) {
          kept = x == a.arg;
        } else {
          some = has_dist(q, h);
          if (in && some) {                // u q(x) < p(x), times both sums
            zp = ((double)lx - (double)a.m) * h.inv;
            kept = uniform(u) * exp2_neg(tab, ((double)dx - (double)q.m) * h.inv) * a.s < exp2_neg(tab, zp) * q.s;
          }
        }
      }
      if (lane == 0) {
        sm_kept[wave] = kept, sm_rest[wave] = some && !kept;
        sm_p[wave] = a, sm_q[wave] = q;
        if (kept) sm_z[j - 1] = zp, sm_s[j - 1] = a.s;
      }
    } else if (lane == 0) {
      sm_kept[wave] = 0;
    }
    __syncthreads();
    int w = 0;
    while (w < AC_WAVES && sm_kept[w]) ++w;
    if (w < AC_WAVES) {
      at = j0 + w - 1;
      rest = sm_rest[w];
      tp = sm_p[w], tq = sm_q[w];
      break;
    }
    __syncthreads();
  }
  const int r = sr.r0 + at;
  const float u = p.u[sr.r0];
  int token;
  if (rest) {
    const TL* rp = (const TL*)p.logits + (long)r * p.row;
    const TD* rq = (const TD*)p.draft + (long)(r + 1) * p.draft_row;
    // times p's sum, so that equal logits of the target weigh exactly 1 and their running sums are exact
    const double iq = tp.s / tq.s;
    const Weigh wp(tp.m, h), wq(tq.m, h);
    auto more = [&](int i) {
      const double d = wp(tab, logit(rp, i)) - wq(tab, logit(rq, i)) * iq;
      return d > 0.0 ? d : 0.0;
    };
    // a wave's part of the chunk: its share of 8, in runs
    constexpr int SHARE = AC_CHUNK / AC_WAVES;
    double sum = 0.0;
    const int first = chunk * AC_CHUNK + wave * SHARE + lane;
#pragma unroll
    for (int i = 0; i < SHARE / 64; ++i) {
      const double w = more(min(first + 64 * i, p.vocab - 1));
      sum += first + 64 * i < p.vocab ? w : 0.0;
    }
    sum = wave_sum64(sum);
    const int shares = p.chunks * AC_WAVES;
    double* parts = p.rest_sum + (long)b * shares;
    if (lane == 0) put(parts + chunk * AC_WAVES + wave, sum);
    if (arrive(p.counters + b) != (unsigned)p.chunks) return;
    __shared__ double sm_shares[AC_MAX_CHUNKS * AC_SHARES];
    for (int i = threadIdx.x; i < shares; i += AC_TEST) sm_shares[i] = get(parts + i);
    __syncthreads();
    double total = 0.0;
    for (int c = lane; c < shares; c += 64) total += sm_shares[c];
    total = wave_sum64(total);
    if (total > 0.0) {
      const double target = uniform(u) * total;
      double before = 0.0;
      const int c = first_above(shares, target, &before, [&](int i) { return sm_shares[i]; });
      token = draw_in_part<SHARE, AC_TEST>(c * SHARE, p.vocab, target - before, more);
    } else {                               // nothing is left by rounding: p and q are alike
      token = draw_row<AC_TEST, TL>(p, tab, r, tp, h, u);
    }
  } else {
    if (chunk != 0) return;
    token = draw_row<AC_TEST, TL>(p, tab, r, tp, h, u);
  }
  const int i = threadIdx.x;
  if (i == 0) p.n_keep[b] = at + 1;
  if (i < p.r.max_rows) {
    const long o = (long)b * p.r.max_rows + i;
    p.path[o] = i <= at ? i : -1;
    p.tokens[o] = i < at ? p.ids[sr.r0 + i + 1] : i == at ? token : -1;
    p.lp[o] = i < at ? (h.inv == 0.0 ? 0.f : (float)(sm_z[i] * LN2 - log(sm_s[i]))) : i == at ? log_p<TL>(p, r, tp, h, token) : 0.f;
  }
}

// ------------------------------------------------------------------ launch
int accept_chunks(int vocab) { return (vocab + AC_CHUNK - 1) / AC_CHUNK; }

template <typename TL, typename TD>
static hipError_t accept_types(const AcceptArgs& p, hipStream_t s) {
  const long blocks = std::max<long>(1, (long)p.items * p.chunks);
  hipLaunchKernelGGL((accept_stats_kernel<TL, TD>), dim3((unsigned)blocks), dim3(256), 0, s, p);
  if (hipError_t e = hipGetLastError()) return e;
  if (p.r.rows == 0) return hipSuccess;
  // in two dimensions: sequences times chunks times 512 threads may pass the 2^32 of one
  if (p.draft) hipLaunchKernelGGL((accept_draft_kernel<TL, TD>), dim3((unsigned)p.chunks, (unsigned)p.r.batch), dim3(AC_TEST), 0, s, p);
  else hipLaunchKernelGGL((accept_follow_kernel<TL>), dim3((unsigned)p.r.rows), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t accept(const AcceptArgs& p, hipStream_t s) {
  if (p.r.max_rows <= 0 || p.r.max_rows > 64 || p.vocab <= 0 || p.vocab > AC_MAX_CHUNKS * AC_CHUNK) return hipErrorInvalidValue;
  if (p.f32) return p.draft_f32 ? accept_types<float, float>(p, s) : accept_types<float, bf16_t>(p, s);
  return p.draft_f32 ? accept_types<bf16_t, float>(p, s) : accept_types<bf16_t, bf16_t>(p, s);
}

}  // namespace nova
