// Attention of drafted tokens over a paged cache.  Sequence b brings n rows (1 to 64 drafted tokens, a
// tree or a chain), already appended to its cache as tokens ctx .. ctx + n - 1; each row sees every
// token below ctx and those drafted tokens whose bit is set in its mask:
//   out = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale q.k_t - max).
// One pass over the cache with a running maximum and sum (in fp32, base 2).
//  * The rows (token, query head) that share a KV head are the MFMA columns, so K and V are read once
//    for many: S = K Q^T and O^T = V^T P^T.
//  * Which token is which MFMA row is free, so a lane (or lane group) is given consecutive tokens and
//    finds its V of a dimension, [D][16 tokens] in the cache, in 16-byte loads.
//  * e4m3 turns into bf16 exactly on the way to the MFMA: K with its token's scale, V without; V's
//    scale goes onto p, a power of two.  p is rounded to bf16 once (the matrix cores take no other
//    type beside bf16 V); the sum of p keeps fp32.  The f32 cache uses the fp32 matrix instructions.
//  * grid (context splits, KV head x row tiles, sequence); a second kernel joins the splits.
#include <algorithm>

#include "paged.hpp"

namespace nova {

NOVA_DEV f32x4 mfma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

template <typename CT> struct TreeT;
template <> struct TreeT<e4m3_t> { typedef bf16_t act; static constexpr int JN = 4; };
template <> struct TreeT<bf16_t> { typedef bf16_t act; static constexpr int JN = 2; };
template <> struct TreeT<float> { typedef float act; static constexpr int JN = 2; };

// Raw registers of a step: the lane's K rows (MFMA row block j) and V rows (dimension 16 i + col).
template <typename CT, int D> struct TreeRaw {
  static constexpr int JN = TreeT<CT>::JN;
  static constexpr int KW = D * sizeof(CT) / 64;          // 16-byte words of a K row per lane
  static constexpr int VW = 4 * JN * sizeof(CT) / 16;     // of a V row
  u32x4 k[JN][KW];
  u32x4 v[D / 16][VW];
  uint8_t ks[JN];                                         // e4m3: exponent bytes of the lane's K rows
  u32x4 ve;                                               // e4m3: exponent bytes of the lane group's 16 tokens
  bool ok;                                                // the lane group's own block (V) exists
};

// The elements of 16 bytes of V that are not finite, a bit each (e4m3 has NaN only).
template <typename CT> NOVA_DEV uint32_t v_odd(u32x4 q) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  uint32_t is = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = w[i];
    if constexpr (sizeof(CT) == 4) {
      is |= (x & 0x7F800000u) == 0x7F800000u ? 1u << i : 0u;
    } else if constexpr (sizeof(CT) == 2) {
      is |= (x & 0x7F80u) == 0x7F80u ? 1u << 2 * i : 0u;
      is |= (x & 0x7F800000u) == 0x7F800000u ? 2u << 2 * i : 0u;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) is |= ((x >> 8 * e) & 0x7Fu) == 0x7Fu ? 1u << (4 * i + e) : 0u;
    }
  }
  return is;
}
// A V element where it is not finite (as a float), 0 elsewhere.
template <typename CT> NOVA_DEV float odd_value(CT x) {
  if constexpr (sizeof(CT) == 1) return (x.v & 0x7F) == 0x7F ? __uint_as_float(0x7FC00000u) : 0.f;
  else return to_f<CT>(x);
}
// 16 bytes of V with the elements cleared whose bit in `keep` is not set.
template <typename CT> NOVA_DEV u32x4 v_keep(u32x4 q, uint32_t keep) {
  constexpr int EPW = 4 / sizeof(CT);                     // elements per dword
  constexpr uint32_t one = sizeof(CT) == 4 ? ~0u : (1u << (8 * (sizeof(CT) & 3))) - 1u;
  uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < EPW; ++e) m |= ((keep >> (i * EPW + e)) & 1u) ? one << (8 * sizeof(CT) * e % 32) : 0u;
    w[i] &= m;
  }
  return u32x4{w[0], w[1], w[2], w[3]};
}

// A row whose sum of p is 0: zeros where it sees no token, and NaN where it sees some, all with scores of -infinity,
// whose softmax is 0 / 0.  Found out here, at the end and rarely, so that the passes over the cache pay nothing for it.
NOVA_DEV float empty_row(const TreeArgs& p, int b, unsigned long long sees) {
  const SeqRows sr = seq_rows(p.r, b);
  const int total = min(sr.ctx + sr.n, p.r.max_ctx);
  bool any = false;
#pragma unroll 1
  for (int j = max(0, -sr.ctx); j < total - sr.ctx && !any; ++j)
    any = ((sees >> j) & 1) && page_of(p.r, p.c.num_blocks, b, (sr.ctx + j) / PAGE) >= 0;
#pragma unroll 1
  for (int t = 0; t < sr.ctx && !any; t += PAGE) any = page_of(p.r, p.c.num_blocks, b, t / PAGE) >= 0;
  return any ? __uint_as_float(0x7FC00000u) : 0.f;
}
NOVA_DEV unsigned long long seen_by(const TreeArgs& p, const SeqRows& sr, int t) {
  return p.mask ? p.mask[sr.r0 + t] : (2ull << t) - 1;    // of its sequence's drafted tokens, a bit each
}

// Steps of a split: the plan's number of splits shares out the sequence's own steps, `least` at a time.
NOVA_DEV int split_steps(int nsteps, int nsplit, int least) { return max(least, (nsteps + nsplit - 1) / nsplit); }

// ------------------------------------------------------------------ few rows
// One tile of 16 rows: bound by the cache's bytes.  The waves of a workgroup take steps in turn, each from
// memory to its own registers (K of the next step is requested once S is formed, V once it is used).  32 single
// tokens of 28/4 heads of 128 behind 2700 to 3627 e4m3 tokens: 106 MB in 23.4 to 25 us, 4.2 to 4.5 TB/s where a large
// copy reaches 5.0; bf16 209 MB in 42.4 us, 4.9 TB/s.  The fp32 cache's calls are small: 5 tokens behind 96, 6.8 us of latency.
template <typename CT, int D>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
tree_attn_kernel(TreeArgs p, int least) {
  typedef typename TreeT<CT>::act T;
  typedef TreeRaw<CT, D> Raw;
  constexpr bool F32 = sizeof(CT) == 4, Q8 = sizeof(CT) == 1;
  constexpr int JN = Raw::JN, TPG = 4 * JN, STEP = 16 * JN, BPS = STEP / PAGE, ND = D / 16;
  constexpr int NS = D / 32;                              // bf16 k-steps of S
  __shared__ float sm_m[4][16], sm_l[4][16];
  __shared__ float sm_o[4][16][D + 4];
  __shared__ int sm_odd;                                  // some drafted token's V is not finite

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_kv = p.c.n_kv, G = p.n_q / n_kv;
  const int split = blockIdx.x, kvh = blockIdx.y % n_kv, row0 = blockIdx.y / n_kv * 16, b = blockIdx.z;
  const int col = lane & 15, grp = lane >> 4;
  const SeqRows sr = seq_rows(p.r, b);
  const int nrow = sr.n * G;
  if (row0 >= nrow) return;
  const int total = min(sr.ctx + sr.n, p.r.max_ctx);      // the sequence's tokens that exist
  const int nsteps = (total + STEP - 1) / STEP, nblk = min((total + PAGE - 1) / PAGE, p.r.max_blocks);
  const int per = split_steps(nsteps, gridDim.x, least);
  const int step0 = split * per, step1 = min(step0 + per, nsteps);
  const int first = step0 + wave;
  const int n_it = first < step1 ? (step1 - first + 3) / 4 : 0;
  const int* table = p.r.tables + (size_t)b * p.r.max_blocks;

  // block ids of 64 / BPS iterations at a time, one per lane
  int tl = -1, tl_chunk = -1;
  constexpr int IPC = 64 / BPS;
  auto page = [&](int it, int j) -> int {
    if (it / IPC != tl_chunk) {
      tl_chunk = it / IPC;
      const int blk = (first + 4 * (tl_chunk * IPC + lane / BPS)) * BPS + lane % BPS;
      tl = blk < nblk ? table[blk] : -1;
      if ((unsigned)tl >= (unsigned)p.c.num_blocks) tl = -1;
    }
    return __shfl(tl, (it % IPC) * BPS + j, 64);
  };
  Raw raw;
  auto load_k = [&](int it) {
    // MFMA row col of block j is token TPG (col / 4) + 4 j + col % 4 of the step
    const int t = TPG * (col >> 2) + (col & 3);
    const size_t tok = ((size_t)max(page(it, t / PAGE), 0) * n_kv + kvh) * PAGE + t % PAGE;
#pragma unroll
    for (int j = 0; j < JN; ++j) {
      // a lane's 16 bytes of word w: dimensions 64 w + 16 grp .. of e4m3, 32 w + 8 grp .. of bf16, 16 w + 4 grp .. of f32
      const u32x4* kr = reinterpret_cast<const u32x4*>(reinterpret_cast<const CT*>(p.c.k) + (tok + 4 * j) * D) + grp;
#pragma unroll
      for (int w = 0; w < Raw::KW; ++w) raw.k[j][w] = kr[4 * w];
      if constexpr (Q8) raw.ks[j] = p.c.k_exp[tok + 4 * j];
    }
  };
  auto load_v = [&](int it) {
    const int t = TPG * grp, ph = page(it, t / PAGE);
    raw.ok = ph >= 0;
    const size_t tok = ((size_t)max(ph, 0) * n_kv + kvh) * PAGE;
    const CT* vr = reinterpret_cast<const CT*>(p.c.v) + tok * D + (size_t)col * PAGE + t % PAGE;
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int w = 0; w < Raw::VW; ++w) raw.v[i][w] = reinterpret_cast<const u32x4*>(vr + (size_t)16 * i * PAGE)[w];
    if constexpr (Q8) raw.ve = *reinterpret_cast<const u32x4*>(p.c.v_exp + tok);
  };
  if (n_it > 0) {
    load_k(0);
    load_v(0);
  }
  if (tid == 0) sm_odd = 0;
  __syncthreads();

  // this lane's row: its drafted token, its q and what it sees of the drafted ones
  const int rc = min(row0 + col, nrow - 1), mine_t = rc / G;
  const T* qrow = reinterpret_cast<const T*>(p.q) + (sr.r0 + mine_t) * p.q_row + (kvh * G + rc % G) * D;
  const unsigned long long sees = seen_by(p, sr, mine_t);
  // Q^T fragments: the dimensions of each k-step in the order in which K's words hold them
  Frag8 qf[F32 ? 1 : NS];
  f32x4 qx[F32 ? D / 16 : 1];
  if constexpr (F32) {
#pragma unroll
    for (int w = 0; w < D / 16; ++w) qx[w] = *reinterpret_cast<const f32x4*>(qrow + 16 * w + 4 * grp) * (p.scale < 0.f ? -1.f : 1.f);
  } else {
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      qf[s] = *reinterpret_cast<const Frag8*>(qrow + (Q8 ? 64 * (s >> 1) + 16 * grp + 8 * (s & 1) : 32 * s + 8 * grp));
      if (p.scale < 0.f) {                                // |scale| is folded into the exponent below
#pragma unroll
        for (int e = 0; e < 4; ++e) qf[s].w[e] ^= 0x80008000u;
      }
    }
  }

  f32x4 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;                   // l_run: of this lane group's tokens only
  const float scale = fmaxf(fabsf(p.scale) * 1.4426950408889634f, 1e-37f);   // not 0: -infinity stays what it is

  for (int it = 0; it < n_it; ++it) {
    const int mine = (first + 4 * it) * STEP + TPG * grp;         // the lane group's first token
    const bool masked = (first + 4 * it) * STEP + STEP > sr.ctx || !__all(raw.ok);   // drafted tokens, the end, a missing block
    const int valid = !masked ? TPG : raw.ok ? min(max(total - mine, 0), TPG) : 0;
    // S: lane holds scores of its lane group's tokens 4 j + q for row col
    f32x4 sc[JN];
#pragma unroll
    for (int j = 0; j < JN; ++j) {
      sc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < Raw::KW; ++w) {
        const u32x4 x = raw.k[j][w];
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[j] = mfma4(__uint_as_float(x[e]), qx[w][e], sc[j]);
        } else if constexpr (Q8) {
          const float s = exp_scale(raw.ks[j]);
          const Frag8 a{{e4m3_pair<false>(x.x, s), e4m3_pair<true>(x.x, s), e4m3_pair<false>(x.y, s), e4m3_pair<true>(x.y, s)}};
          const Frag8 c{{e4m3_pair<false>(x.z, s), e4m3_pair<true>(x.z, s), e4m3_pair<false>(x.w, s), e4m3_pair<true>(x.w, s)}};
          sc[j] = mfma16(a, qf[2 * w], sc[j]);
          sc[j] = mfma16(c, qf[2 * w + 1], sc[j]);
        } else {
          sc[j] = mfma16(__builtin_bit_cast(Frag8, x), qf[w], sc[j]);
        }
      }
    }
    if (it + 1 < n_it) load_k(it + 1);

    if (masked) {
      // what the lane's row sees of the lane group's tokens, a bit each
      const int dr = mine - sr.ctx;                               // the first token as a drafted one
      const unsigned long long m = dr >= 64 ? 0ull : dr >= 0 ? sees >> dr : dr <= -TPG ? ~0ull : (sees << -dr) | ((1ull << -dr) - 1);
      const uint32_t held = (1u << valid) - 1u, vis = (uint32_t)m & held;
#pragma unroll
      for (int e = 0; e < TPG; ++e) sc[e >> 2][e & 3] = (vis >> e) & 1 ? sc[e >> 2][e & 3] : -INFINITY;
      // Slots past the last token may hold anything: their V is cleared.  A drafted token's V that is not
      // finite concerns the rows that see it and no other, and 0 times infinity is not 0: such elements
      // are cleared too and added when the rows are written.
      const uint32_t drafted = mine >= sr.ctx ? ~0u : mine + TPG <= sr.ctx ? 0u : ~0u << (sr.ctx - mine);
      uint32_t odd = 0;
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int w = 0; w < Raw::VW; ++w) {
          constexpr int N = 16 / sizeof(CT);
          u32x4 v = v_keep<CT>(raw.v[i][w], held >> (w * N));
          const uint32_t is = v_odd<CT>(v) & (drafted >> (w * N));
          if (is) v = v_keep<CT>(v, ~is);
          odd |= is;
          raw.v[i][w] = v;
        }
      if (odd) sm_odd = 1;
    }

    // softmax; p as the MFMA's P^T operand (tokens 8 h .. 8 h + 7 of the lane group).  The sums move to a new
    // maximum only when it exceeds theirs by 2^8: until then p is at most 2^8, which rounds no worse.
    float s[TPG];
    float tmax = -INFINITY;
#pragma unroll
    for (int e = 0; e < TPG; ++e) tmax = fmaxf(tmax, sc[e >> 2][e & 3]);
    tmax = fmaxf(tmax, __shfl_xor(tmax, 16, 64));
    tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
    const float m_new = fmaxf(m_run, tmax * scale);
    if (__any(m_new > m_run + 8.f)) {
      const float corr = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
      m_run = m_new;
      l_run *= corr;
#pragma unroll
      for (int i = 0; i < ND; ++i) o[i] *= corr;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;         // nothing seen yet: every p is 0
#pragma unroll
    for (int e = 0; e < TPG; ++e) {
      s[e] = __builtin_amdgcn_exp2f(fmaf(sc[e >> 2][e & 3], scale, -m_use));
      l_run += s[e];
    }
    Frag8 pf[F32 ? 1 : JN / 2];
    if constexpr (!F32) {
      if constexpr (Q8) {
#pragma unroll
        for (int e = 0; e < TPG; ++e) {
          const float vs = exp_scale((raw.ve[e >> 2] >> (8 * (e & 3))) & 255u);
          s[e] = e < valid ? s[e] * vs : 0.f;
        }
      }
#pragma unroll
      for (int h = 0; h < JN / 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) pf[h].w[e] = pack2(s[8 * h + 2 * e], s[8 * h + 2 * e + 1]);
    }
    // O^T += V^T P^T
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < TPG; ++e) o[i] = mfma4(__uint_as_float(raw.v[i][e >> 2][e & 3]), s[e], o[i]);
      } else if constexpr (Q8) {
        const u32x4 x = raw.v[i][0];
        const Frag8 a{{e4m3_pair<false>(x.x, 1.f), e4m3_pair<true>(x.x, 1.f), e4m3_pair<false>(x.y, 1.f), e4m3_pair<true>(x.y, 1.f)}};
        const Frag8 c{{e4m3_pair<false>(x.z, 1.f), e4m3_pair<true>(x.z, 1.f), e4m3_pair<false>(x.w, 1.f), e4m3_pair<true>(x.w, 1.f)}};
        o[i] = mfma16(a, pf[0], o[i]);
        o[i] = mfma16(c, pf[JN / 2 - 1], o[i]);
      } else {
        o[i] = mfma16(__builtin_bit_cast(Frag8, raw.v[i][0]), pf[0], o[i]);
      }
    }
    if (it + 1 < n_it) load_v(it + 1);
  }

  // the lane groups' sums, then the four waves
  const int nsplit = gridDim.x;
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  if (grp == 0) { sm_m[wave][col] = m_run; sm_l[wave][col] = l_run; }
#pragma unroll
  for (int i = 0; i < ND; ++i) *reinterpret_cast<f32x4*>(&sm_o[wave][col][16 * i + 4 * grp]) = o[i];
  __syncthreads();
  for (int idx = tid; idx < 16 * D; idx += 256) {
    const int c = idx / D, d = idx % D, r = row0 + c;
    if (r >= nrow) break;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, sm_m[w][c]);
    const float mu = M == -INFINITY ? 0.f : M;
    float L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm_m[w][c] - mu);
      L += f * sm_l[w][c];
      O += f * sm_o[w][c][d];
    }
    const long t = sr.r0 + r / G;
    if (sm_odd) {
      const unsigned long long see = seen_by(p, sr, r / G);
#pragma unroll 1
      for (int j = max(0, step0 * STEP - sr.ctx); j < min(total, step1 * STEP) - sr.ctx; ++j) {
        const int tok = sr.ctx + j, ph = page_of(p.r, p.c.num_blocks, b, tok / PAGE);
        if (!((see >> j) & 1) || ph < 0) continue;
        const float v = odd_value<CT>(reinterpret_cast<const CT*>(p.c.v)[(((size_t)ph * n_kv + kvh) * D + d) * PAGE + tok % PAGE]);
        if (!(fabsf(v) < INFINITY)) O += v;
      }
    }
    const int head = kvh * G + r % G;
    if (nsplit == 1) {
      reinterpret_cast<T*>(p.out)[t * p.out_row + head * D + d] = from_f<T>(L == 0.f ? empty_row(p, b, seen_by(p, sr, r / G)) : O / L);
    } else {
      float* part = p.partial + ((t * p.n_q + head) * nsplit + split) * (D + 4);
      part[4 + d] = O;
      if (d == 0) { part[0] = M; part[1] = L; }
    }
  }
}

// ------------------------------------------------------------------ many rows
// Above 16 rows of a KV head the products outweigh the loads, and the waves share K and V: workgroup of
// 4 waves x 32 rows, 64 tokens at a time staged in LDS as bf16 (8-bit ones are converted once for
// the four waves), two buffers, so that a step costs one barrier and the next step's loads are in flight
// during its products (32x32x16: S = K Q^T, O^T = V^T P^T).  S's rows are read in the order in which
// lane half h then holds tokens 16 u + 8 h + e of each 32, the ones that it hands to the second product.
// 16-byte pieces are swizzled by their row so that a read covers every bank once.
// Two sequences of 64 and 48 tokens behind 32700 and 28613 (28/4 heads of 128, e4m3): 5.0e10 operations in
// 86 us, 0.58 PFLOP/s.  Of its cycles the MFMAs are busy for 24% and LDS for 30% (and 7% of bank conflicts), and vector
// instructions issue in 32%: none of them bounds it, the two waves of a SIMD do, whose chains (scores, exponentials,
// conversion, product, barrier) cover each other's waits in part; 31% of their time is waiting.
// 64 rows a wave halve the LDS reads, but leave one wave a SIMD, whose vector instructions issue every 5 clocks
// instead of 4 and wait alone: 116 us.
// Eight sequences of 9 to 16 tokens behind 1222 to 1564 (bf16): 17 us, four steps of 1.7 us, the rest
// launch and first loads.
// HALF (up to 64 rows): waves 0 and 1 take the first 32 tokens of every step, waves 2 and 3 the others for the same
// rows, and the pairs join at the end.  Five tokens of 28/4 heads (35 rows), 32 sequences behind 1800 e4m3 tokens:
// 24.9 us, with two waves idle 27.9; one sequence behind 30000 25.8 and 28.1; but where a workgroup has a step or
// two the join costs 0.4 us more than it gains.
template <typename CT, int D, bool HALF>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
tree_wide_kernel(TreeArgs p, int least) {
  constexpr bool Q8 = sizeof(CT) == 1;
  constexpr int STEP = 64, ND = D / 32, NS = D / 16;
  constexpr int LW = STEP * D * sizeof(CT) / 16 / 256;            // 16-byte loads of a thread, for K and for V
  constexpr int KPT = D * sizeof(CT) / 16;                        // of a K row
  constexpr int VPT = PAGE * sizeof(CT) / 16;                     // of a V row of a block
  // K [2][64 tokens][D] and V [2][D][64 tokens] in bf16, byte-addressed: the 16-byte piece c of a row sits at
  // c ^ x(row), so pieces 2 n + h of a row are one address, of piece h, with n << 5 toggled
  constexpr int KBUF = STEP * D * 2, VBUF = D * STEP * 2;
  __shared__ __align__(1024) unsigned char smem[2 * KBUF + 2 * VBUF];
  __shared__ __align__(16) float sm_vs[2][STEP + 64];
  __shared__ int sm_odd;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_kv = p.c.n_kv, G = p.n_q / n_kv;
  const int split = blockIdx.x, kvh = blockIdx.y % n_kv, tile = blockIdx.y / n_kv, b = blockIdx.z;
  const int col = lane & 31, half = lane >> 5;
  const SeqRows sr = seq_rows(p.r, b);
  const int nrow = sr.n * G, row0 = tile * 128, rows_of = HALF ? wave & 1 : wave, second = HALF ? wave >> 1 : 0;
  if (row0 >= nrow) return;
  const int total = min(sr.ctx + sr.n, p.r.max_ctx);      // the sequence's tokens that exist
  const int nsteps = (total + STEP - 1) / STEP;
  const int per = split_steps(nsteps, gridDim.x, least);
  const int step0 = split * per, step1 = min(step0 + per, nsteps);
  const bool active = row0 + 32 * rows_of < nrow;
  const int row = row0 + 32 * rows_of + col, rc = min(row, nrow - 1);
  const int t = rc / G, head = kvh * G + rc % G;
  const unsigned long long sees = seen_by(p, sr, t);
  if (tid == 0) sm_odd = 0;

  // Block ids of 16 steps at a time, one per lane (those that exist), the next 16 requested ahead: a
  // step's loads wait for no table load.  A wave's u-th 16-byte load of K and of V lies in one block.
  const int* table = p.r.tables + (size_t)b * p.r.max_blocks;
  const int nblk = (total + PAGE - 1) / PAGE;
  auto entries = [&](int step) -> int {
    const int blk = 4 * step + lane;
    const int ph = blk < min(nblk, p.r.max_blocks) ? table[blk] : -1;
    return (unsigned)ph < (unsigned)p.c.num_blocks ? ph : -1;
  };
  int tl = entries(step0), tl_next = entries(step0 + 16);
  constexpr int BB = D * sizeof(CT);                              // 16-byte pieces of a block's K, and of its V
  constexpr int UB = 4 / LW;                                      // blocks that a load of the workgroup covers
  const int wblk = __builtin_amdgcn_readfirstlane(tid / BB % UB), piece = tid % BB;
  u32x4 rk[LW], rv[LW];
  uint8_t rks[Q8 ? LW : 1], rvs[Q8 ? LW : 1];                     // exponent bytes: nothing waits for the loads here
  unsigned exists = 0;                                            // of the loaded step's 4 blocks, a bit each
  auto advance = [&](int step) {                                  // before the load of a step whose ids are the next 16's
    if (((step - step0) & 15) == 0) {
      tl = tl_next;
      tl_next = entries(step + 16);
    }
  };
  auto load = [&](int step) {
    const int at = 4 * ((step - step0) & 15);
    exists = (unsigned)(__ballot(tl >= 0) >> at) & 15u;
#pragma unroll
    for (int u = 0; u < LW; ++u) {
      const int ph = max(__builtin_amdgcn_readlane(tl, at + UB * u + wblk), 0);
      const size_t blk = (size_t)ph * n_kv + kvh;
      unsigned off = piece;
      asm volatile("" : "+v"(off));                               // uniform base + 32-bit offset, not a 64-bit address kept per pool
      rk[u] = (reinterpret_cast<const u32x4*>(p.c.k) + blk * BB)[off];
      rv[u] = (reinterpret_cast<const u32x4*>(p.c.v) + blk * BB)[off];
      if constexpr (Q8) {
        rks[u] = (p.c.k_exp + blk * PAGE)[off / KPT];
        rvs[u] = (p.c.v_exp + blk * PAGE)[off % PAGE];
      }
    }
  };
  auto keep_of = [&](int step) -> unsigned long long {            // tokens inside the sequence, in blocks that exist
    const int left = total - step * STEP;
    if (left >= STEP && exists == 15u) return ~0ull;
    unsigned long long m = left >= 64 ? ~0ull : (1ull << left) - 1;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (!((exists >> j) & 1)) m &= ~(0xFFFFull << (16 * j));
    return m;
  };
  auto kat = [&](int r, int c) { return r * (2 * D) + ((D == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7)) << 4); };
  auto vat = [&](int d, int c) { return d * (2 * STEP) + ((c ^ ((d >> 1) & 7)) << 4); };
  auto masked_step = [&](int step, unsigned long long keep) { return (step + 1) * STEP > sr.ctx || keep != ~0ull; };
  // Slots that hold no token are cleared, and drafted values that are not finite, which concern the rows
  // that see them only, are added when the rows are written.
  auto clean = [&](int step, unsigned long long keep) {
#pragma unroll
    for (int u = 0; u < LW; ++u) {
      constexpr int N = 16 / sizeof(CT);
      const int j = UB * u + wblk, t0 = PAGE * j + piece % VPT * N;
      const int first = sr.ctx - (step * STEP + t0);              // its first drafted token
      u32x4 v = v_keep<CT>(rv[u], (uint32_t)(keep >> t0));
      const uint32_t odd = v_odd<CT>(v) & (first >= N ? 0u : ~0u << max(first, 0));
      if (odd) {
        v = v_keep<CT>(v, ~odd);
        sm_odd = 1;
      }
      rv[u] = v;
      if constexpr (Q8)
        if (!((keep >> (PAGE * j + piece % PAGE)) & 1)) rvs[u] = 0;     // its scale may be anything: 0
    }
  };
  // where the thread's first load goes; its u-th lies UB blocks on: 16 UB rows of K (the same x), 2 UB pieces of V
  const int kw = kat(PAGE * wblk + piece / KPT, (Q8 ? 2 : 1) * (piece % KPT));
  const int vw = 2 * KBUF + vat(piece / VPT, 2 * wblk + piece % VPT);
  auto store = [&](int buf) {
#pragma unroll
    for (int u = 0; u < LW; ++u) {
      const int ka = kw + buf * KBUF + u * UB * PAGE * 2 * D, va = (vw + buf * VBUF) ^ (u * UB << 5);
      if constexpr (Q8) {
        const u32x4 a = rk[u], v = rv[u];
        const float s = exp_scale(rks[u]);
        *reinterpret_cast<u32x4*>(smem + ka) = u32x4{e4m3_pair<false>(a.x, s), e4m3_pair<true>(a.x, s), e4m3_pair<false>(a.y, s), e4m3_pair<true>(a.y, s)};
        *reinterpret_cast<u32x4*>(smem + (ka ^ 16)) = u32x4{e4m3_pair<false>(a.z, s), e4m3_pair<true>(a.z, s), e4m3_pair<false>(a.w, s), e4m3_pair<true>(a.w, s)};
        *reinterpret_cast<u32x4*>(smem + va) = u32x4{e4m3_pair<false>(v.x, 1.f), e4m3_pair<true>(v.x, 1.f), e4m3_pair<false>(v.y, 1.f), e4m3_pair<true>(v.y, 1.f)};
        *reinterpret_cast<u32x4*>(smem + (va ^ 16)) = u32x4{e4m3_pair<false>(v.z, 1.f), e4m3_pair<true>(v.z, 1.f), e4m3_pair<false>(v.w, 1.f), e4m3_pair<true>(v.w, 1.f)};
        sm_vs[buf][piece < PAGE ? PAGE * (UB * u + wblk) + piece : STEP + lane] = exp_scale(rvs[u]);     // the others write nowhere
      } else {
        *reinterpret_cast<u32x4*>(smem + ka) = rk[u];
        *reinterpret_cast<u32x4*>(smem + va) = rv[u];
      }
    }
  };

  if (step0 < step1) load(step0);
  const bf16_t* qrow = reinterpret_cast<const bf16_t*>(p.q) + (sr.r0 + t) * p.q_row + head * D;
  Frag8 qf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    qf[s] = *reinterpret_cast<const Frag8*>(qrow + 16 * s + 8 * half);
    if (p.scale < 0.f) {                                          // |scale| is folded into the exponent below
#pragma unroll
      for (int e = 0; e < 4; ++e) qf[s].w[e] ^= 0x80008000u;
    }
  }
  f32x16 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;                           // l_run: of this lane half's tokens
  const float scale = fmaxf(fabsf(p.scale) * 1.4426950408889634f, 1e-37f);   // not 0: -infinity stays what it is
  __syncthreads();                                                // sm_odd is cleared
  unsigned long long keep = 0, keep_next = 0;                     // of the step at hand and of the one in registers
  if (step0 < step1) {
    keep = keep_of(step0);
    if (masked_step(step0, keep)) clean(step0, keep);
    store(0);
    if (step0 + 1 < step1) {
      load(step0 + 1);
      keep_next = keep_of(step0 + 1);
    }
  }
  __syncthreads();

  // MFMA row m of S is token tau of its 32
  const int tau = 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
  // A step is two halves of 32 tokens, so that matrix and vector instructions of one wave run side by
  // side: S of the first half beside the conversion of the next step into the other buffer, S of the second
  // beside the exponentials of the first, V^T P^T of the first beside those of the second; then the
  // step's one barrier, and V^T P^T of the second beside the loads of the step after next.  The LDS
  // reads of a product run L ahead of its MFMAs, over the steps' ends: V's last ones are read before
  // the barrier, after which nothing reads the step's buffer.  Left alone, the scheduler does neither.
  const int kr = kat(tau, half) + second * 32 * 2 * D, vr = (2 * KBUF + vat(col, half)) ^ (second * 2 << 5);
  auto k_read = [&](int buf, int x) {                             // x: 32-token half of the step and k-step
    return *reinterpret_cast<const Frag8*>(smem + ((kr + buf * KBUF) ^ (x % NS << 5)) + x / NS * 32 * 2 * D);
  };
  auto v_read = [&](int buf, int x) {                             // x: 16 tokens and 32 dimensions
    return *reinterpret_cast<const Frag8*>(smem + ((vr + buf * VBUF) ^ (x / ND << 5)) + x % ND * 32 * 2 * STEP);
  };
  constexpr int NK = HALF ? NS : 2 * NS, NF = NK + (HALF ? 2 : 4) * ND;   // operands of a step: K's, then V's (NS == 2 ND)
  constexpr int L = 2 * ND;                                       // divides NK and NF
  Frag8 f[L];
  auto read = [&](int buf, int x) { f[x % L] = x < NK ? k_read(buf, x) : x < NF ? v_read(buf, x - NK) : k_read(buf ^ 1, x - NF); };
  // scores of one half: seen or not, and whether the running maximum has to move
  auto hide = [&](f32x16& sc, uint32_t seen) {
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = seen & (1u << (16 * (r >> 3) + (r & 7))) ? sc[r] : -INFINITY;
  };
  auto top_of = [&](const f32x16& sc) {
    float m = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) m = fmaxf(m, sc[r]);
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])) * scale;   // both lane halves'
  };
  // p of elements e0 .. e0 + n - 1 of a half, packed as the second product's operand once 8 are there
  float px[8], rs = 0.f;
  auto expo = [&](const f32x16& sc, int buf, int h0, int e0, int n, float m, Frag8 (&pf)[2]) {
#pragma unroll
    for (int e = e0; e < e0 + n; ++e) {
      px[e & 7] = __builtin_amdgcn_exp2f(fmaf(sc[e], scale, -m));
      rs += px[e & 7];
      if ((e & 7) != 7) continue;
      const int h = e >> 3;                                       // 16 tokens
      if constexpr (Q8) {
        const float4 a = *reinterpret_cast<const float4*>(&sm_vs[buf][16 * (h0 + h) + 8 * half]);
        const float4 c = *reinterpret_cast<const float4*>(&sm_vs[buf][16 * (h0 + h) + 8 * half + 4]);
        px[0] *= a.x, px[1] *= a.y, px[2] *= a.z, px[3] *= a.w, px[4] *= c.x, px[5] *= c.y, px[6] *= c.z, px[7] *= c.w;
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) pf[h].w[w] = pack2(px[2 * w], px[2 * w + 1]);
      // computed here, beside the MFMAs, and not where it is used
      asm volatile("" : "+v"(pf[h].w[0]), "+v"(pf[h].w[1]), "+v"(pf[h].w[2]), "+v"(pf[h].w[3]));
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto base_of = [&]() { return m_run == -INFINITY ? 0.f : m_run; };   // nothing seen yet: every p is 0
  if (active) {
#pragma unroll
    for (int x = 0; x < L; ++x) read(0, x);
  }
  for (int step = step0; step < step1; ++step) {
    const int buf = (step - step0) & 1;
    if (step + 1 < step1 && masked_step(step + 1, keep_next)) clean(step + 1, keep_next);
    const int then = min(step + 2, step1 - 1);                    // at the end the last step once more: the loads stay in line
    if (step + 2 < step1) advance(step + 2);
    if (active) {
      const bool masked = masked_step(step, keep);
      unsigned long long vis = ~0ull;
      if (masked) {                                               // drafted tokens, the end, or a missing block
        const int dr = step * STEP - sr.ctx;                      // the step's first token as a drafted one
        vis = dr >= 64 ? 0ull : dr >= 0 ? sees >> dr : dr <= -64 ? ~0ull : (sees << -dr) | ((1ull << -dr) - 1);
        vis = (vis & keep) >> (8 * half + 32 * second);
      }
      f32x16 s0, s1;
      Frag8 p0[2], p1[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) s0[r] = s1[r] = 0.f;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < NS; ++x) {
        s0 = mfma32(f[x % L], qf[x], s0);
        read(buf, x + L);
      }
      store(buf ^ 1);                                             // after the last step: stale, and never used
      __builtin_amdgcn_sched_barrier(0);
      if (masked) hide(s0, (uint32_t)vis);
      // the sums move to a new maximum only when it exceeds theirs by 2^8: until then p is at most
      // 2^8, which rounds no worse, and the accumulators are left alone at most steps
      float top = fmaxf(m_run, top_of(s0));
      if (__any(top > m_run + 8.f)) {
        const float corr = __builtin_amdgcn_exp2f(m_run - (top == -INFINITY ? 0.f : top));
        m_run = top;
        l_run *= corr;
#pragma unroll
        for (int i = 0; i < ND; ++i) o[i] *= corr;
      }
      if constexpr (HALF) {
        const float base = base_of();
        rs = 0.f;
        __builtin_amdgcn_sched_barrier(0);
        expo(s0, buf, 2 * second, 0, 16, base, p0);
        l_run += rs;
        __syncthreads();
#pragma unroll
        for (int x = 0; x < 2 * ND; ++x) {
          o[x % ND] = mfma32(f[(NK + x) % L], p0[x / ND], o[x % ND]);
          read(buf, NK + x + L);
        }
      } else {
        const float base0 = base_of();
        rs = 0.f;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = NS; x < NK; ++x) {
          s1 = mfma32(f[x % L], qf[x - NS], s1);
          read(buf, x + L);
          expo(s0, buf, 0, (x - NS) * (16 / NS), 16 / NS, base0, p0);
        }
        l_run += rs;
        if (masked) hide(s1, (uint32_t)(vis >> 32));
        top = fmaxf(m_run, top_of(s1));
        const bool move = __any(top > m_run + 8.f);
        float corr = 1.f;
        if (move) {                                               // applied once the first half is added
          corr = __builtin_amdgcn_exp2f(m_run - (top == -INFINITY ? 0.f : top));
          m_run = top;
          l_run *= corr;
        }
        const float base1 = base_of();
        rs = 0.f;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < 2 * ND; ++x) {
          o[x % ND] = mfma32(f[(NK + x) % L], p0[x / ND], o[x % ND]);
          read(buf, NK + x + L);
          expo(s1, buf, 2, x * (8 / ND), 8 / ND, base1, p1);
        }
        l_run += rs;
        if (move) {
#pragma unroll
          for (int i = 0; i < ND; ++i) o[i] *= corr;
        }
        __syncthreads();
#pragma unroll
        for (int x = 2 * ND; x < 4 * ND; ++x) {
          o[x % ND] = mfma32(f[(NK + x) % L], p1[x / ND - 2], o[x % ND]);
          read(buf, NK + x + L);
        }
      }
      load(then);
      __builtin_amdgcn_sched_barrier(0);
    } else {
      store(buf ^ 1);
      __syncthreads();
      load(then);
    }
    keep = keep_next;
    keep_next = keep_of(then);
  }
  if constexpr (HALF) {                                           // nothing reads the steps' buffers any more after the barrier
    float* other = reinterpret_cast<float*>(smem) + rows_of * (16 * ND + 2) * 64 + lane;
    __syncthreads();
    if (second) {
      other[0] = m_run, other[64] = l_run;
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) other[64 * (2 + 16 * i + r)] = o[i][r];
    }
    __syncthreads();
    if (second) return;
    const float m = other[0], top = fmaxf(m, m_run), mu = top == -INFINITY ? 0.f : top;
    const float mine = __builtin_amdgcn_exp2f(m_run - mu), its = __builtin_amdgcn_exp2f(m - mu);
    l_run = l_run * mine + other[64] * its;
    m_run = top;
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] = o[i][r] * mine + other[64 * (2 + 16 * i + r)] * its;
  }
  if (!active || row >= nrow) return;
  float l = l_run;
  l += __shfl_xor(l, 32, 64);
  if (sm_odd) {
    const int j0 = max(0, step0 * STEP - sr.ctx), j1 = min(total, step1 * STEP) - sr.ctx;
#pragma unroll 1
    for (int j = j0; j < j1; ++j) {
      const int tok = sr.ctx + j, ph = page_of(p.r, p.c.num_blocks, b, tok / PAGE);
      if (!((sees >> j) & 1) || ph < 0) continue;
      const CT* vb = reinterpret_cast<const CT*>(p.c.v) + ((size_t)ph * n_kv + kvh) * D * PAGE + tok % PAGE;
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        __builtin_amdgcn_sched_barrier(0);                        // few loads at a time: rare, and it must not cost registers
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float v = odd_value<CT>(vb[(size_t)(32 * i + 8 * (r >> 2) + 4 * half + (r & 3)) * PAGE]);
          if (!(fabsf(v) < INFINITY)) o[i][r] += v;
        }
      }
    }
  }
  const int nsplit = gridDim.x;
  const long rh = (sr.r0 + t) * (long)p.n_q + head;
  if (nsplit == 1) {
    bf16_t* out = reinterpret_cast<bf16_t*>(p.out) + (sr.r0 + t) * p.out_row + head * D + 4 * half;
    const float inv = l == 0.f ? empty_row(p, b, sees) : 1.f / l;
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<uint2*>(out + 32 * i + 2 * r) = make_uint2(pack2(o[i][r] * inv, o[i][r + 1] * inv), pack2(o[i][r + 2] * inv, o[i][r + 3] * inv));
  } else {
    float* part = p.partial + (rh * nsplit + split) * (D + 4);
    if (half == 0) *reinterpret_cast<float2*>(part) = make_float2(m_run, l);
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<float4*>(part + 4 + 32 * i + 2 * r + 4 * half) = make_float4(o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]);
  }
}

// Joins the splits of a row and head: a wave each, D / 64 dimensions per lane.  Bound by latency: 4 to 5 us with 4
// to 7 splits, 6.3 us where 3584 rows and heads have 16.
template <typename T, int D>
__global__ void __launch_bounds__(256) tree_combine_kernel(TreeArgs p, int nsplit) {
  const int lane = threadIdx.x & 63;
  const SeqRows sr = seq_rows(p.r, blockIdx.y);
  const int i = blockIdx.x * 4 + (threadIdx.x >> 6);     // row of the sequence and head
  if (i >= sr.n * p.n_q) return;
  const long t = sr.r0 + i / p.n_q;
  const int head = i % p.n_q;
  const float* part = p.partial + (t * p.n_q + head) * nsplit * (D + 4);
  const float m = lane < nsplit ? part[lane * (D + 4)] : -INFINITY;
  const float l = lane < nsplit ? part[lane * (D + 4) + 1] : 0.f;
  const float M = wave_max(m);
  const float f = M == -INFINITY ? 0.f : exp2f(m - M);
  const float L = wave_sum(f * l);
  float o[D / 64] = {};
  for (int s0 = 0; s0 < nsplit; s0 += 8) {                // 8 splits' loads at a time
    float v[8][D / 64];
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
      for (int d = 0; d < D / 64; ++d) v[s][d] = s0 + s < nsplit ? part[(s0 + s) * (D + 4) + 4 + lane + 64 * d] : 0.f;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), min(s0 + s, 63)));
#pragma unroll
      for (int d = 0; d < D / 64; ++d) o[d] += w * v[s][d];
    }
  }
  const float empty = L == 0.f ? empty_row(p, blockIdx.y, seen_by(p, sr, i / p.n_q)) : 0.f;
#pragma unroll
  for (int d = 0; d < D / 64; ++d)
    reinterpret_cast<T*>(p.out)[t * p.out_row + head * D + lane + 64 * d] = from_f<T>(L == 0.f ? empty : o[d] / L);
}

// The kernel, the workgroups that a KV head's rows take, and the splits of the context: as many as give every
// compute unit two workgroups, of `least` steps at least.
//  * few rows: 4, one for each wave (1530 tokens, 32 sequences: 2 and 3 steps cost up to 1.5 us more).  A context of
//    two steps a wave is not split, nor one of four where the workgroups fill half the compute units (one token behind
//    400 in e4m3: 8.9 us, and 10.1 with two splits and their join; 32 sequences of one behind 1000: 13.0 and 14.6; but
//    one behind 1000: 11.8 and 10.7).
//  * many rows: a split's steps follow one another (1.7 us each), but every split is one more to join.  While there are
//    few workgroups short splits win (5 tokens behind 1000, one sequence: 10.9 us with 1, 14.2 with 4; 64 behind
//    600: 16.5 with 1, 14.3 with 2, 16.0 with 4), with many of them 4 do (5 behind 8000: 18.0 with 2, 16.6 with 4): as
//    many steps as keep the workgroups at half the compute units, 4 at most.
constexpr int LEAST_STEPS = 4;
struct TreePlan { bool wide, half; int tiles, nsplit, least; };
static TreePlan tree_plan(int type, int n_kv, int n_q, int batch, int max_rows, int max_ctx, int cus) {
  TreePlan t;
  const int rows = max_rows * (n_q / n_kv);
  t.wide = type != CACHE_F32 && rows > 16;
  t.tiles = (rows + (t.wide ? 127 : 15)) / (t.wide ? 128 : 16);
  const int step = t.wide || type == CACHE_E4M3 ? 64 : 32;
  const int steps = (max_ctx + step - 1) / step;
  const long wgs = (long)batch * n_kv * t.tiles, want = (2L * cus + wgs - 1) / wgs;
  if (t.wide) t.least = (int)std::min<long>(LEAST_STEPS, std::max(1L, (2 * wgs * steps + cus - 1) / cus));
  else t.least = steps <= 8 || (steps <= 16 && 2 * wgs >= cus) ? std::max(steps, LEAST_STEPS) : LEAST_STEPS;
  t.half = t.wide && rows <= 64 && t.least == LEAST_STEPS;
  t.nsplit = (int)std::max(1L, std::min({want, 64L, (steps + t.least - 1L) / t.least}));
  return t;
}

size_t tree_partial_floats(int type, int n_kv, int n_q, int D, int batch, int rows, int max_rows, int max_ctx, int cus) {
  const TreePlan t = tree_plan(type, n_kv, n_q, batch, max_rows, max_ctx, cus);
  return t.nsplit > 1 ? (size_t)rows * n_q * t.nsplit * (D + 4) : 0;
}

template <typename CT, int D>
static hipError_t tree_launch(const TreeArgs& p, const TreePlan& t, hipStream_t s) {
  typedef typename TreeT<CT>::act T;
  const dim3 grid(t.nsplit, p.c.n_kv * t.tiles, p.r.batch);
  if constexpr (sizeof(CT) < 4) {
    if (t.half) hipLaunchKernelGGL((tree_wide_kernel<CT, D, true>), grid, dim3(256), 0, s, p, t.least);
    else if (t.wide) hipLaunchKernelGGL((tree_wide_kernel<CT, D, false>), grid, dim3(256), 0, s, p, t.least);
    else hipLaunchKernelGGL((tree_attn_kernel<CT, D>), grid, dim3(256), 0, s, p, t.least);
  } else {
    hipLaunchKernelGGL((tree_attn_kernel<CT, D>), grid, dim3(256), 0, s, p, t.least);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || t.nsplit == 1) return e;
  hipLaunchKernelGGL((tree_combine_kernel<T, D>), dim3((p.r.max_rows * p.n_q + 3) / 4, p.r.batch), dim3(256), 0, s, p, t.nsplit);
  return hipGetLastError();
}

hipError_t tree_attention(const TreeArgs& p, int cus, hipStream_t s) {
  if (p.r.rows <= 0) return hipSuccess;
  const TreePlan t = tree_plan(p.c.type, p.c.n_kv, p.n_q, p.r.batch, p.r.max_rows, p.r.max_ctx, cus);
  if (t.nsplit > 1 && !p.partial) return hipErrorInvalidValue;
  const bool d128 = p.c.D == 128;
  if (!d128 && p.c.D != 64) return hipErrorInvalidValue;
  switch (p.c.type) {
    case CACHE_BF16: return d128 ? tree_launch<bf16_t, 128>(p, t, s) : tree_launch<bf16_t, 64>(p, t, s);
    case CACHE_F32: return d128 ? tree_launch<float, 128>(p, t, s) : tree_launch<float, 64>(p, t, s);
    case CACHE_E4M3: return d128 ? tree_launch<e4m3_t, 128>(p, t, s) : tree_launch<e4m3_t, 64>(p, t, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace nova
