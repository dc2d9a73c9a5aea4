// Attention of drafted tokens over a paged cache.  Sequence b brings n rows (1 to 64 drafted tokens, a
// tree or a chain), already appended to its cache as tokens ctx .. ctx + n - 1; each row sees every
// token below ctx and those drafted tokens whose bit is set in its mask:
//   out = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale q.k_t - max).
// One pass over the cache with a running maximum and sum (in fp32, base 2).
//  * The rows (token, query head) that share a KV head are the MFMA columns, 16 to a tile, so K and V
//    are read once for NQ tiles: S = K Q^T and O^T = V^T P^T.
//  * A wave takes a step of 4 JN tokens per lane group (JN row blocks of S): which token is which MFMA
//    row is free, so lane group g takes the step's tokens 4 JN g .. and finds its V of a dimension in
//    one 16-byte load (e4m3: 16 tokens of a block, bf16: 8, f32: two loads of 4).
//  * e4m3 turns into bf16 exactly on the way to the MFMA: K with its token's scale, V without; V's
//    scale goes onto p, a power of two.  p is rounded to bf16 once (the matrix cores take no other
//    type beside bf16 V); the sum of p keeps fp32.  The f32 cache uses the fp32 matrix instructions.
//  * grid (context splits, KV head x row tiles, sequence); the waves of a workgroup share a split and
//    are merged through LDS, the splits by a second kernel.
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
  uint4 k[JN][KW];
  uint4 v[D / 16][VW];
  float ks[JN];                                           // e4m3: scale of the lane's K rows
  uint4 ve;                                               // e4m3: exponent bytes of the lane group's 16 tokens
  bool ok;                                                // the lane group's own block (V) exists
};

// The elements of a lane's V words that are not finite, a bit each (e4m3 has NaN only).
template <typename CT, int VW> NOVA_DEV uint32_t v_odd(const uint4 (&v)[VW]) {
  uint32_t is = 0;
#pragma unroll
  for (int w = 0; w < 4 * VW; ++w) {
    const uint32_t x = (w & 3) == 0 ? v[w / 4].x : (w & 3) == 1 ? v[w / 4].y : (w & 3) == 2 ? v[w / 4].z : v[w / 4].w;
    if constexpr (sizeof(CT) == 4) {
      is |= (x & 0x7F800000u) == 0x7F800000u ? 1u << w : 0u;
    } else if constexpr (sizeof(CT) == 2) {
      is |= (x & 0x7F80u) == 0x7F80u ? 1u << 2 * w : 0u;
      is |= (x & 0x7F800000u) == 0x7F800000u ? 2u << 2 * w : 0u;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) is |= ((x >> 8 * e) & 0x7Fu) == 0x7Fu ? 1u << (4 * w + e) : 0u;
    }
  }
  return is;
}
// Clears the elements of a lane's V words whose bit in `keep` is not set.
template <typename CT, int VW> NOVA_DEV void v_keep(uint4 (&v)[VW], uint32_t keep) {
  constexpr int EPW = 4 / sizeof(CT);
#pragma unroll
  for (int w = 0; w < 4 * VW; ++w) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < EPW; ++e) {
      constexpr uint32_t one = sizeof(CT) == 4 ? ~0u : (1u << (8 * (sizeof(CT) & 3))) - 1u;
      m |= ((keep >> (w * EPW + e)) & 1u) ? one << (8 * sizeof(CT) * e % 32) : 0u;
    }
    uint32_t& x = (w & 3) == 0 ? v[w / 4].x : (w & 3) == 1 ? v[w / 4].y : (w & 3) == 2 ? v[w / 4].z : v[w / 4].w;
    x &= m;
  }
}

template <typename CT, int D, int NQ>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(NQ > 2 ? 1 : 2)))
tree_attn_kernel(TreeArgs p, int steps_per_split) {
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
  const int split = blockIdx.x, kvh = blockIdx.y % n_kv, tile = blockIdx.y / n_kv, b = blockIdx.z;
  const int col = lane & 15, grp = lane >> 4;
  const SeqRows sr = seq_rows(p.r, b);
  const int nrow = sr.n * G, row0 = tile * 16 * NQ;
  if (row0 >= nrow) return;
  const int total = sr.ctx + sr.n;
  const int nsteps = (total + STEP - 1) / STEP, nblk = (total + PAGE - 1) / PAGE;
  const int step0 = split * steps_per_split, step1 = min(step0 + steps_per_split, nsteps);
  const int first = step0 + wave;
  const int n_it = first < step1 ? (step1 - first + 3) / 4 : 0;
  const int* table = p.r.tables + (size_t)b * p.r.max_blocks;

  // this lane's row of each tile: its drafted token and what it sees of the drafted ones
  const T* qrow[NQ];
  unsigned long long sees[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = row0 + 16 * n + col, t = min(r, nrow - 1) / G;
    const int head = kvh * G + min(r, nrow - 1) % G;
    qrow[n] = reinterpret_cast<const T*>(p.q) + (sr.r0 + t) * p.q_row + head * D;
    sees[n] = p.mask ? p.mask[sr.r0 + t] : (2ull << t) - 1;
  }

  // block ids of 64 / BPS iterations at a time, one per lane
  int tl = -1, tl_chunk = -1;
  constexpr int IPC = 64 / BPS;
  auto page = [&](int it, int j) -> int {
    if (it / IPC != tl_chunk) {
      tl_chunk = it / IPC;
      const int blk = (first + 4 * (tl_chunk * IPC + lane / BPS)) * BPS + lane % BPS;
      tl = blk < nblk && blk < p.r.max_blocks ? table[blk] : -1;
      if ((unsigned)tl >= (unsigned)p.c.num_blocks) tl = -1;
    }
    return __shfl(tl, (it % IPC) * BPS + j, 64);
  };
  if (tid == 0) sm_odd = 0;
  __syncthreads();

  Raw raw;
  auto load_k = [&](int it) {
    // MFMA row col of block j is token TPG (col / 4) + 4 j + col % 4 of the step
    const int t = TPG * (col >> 2) + (col & 3);
    const size_t tok = ((size_t)max(page(it, t / PAGE), 0) * n_kv + kvh) * PAGE + t % PAGE;
#pragma unroll
    for (int j = 0; j < JN; ++j) {
      // a lane's 16 bytes of word w: dimensions 64 w + 16 grp .. of e4m3, 32 w + 8 grp .. of bf16, 16 w + 4 grp .. of f32
      const uint4* kr = reinterpret_cast<const uint4*>(reinterpret_cast<const CT*>(p.c.k) + (tok + 4 * j) * D) + grp;
#pragma unroll
      for (int w = 0; w < Raw::KW; ++w) raw.k[j][w] = kr[4 * w];
      if constexpr (Q8) raw.ks[j] = exp_scale(p.c.k_exp[tok + 4 * j]);
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
      for (int w = 0; w < Raw::VW; ++w) raw.v[i][w] = reinterpret_cast<const uint4*>(vr + (size_t)16 * i * PAGE)[w];
    if constexpr (Q8) raw.ve = *reinterpret_cast<const uint4*>(p.c.v_exp + tok);
  };
  if (n_it > 0) {
    load_k(0);
    load_v(0);
  }

  // Q^T fragments: the dimensions of each k-step in the order in which K's words hold them
  Frag8 qf[NQ][F32 ? 1 : NS];
  float4 qx[NQ][F32 ? D / 16 : 1];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    if constexpr (F32) {
#pragma unroll
      for (int w = 0; w < D / 16; ++w) qx[n][w] = *reinterpret_cast<const float4*>(qrow[n] + 16 * w + 4 * grp);
    } else {
#pragma unroll
      for (int s = 0; s < NS; ++s)
        qf[n][s] = *reinterpret_cast<const Frag8*>(qrow[n] + (Q8 ? 64 * (s >> 1) + 16 * grp + 8 * (s & 1) : 32 * s + 8 * grp));
    }
  }

  f32x4 o[NQ][ND];
  float m_run[NQ], l_run[NQ];                             // l_run: of this lane group's tokens only
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = -INFINITY;
    l_run[n] = 0.f;
#pragma unroll
    for (int i = 0; i < ND; ++i) o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float scale = p.scale * 1.4426950408889634f;

  // V^T P^T of one dimension block added to its accumulators: `v` the lane's words, `pt` P^T
  auto add_pv = [&](const uint4 (&v)[Raw::VW], const auto& pt, f32x4 (&acc)[NQ]) {
    if constexpr (F32) {
      float f[TPG];
      __builtin_memcpy(f, v, sizeof f);
#pragma unroll
      for (int e = 0; e < TPG; ++e)
#pragma unroll
        for (int n = 0; n < NQ; ++n) acc[n] = mfma4(f[e], pt[n][e], acc[n]);
    } else if constexpr (Q8) {
      const uint4 x = v[0];
      const Frag8 a{{e4m3_pair<false>(x.x, 1.f), e4m3_pair<true>(x.x, 1.f), e4m3_pair<false>(x.y, 1.f), e4m3_pair<true>(x.y, 1.f)}};
      const Frag8 c{{e4m3_pair<false>(x.z, 1.f), e4m3_pair<true>(x.z, 1.f), e4m3_pair<false>(x.w, 1.f), e4m3_pair<true>(x.w, 1.f)}};
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        acc[n] = mfma16(a, pt[n][0], acc[n]);
        acc[n] = mfma16(c, pt[n][JN / 2 - 1], acc[n]);
      }
    } else {
#pragma unroll
      for (int n = 0; n < NQ; ++n) acc[n] = mfma16(__builtin_bit_cast(Frag8, v[0]), pt[n][0], acc[n]);
    }
  };

  // One step.  MASKED: it holds drafted tokens, the sequence's end or a missing block.
  auto step = [&](int it, auto masked_) {
    constexpr bool MASKED = decltype(masked_)::value;
    const int mine = (first + 4 * it) * STEP + TPG * grp;        // the lane group's first token
    const int valid = !MASKED ? TPG : raw.ok ? min(max(total - mine, 0), TPG) : 0;
    // S: lane holds scores of its lane group's tokens 4 j + q for row col
    f32x4 sc[NQ][JN];
#pragma unroll
    for (int j = 0; j < JN; ++j) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) sc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < Raw::KW; ++w) {
        const uint4 x = raw.k[j][w];
        if constexpr (F32) {
          const float f[4] = {__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w)};
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            sc[n][j] = mfma4(f[0], qx[n][w].x, sc[n][j]);
            sc[n][j] = mfma4(f[1], qx[n][w].y, sc[n][j]);
            sc[n][j] = mfma4(f[2], qx[n][w].z, sc[n][j]);
            sc[n][j] = mfma4(f[3], qx[n][w].w, sc[n][j]);
          }
        } else if constexpr (Q8) {
          const float s = raw.ks[j];
          const Frag8 a{{e4m3_pair<false>(x.x, s), e4m3_pair<true>(x.x, s), e4m3_pair<false>(x.y, s), e4m3_pair<true>(x.y, s)}};
          const Frag8 c{{e4m3_pair<false>(x.z, s), e4m3_pair<true>(x.z, s), e4m3_pair<false>(x.w, s), e4m3_pair<true>(x.w, s)}};
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            sc[n][j] = mfma16(a, qf[n][2 * w], sc[n][j]);
            sc[n][j] = mfma16(c, qf[n][2 * w + 1], sc[n][j]);
          }
        } else {
          const Frag8 a = __builtin_bit_cast(Frag8, x);
#pragma unroll
          for (int n = 0; n < NQ; ++n) sc[n][j] = mfma16(a, qf[n][w], sc[n][j]);
        }
      }
    }
    if (it + 1 < n_it) load_k(it + 1);

    // what row n sees of the lane group's tokens, a bit each
    uint32_t vis[NQ];
    if constexpr (MASKED) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int dr = mine - sr.ctx;                            // the first token as a drafted one
        const unsigned long long m = dr >= 64 ? 0ull : dr >= 0 ? sees[n] >> dr : dr <= -TPG ? ~0ull : (sees[n] << -dr) | ((1ull << -dr) - 1);
        vis[n] = (uint32_t)m & ((1u << valid) - 1u);
      }
      // slots past the last token may hold anything: their V is cleared
#pragma unroll
      for (int i = 0; i < ND; ++i) v_keep<CT>(raw.v[i], (1u << valid) - 1u);
      // A drafted token's V that is not finite concerns the rows that see it and no other, and 0 times
      // infinity is not 0: such elements are cleared here too and added when the rows are written.
      if (mine + TPG > sr.ctx) {
        const uint32_t drafted = mine >= sr.ctx ? ~0u : ~0u << (sr.ctx - mine);
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
          const uint32_t is = v_odd<CT>(raw.v[i]) & drafted;
          if (is) v_keep<CT>(raw.v[i], ~is);
          odd |= is;
        }
        if (odd) sm_odd = 1;
      }
    }

    // softmax of each row tile; p as the MFMA's P^T operand (tokens 8 h .. 8 h + 7 of the lane group)
    Frag8 pf[NQ][F32 ? 1 : JN / 2];
    float px[NQ][F32 ? TPG : 1];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float s[TPG];
      float tmax = -INFINITY;
#pragma unroll
      for (int e = 0; e < TPG; ++e) {
        s[e] = sc[n][e >> 2][e & 3] * scale;
        if constexpr (MASKED) s[e] = (vis[n] >> e) & 1 ? s[e] : -INFINITY;
        tmax = fmaxf(tmax, s[e]);
      }
      tmax = fmaxf(tmax, __shfl_xor(tmax, 16, 64));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
      const float m_new = fmaxf(m_run[n], tmax);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;      // nothing seen yet: every p is 0
      const float corr = exp2f(m_run[n] - m_use);
      m_run[n] = m_new;
      float rs = 0.f;
#pragma unroll
      for (int e = 0; e < TPG; ++e) {
        s[e] = exp2f(s[e] - m_use);
        rs += s[e];
      }
      l_run[n] = l_run[n] * corr + rs;
      if (__any(corr != 1.f)) {
#pragma unroll
        for (int i = 0; i < ND; ++i) o[n][i] *= corr;
      }
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < TPG; ++e) px[n][e] = s[e];
      } else {
        if constexpr (Q8) {
          const uint32_t w[4] = {raw.ve.x, raw.ve.y, raw.ve.z, raw.ve.w};
#pragma unroll
          for (int e = 0; e < TPG; ++e) {
            const float vs = exp_scale((w[e >> 2] >> (8 * (e & 3))) & 255u);
            s[e] = !MASKED || e < valid ? s[e] * vs : 0.f;
          }
        }
#pragma unroll
        for (int h = 0; h < JN / 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) pf[n][h].w[e] = pack2(s[8 * h + 2 * e], s[8 * h + 2 * e + 1]);
      }
    }
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      f32x4 acc[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) acc[n] = o[n][i];
      if constexpr (F32) add_pv(raw.v[i], px, acc);
      else add_pv(raw.v[i], pf, acc);
#pragma unroll
      for (int n = 0; n < NQ; ++n) o[n][i] = acc[n];
    }
    if (it + 1 < n_it) load_v(it + 1);
  };

  for (int it = 0; it < n_it; ++it) {
    if ((first + 4 * it) * STEP + STEP > sr.ctx || !__all(raw.ok)) step(it, std::true_type{});
    else step(it, std::false_type{});
  }

  // the lane groups' sums, then the four waves, one row tile at a time
  const int nsplit = gridDim.x;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    if (row0 + 16 * n >= nrow) break;
    float l = l_run[n];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (n > 0) __syncthreads();
    if (grp == 0) { sm_m[wave][col] = m_run[n]; sm_l[wave][col] = l; }
#pragma unroll
    for (int i = 0; i < ND; ++i) *reinterpret_cast<f32x4*>(&sm_o[wave][col][16 * i + 4 * grp]) = o[n][i];
    __syncthreads();
    for (int idx = tid; idx < 16 * D; idx += 256) {
      const int c = idx / D, d = idx % D, r = row0 + 16 * n + c;
      if (r >= nrow) break;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < 4; ++w) M = fmaxf(M, sm_m[w][c]);
      const float mu = M == -INFINITY ? 0.f : M;
      float L = 0.f, O = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = exp2f(sm_m[w][c] - mu);
        L += f * sm_l[w][c];
        O += f * sm_o[w][c][d];
      }
      const long t = sr.r0 + r / G;
      if (sm_odd) {
        const unsigned long long see = p.mask ? p.mask[t] : (2ull << (r / G)) - 1;
#pragma unroll 1
        for (int j = max(0, step0 * STEP - sr.ctx); j < min(sr.n, step1 * STEP - sr.ctx); ++j) {
          const int tok = sr.ctx + j, ph = page_of(p.r, p.c.num_blocks, b, tok / PAGE);
          if (!((see >> j) & 1) || ph < 0) continue;
          const CT x = reinterpret_cast<const CT*>(p.c.v)[(((size_t)ph * n_kv + kvh) * D + d) * PAGE + tok % PAGE];
          float v;
          if constexpr (Q8) v = (x.v & 0x7F) == 0x7F ? __uint_as_float(0x7FC00000u) : 0.f;
          else v = to_f<CT>(x);
          if (!(fabsf(v) < INFINITY)) O += v;
        }
      }
      const int head = kvh * G + r % G;
      if (nsplit == 1) {
        reinterpret_cast<T*>(p.out)[t * p.out_row + head * D + d] = from_f<T>(L == 0.f ? 0.f : O / L);
      } else {
        float* part = p.partial + ((t * p.n_q + head) * nsplit + split) * (D + 4);
        part[4 + d] = O;
        if (d == 0) { part[0] = M; part[1] = L; }
      }
    }
  }
}

// Joins the splits of one row and head: one wave, D / 64 dimensions per lane.
template <typename T, int D>
__global__ void __launch_bounds__(256) tree_combine_kernel(TreeArgs p, int nsplit, long row_heads) {
  const int lane = threadIdx.x & 63;
  const long rh = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (rh >= row_heads) return;
  const long t = rh / p.n_q;
  const int head = (int)(rh % p.n_q);
  if (p.r.row_start) {                                   // rows of no sequence are left as they were
    int lo = 0, hi = p.r.batch;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (p.r.row_start[mid + 1] <= t) lo = mid + 1;
      else hi = mid;
    }
    if (lo >= p.r.batch) return;
    const SeqRows sr = seq_rows(p.r, lo);
    if (t < sr.r0 || t >= sr.r0 + sr.n) return;
  }
  const float* part = p.partial + rh * nsplit * (D + 4);
  const float m = lane < nsplit ? part[lane * (D + 4)] : -INFINITY;
  const float l = lane < nsplit ? part[lane * (D + 4) + 1] : 0.f;
  const float M = wave_max(m);
  const float f = M == -INFINITY ? 0.f : exp2f(m - M);
  const float L = wave_sum(f * l);
  float o[D / 64] = {};
  for (int s = 0; s < nsplit; ++s) {
    const float w = __shfl(f, s, 64);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) o[i] += w * part[s * (D + 4) + 4 + lane + 64 * i];
  }
#pragma unroll
  for (int i = 0; i < D / 64; ++i)
    reinterpret_cast<T*>(p.out)[t * p.out_row + head * D + lane + 64 * i] = from_f<T>(L == 0.f ? 0.f : o[i] / L);
}

// Row tiles (of 16) that a workgroup takes, and the splits of the context.
struct TreePlan { int nq, tiles, nsplit, per; };
static TreePlan tree_plan(int type, int n_kv, int n_q, int batch, int max_rows, int max_ctx, int cus) {
  TreePlan t;
  const int rows = max_rows * (n_q / n_kv);
  t.nq = type == CACHE_F32 ? 1 : rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  t.tiles = (rows + 16 * t.nq - 1) / (16 * t.nq);
  const int step = type == CACHE_E4M3 ? 64 : 32;
  const int steps = (max_ctx + step - 1) / step;
  const int base = batch * n_kv * t.tiles;
  const int want = std::max(1, (2 * cus + base - 1) / base);
  t.per = std::max(4, (steps + want - 1) / want);
  t.nsplit = (steps + t.per - 1) / t.per;
  while (t.nsplit > 64) t.nsplit = (steps + ++t.per - 1) / t.per;
  return t;
}

size_t tree_partial_floats(int type, int n_kv, int n_q, int D, int batch, int rows, int max_rows, int max_ctx, int cus) {
  const TreePlan t = tree_plan(type, n_kv, n_q, batch, max_rows, max_ctx, cus);
  return t.nsplit > 1 ? (size_t)rows * n_q * t.nsplit * (D + 4) : 0;
}

template <typename CT, int D, int NQ>
static hipError_t tree_launch(const TreeArgs& p, const TreePlan& t, hipStream_t s) {
  typedef typename TreeT<CT>::act T;
  hipLaunchKernelGGL((tree_attn_kernel<CT, D, NQ>), dim3(t.nsplit, p.c.n_kv * t.tiles, p.r.batch), dim3(256), 0, s, p, t.per);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || t.nsplit == 1) return e;
  const long rh = (long)p.r.rows * p.n_q;
  hipLaunchKernelGGL((tree_combine_kernel<T, D>), dim3((unsigned)((rh + 3) / 4)), dim3(256), 0, s, p, t.nsplit, rh);
  return hipGetLastError();
}
template <typename CT, int D>
static hipError_t tree_tiles(const TreeArgs& p, const TreePlan& t, hipStream_t s) {
  if (t.nq == 1) return tree_launch<CT, D, 1>(p, t, s);
  if constexpr (sizeof(CT) < 4) {
    if (t.nq == 2) return tree_launch<CT, D, 2>(p, t, s);
    return tree_launch<CT, D, 4>(p, t, s);
  }
  return hipErrorInvalidValue;
}

hipError_t tree_attention(const TreeArgs& p, int cus, hipStream_t s) {
  if (p.r.rows <= 0) return hipSuccess;
  const TreePlan t = tree_plan(p.c.type, p.c.n_kv, p.n_q, p.r.batch, p.r.max_rows, p.r.max_ctx, cus);
  if (t.nsplit > 1 && !p.partial) return hipErrorInvalidValue;
  const bool wide = p.c.D == 128;
  if (!wide && p.c.D != 64) return hipErrorInvalidValue;
  switch (p.c.type) {
    case CACHE_BF16: return wide ? tree_tiles<bf16_t, 128>(p, t, s) : tree_tiles<bf16_t, 64>(p, t, s);
    case CACHE_F32: return wide ? tree_tiles<float, 128>(p, t, s) : tree_tiles<float, 64>(p, t, s);
    case CACHE_E4M3: return wide ? tree_tiles<e4m3_t, 128>(p, t, s) : tree_tiles<e4m3_t, 64>(p, t, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace nova
