// Operators on the paged KV cache outside the fused decode step: rotary embedding of new rows with
// their K and V written (in 8 bits: quantised) into the cache, and cached rows read back.
//
// An e4m3 cache keeps each token's K (and V) of a head as D numbers q_c and one exponent e: the value
// is q_c 2^e.  e is the smallest one with max|x| <= 448 2^e, so the scaling is exact, every value is
// rounded once (4 significant bits), and what is read back is exact in bf16.  A power of two costs
// nothing in precision (e4m3 has its own exponent) and lets the readers apply it as an exponent.
// Writing rows that were read back stores the same values again.
#include <algorithm>

#include "paged.hpp"

namespace nova {

constexpr int MIN_SCALE_EXP = -100;      // so that every value read back is a normal bf16
// The largest float below 248 2^120.  With the largest scale, 2^120, a value from there on would round to 256 2^120,
// which no float holds; taken back to it, it rounds to 240 2^120, within half a step (2^-4) like any other.
constexpr float MAX_QUANT = 0x1.effffep127f;

// sin and cos of 2 pi t.  t is reduced in double to a quarter turn, the rest is at most pi/4, where
// the Taylor series to x^9 and x^10 are within 2e-9 and 2e-10 of the functions: what remains is
// fp32 rounding at any position.
NOVA_DEV void turn_sincos(double t, float* sn, float* cs) {
  const double r = 4.0 * (t - floor(t)), q = rint(r);
  const float x = (float)((r - q) * 1.5707963267948966);
  const float z = x * x;
  const float s = x + x * z * fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const int k = (int)q & 3;
  const float a = (k & 1) ? c : s, b = (k & 1) ? s : c;
  *sn = (k & 2) ? -a : a;
  *cs = (k == 1 || k == 2) ? -b : b;
}

// Smallest e >= MIN_SCALE_EXP with amax <= 448 2^e (448 = 1.75 2^8): amax's exponent less 8, one more
// where its mantissa is above 1.75.
NOVA_DEV int scale_exp(float amax) {
  const int e = (int)((__float_as_uint(amax) + 0x1FFFFFu) >> 23) - 127 - 8;
  return max(e, MIN_SCALE_EXP);
}

template <typename T> NOVA_DEV void load8(const T* p, float* x) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(p);
    *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(p + 4);
  } else {
    const Frag8 f = *reinterpret_cast<const Frag8*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(f.w[i] << 16);
      x[2 * i + 1] = __uint_as_float(f.w[i] & 0xFFFF0000u);
    }
  }
}
template <typename T> struct Raw8;
template <> struct Raw8<bf16_t> { u32x4 a; };
template <> struct Raw8<float> { f32x4 a, b; };
NOVA_DEV Raw8<bf16_t> load_raw(const bf16_t* p) { return {*reinterpret_cast<const u32x4*>(p)}; }
NOVA_DEV Raw8<float> load_raw(const float* p) { return {reinterpret_cast<const f32x4*>(p)[0], reinterpret_cast<const f32x4*>(p)[1]}; }
NOVA_DEV void unpack8(const Raw8<bf16_t>& r, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(r.a[i] << 16);
    x[2 * i + 1] = __uint_as_float(r.a[i] & 0xFFFF0000u);
  }
}
NOVA_DEV void unpack8(const Raw8<float>& r, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = r.a[i], x[4 + i] = r.b[i];
}
template <typename T> NOVA_DEV void store8(T* p, const float* x) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = *reinterpret_cast<const float4*>(x);
    *reinterpret_cast<float4*>(p + 4) = *reinterpret_cast<const float4*>(x + 4);
  } else {
    Frag8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.w[i] = pack2(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<Frag8*>(p) = f;
  }
}
// Eight values as e4m3 with scale 2^-e; NaN and infinities become NaN (e4m3 has no infinity).
NOVA_DEV uint2 quant8(const float* x, float inv) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = fabsf(x[i]) < INFINITY ? __builtin_amdgcn_fmed3f(x[i], -MAX_QUANT, MAX_QUANT) * inv : __uint_as_float(0x7FC00000u);
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// Orders a wave's own LDS writes before its own LDS reads (no other wave touches the buffer).
NOVA_DEV void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ------------------------------------------------------------------ rotary embedding and append
// Workgroup (block of 16 cache slots, group of heads): a wave takes one head of the block's rows at a
// time, D / 8 lanes per row with 16-byte loads.  The rows' sines and cosines are computed once per
// workgroup into LDS.  Pairs of the half layout lie D/8 or fewer lanes apart and are exchanged by a
// shuffle; the maximum of a row is a shuffle reduction over its lanes.  V is turned to [D][16]
// through wave-private LDS: a whole block leaves as 16 tokens per lane, a part of one per element.
// Bound by HBM for prompts (3579 tokens of 28 + 2 x 4 heads of 128 in bf16 into an e4m3 cache: 62 MB in 16.5 to
// 17.8 us, 3.6 TB/s where a large copy reaches 5.0), by latency for a decode step (32 tokens: 7.3 us, a chain
// of row starts, table, rows and stores; six sequences' drafts of 8 to 13: 6.4 us).
template <typename TI, typename TO, typename CT, int D>
__global__ void __launch_bounds__(256) kv_append_kernel(AppendArgs p, int heads_per_wg) {
  constexpr int LPR = D / 8, RPI = 64 / LPR, NI = PAGE / RPI;
  constexpr bool Q8 = sizeof(CT) == 1;
  __shared__ __align__(16) float sm_cs[PAGE][64], sm_sn[PAGE][64];
  __shared__ __align__(16) CT sm_v[4][PAGE][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b, blk;
  const SeqRows sr = find_tile(p.r, blockIdx.x, &b, &blk);
  if (b < 0) return;
  const int t0 = blk * PAGE - sr.ctx;                    // row of the sequence at slot 0 of the block
  const int lo = max(-t0, 0), hi = min(sr.n - t0, PAGE); // slots lo .. hi - 1 get rows,
  const int kept = min(hi, p.r.max_ctx - blk * PAGE);    // of which the cache keeps those below `kept`
  const int ph = page_of(p.r, p.c.num_blocks, b, blk);
  const int n_kv = p.c.n_kv, heads = 2 * n_kv + (p.q ? p.n_q : 0);
  const int h0 = blockIdx.y * heads_per_wg, h1 = min(h0 + heads_per_wg, heads);

  // The rows of a head, D / 8 lanes each, as loaded; rows that are not live read as zeros.
  const int sub = lane % LPR, rr = lane / LPR;
  Raw8<TI> raw[NI];
  auto request = [&](int h) {
    const bool is_k = h < n_kv, is_v = !is_k && h < 2 * n_kv;
    const TI* src = reinterpret_cast<const TI*>(is_k ? p.k : is_v ? p.v : p.q);
    const long row = is_k ? p.k_row : is_v ? p.v_row : p.q_row;
    const int hh = is_k ? h : is_v ? h - n_kv : h - 2 * n_kv;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int slot = i * RPI + rr;
      raw[i] = slot >= lo && slot < hi ? load_raw(src + (sr.r0 + t0 + slot) * row + hh * D + 8 * sub) : Raw8<TI>{};
    }
  };
  if (h0 + wave < h1) request(h0 + wave);                // in flight while the angles are computed

  if (p.rot > 0 && !(h0 >= n_kv && h1 <= 2 * n_kv)) {    // heads in the order k, v, q: some head rotates
    const int half = p.rot >> 1;
    for (int i = threadIdx.x; i < PAGE * 64; i += 256) {
      const int slot = i >> 6, c = i & 63;
      if (slot < lo || slot >= hi || c >= half) continue;
      const int pos = p.pos ? p.pos[sr.r0 + t0 + slot] : blk * PAGE + slot;
      float sn, cs;
      turn_sincos((double)pos * p.turns[c], &sn, &cs);
      sm_sn[slot][c] = sn * p.mscale;
      sm_cs[slot][c] = cs * p.mscale;
    }
  }
  __syncthreads();

  for (int h = h0 + wave; h < h1; h += 4) {
    const bool is_k = h < n_kv, is_v = !is_k && h < 2 * n_kv;
    const int hh = is_k ? h : is_v ? h - n_kv : h - 2 * n_kv;
    float x[NI][8];
#pragma unroll
    for (int i = 0; i < NI; ++i) unpack8(raw[i], x[i]);
    if (h + 4 < h1) request(h + 4);                      // the next head's rows, during this one's work
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int slot = i * RPI + rr;
      const bool live = slot >= lo && slot < hi;
      if (!is_v && p.rot > 0) {
        if (p.interleaved) {
          if (8 * sub < p.rot) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float c = sm_cs[slot][4 * sub + e], s = sm_sn[slot][4 * sub + e];
              const float a = x[i][2 * e], o = x[i][2 * e + 1];
              x[i][2 * e] = a * c - o * s;
              x[i][2 * e + 1] = o * c + a * s;
            }
          }
        } else {
          const int hl = p.rot >> 4;                     // lanes that hold the first half
          const bool first = sub < hl, second = !first && sub < 2 * hl;
          const int from = lane + (first ? hl : second ? -hl : 0);
          const int c0 = 8 * (first ? sub : sub - hl);
          float o[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = __shfl(x[i][e], from, 64);
          if (first || second) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float c = sm_cs[slot][c0 + e], s = sm_sn[slot][c0 + e];
              x[i][e] = first ? x[i][e] * c - o[e] * s : x[i][e] * c + o[e] * s;
            }
          }
        }
      }
      if (!is_k && !is_v) {
        if (live) store8(reinterpret_cast<TO*>(p.q_out) + (sr.r0 + t0 + slot) * p.q_out_row + hh * D + 8 * sub, x[i]);
        continue;
      }
      if (ph < 0) continue;                              // no such block: the row is not kept
      const bool keep = slot >= lo && slot < kept;
      const size_t tok = ((size_t)ph * n_kv + hh) * PAGE + slot;
      if constexpr (Q8) {
        float amax = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float a = fabsf(x[i][e]);
          amax = a < INFINITY ? fmaxf(amax, a) : amax;
        }
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o, 64));
        const int e = scale_exp(amax);
        const uint2 w = quant8(x[i], exp_scale(127 - e));
        if (keep && sub == 0) (is_k ? p.c.k_exp : p.c.v_exp)[tok] = (uint8_t)(e + 127);
        if (is_k) {
          if (keep) *reinterpret_cast<uint2*>((uint8_t*)p.c.k + tok * D + 8 * sub) = w;
        } else {
          *reinterpret_cast<uint2*>(&sm_v[wave][slot][8 * sub]) = w;
        }
      } else {
        if (is_k) {
          if (keep) store8(reinterpret_cast<CT*>(p.c.k) + tok * D + 8 * sub, x[i]);
        } else {
          store8(&sm_v[wave][slot][8 * sub], x[i]);
        }
      }
    }
    if (is_v && ph >= 0) {
      wave_lds_fence();
      CT* vb = reinterpret_cast<CT*>(p.c.v) + ((size_t)ph * n_kv + hh) * PAGE * D;
#pragma unroll
      for (int d = lane; d < D; d += 64) {
        if (kept - lo == PAGE) {
          CT t[PAGE];
#pragma unroll
          for (int j = 0; j < PAGE; ++j) t[j] = sm_v[wave][j][d];
          constexpr int N16 = PAGE * sizeof(CT) / 16;
          uint4 w[N16];
          __builtin_memcpy(w, t, sizeof t);
#pragma unroll
          for (int j = 0; j < N16; ++j) reinterpret_cast<uint4*>(vb + (size_t)d * PAGE)[j] = w[j];
        } else {
          for (int j = lo; j < kept; ++j) vb[(size_t)d * PAGE + j] = sm_v[wave][j][d];
        }
      }
      wave_lds_fence();
    }
  }
}

template <typename TI, typename TO, typename CT>
static hipError_t append_launch(const AppendArgs& p, int cus, hipStream_t s) {
  const long tiles = std::min<long>(p.r.rows, p.r.rows / PAGE + 2L * p.r.batch);
  const int heads = 2 * p.c.n_kv + (p.q ? p.n_q : 0);
  // Heads are cut into groups that each compute the rows' sines and cosines: one head a wave while the blocks
  // are few, fewer and larger groups once the workgroups are 2.5 for each compute unit (3579 tokens of
  // 36 heads: 9 groups 18.7 us, 5 17.6, 3 16.1, 1 25.6; 32 single tokens: 6.9, 9.0, 10.4, 18.6).
  const long most = (heads + 3) / 4, groups = std::min(most, std::max(1L, (5L * cus / 2 + tiles - 1) / tiles));
  const int per = (int)(((heads + groups - 1) / groups + 3) / 4 * 4);
  const dim3 grid((unsigned)tiles, (heads + per - 1) / per);
  if (p.c.D == 64) hipLaunchKernelGGL((kv_append_kernel<TI, TO, CT, 64>), grid, dim3(256), 0, s, p, per);
  else hipLaunchKernelGGL((kv_append_kernel<TI, TO, CT, 128>), grid, dim3(256), 0, s, p, per);
  return hipGetLastError();
}

template <typename CT>
static hipError_t append_types(const AppendArgs& p, int cus, hipStream_t s) {
  if (p.in_f32) return p.q_out_f32 ? append_launch<float, float, CT>(p, cus, s) : append_launch<float, bf16_t, CT>(p, cus, s);
  return p.q_out_f32 ? append_launch<bf16_t, float, CT>(p, cus, s) : append_launch<bf16_t, bf16_t, CT>(p, cus, s);
}

hipError_t kv_append(const AppendArgs& p, int cus, hipStream_t s) {
  if (p.r.rows <= 0) return hipSuccess;
  if ((p.c.D != 64 && p.c.D != 128) || p.rot < 0 || p.rot > p.c.D || p.rot % 16) return hipErrorInvalidValue;
  switch (p.c.type) {
    case CACHE_BF16: return append_types<bf16_t>(p, cus, s);
    case CACHE_F32: return append_types<float>(p, cus, s);
    case CACHE_E4M3: return append_types<e4m3_t>(p, cus, s);
  }
  return hipErrorInvalidValue;
}

// ------------------------------------------------------------------ reading rows back
// Eight cached values as floats.
template <typename CT> NOVA_DEV void cached8(const CT* p, float scale, float* x) {
  if constexpr (sizeof(CT) == 1) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    const uint32_t a[4] = {e4m3_pair<false>(w.x, scale), e4m3_pair<true>(w.x, scale), e4m3_pair<false>(w.y, scale),
                           e4m3_pair<true>(w.y, scale)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(a[i] << 16);
      x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    }
  } else {
    load8(p, x);
  }
}

NOVA_DEV float cached1(e4m3_t x, float scale) { return __uint_as_float(e4m3_pair<false>(x.v, scale) << 16); }
template <typename T> NOVA_DEV float cached1(T x, float) { return to_f<T>(x); }

// Consecutive rows: workgroup (block of 16 slots, group of K and V heads), a wave per head.  K rows are
// copied with 8 elements per lane; a V block [D][16] is read whole, 16 tokens per lane, and turned
// through wave-private LDS.  Rows whose token does not exist read as zeros.  Bound by HBM: 32 sequences of 1846
// to 3579 tokens from e4m3 to bf16, 261 MB in 51 us, 5.1 TB/s, a large copy's rate.
template <typename CT, typename TO, int D>
__global__ void __launch_bounds__(256) kv_gather_kernel(GatherArgs p) {
  constexpr int LPR = D / 8, RPI = 64 / LPR, NI = PAGE / RPI;
  __shared__ __align__(16) CT sm_v[4][PAGE][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b, blk;
  const SeqRows sr = find_tile(p.r, blockIdx.x, &b, &blk);
  if (b < 0) return;
  const int t0 = blk * PAGE - sr.ctx;
  const int lo = max(-t0, 0), hi = min(sr.n - t0, PAGE);
  const int ph = page_of(p.r, p.c.num_blocks, b, blk), held = p.r.max_ctx - blk * PAGE;
  const int sub = lane % LPR, rr = lane / LPR, n_kv = p.c.n_kv;
  const int h = blockIdx.y * 4 + wave;
  if (h >= 2 * n_kv) return;
  const bool is_k = h < n_kv;
  const int hh = is_k ? h : h - n_kv;
  const size_t tok0 = ((size_t)max(ph, 0) * n_kv + hh) * PAGE;
  if (!is_k && ph >= 0) {
    const CT* vb = reinterpret_cast<const CT*>(p.c.v) + tok0 * D;
#pragma unroll
    for (int d = lane; d < D; d += 64) {
      constexpr int N16 = PAGE * sizeof(CT) / 16;
      uint4 w[N16];
#pragma unroll
      for (int j = 0; j < N16; ++j) w[j] = reinterpret_cast<const uint4*>(vb + (size_t)d * PAGE)[j];
      CT t[PAGE];
      __builtin_memcpy(t, w, sizeof t);
#pragma unroll
      for (int j = 0; j < PAGE; ++j) sm_v[wave][j][d] = t[j];
    }
    wave_lds_fence();
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int slot = i * RPI + rr;
    if (slot < lo || slot >= hi) continue;
    float x[8] = {};
    if (ph >= 0 && slot < held) {
      float scale = 1.f;
      if constexpr (sizeof(CT) == 1) scale = exp_scale((is_k ? p.c.k_exp : p.c.v_exp)[tok0 + slot]);
      if (is_k) cached8(reinterpret_cast<const CT*>(p.c.k) + (tok0 + slot) * D + 8 * sub, scale, x);
      else cached8(&sm_v[wave][slot][8 * sub], scale, x);
    }
    const long r = sr.r0 + t0 + slot;
    store8(reinterpret_cast<TO*>(is_k ? p.k : p.v) + r * (is_k ? p.k_row : p.v_row) + hh * D + 8 * sub, x);
  }
}

// Rows by token number: workgroup (group of rows, group of heads), D / 8 lanes per row and head.  A V row lies 16
// elements apart, so its lanes take one element each, neighbours side by side: a load touches 16 (e4m3) or 32
// (bf16) lines of 64 bytes, not 64 as with 8 elements a lane.  For a handful of accepted tokens bound by latency (eight
// sequences' accepted tokens, 36 of 4 KV heads: 4.1 us), for many by V's lines, of which a token uses a sixteenth
// (32 sequences' 750 to 1500 tokens anywhere among 2000, e4m3: 49.7 us, 64.1 with 8 elements a lane; bf16 74.4 and 81.9).
template <typename CT, typename TO, int D>
__global__ void __launch_bounds__(256) kv_pick_kernel(GatherArgs p) {
  constexpr int LPR = D / 8, ROWS = 64 / LPR;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sub = lane % LPR, n_kv = p.c.n_kv;
  const int r0 = blockIdx.x * ROWS, r = r0 + lane / LPR, h = blockIdx.y * 4 + wave;
  if (h >= 2 * n_kv) return;
  const bool is_k = h < n_kv;
  const int hh = is_k ? h : h - n_kv;
  int b = 0;
  if (p.r.row_start) {                                   // sequences that end at or before row r
    int lo = 0, hi = p.r.batch;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (p.r.row_start[mid + 1] <= r) lo = mid + 1;
      else hi = mid;
    }
    b = lo;
  } else {
    b = r / p.r.max_rows;
  }
  bool live = r < p.r.rows && b < p.r.batch;
  int ph = -1, slot = 0;
  if (live) {
    const SeqRows sr = seq_rows(p.r, b);
    live = r >= sr.r0 && r < sr.r0 + sr.n;
    const int t = live ? p.slots[r] : -1;
    ph = t < 0 ? -1 : page_of(p.r, p.c.num_blocks, b, t / PAGE);
    slot = t < 0 ? 0 : t % PAGE;
  }
  const size_t tok = ((size_t)max(ph, 0) * n_kv + hh) * PAGE + slot;
  float scale = 1.f;
  if constexpr (sizeof(CT) == 1)
    if (ph >= 0) scale = exp_scale((is_k ? p.c.k_exp : p.c.v_exp)[tok]);
  if (is_k) {
    if (!live) return;
    float x[8] = {};
    if (ph >= 0) cached8(reinterpret_cast<const CT*>(p.c.k) + tok * D + 8 * sub, scale, x);
    store8(reinterpret_cast<TO*>(p.k) + r * p.k_row + hh * D + 8 * sub, x);
    return;
  }
  CT v[ROWS][D / 64];
  float x[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {                       // the rows' loads together
    const int phi = __shfl(ph, i * LPR, 64), si = __shfl(slot, i * LPR, 64);
    x[i] = phi >= 0 ? __shfl(scale, i * LPR, 64) : 0.f;
    const CT* vb = reinterpret_cast<const CT*>(p.c.v) + ((size_t)max(phi, 0) * n_kv + hh) * PAGE * D + si;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) v[i][j] = vb[(size_t)(lane + 64 * j) * PAGE];
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    if (!__shfl((int)live, i * LPR, 64)) continue;
    TO* out = reinterpret_cast<TO*>(p.v) + (long)(r0 + i) * p.v_row + hh * D + lane;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) out[64 * j] = from_f<TO>(x[i] != 0.f ? cached1(v[i][j], x[i]) : 0.f);
  }
}

template <typename CT, typename TO, int D>
static hipError_t gather_launch(const GatherArgs& p, hipStream_t s) {
  const unsigned y = (2 * p.c.n_kv + 3) / 4;
  if (p.slots) {
    constexpr int ROWS = 64 / (D / 8);
    hipLaunchKernelGGL((kv_pick_kernel<CT, TO, D>), dim3((p.r.rows + ROWS - 1) / ROWS, y), dim3(256), 0, s, p);
  } else {
    const long tiles = std::min<long>(p.r.rows, p.r.rows / PAGE + 2L * p.r.batch);
    hipLaunchKernelGGL((kv_gather_kernel<CT, TO, D>), dim3((unsigned)tiles, y), dim3(256), 0, s, p);
  }
  return hipGetLastError();
}
template <typename CT>
static hipError_t gather_types(const GatherArgs& p, hipStream_t s) {
  if (p.c.D == 64) return p.out_f32 ? gather_launch<CT, float, 64>(p, s) : gather_launch<CT, bf16_t, 64>(p, s);
  return p.out_f32 ? gather_launch<CT, float, 128>(p, s) : gather_launch<CT, bf16_t, 128>(p, s);
}

hipError_t kv_gather(const GatherArgs& p, hipStream_t s) {
  if (p.r.rows <= 0) return hipSuccess;
  if (p.c.D != 64 && p.c.D != 128) return hipErrorInvalidValue;
  switch (p.c.type) {
    case CACHE_BF16: return gather_types<bf16_t>(p, s);
    case CACHE_F32: return gather_types<float>(p, s);
    case CACHE_E4M3: return gather_types<e4m3_t>(p, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace nova
