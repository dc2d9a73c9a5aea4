// Low-rank adapters of many requests beside a projection that they share: with i the adapter of a row's sequence,
//   out = base + s_i B_i (A_i x),   A_i [rank][K], B_i [N][rank].
//  * shrink: h = A_i x per row, tiles of a sequence's rows times a slice of K, fp32 partials [slice][row][rank];
//  * expand: the slices summed in order, times s_i, then B_i h onto base, rounded once.
// The ranks are far below what would make this compute-bound: it is bound by reading x, base and the adapters and by
// writing out.  The matrix cores take bf16, so h goes to them as a sum of bf16 parts, an MFMA each: two (a relative error
// of 2^-16 instead of a bf16 rounding's 2^-8) where out is bf16, three (all 24 bits) where it is fp32.  x in fp32 likewise.
#include <algorithm>

#include "paged.hpp"

namespace nova {

constexpr int LO_ROWS = 64;                // rows of a tile of long sequences
constexpr int LO_STEP = 16;                // of a tile of short ones

// The tile-th tile of `rows` rows of the batch's sequences, counted over them: its sequence (-1: none) and first row.
template <int TM> NOVA_DEV SeqRows find_row_tile(const BatchRows& p, int tile, int* b, int* row) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int base = 0; base < p.batch; base += 64) {
    const int i = base + lane;
    const SeqRows s = i < p.batch ? seq_rows(p, i) : SeqRows{0, 0, 0};
    const int tiles = (s.n + TM - 1) / TM;
    int sum = tiles;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(sum, o, 64);
      if (lane >= o) sum += up;
    }
    const unsigned long long m = __ballot(before + sum > tile);
    if (m) {
      const int l = __ffsll(m) - 1;
      SeqRows f;
      f.r0 = __builtin_amdgcn_readlane(s.r0, l);
      f.n = __builtin_amdgcn_readlane(s.n, l);
      f.ctx = 0;
      *b = base + l;
      *row = (tile - (before + __builtin_amdgcn_readlane(sum - tiles, l))) * TM;
      return f;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  *b = -1;
  *row = 0;
  return SeqRows{0, 0, 0};
}

// What a bf16 rounding of v leaves; nothing of what is not finite.
NOVA_DEV float rest_of(float v, float rounded) { return fabsf(rounded) < INFINITY ? v - rounded : 0.f; }

// Eight floats as a sum of N operands of bf16, each the rounded rest of those before it.
template <int N> NOVA_DEV void split_parts(float* x, Frag8* f) {
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[n].w[i] = pack2(x[2 * i], x[2 * i + 1]);
      x[2 * i] = rest_of(x[2 * i], __uint_as_float(f[n].w[i] << 16));
      x[2 * i + 1] = rest_of(x[2 * i + 1], __uint_as_float(f[n].w[i] & 0xFFFF0000u));
    }
}
// Eight elements of x as N operands (of bf16 there is one).
template <int N> NOVA_DEV void load_x(const bf16_t* p, Frag8* f) { f[0] = *reinterpret_cast<const Frag8*>(p); }
template <int N> NOVA_DEV void load_x(const float* p, Frag8* f) {
  float x[8];
  *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(p);
  *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(p + 4);
  split_parts<N>(x, f);
}

// ------------------------------------------------------------------ h = A x
// Workgroup: (tile of TM rows, slice of K).  Lane (row or rank column = lane % 16, k group = lane / 16) loads 16 bytes
// of its row of x and of A per 32 k.  TM = 16: the waves take the k steps in turn and their sums are joined in LDS;
// TM = 64: each wave has 16 rows of its own.
template <typename TX, int NX, int RT, int TM>
__global__ void __launch_bounds__(256) lora_shrink_kernel(LoraArgs p) {
  constexpr bool ROWS4 = TM == LO_ROWS;
  __shared__ float sm[ROWS4 ? 1 : 4][ROWS4 ? 1 : 16][16 * RT + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  int b, row0;
  const SeqRows sr = find_row_tile<TM>(p.r, blockIdx.x, &b, &row0);
  if (b < 0) return;
  const int i = p.which[b];
  if ((unsigned)i >= (unsigned)p.n) return;
  if (ROWS4) row0 += 16 * wave;
  const int k0 = blockIdx.y * p.kslice, k1 = min(p.k, k0 + p.kslice);
  const bf16_t* A = p.a + (size_t)i * p.rank * p.k;
  const TX* x = reinterpret_cast<const TX*>(p.x) + (sr.r0 + row0 + col) * p.x_row;
  const bool live = row0 + col < sr.n;
  f32x4 acc[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (row0 < sr.n) {
    constexpr int STEP = ROWS4 ? 32 : 128;
#pragma unroll 2
    for (int kk = k0 + (ROWS4 ? 0 : 32 * wave); kk < k1; kk += STEP) {
      const int k = kk + 8 * grp;
      const bool in = k < k1;
      Frag8 f[NX], a[RT];
#pragma unroll
      for (int n = 0; n < NX; ++n) f[n] = zero_frag();
      if (in && live) load_x<NX>(x + k, f);
#pragma unroll
      for (int t = 0; t < RT; ++t)
        a[t] = in && 16 * t + col < p.rank ? *reinterpret_cast<const Frag8*>(A + (size_t)(16 * t + col) * p.k + k) : zero_frag();
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int n = 0; n < NX; ++n) acc[t] = mfma16(f[n], a[t], acc[t]);
    }
  }
  // acc[t][e]: row 4 grp + e, rank column 16 t + col
  float* h = p.part + ((size_t)blockIdx.y * p.r.rows + sr.r0 + row0) * p.rank;
  if constexpr (ROWS4) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (row0 + 4 * grp + e < sr.n && 16 * t + col < p.rank) h[(size_t)(4 * grp + e) * p.rank + 16 * t + col] = acc[t][e];
  } else {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) sm[wave][4 * grp + e][16 * t + col] = acc[t][e];
    __syncthreads();
    for (int w = threadIdx.x; w < 16 * 16 * RT; w += 256) {
      const int rr = w / (16 * RT), c = w % (16 * RT);
      if (row0 + rr < sr.n && c < p.rank) h[(size_t)rr * p.rank + c] = (sm[0][rr][c] + sm[1][rr][c]) + (sm[2][rr][c] + sm[3][rr][c]);
    }
  }
}

// ------------------------------------------------------------------ out = base + s B h
// Eight elements of base as loaded, and as floats.
template <typename T> struct Out8;
template <> struct Out8<bf16_t> { u32x4 w; };
template <> struct Out8<float> { f32x4 a, b; };
NOVA_DEV Out8<bf16_t> load_out8(const bf16_t* p) { return {*reinterpret_cast<const u32x4*>(p)}; }
NOVA_DEV Out8<float> load_out8(const float* p) { return {reinterpret_cast<const f32x4*>(p)[0], reinterpret_cast<const f32x4*>(p)[1]}; }
NOVA_DEV void unpack_out8(const Out8<bf16_t>& r, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(r.w[i] << 16);
    x[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
  }
}
NOVA_DEV void unpack_out8(const Out8<float>& r, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = r.a[i], x[4 + i] = r.b[i];
}
template <typename T> NOVA_DEV void store_out8(T* p, const float* x) {
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

// Workgroup: (tile of TM rows, `cols` columns); a wave takes 64 columns at a time.  Which column of B is which MFMA row
// is free, so two tiles give a lane 8 consecutive columns of its row of out, and the four lane groups 32: 64 bytes of a
// row side by side in one instruction.  The rows of base of all row tiles are requested before the first product.  K (here the rank) is 32 a
// step.
template <typename TO, int RT, int TM>
__global__ void __launch_bounds__(256) lora_expand_kernel(LoraArgs p) {
  constexpr int KS = (RT + 1) / 2;                           // steps of 32 of the rank
  constexpr int LD = 32 * KS + 8;                            // row pitch in LDS (16 bytes more: rows on other banks)
  constexpr int NH = sizeof(TO) == 4 ? 3 : 2;                // parts of h
  __shared__ __align__(16) bf16_t sm[NH][TM][LD];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  int b, row0;
  const SeqRows sr = find_row_tile<TM>(p.r, blockIdx.x, &b, &row0);
  if (b < 0) return;
  const int i = p.which[b], rows = min(TM, sr.n - row0);
  const bool has = (unsigned)i < (unsigned)p.n;
  const long r0 = sr.r0 + row0;
  const TO* base = reinterpret_cast<const TO*>(p.base);
  TO* out = reinterpret_cast<TO*>(p.out);
  if (!has && base == out) return;                           // nothing is added
  if (has) {
    const float scale = p.scale ? p.scale[i] : 1.f;
    for (int w = threadIdx.x; w < TM * 32 * KS; w += 256) {
      const int rr = w / (32 * KS), c = w % (32 * KS);
      float h = 0.f;
      if (rr < rows && c < p.rank)
        for (int s = 0; s < p.slices; ++s) h += p.part[((size_t)s * p.r.rows + r0 + rr) * p.rank + c];
      h *= scale;
#pragma unroll
      for (int n = 0; n < NH; ++n) {
        const bf16_t part = f2bf(h);
        sm[n][rr][c] = part;
        h = rest_of(h, bf2f(part));
      }
    }
    __syncthreads();
  }
  const bf16_t* B = p.b + (has ? (size_t)i * p.nout * p.rank : 0);
  const int n_end = min(p.nout, (int)(blockIdx.y + 1) * p.cols);
  for (int n0 = blockIdx.y * p.cols + 64 * wave; n0 < n_end; n0 += 256) {
    Out8<TO> old[TM / 16][2];
#pragma unroll
    for (int rt = 0; rt < TM / 16; ++rt)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int rr = 16 * rt + col, n = n0 + 32 * q + 8 * grp;
        old[rt][q] = base && rr < rows && n < p.nout ? load_out8(base + (r0 + rr) * p.base_row + n) : Out8<TO>{};
      }
    // tile t = 2 q + h, MFMA row m: column n0 + 32 q + 8 (m / 4) + 4 h + m % 4, so that lane group g holds 32 q + 8 g ..
    Frag8 bf[KS][4];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int n = n0 + 32 * (t >> 1) + 8 * (col >> 2) + 4 * (t & 1) + (col & 3), k = 32 * ks + 8 * grp;
        bf[ks][t] = has && n < p.nout && k < p.rank ? *reinterpret_cast<const Frag8*>(B + (size_t)n * p.rank + k) : zero_frag();
      }
#pragma unroll
    for (int rt = 0; rt < TM / 16; ++rt) {
      if (16 * rt >= rows) break;
      const int rr = 16 * rt + col;
      f32x4 acc[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (has) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          Frag8 h[NH];
#pragma unroll
          for (int q = 0; q < NH; ++q) h[q] = *reinterpret_cast<const Frag8*>(&sm[q][rr][32 * ks + 8 * grp]);
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int q = 0; q < NH; ++q) acc[t] = mfma16(bf[ks][t], h[q], acc[t]);
        }
      }
      if (rr >= rows) continue;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int n = n0 + 32 * q + 8 * grp;
        if (n >= p.nout) continue;
        float y[8];
        unpack_out8(old[rt][q], y);
        if (has)
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] += acc[2 * q + (e >> 2)][e & 3];
        store_out8(out + (r0 + rr) * p.out_row + n, y);
      }
    }
  }
}

// ------------------------------------------------------------------ launch
// Tiles of 64 rows where the sequences have that many on average, else of 16.
static bool lora_long(const LoraArgs& p) { return p.r.rows >= LO_ROWS / 2 * (long)p.r.batch; }
static long lora_tiles(const LoraArgs& p) {
  const int tm = lora_long(p) ? LO_ROWS : LO_STEP;
  return std::min<long>(p.r.rows, p.r.rows / tm + p.r.batch);
}
// Slices of K: two workgroups for each compute unit, each of at least 512 of K.
int lora_slices(const LoraArgs& p, int cus) {
  const long want = (2l * cus + lora_tiles(p) - 1) / std::max(1l, lora_tiles(p));
  return (int)std::max(1l, std::min<long>(want, (p.k + 511) / 512));
}

template <typename TX, typename TO, int RT, int TM>
static hipError_t lora_launch(const LoraArgs& p, int cus, hipStream_t s) {
  const unsigned tiles = (unsigned)lora_tiles(p);
  constexpr int NX = sizeof(TX) == 2 ? 1 : sizeof(TO) == 2 ? 2 : 3;
  hipLaunchKernelGGL((lora_shrink_kernel<TX, NX, RT, TM>), dim3(tiles, p.slices), dim3(256), 0, s, p);
  if (hipError_t e = hipGetLastError()) return e;
  // columns of a workgroup: eight workgroups for each compute unit, whole steps of 256
  LoraArgs q = p;
  const long steps = (p.nout + 255) / 256, groups = std::min(steps, std::max(1l, 8l * cus / tiles));
  q.cols = (int)((steps + groups - 1) / groups * 256);
  hipLaunchKernelGGL((lora_expand_kernel<TO, RT, TM>), dim3(tiles, (p.nout + q.cols - 1) / q.cols), dim3(256), 0, s, q);
  return hipGetLastError();
}
template <typename TX, typename TO, int TM>
static hipError_t lora_rank(const LoraArgs& p, int cus, hipStream_t s) {
  if (p.rank <= 16) return lora_launch<TX, TO, 1, TM>(p, cus, s);
  if (p.rank <= 32) return lora_launch<TX, TO, 2, TM>(p, cus, s);
  if (p.rank <= 64) return lora_launch<TX, TO, 4, TM>(p, cus, s);
  return lora_launch<TX, TO, 8, TM>(p, cus, s);
}
template <typename TX, typename TO>
static hipError_t lora_types(const LoraArgs& p, int cus, hipStream_t s) {
  return lora_long(p) ? lora_rank<TX, TO, LO_ROWS>(p, cus, s) : lora_rank<TX, TO, LO_STEP>(p, cus, s);
}
hipError_t lora(const LoraArgs& p, int cus, hipStream_t s) {
  if (p.r.rows <= 0) return hipSuccess;
  if (p.rank <= 0 || p.rank > 128 || p.rank % 8 || p.k % 8 || p.nout % 8) return hipErrorInvalidValue;
  LoraArgs q = p;
  q.slices = lora_slices(p, cus);
  q.kslice = ((p.k + q.slices - 1) / q.slices + 31) / 32 * 32;
  if (p.x_f32) return p.out_f32 ? lora_types<float, float>(q, cus, s) : lora_types<float, bf16_t>(q, cus, s);
  return p.out_f32 ? lora_types<bf16_t, float>(q, cus, s) : lora_types<bf16_t, bf16_t>(q, cus, s);
}

}  // namespace nova
