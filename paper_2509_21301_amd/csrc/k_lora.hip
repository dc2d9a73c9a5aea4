// Low-rank adapters of many requests beside a projection that they share: with i the adapter of a row's sequence,
//   out = base + s_i B_i (A_i x),   A_i [rank][K], B_i [N][rank].
//  * shrink: h = A_i x per row, tiles of a sequence's rows times a slice of K, fp32 partials [slice][row][rank];
//  * join (long sequences): the slices summed in order;
//  * expand: B_i h, times s_i, onto base, rounded once.  Short tiles sum the slices themselves (a launch less).
// The ranks are far below what would make this compute-bound: it is bound by reading x, base and the adapters and by
// writing out.  The matrix cores take bf16, so h, and x in fp32, go to them as a sum of three bf16 parts, which hold all 24
// bits, an MFMA each.
#include <algorithm>

#include "paged.hpp"

namespace nova {

constexpr int LO_STEP = 16;                // rows of a tile of short sequences; long ones have 64 or 128

// Orders a wave's own LDS writes before its own LDS reads.
NOVA_DEV void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

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

// An fp32 number is the sum of three of bf16, 8 of its 24 bits each (what is below bf16's smallest number, 2^-133, is left
// out): cut off, not rounded, so that no part of a finite number is infinite.  The upper halves of two floats in a dword (a's in the low half), those halves as floats, and what
// they leave (of infinity nothing; of NaN NaN).
constexpr int LO_PARTS = 3;
NOVA_DEV uint32_t top2(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
NOVA_DEV float top(float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); }
NOVA_DEV float rest_of(float v) {
  const float t = top(v);
  return v == t ? 0.f : v - t;
}

// Eight floats as a sum of N operands of bf16.
template <int N> NOVA_DEV void split_parts(float* x, Frag8* f) {
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[n].w[i] = top2(x[2 * i], x[2 * i + 1]);
      x[2 * i] = rest_of(x[2 * i]);
      x[2 * i + 1] = rest_of(x[2 * i + 1]);
    }
}

// Eight elements of x as loaded, and as N operands.
template <typename T> struct Raw;
template <> struct Raw<bf16_t> { Frag8 f; };
template <> struct Raw<float> { f32x4 a, b; };
NOVA_DEV Raw<bf16_t> load_raw_x(const bf16_t* p) { return {*reinterpret_cast<const Frag8*>(p)}; }
NOVA_DEV Raw<float> load_raw_x(const float* p) { return {reinterpret_cast<const f32x4*>(p)[0], reinterpret_cast<const f32x4*>(p)[1]}; }
template <int N> NOVA_DEV void split_raw(const Raw<bf16_t>& r, Frag8* f) { f[0] = r.f; }
template <int N> NOVA_DEV void split_raw(const Raw<float>& r, Frag8* f) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = r.a[i], x[4 + i] = r.b[i];
  split_parts<N>(x, f);
}

// ------------------------------------------------------------------ h = A x, short sequences
// Workgroup: (tile of 16 rows, slice of K); its waves take the k steps in turn and their sums are joined in LDS.  Lane (row
// or rank column = lane % 16, k group = lane / 16) loads 16 bytes of its row of x and of A per 32 k.
template <typename TX, int NX, int RT>
__global__ void __launch_bounds__(256) lora_shrink_kernel(LoraArgs p) {
  constexpr int AHEAD = RT * NX >= 8 ? 2 : 4;                // steps whose loads are requested together
  __shared__ float sm[4][16][16 * RT + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  int b, row0;
  const SeqRows sr = find_row_tile<LO_STEP>(p.r, blockIdx.x, &b, &row0);
  if (b < 0) return;
  const int i = p.which[b];
  if ((unsigned)i >= (unsigned)p.n) return;
  const int k0 = blockIdx.y * p.kslice, k1 = min(p.k, k0 + p.kslice);
  const bf16_t* A = p.a + (size_t)i * p.rank * p.k;
  // Rows behind the tile's last and ranks behind the adapter's repeat the last one: what comes of them is not stored.
  const TX* x = reinterpret_cast<const TX*>(p.x) + (long)(sr.r0 + min(row0 + col, sr.n - 1)) * p.x_row;
  const bf16_t* ar[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) ar[t] = A + (size_t)min(16 * t + col, p.rank - 1) * p.k;
  f32x4 acc[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto step = [&](int kk, bool whole) {                      // k kk .. kk + 31, of which those below k1
    const int k = kk + 8 * grp;
    const bool in = whole || k < k1;
    const int at = in ? k : 0;
    Frag8 f[NX], a[RT];
    split_raw<NX>(load_raw_x(x + at), f);
#pragma unroll
    for (int t = 0; t < RT; ++t) a[t] = *reinterpret_cast<const Frag8*>(ar[t] + at);
    if (!whole) {
#pragma unroll
      for (int n = 0; n < NX; ++n) f[n] = in ? f[n] : zero_frag();
#pragma unroll
      for (int t = 0; t < RT; ++t) a[t] = in ? a[t] : zero_frag();
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int n = 0; n < NX; ++n) acc[t] = mfma16(f[n], a[t], acc[t]);
  };
  int kk = k0 + 32 * wave;
#pragma unroll AHEAD
  for (; kk + 32 <= k1; kk += 128) step(kk, true);
  if (kk < k1) step(kk, false);
  // acc[t][e]: row 4 grp + e, rank column 16 t + col
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) sm[wave][4 * grp + e][16 * t + col] = acc[t][e];
  __syncthreads();
  float* h = p.part + ((size_t)blockIdx.y * p.r.rows + sr.r0 + row0) * p.rank;
  for (int w = threadIdx.x; w < 16 * 16 * RT; w += 256) {
    const int rr = w / (16 * RT), c = w % (16 * RT);
    if (row0 + rr < sr.n && c < p.rank) h[(size_t)rr * p.rank + c] = (sm[0][rr][c] + sm[1][rr][c]) + (sm[2][rr][c] + sm[3][rr][c]);
  }
}

// ------------------------------------------------------------------ h = A x, long sequences
// Workgroup: (tile of 64 RW rows, slice of K), RW blocks of 16 rows a wave.  64 of K at a time go through LDS, loaded a
// step ahead: an MFMA operand has neighbouring lanes in different rows, and read straight from memory each of its 16 bytes
// is an access of its own to the address unit (54 of 64 a load, and the unit busy for 78% of the time).  16-byte chunks of
// a row are turned by its number (chunk c of row r at c ^ (r & 7)): no bank conflicts.  3751 rows of 3584 to rank 64: 13.4
// us, 27 from memory; the floor, reading x, is 5.3.
template <typename TX, int NX, int RT, int RW>
__global__ void __launch_bounds__(256) lora_down_kernel(LoraArgs p) {
  constexpr int TM = 64 * RW, XC = TM * 8 / 256, AC = (16 * RT * 8 + 255) / 256;   // chunks of a thread: x, A
  constexpr int NB = NX == 1 ? 2 : 1;                        // buffers; x in parts leaves room for one
  __shared__ __align__(16) Frag8 sm_x[NB][NX][TM][8];
  __shared__ __align__(16) Frag8 sm_a[NB][16 * RT][8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  int b, row0;
  const SeqRows sr = find_row_tile<TM>(p.r, blockIdx.x, &b, &row0);
  if (b < 0) return;
  const int i = p.which[b];
  if ((unsigned)i >= (unsigned)p.n) return;
  const int k0 = blockIdx.y * p.kslice, k1 = min(p.k, k0 + p.kslice);
  // Rows behind the tile's last and ranks behind the adapter's repeat the last one: what comes of them is not stored.
  const TX* x = reinterpret_cast<const TX*>(p.x) + (long)(sr.r0 + row0) * p.x_row;
  const bf16_t* A = p.a + (size_t)i * p.rank * p.k;
  const int rows = min(TM, sr.n - row0), chunk = threadIdx.x & 7, first = threadIdx.x >> 3;
  Raw<TX> rx[XC];
  Frag8 ra[AC];
  auto request = [&](int kk) {
    const int k = min(kk + 8 * chunk, k1 - 8);
#pragma unroll
    for (int j = 0; j < XC; ++j) rx[j] = load_raw_x(x + (long)min(first + 32 * j, rows - 1) * p.x_row + k);
#pragma unroll
    for (int j = 0; j < AC; ++j) ra[j] = *reinterpret_cast<const Frag8*>(A + (size_t)min(first + 32 * j, p.rank - 1) * p.k + k);
  };
  auto keep = [&](int kk, int buf) {
    const bool in = kk + 8 * chunk < k1;                     // what lies behind the slice is zero
#pragma unroll
    for (int j = 0; j < XC; ++j) {
      const int r = first + 32 * j;
      Frag8 f[NX];
      split_raw<NX>(rx[j], f);
#pragma unroll
      for (int n = 0; n < NX; ++n) sm_x[buf][n][r][chunk ^ (r & 7)] = in ? f[n] : zero_frag();
    }
#pragma unroll
    for (int j = 0; j < AC; ++j) {
      const int r = first + 32 * j;
      if (16 * RT % 32 == 0 || r < 16 * RT) sm_a[buf][r][chunk ^ (r & 7)] = in ? ra[j] : zero_frag();
    }
  };
  f32x4 acc[RW][RT];
#pragma unroll
  for (int w = 0; w < RW; ++w)
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[w][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (k0 < k1) request(k0);
  for (int kk = k0, buf = 0; kk < k1; kk += 64, buf ^= NB - 1) {
    if (NB == 1 && kk > k0) __syncthreads();
    keep(kk, buf);
    if (kk + 64 < k1) request(kk + 64);
    __syncthreads();                       // of two buffers a wave one step ahead writes the other
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Frag8 a[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) a[t] = sm_a[buf][16 * t + col][(4 * s + grp) ^ (col & 7)];
#pragma unroll
      for (int w = 0; w < RW; ++w)
#pragma unroll
        for (int n = 0; n < NX; ++n) {
          const Frag8 f = sm_x[buf][n][16 * (RW * wave + w) + col][(4 * s + grp) ^ (col & 7)];
#pragma unroll
          for (int t = 0; t < RT; ++t) acc[w][t] = mfma16(f, a[t], acc[w][t]);
        }
    }
  }
  // acc[w][t][e]: row 16 (RW wave + w) + 4 grp + e, rank column 16 t + col
  float* h = p.part + ((size_t)blockIdx.y * p.r.rows + sr.r0 + row0) * p.rank;
#pragma unroll
  for (int w = 0; w < RW; ++w)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 16 * (RW * wave + w) + 4 * grp + e;
#pragma unroll
      for (int t = 0; t < RT; ++t)
        if (r < rows && 16 * t + col < p.rank) h[(size_t)r * p.rank + 16 * t + col] = acc[w][t][e];
    }
}

// ------------------------------------------------------------------ h joined
// Thread: four ranks of a row, [row][32 KS] with zeros behind the rank, in fp32: the expand reads every row once for each of
// its columns' workgroups, and parts would be half as much again.  Rows without an adapter (whose partials nobody wrote) give
// what nobody reads.
template <int KS>
__global__ void __launch_bounds__(256) lora_join_kernel(LoraArgs p) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x, row = i / (8 * KS);
  const int c = (int)(i % (8 * KS)) * 4;
  if (row >= p.r.rows) return;
  f32x4 h{0.f, 0.f, 0.f, 0.f};
  if (c < p.rank) {
#pragma unroll 4
    for (int s = 0; s < p.slices; ++s) h += *reinterpret_cast<const f32x4*>(p.part + ((size_t)s * p.r.rows + row) * p.rank + c);
  }
  *reinterpret_cast<f32x4*>(p.joined + row * (32 * KS) + c) = h;
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

// Chunk c of column n of B in LDS (CH chunks of 16 bytes a column) lies so that eight neighbouring columns' chunks are on
// different banks.
template <int CH> NOVA_DEV int turn_chunk(int n, int c) { return CH >= 8 ? c ^ (n & 7) : CH == 4 ? c ^ ((n >> 1) & 3) : c ^ ((n >> 2) & 1); }

// ---- short sequences
// Workgroup: (tile of 16 rows, `cols` columns); a wave takes 64 columns at a time, whose B it loads in one run and turns
// into MFMA operands in LDS of its own, a step ahead; the first step's loads are on their way while h is summed.  Which
// column of B is which MFMA row is free, so two tiles give a lane 8 consecutive columns of its row of out.  K (here the
// rank) is 32 a step.  Bound by latency: 32 tokens with an adapter each of rank 16 onto 4608 columns 5.3 to 6.3 us (the kernel
// above 3.6), onto 37888 columns 14.7 us, 2.7 TB/s of adapters.
template <typename TO, int RT>
__global__ void __launch_bounds__(256) lora_expand_kernel(LoraArgs p) {
  constexpr int KS = (RT + 1) / 2;                           // steps of 32 of the rank
  constexpr int LD = 32 * KS + 8;                            // row pitch of h in LDS (16 bytes more: rows on other banks)
  constexpr int CH = 2 * RT;                                 // chunks of a column of B, and of a lane
  __shared__ __align__(16) bf16_t sm[LO_PARTS][LO_STEP][LD];
  __shared__ __align__(16) Frag8 sm_b[4][64][CH];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  int b, row0;
  const SeqRows sr = find_row_tile<LO_STEP>(p.r, blockIdx.x, &b, &row0);
  if (b < 0) return;
  const int i = p.which[b], rows = min(LO_STEP, sr.n - row0);
  const bool has = (unsigned)i < (unsigned)p.n;
  const long r0 = sr.r0 + row0;
  const TO* base = reinterpret_cast<const TO*>(p.base);
  TO* out = reinterpret_cast<TO*>(p.out);
  if (!has && base == out) return;                           // nothing is added
  const bf16_t* B = p.b + (has ? (size_t)i * p.nout * p.rank : 0);
  Frag8 rb[CH];
  Out8<TO> next[2], old[2];
  // Rows behind the tile's last and columns and ranks behind the last repeat what is there.
  auto request = [&](int n0) {
    if (has)
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const int w = lane + 64 * j;
        rb[j] = *reinterpret_cast<const Frag8*>(B + (size_t)min(n0 + w / CH, p.nout - 1) * p.rank + min(8 * (w % CH), p.rank - 8));
      }
    if (base) {
#pragma unroll
      for (int q = 0; q < 2; ++q) next[q] = load_out8(base + (r0 + min(col, rows - 1)) * p.base_row + min(n0 + 32 * q + 8 * grp, p.nout - 8));
    } else {
      next[0] = next[1] = Out8<TO>{};
    }
  };
  const int n_end = min(p.nout, (int)(blockIdx.y + 1) * p.cols);
  int n0 = blockIdx.y * p.cols + 64 * wave;
  if (n0 < n_end) request(n0);
  const float scale = has && p.scale ? p.scale[i] : 1.f;
  if (has) {
    for (int w = threadIdx.x; w < LO_STEP * 32 * KS; w += 256) {
      const int rr = w / (32 * KS), c = w % (32 * KS);
      float h = 0.f;
      if (rr < rows && c < p.rank) {
#pragma unroll 8
        for (int s = 0; s < p.slices; ++s) h += p.part[((size_t)s * p.r.rows + r0 + rr) * p.rank + c];
      }
#pragma unroll
      for (int n = 0; n < LO_PARTS; ++n) {
        sm[n][rr][c] = (bf16_t)(__float_as_uint(h) >> 16);
        h = rest_of(h);
      }
    }
    __syncthreads();
  }
  for (; n0 < n_end; n0 += 256) {
    if (has) {
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const int w = lane + 64 * j, n = w / CH, c = w % CH;
        sm_b[wave][n][turn_chunk<CH>(n, c)] = 8 * c < p.rank ? rb[j] : zero_frag();
      }
    }
    old[0] = next[0], old[1] = next[1];
    if (n0 + 256 < n_end) request(n0 + 256);
    wave_fence();
    f32x4 acc[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (has) {
      // tile t = 2 q + h, MFMA row m: column 32 q + 8 (m / 4) + 4 h + m % 4 of the step, so that lane group g holds 32 q + 8 g ..
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        Frag8 h[LO_PARTS];
#pragma unroll
        for (int q = 0; q < LO_PARTS; ++q) h[q] = *reinterpret_cast<const Frag8*>(&sm[q][col][32 * ks + 8 * grp]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int n = 32 * (t >> 1) + 8 * (col >> 2) + 4 * (t & 1) + (col & 3), c = 4 * ks + grp;
          const Frag8 f = CH >= 4 || grp < 2 ? sm_b[wave][n][turn_chunk<CH>(n, CH >= 4 ? c : c & 1)] : zero_frag();
#pragma unroll
          for (int q = 0; q < LO_PARTS; ++q) acc[t] = mfma16(f, h[q], acc[t]);
        }
      }
    }
    wave_fence();                          // the next step writes there
    if (col < rows) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int n = n0 + 32 * q + 8 * grp;
        if (n >= p.nout) continue;
        float y[8];
        unpack_out8(old[q], y);
        if (has)
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] += scale * acc[2 * q + (e >> 2)][e & 3];
        store_out8(out + (r0 + col) * p.out_row + n, y);
      }
    }
  }
}

// ---- long sequences
// 16 bytes of base as loaded, and as floats.
template <typename T> NOVA_DEV void unpack16(const u32x4& w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      x[i] = __uint_as_float(w[i]);
    } else {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}
template <typename T> NOVA_DEV u32x4 pack16(const float* x) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(x[i]) : pack2(x[2 * i], x[2 * i + 1]);
  return w;
}

// Workgroup: (tile of 64 RW rows, `cols` columns), RW blocks of 16 rows a wave, whose h stays in registers.  64 columns of
// B at a time go through LDS for all four waves, loaded a step ahead (turned as in the kernel above), and what they give
// goes back through LDS, so that base and out are read and written in runs of a row's 64 columns: see there.  3751 rows onto
// 37888 columns in bf16, rank 64: 117 to 132 us, 4.3 to 4.9 TB/s of 5.1 that a large copy reaches (162 us with operands
// and rows straight from memory); rank 16 110, rank 128 (one block) 156 to 181, fp32 228 us.  Rows that start off a line of
// 128 bytes (37896 columns) share each line between two steps: 182 us.
template <typename TO, int RT, int RW>
__global__ void __launch_bounds__(256) lora_up_kernel(LoraArgs p) {
  constexpr int KS = (RT + 1) / 2, TM = 64 * RW;
  constexpr int CH = 2 * RT, BC = 64 * CH / 256 > 0 ? 64 * CH / 256 : 1;   // chunks of a column of B; of a thread
  constexpr int E = 16 / sizeof(TO), LPR = 64 / E, RPI = 64 / LPR, IT = 16 / RPI;   // of out: elements and lanes of a row, rows of an instruction
  constexpr int LD = 68;                                     // floats of a row in LDS
  __shared__ __align__(16) Frag8 sm_b[2][64][CH];
  __shared__ __align__(16) float sm_o[4][16][LD];
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
  const float scale = has && p.scale ? p.scale[i] : 1.f;
  const bf16_t* B = p.b + (has ? (size_t)i * p.nout * p.rank : 0);
  Frag8 h[RW][KS][LO_PARTS];
#pragma unroll
  for (int w = 0; w < RW; ++w)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (has) unpack_out8(load_out8(p.joined + (r0 + min(16 * (RW * wave + w) + col, rows - 1)) * (32 * KS) + 32 * ks + 8 * grp), y);
      split_parts<LO_PARTS>(y, h[w][ks]);
    }
  const int bn = threadIdx.x / CH, bc = threadIdx.x % CH;    // the thread's first column and chunk
  Frag8 rb[BC];
  u32x4 old[RW][IT], next[RW][IT];
  const int orow = lane / LPR, ocol = lane % LPR * E;        // of an instruction
  auto request = [&](int n0) {
    if (has) {
#pragma unroll
      for (int j = 0; j < BC; ++j) {
        const int n = bn + 256 / CH * j;
        rb[j] = *reinterpret_cast<const Frag8*>(B + (size_t)min(n0 + n, p.nout - 1) * p.rank + min(8 * bc, p.rank - 8));
      }
    }
    if (base) {
#pragma unroll
      for (int w = 0; w < RW; ++w)
#pragma unroll
        for (int j = 0; j < IT; ++j)
          next[w][j] = *reinterpret_cast<const u32x4*>(base + (r0 + min(16 * (RW * wave + w) + RPI * j + orow, rows - 1)) * p.base_row + min(n0 + ocol, p.nout - E));
    } else {
#pragma unroll
      for (int w = 0; w < RW; ++w)
#pragma unroll
        for (int j = 0; j < IT; ++j) next[w][j] = u32x4{0u, 0u, 0u, 0u};
    }
  };
  const int n_begin = blockIdx.y * p.cols, n_end = min(p.nout, n_begin + p.cols);
  request(n_begin);
  for (int n0 = n_begin, buf = 0; n0 < n_end; n0 += 64, buf ^= 1) {
    if (has && (64 * CH >= 256 || threadIdx.x < 64 * CH)) {
#pragma unroll
      for (int j = 0; j < BC; ++j) {
        const int n = bn + 256 / CH * j;
        sm_b[buf][n][turn_chunk<CH>(n, bc)] = 8 * bc < p.rank ? rb[j] : zero_frag();
      }
    }
#pragma unroll
    for (int w = 0; w < RW; ++w)
#pragma unroll
      for (int j = 0; j < IT; ++j) old[w][j] = next[w][j];
    if (n0 + 64 < n_end) request(n0 + 64);
    __syncthreads();                       // a wave one step ahead writes the other buffer
    f32x4 acc[RW][4];
#pragma unroll
    for (int w = 0; w < RW; ++w)
#pragma unroll
      for (int t = 0; t < 4; ++t) acc[w][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (has) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int n = 16 * t + col, c = 4 * ks + grp;
          const Frag8 f = CH >= 4 || grp < 2 ? sm_b[buf][n][turn_chunk<CH>(n, CH >= 4 ? c : c & 1)] : zero_frag();
#pragma unroll
          for (int w = 0; w < RW; ++w)
#pragma unroll
            for (int q = 0; q < LO_PARTS; ++q) acc[w][t] = mfma16(f, h[w][ks][q], acc[w][t]);
        }
    }
    // acc[w][t][e]: row 16 (RW wave + w) + col, column 16 t + 4 grp + e
#pragma unroll
    for (int w = 0; w < RW; ++w) {
      if (16 * (RW * wave + w) >= rows) break;
#pragma unroll
      for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4*>(&sm_o[wave][col][16 * t + 4 * grp]) = acc[w][t];
      wave_fence();
#pragma unroll
      for (int j = 0; j < IT; ++j) {
        const int rr = RPI * j + orow, r = 16 * (RW * wave + w) + rr;
        float y[E];
        unpack16<TO>(old[w][j], y);
        if (has)
#pragma unroll
          for (int e = 0; e < E; e += 4) {
            const f32x4 d = *reinterpret_cast<const f32x4*>(&sm_o[wave][rr][ocol + e]);
#pragma unroll
            for (int x = 0; x < 4; ++x) y[e + x] += scale * d[x];
          }
        if (r < rows && n0 + ocol < p.nout) *reinterpret_cast<u32x4*>(out + (r0 + r) * p.out_row + n0 + ocol) = pack16<TO>(y);
      }
      wave_fence();
    }
  }
}

// ------------------------------------------------------------------ launch
// Blocks of 16 rows a wave of the kernels for long sequences takes (0: those for short ones): long ones by the rows that a
// sequence has on average, two blocks, which read B half as often, where the result is large and h of both leaves registers
// enough.  us of a call in a graph with 0 / 1 / 2:
//  * onto 37888 columns: 8 sequences of 24 rows at rank 16 20 / 21 / 29; one of 2000 at rank 64 147 / 84 / 86, with 31 of one
//    row beside it 157 / 110 / 120, with 127 187 / 181 / 241; 64 of one row at rank 16 24 / 45 / 73;
//  * with 1 / 2 onto 37888 columns: one of 600 rows at rank 64 35 / 38, of 4000 153 / 147, at rank 128 191 / 184 (fp32 285 /
//    308); 8 of 140 63 / 74; 3751 rows at rank 64 onto 3584 33 / 36, in fp32 onto 4608 60 / 66.
static int lora_blocks(const LoraArgs& p) {
  const long rows = p.r.rows, batch = p.r.batch;
  if (rows < 32 * batch) return 0;
  return rows >= 128 * batch && rows * p.nout >= 100000000 && p.rank <= 64 ? 2 : 1;
}
static long lora_tiles(const LoraArgs& p) {
  const int rw = lora_blocks(p), tm = rw ? 64 * rw : LO_STEP;
  return std::min<long>(p.r.rows, p.r.rows / tm + p.r.batch);
}
// Slices of K: four workgroups for each compute unit, each of at least 256 of K where h is joined, 512 where every
// workgroup of the expand sums the slices.
static int lora_slices(const LoraArgs& p, int cus) {
  const long tiles = std::max(1l, lora_tiles(p)), want = (4l * cus + tiles - 1) / tiles, least = lora_blocks(p) ? 256 : 512;
  return (int)std::max(1l, std::min<long>(want, (p.k + least - 1) / least));
}
static size_t joined_at(const LoraArgs& p, int slices) { return ((size_t)slices * p.r.rows * p.rank * sizeof(float) + 255) / 256 * 256; }
size_t lora_bytes(const LoraArgs& p, int cus) {
  // and h, of the rank rounded up to the widths that the kernels have
  const int wide = p.rank <= 32 ? 32 : p.rank <= 64 ? 64 : 128;
  return joined_at(p, lora_slices(p, cus)) + (lora_blocks(p) ? (size_t)p.r.rows * wide * sizeof(float) : 0);
}

template <typename TX, typename TO, int RT, int RW>
static hipError_t lora_launch(const LoraArgs& p, int cus, hipStream_t s) {
  constexpr int NX = sizeof(TX) == 2 ? 1 : LO_PARTS;
  const unsigned tiles = (unsigned)lora_tiles(p);
  const dim3 slices(tiles, p.slices);
  if constexpr (RW == 0) {
    hipLaunchKernelGGL((lora_shrink_kernel<TX, NX, RT>), slices, dim3(256), 0, s, p);
  } else {
    constexpr int KS = (RT + 1) / 2;
    hipLaunchKernelGGL((lora_down_kernel<TX, NX, RT, RW>), slices, dim3(256), 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL((lora_join_kernel<KS>), dim3((unsigned)(((long)p.r.rows * 8 * KS + 255) / 256)), dim3(256), 0, s, p);
  }
  if (hipError_t e = hipGetLastError()) return e;
  // columns of a workgroup: whole steps, twelve workgroups for each compute unit (3751 rows onto 37888 columns at rank 64:
  // 147 us a call, 150 with eight, 168 with four)
  LoraArgs q = p;
  const int step = RW ? 64 : 256;
  const long steps = (p.nout + step - 1) / step, groups = std::min(steps, std::max(1l, 12l * cus / tiles));
  q.cols = (int)((steps + groups - 1) / groups * step);
  const dim3 grid(tiles, (p.nout + q.cols - 1) / q.cols);
  if constexpr (RW == 0) hipLaunchKernelGGL((lora_expand_kernel<TO, RT>), grid, dim3(256), 0, s, q);
  else hipLaunchKernelGGL((lora_up_kernel<TO, RT, RW>), grid, dim3(256), 0, s, q);
  return hipGetLastError();
}
template <typename TX, typename TO, int RW>
static hipError_t lora_rank(const LoraArgs& p, int cus, hipStream_t s) {
  if (p.rank <= 16) return lora_launch<TX, TO, 1, RW>(p, cus, s);
  if (p.rank <= 32) return lora_launch<TX, TO, 2, RW>(p, cus, s);
  if (p.rank <= 64) return lora_launch<TX, TO, 4, RW>(p, cus, s);
  return lora_launch<TX, TO, 8, RW == 2 ? 1 : RW>(p, cus, s);   // lora_blocks(): two up to rank 64
}
template <typename TX, typename TO>
static hipError_t lora_types(const LoraArgs& p, int cus, hipStream_t s) {
  switch (lora_blocks(p)) {
    case 0: return lora_rank<TX, TO, 0>(p, cus, s);
    case 1: return lora_rank<TX, TO, 1>(p, cus, s);
    default: return lora_rank<TX, TO, 2>(p, cus, s);
  }
}
hipError_t lora(const LoraArgs& p, int cus, hipStream_t s) {
  if (p.r.rows <= 0) return hipSuccess;
  if (p.rank <= 0 || p.rank > 128 || p.rank % 8 || p.k % 8 || p.nout % 8) return hipErrorInvalidValue;
  LoraArgs q = p;
  q.slices = lora_slices(p, cus);
  q.joined = (float*)((char*)p.part + joined_at(p, q.slices));
  q.kslice = ((p.k + q.slices - 1) / q.slices + 63) / 64 * 64;
  if (p.x_f32) return p.out_f32 ? lora_types<float, float>(q, cus, s) : lora_types<float, bf16_t>(q, cus, s);
  return p.out_f32 ? lora_types<bf16_t, float>(q, cus, s) : lora_types<bf16_t, bf16_t>(q, cus, s);
}

}  // namespace nova
