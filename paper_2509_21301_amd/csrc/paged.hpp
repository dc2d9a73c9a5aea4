// Device-side view of a paged KV cache layer and of a batch of rows over it, shared by the cache and
// tree-attention kernels.  Everything read from device arrays (row starts, contexts, block ids) is
// clamped or checked before it becomes an address, so no array content leads outside the buffers.
#pragma once
#include "common.hpp"
#include "kernels.hpp"

namespace nova {

constexpr int PAGE = 16;                 // tokens per block
struct e4m3_t { uint8_t v; };            // one OCP e4m3 number; its token's scale is kept beside the pool

// One sequence's rows: global rows r0 .. r0 + n - 1 are its tokens ctx .. ctx + n - 1.  Tokens outside 0 .. max_ctx - 1
// do not exist: ctx is between -n and max_ctx, so that what lies outside is neither kept nor seen.
struct SeqRows { int r0, n, ctx; };

NOVA_DEV SeqRows seq_rows(const BatchRows& p, int b) {
  SeqRows s;
  if (p.row_start) {
    s.r0 = min(max(p.row_start[b], 0), p.rows);
    s.n = min(max(p.row_start[b + 1], s.r0), p.rows) - s.r0;
  } else {
    s.r0 = b * p.max_rows;               // every sequence has max_rows rows
    s.n = p.max_rows;
  }
  s.n = min(s.n, p.max_rows);
  s.ctx = p.ctx ? min(max(p.ctx[b], -s.n), p.max_ctx) : 0;
  return s;
}

// Block of a token, rounded down (a token before the sequence is in block -1 or below).
NOVA_DEV int block_of(int t) { return t >> 4; }
static_assert(PAGE == 16);

// The tile-th of all 16-token cache blocks that the batch's rows touch, counted over the sequences:
// its sequence in *b (-1: the batch has fewer tiles) and the block's number in the sequence in *blk.
// Every lane of a wave returns the same; 64 sequences are looked at a time.
NOVA_DEV SeqRows find_tile(const BatchRows& p, int tile, int* b, int* blk) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int base = 0; base < p.batch; base += 64) {
    const int i = base + lane;
    SeqRows s{0, 0, 0};
    int tiles = 0;
    if (i < p.batch) {
      s = seq_rows(p, i);
      tiles = s.n > 0 ? block_of(s.ctx + s.n - 1) - block_of(s.ctx) + 1 : 0;
    }
    int sum = tiles;                     // inclusive prefix sum over the lanes
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
      f.ctx = __builtin_amdgcn_readlane(s.ctx, l);
      *b = base + l;
      *blk = block_of(f.ctx) + tile - (before + __builtin_amdgcn_readlane(sum - tiles, l));
      return f;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  *b = -1;
  *blk = 0;
  return SeqRows{0, 0, 0};
}

// Physical block of the sequence's blk-th block, -1 where the table does not reach it or names none.
NOVA_DEV int page_of(const BatchRows& p, int num_blocks, int b, int blk) {
  if (blk < 0 || blk >= p.max_blocks) return -1;
  const int ph = p.tables[(size_t)b * p.max_blocks + blk];
  return (unsigned)ph < (unsigned)num_blocks ? ph : -1;
}

// 2^e from the byte e + 127 that an 8-bit cache keeps for a token and head.
NOVA_DEV float exp_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two e4m3 numbers (the low or the high half of a dword) times a power of two, as two bf16 in a dword:
// exact, since e4m3 has 4 significant bits.
template <bool HI> NOVA_DEV uint32_t e4m3_pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}

}  // namespace nova
