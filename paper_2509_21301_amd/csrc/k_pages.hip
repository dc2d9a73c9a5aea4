// Pages of a paged cache on the device: blocks taken for tokens to come, sequences forked (whole pages shared, the
// last one copied), given up, the pool's used blocks moved to its front, blocks copied by number, and the accepted
// rows of drafted trees moved next to their context.  refs[block] counts the table entries that name a block; a block
// with none is free.  What is taken is always the lowest free blocks in the order of the requests, so results do not
// depend on scheduling.
//
// A plan (who gets which block) is one workgroup of 1024 threads: prefix sums over the requests and over the pool,
// bound by the latency of their few steps.  Moving the pages themselves, in every layer, is the second launch, bound
// by HBM.
#include <algorithm>

#include "paged.hpp"

namespace nova {

constexpr int PLAN = 1024;

// Exclusive prefix sum over the workgroup's threads, and the total.
template <typename T> NOVA_DEV T block_scan(T v, T* total) {
  __shared__ T sm[PLAN / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T up = __shfl_up(s, o, 64);
    if (lane >= o) s += up;
  }
  __syncthreads();
  if (lane == 63) sm[wave] = s;
  __syncthreads();
  T before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < PLAN / 64; ++w) {
    if (w < wave) before += sm[w];
    sum += sm[w];
  }
  *total = sum;
  return before + s - v;
}

// A span of PLAN * E consecutive blocks: a wave has 64 E of them, 64 at a time, and which of those satisfy is(count) as a
// mask each.
template <int E, typename F> NOVA_DEV void span_masks(const int* refs, int num_blocks, int base, unsigned long long (&m)[E], F&& is) {
  int v[E];
  const int first = base + (threadIdx.x >> 6) * (64 * E) + (threadIdx.x & 63);
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = refs[min(first + 64 * i, num_blocks - 1)];   // the loads together
#pragma unroll
  for (int i = 0; i < E; ++i) m[i] = __ballot(first + 64 * i < num_blocks && is(v[i]));
}
template <int E> NOVA_DEV int mask_count(const unsigned long long (&m)[E]) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) n += __popcll(m[i]);
  return n;
}
// Calls f(rank, block) for every block of the span in the masks, ranks from `before` on; returns the rank behind them.
template <int E, typename F> NOVA_DEV int span_ranks(const unsigned long long (&m)[E], int base, int before, F&& f) {
  __shared__ int sm[PLAN / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  if (lane == 0) sm[wave] = mask_count(m);
  __syncthreads();
  int at = before, end = before;
#pragma unroll
  for (int w = 0; w < PLAN / 64; ++w) {
    if (w < wave) at += sm[w];
    end += sm[w];
  }
#pragma unroll
  for (int i = 0; i < E; ++i) {
    if (m[i] >> lane & 1) f(at + __popcll(m[i] & ((1ull << lane) - 1)), base + (wave * E + i) * 64 + lane);
    at += __popcll(m[i]);
  }
  return end;
}

// The lowest `want` free blocks of the pool into list[]; returns how many there are (at most `want`).  (64 sequences of a
// pool of 100000 blocks that take one each: 38 us with what they give back.)
template <int E> NOVA_DEV int free_blocks(const int* refs, int num_blocks, int want, int* list) {
  int got = 0;
  for (long base = 0; base < num_blocks && got < want; base += PLAN * E) {
    unsigned long long m[E];
    span_masks(refs, num_blocks, (int)base, m, [](int n) { return n <= 0; });
    got = span_ranks(m, (int)base, got, [&](int rank, int block) {
      if (rank < want) list[rank] = block;
    });
  }
  __syncthreads();                          // list[] is read by other threads
  return min(got, want);
}

NOVA_DEV bool in_pool(int block, int num_blocks) { return (unsigned)block < (unsigned)num_blocks; }

// ------------------------------------------------------------------ blocks for tokens to come
// A wave per sequence counts the entries below need / 16 that name no block; a sequence is served if it and those
// before it find enough free blocks.
template <int E> __global__ void __launch_bounds__(PLAN) pages_extend_kernel(PagesArgs p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int b = wave; b < p.n; b += PLAN / 64) {
    const int need = p.lens[b];
    const long blocks = need <= 0 ? 0 : ((long)need + PAGE - 1) / PAGE;
    int miss = 0;
    if (blocks <= p.max_blocks)
      for (int e = lane; e < blocks; e += 64) miss += !in_pool(p.tables[(long)b * p.max_blocks + e], p.num_blocks);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) miss += __shfl_xor(miss, o, 64);
    if (lane == 0) p.want[b] = blocks > p.max_blocks ? -1 : miss;       // -1: the table is too short
  }
  __syncthreads();
  long asked = 0;
  for (int b0 = 0; b0 < p.n; b0 += PLAN) {
    const int b = b0 + threadIdx.x;
    long total;
    const long before = block_scan<long>(b < p.n ? max(p.want[b], 0) : 0, &total);
    if (b < p.n) p.rank[b] = (int)min(asked + before, 0x7FFFFFFFL);
    asked += total;
  }
  const int found = free_blocks<E>(p.refs, p.num_blocks, (int)min(asked, (long)p.num_blocks), p.list);
  for (int b = wave; b < p.n; b += PLAN / 64) {
    const int want = p.want[b], rank = p.rank[b];
    const bool ok = want == 0 || (want > 0 && (long)rank + want <= found);
    if (lane == 0) p.done[b] = ok;
    if (!ok || want == 0) continue;
    const int blocks = (int)(((long)p.lens[b] + PAGE - 1) / PAGE);
    int at = rank;
    for (int e0 = 0; e0 < blocks; e0 += 64) {
      const int e = e0 + lane;
      int* entry = p.tables + (long)b * p.max_blocks + e;
      const bool miss = e < blocks && !in_pool(*entry, p.num_blocks);
      const unsigned long long m = __ballot(miss);
      if (miss) {
        const int block = p.list[at + __popcll(m & ((1ull << lane) - 1))];
        *entry = block;
        p.refs[block] = 1;
      }
      at += __popcll(m);
    }
  }
}

// ------------------------------------------------------------------ forks
// Fork i: row dst[i] of the tables becomes the first lens[i] tokens of row src[i].  Refused (done 0, nothing changed):
// rows outside the tables, a target that is any request's source (so no source is overwritten, whatever the order) or an
// earlier request's target (be that one served or not), lengths that the source's pages do not cover, and forks behind the
// pool's last free block.
constexpr int MAX_BATCH = 1 << 16;
template <int E> __global__ void __launch_bounds__(PLAN) pages_fork_kernel(PagesArgs p) {
  __shared__ unsigned sm_source[MAX_BATCH / 32];            // a bit for every row: it is a source
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int b = threadIdx.x; b < p.batch; b += PLAN) __hip_atomic_store(p.claim + b, 0x7FFFFFFF, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  for (int w = threadIdx.x; w < (p.batch + 31) / 32; w += PLAN) sm_source[w] = 0u;
  __syncthreads();
  for (int i = threadIdx.x; i < p.n; i += PLAN) {
    const int src = p.src[i], dst = p.dst[i];
    if ((unsigned)src < (unsigned)p.batch) atomicOr(sm_source + (src >> 5), 1u << (src & 31));
    if ((unsigned)dst < (unsigned)p.batch) __hip_atomic_fetch_min(p.claim + dst, i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  for (int i = wave; i < p.n; i += PLAN / 64) {
    const int src = p.src[i], dst = p.dst[i], len = p.lens[i];
    const long blocks = ((long)len + PAGE - 1) / PAGE;
    bool ok = (unsigned)src < (unsigned)p.batch && (unsigned)dst < (unsigned)p.batch && len >= 0 && blocks <= p.max_blocks;
    if (ok) ok = __hip_atomic_load(p.claim + dst, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i &&
                 !(sm_source[dst >> 5] >> (dst & 31) & 1);
    bool miss = false;
    if (ok)
      for (int e = lane; e < blocks; e += 64) miss |= !in_pool(p.tables[(long)src * p.max_blocks + e], p.num_blocks);
    if (__ballot(miss)) ok = false;
    if (lane == 0) p.want[i] = ok ? len % PAGE > 0 : -1;
  }
  __syncthreads();
  int asked = 0;
  for (int i0 = 0; i0 < p.n; i0 += PLAN) {
    const int i = i0 + threadIdx.x;
    int total;
    const int before = block_scan(i < p.n ? max(p.want[i], 0) : 0, &total);
    if (i < p.n) p.rank[i] = asked + before;
    asked += total;
  }
  const int found = free_blocks<E>(p.refs, p.num_blocks, min(asked, p.num_blocks), p.list);
  for (int i = threadIdx.x; i < p.n; i += PLAN) {
    const int want = p.want[i], rank = p.rank[i];
    const bool ok = want == 0 || (want == 1 && rank < found);
    int from = -1, to = -1;
    if (ok && want) from = p.tables[(long)p.src[i] * p.max_blocks + p.lens[i] / PAGE], to = p.list[rank];
    p.done[i] = ok, p.from[i] = from, p.to[i] = to;
  }
}

// ------------------------------------------------------------------ pages given up
// Request i with lens keeps the pages of row src[i]'s first lens[i] tokens.  What the row appends next goes into the page
// that is kept in part, so that has to be the row's own: one that other entries name too is refused, by the counts
// before anything is given up (a launch of its own, since requests of one call may share pages).
__global__ void __launch_bounds__(256) pages_trim_kernel(PagesArgs p) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= p.n) return;
  const int row = p.src[i], len = max(p.lens[i], 0), last = len / PAGE;     // the page that holds token len
  bool ok = (unsigned)row < (unsigned)p.batch;
  if (ok && len % PAGE && last < p.max_blocks) {
    const int block = p.tables[(long)row * p.max_blocks + last];
    ok = !in_pool(block, p.num_blocks) || p.refs[block] <= 1;
  }
  p.done[i] = ok;
}

// Row src[i] of the tables keeps the pages of its first lens[i] tokens (lens null: none).  An entry is taken out of
// the table by one thread, whoever else is at it.
__global__ void __launch_bounds__(256) pages_free_kernel(PagesArgs p) {
  const int row = p.src[blockIdx.y];
  if ((unsigned)row >= (unsigned)p.batch || (p.lens && !p.done[blockIdx.y])) return;
  const int len = p.lens ? max(p.lens[blockIdx.y], 0) : 0;
  const int keep = (int)(((long)len + PAGE - 1) / PAGE);
  for (int e = keep + blockIdx.x * 256 + threadIdx.x; e < p.max_blocks; e += gridDim.x * 256) {
    int* entry = p.tables + (long)row * p.max_blocks + e;
    if (*entry == -1) continue;
    const int block = atomicExch(entry, -1);
    if (in_pool(block, p.num_blocks)) atomicSub(p.refs + block, 1);
  }
}

// ------------------------------------------------------------------ the pool's used blocks to its front
// Of `live` used blocks those at live and above move to the free ones below it, in order: from[i] to to[i].  place[b]: -1
// where block b is free, b where it stays, -2 - i where it is move i.
template <int E> __global__ void __launch_bounds__(PLAN) pages_compact_kernel(PagesArgs p) {
  __shared__ int sm[PLAN / 64];
  int used = 0;
  unsigned long long m[E];
  for (long base = 0; base < p.num_blocks; base += PLAN * E) {
    span_masks(p.refs, p.num_blocks, (int)base, m, [](int n) { return n > 0; });
    used += mask_count(m);
  }
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = used;
  __syncthreads();
  int live = 0;
#pragma unroll
  for (int w = 0; w < PLAN / 64; ++w) live += sm[w];
  int holes = 0, movers = 0;
  for (long base = 0; base < p.num_blocks; base += PLAN * E) {
    unsigned long long h[E], v[E];
    span_masks(p.refs, p.num_blocks, (int)base, m, [](int n) { return n > 0; });
    const int first = (int)base + (threadIdx.x >> 6) * (64 * E), lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      // of blocks first + 64 i ..: those below live, and those that there are
      const long below = (long)live - first - 64 * i, there = (long)p.num_blocks - first - 64 * i;
      const unsigned long long lo = below <= 0 ? 0 : below >= 64 ? ~0ull : (1ull << below) - 1;
      h[i] = ~m[i] & lo & (there <= 0 ? 0 : there >= 64 ? ~0ull : (1ull << there) - 1);
      v[i] = m[i] & ~lo;
      const int block = first + 64 * i + lane;
      if (block < p.num_blocks && !(v[i] >> lane & 1)) p.place[block] = m[i] >> lane & 1 ? block : -1;
    }
    if (base < live) holes = span_ranks(h, (int)base, holes, [&](int rank, int block) { p.to[rank] = block; });
    if (base + PLAN * E > live)
      movers = span_ranks(v, (int)base, movers, [&](int rank, int block) {
        p.from[rank] = block;
        p.place[block] = -2 - rank;
      });
  }
  if (threadIdx.x == 0) {
    *p.moves = movers;
    *p.live = live;
  }
}

// ------------------------------------------------------------------ blocks moved, in every layer
// Units (move, layer, K or V) are dealt to the workgroups; a lane has up to four 16-byte loads in flight.  Moves: from[i] to
// to[i]; either outside its pool: none.  Bound by HBM: 380 blocks of 28 layers in bf16, 697 MB read and written in 136 to 140
// us, 5.0 TB/s, a large copy's rate.
NOVA_DEV void copy_bytes(const char* from, char* to, long bytes) {
  const u32x4* f = reinterpret_cast<const u32x4*>(from);
  u32x4* t = reinterpret_cast<u32x4*>(to);
  const long n = bytes / 16;
  long i = threadIdx.x;
  for (; i + 3 * 256 < n; i += 4 * 256) {
    const u32x4 a = f[i], b = f[i + 256], c = f[i + 512], d = f[i + 768];
    t[i] = a, t[i + 256] = b, t[i + 512] = c, t[i + 768] = d;
  }
  for (; i < n; i += 256) t[i] = f[i];
}
NOVA_DEV void copy_unit(const CopyArgs& p, long unit) {
  const int side = unit & 1, layer = (unit >> 1) % p.layers;
  const long i = (unit >> 1) / p.layers;
  const int from = p.from[i], to = p.to[i];
  if (!in_pool(from, p.src.num_blocks) || !in_pool(to, p.dst.num_blocks)) return;
  const char* s = (const char*)(side ? p.src.v : p.src.k) + ((size_t)layer * p.src.num_blocks + from) * p.page;
  char* d = (char*)(side ? p.dst.v : p.dst.k) + ((size_t)layer * p.dst.num_blocks + to) * p.page;
  if (s == d) return;
  copy_bytes(s, d, p.page);
  if (!p.src.k_exp) return;
  const int n = p.src.n_kv * PAGE;
  copy_bytes((const char*)(side ? p.src.v_exp : p.src.k_exp) + ((size_t)layer * p.src.num_blocks + from) * n,
             (char*)(side ? p.dst.v_exp : p.dst.k_exp) + ((size_t)layer * p.dst.num_blocks + to) * n, n);
}
// A fork's pages, with its tables and counts: behind the workgroups that copy there is one for each request's row.  (One
// workgroup of the plan would add to 7000 counts of 32 branches of 3579 tokens in 12 us.)
__global__ void __launch_bounds__(256) fork_move_kernel(CopyArgs p, PagesArgs g, int copiers) {
  if (blockIdx.x >= (unsigned)copiers) {
    const int i = blockIdx.x - copiers;
    if (!g.done[i]) return;
    const int full = g.lens[i] / PAGE, to = g.to[i];
    const int* theirs = g.tables + (long)g.src[i] * g.max_blocks;
    int* mine = g.tables + (long)g.dst[i] * g.max_blocks;
    for (int e = threadIdx.x; e < g.max_blocks; e += 256) {
      const int block = e < full ? theirs[e] : e == full ? to : -1;
      mine[e] = block;
      if (e < full) atomicAdd(g.refs + block, 1);
    }
    if (threadIdx.x == 0 && to >= 0) atomicExch(g.refs + to, 1);
    return;
  }
  const long units = 2l * p.layers * p.n;
  for (long u = blockIdx.x; u < units; u += copiers) copy_unit(p, u);
}

__global__ void __launch_bounds__(256) copy_pages_kernel(CopyArgs p) {
  const long units = 2l * p.layers * p.n;
  for (long u = blockIdx.x; u < units; u += gridDim.x) copy_unit(p, u);
}

// A compaction's pages, with its tables and counts: the first workgroups take those.
__global__ void __launch_bounds__(256) compact_move_kernel(CopyArgs p, PagesArgs g) {
  const int moves = *p.moves;
  const long entries = (long)g.batch * g.max_blocks, stride = (long)gridDim.x * 256, t0 = (long)blockIdx.x * 256 + threadIdx.x;
  for (long i = t0; i < entries; i += stride) {
    const int block = g.tables[i], at = in_pool(block, g.num_blocks) ? g.place[block] : -1;
    g.tables_out[i] = at <= -2 ? p.to[-2 - at] : at;
  }
  for (long i = t0; i < moves; i += stride) {
    const int from = p.from[i], to = p.to[i], n = g.refs[from];
    g.refs_out[to] = n;
    g.refs_out[from] = 0;
  }
  const int live = *g.live;
  for (long b = t0; b < g.num_blocks; b += stride) {
    const int at = g.place[b];
    if (at == b) g.refs_out[b] = g.refs[b];
    else if (at == -1 && b >= live) g.refs_out[b] = 0;      // free before and after; the others are above
  }
  const long units = 2l * p.layers * moves;
  for (long u = blockIdx.x; u < units; u += gridDim.x) copy_unit(p, u);
}

// ------------------------------------------------------------------ accepted rows
// Workgroup: a KV head of a layer of a sequence.  Row path[i] of the sequence's rows becomes row i, for i below n_keep:
// what is read, K and V, is held in LDS until every read is done, so a path may have any order.  Bound by a chain of
// dependent loads (sequence and path, table, rows): 32 sequences with trees of 64 rows over 28 layers of 4 heads in
// 7.8 us (9.6 with all 64 rows in LDS).
constexpr int KEEP_ROWS = 16;              // rows in LDS: a workgroup of 64 would leave room for four on a compute unit
template <typename CT, int D>
__global__ void __launch_bounds__(128) kv_keep_kernel(KeepArgs p) {
  extern __shared__ __align__(16) char sm_raw[];
  CT* sm_k = reinterpret_cast<CT*>(sm_raw);                 // [KEEP_ROWS][D], K then V
  CT* sm_v = sm_k + KEEP_ROWS * D;
  __shared__ long sm_from[64], sm_to[64];                   // places of the rows that move: block * 16 + slot in the layer
  __shared__ int sm_moves;
  __shared__ uint8_t sm_exp[2][64];
  const int n_kv = p.c.n_kv, h = blockIdx.x % n_kv, layer = blockIdx.x / n_kv % p.layers, b = blockIdx.x / n_kv / p.layers;
  if (threadIdx.x < 64) {
    const int i = threadIdx.x;
    int j = p.path && i < p.r.max_rows ? p.path[(long)b * p.r.max_rows + i] : -1;
    const int n_keep = p.n_keep[b], ctx = p.r.ctx ? p.r.ctx[b] : 0;
    const SeqRows sr = seq_rows(p.r, b);
    const int kept = min(max(n_keep, 0), sr.n);
    if (p.ctx_out && h == 0 && layer == 0 && i == 0) p.ctx_out[b] = ctx + kept;
    // where tokens lie, -1 where there are none
    auto place = [&](int t) -> long {
      if (t < 0 || t >= p.r.max_ctx) return -1;
      const int ph = page_of(p.r, p.c.num_blocks, b, t / PAGE);
      return ph < 0 ? -1 : (long)ph * PAGE + t % PAGE;
    };
    bool moves = i < kept && (unsigned)j < (unsigned)sr.n && j != i;
    if (__ballot(moves)) {
      const long from = moves ? place(sr.ctx + j) : -1, to = moves ? place(sr.ctx + i) : -1;
      moves = from >= 0 && to >= 0;
      const unsigned long long m = __ballot(moves);
      if (moves) {
        const int at = __popcll(m & ((1ull << i) - 1));
        sm_from[at] = from, sm_to[at] = to;
      }
      if (i == 0) sm_moves = __popcll(m);
    } else if (i == 0) {
      sm_moves = 0;
    }
  }
  __syncthreads();
  const int n = sm_moves;
  if (n == 0) return;
  const size_t base = (size_t)layer * p.c.num_blocks;
  constexpr int WORDS = D * sizeof(CT) / 16;                // 16-byte words of a K row
  CT* kc = reinterpret_cast<CT*>(p.c.k);
  CT* vc = reinterpret_cast<CT*>(p.c.v);
  auto k_at = [&](long at, int w) { return reinterpret_cast<u32x4*>(kc + (((base + at / PAGE) * n_kv + h) * PAGE + at % PAGE) * D) + w; };
  auto v_at = [&](long at, int d) { return vc + (((base + at / PAGE) * n_kv + h) * D + d) * PAGE + at % PAGE; };
  auto exp_at = [&](int side, long at) { return (side ? p.c.v_exp : p.c.k_exp) + ((base + at / PAGE) * n_kv + h) * PAGE + at % PAGE; };
  // More rows than the LDS holds go by parts of their columns, which do not depend on one another.
  const int parts = n <= KEEP_ROWS ? 0 : n <= 2 * KEEP_ROWS ? 1 : 2;      // 2^parts of them
  const int words = WORDS >> parts, dims = D >> parts, wl = __builtin_ctz(words), dl = __builtin_ctz(dims);
  for (int part = 0; part < 1 << parts; ++part) {
    const int w0 = part * words, d0 = part * dims;
    if (part) __syncthreads();
    for (int i = threadIdx.x; i < n * words; i += 128) reinterpret_cast<u32x4*>(sm_k)[i] = *k_at(sm_from[i >> wl], w0 + (i & (words - 1)));
    for (int i = threadIdx.x; i < n * dims; i += 128) sm_v[i] = *v_at(sm_from[i >> dl], d0 + (i & (dims - 1)));
    if (sizeof(CT) == 1 && part == 0 && (int)threadIdx.x < 2 * n) sm_exp[threadIdx.x & 1][threadIdx.x >> 1] = *exp_at(threadIdx.x & 1, sm_from[threadIdx.x >> 1]);
    __syncthreads();
    for (int i = threadIdx.x; i < n * words; i += 128) *k_at(sm_to[i >> wl], w0 + (i & (words - 1))) = reinterpret_cast<const u32x4*>(sm_k)[i];
    for (int i = threadIdx.x; i < n * dims; i += 128) *v_at(sm_to[i >> dl], d0 + (i & (dims - 1))) = sm_v[i];
    if (sizeof(CT) == 1 && part == 0 && (int)threadIdx.x < 2 * n) *exp_at(threadIdx.x & 1, sm_to[threadIdx.x >> 1]) = sm_exp[threadIdx.x & 1][threadIdx.x >> 1];
  }
}

// ------------------------------------------------------------------ launch
// Blocks that a thread of a plan looks at at a time: more where the pool is large, so that its counts are on their way
// together; a small pool's few have their ends sooner (64 blocks compacted: 3 us with 1, 10 us with 16; 100000: 99 us
// with 16).
#define PLAN_LAUNCH(kernel)                                                                                            \
  do {                                                                                                                 \
    if (p.num_blocks <= PLAN) hipLaunchKernelGGL((kernel<1>), dim3(1), dim3(PLAN), 0, s, p);                          \
    else if (p.num_blocks <= 16 * PLAN) hipLaunchKernelGGL((kernel<4>), dim3(1), dim3(PLAN), 0, s, p);                \
    else hipLaunchKernelGGL((kernel<16>), dim3(1), dim3(PLAN), 0, s, p);                                               \
    return hipGetLastError();                                                                                          \
  } while (0)
hipError_t pages_extend(const PagesArgs& p, hipStream_t s) { PLAN_LAUNCH(pages_extend_kernel); }
hipError_t pages_fork(const PagesArgs& p, hipStream_t s) {
  if (p.batch > MAX_BATCH) return hipErrorInvalidValue;
  PLAN_LAUNCH(pages_fork_kernel);
}
hipError_t pages_compact(const PagesArgs& p, hipStream_t s) { PLAN_LAUNCH(pages_compact_kernel); }
hipError_t pages_free(const PagesArgs& p, hipStream_t s) {
  if (p.lens) {
    hipLaunchKernelGGL(pages_trim_kernel, dim3((p.n + 255) / 256), dim3(256), 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
  }
  const int x = std::min(64, (p.max_blocks + 255) / 256);
  hipLaunchKernelGGL(pages_free_kernel, dim3(x, p.n), dim3(256), 0, s, p);
  return hipGetLastError();
}
// Eight workgroups for each compute unit take the units in turn.
static unsigned copy_grid(long units, int cus) { return (unsigned)std::max(1l, std::min(units, 8l * cus)); }

hipError_t copy_pages(const CopyArgs& p, int cus, hipStream_t s) {
  if (p.n <= 0) return hipSuccess;
  hipLaunchKernelGGL(copy_pages_kernel, dim3(copy_grid(2l * p.layers * p.n, cus)), dim3(256), 0, s, p);
  return hipGetLastError();
}
hipError_t fork_move(const CopyArgs& p, const PagesArgs& g, int cus, hipStream_t s) {
  const int copiers = (int)copy_grid(2l * p.layers * p.n, cus);
  hipLaunchKernelGGL(fork_move_kernel, dim3(copiers + g.n), dim3(256), 0, s, p, g, copiers);
  return hipGetLastError();
}
hipError_t compact_move(const CopyArgs& p, const PagesArgs& g, int cus, hipStream_t s) {
  const long units = std::max(2l * p.layers * (g.num_blocks / 2), ((long)g.batch * g.max_blocks + 255) / 256);
  hipLaunchKernelGGL(compact_move_kernel, dim3(copy_grid(units, cus)), dim3(256), 0, s, p, g);
  return hipGetLastError();
}

template <typename CT> static hipError_t keep_launch(const KeepArgs& p, hipStream_t s) {
  const dim3 grid((unsigned)((long)p.r.batch * p.layers * p.c.n_kv));
  const size_t lds = (size_t)2 * KEEP_ROWS * p.c.D * sizeof(CT);
  if (p.c.D == 64) hipLaunchKernelGGL((kv_keep_kernel<CT, 64>), grid, dim3(128), lds, s, p);
  else hipLaunchKernelGGL((kv_keep_kernel<CT, 128>), grid, dim3(128), lds, s, p);
  return hipGetLastError();
}
hipError_t kv_keep(const KeepArgs& p, hipStream_t s) {
  if ((p.c.D != 64 && p.c.D != 128) || p.r.max_rows > 64) return hipErrorInvalidValue;
  switch (p.c.type) {
    case CACHE_BF16: return keep_launch<bf16_t>(p, s);
    case CACHE_F32: return keep_launch<float>(p, s);
    case CACHE_E4M3: return keep_launch<e4m3_t>(p, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace nova
