// Blocks that several rows hold (include/br_kv.h): rows that take over others' (br_kv_fork), blocks that move to the lowest ids
// (br_kv_compact), and their keys and values (br_kv_copy).
#include "br_kv_device.h"

// Rows' entries are dealt to parts of waves, G lanes each, `slices` of them to a row, G entries at a time in turns: f(row, its worker, the
// first entry of this lane).
template <int G, class Fn>
__device__ __forceinline__ void br_kv_rows(const BrKvTables &t, int slices, Fn &&f) {
  const int lane = threadIdx.x & (G - 1), rows = t.W * t.B;
  const long long all = (long long)rows * slices, step = (long long)gridDim.x * (256 / G);
  for (long long at = (long long)blockIdx.x * (256 / G) + threadIdx.x / G; at < all; at += step) {
    const int r = (int)(at / slices);
    f(r, r / t.B, (int)(at - (long long)r * slices) * G + lane);
  }
}

// What row r of worker w becomes: tokens, -1 where it stays as it is; f: whose.
__device__ __forceinline__ int br_kv_forked(const BrKvTables &t, int w, int r, int f, const int *len) {
  if ((unsigned)f >= (unsigned)t.B) return -1;
  const int n = br_kv_len(t, w * t.B + f), cut = len ? len[r] : -1;
  return cut >= 0 ? min(n, cut) : n;
}

// Four entries of a row, j, j + step, ..., below `blocks`: asked for, all before any is acted on; then what is to come (-> x.table), counted, bit k of the
// result: entry k changes.
struct BrKvFour {
  int id[4], was[4];
  __device__ __forceinline__ void ask(const BrKvTables &t, int r, long long src, int j, int step, int blocks) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = min(j + k * step, blocks - 1);
      id[k] = t.table[src + e], was[k] = t.table[(long long)r * t.max_blocks + e];
    }
  }
  __device__ __forceinline__ unsigned take(const BrKvTables &t, const BrKvNext &x, int w, int r, int j, int step, int had, int blocks) const {
    unsigned changes = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = j + k * step;
      if (e == blocks - 1) t.tail[r] = id[k];
      if (e >= blocks || (e < had && was[k] == id[k])) continue;
      changes |= 1u << k;
      x.table[(long long)r * t.max_blocks + e] = id[k];
      if ((unsigned)id[k] < (unsigned)t.n_blocks) atomicAdd(&t.holders[(long long)w * t.n_blocks + id[k]], 1);
    }
    return changes;
  }
};

// ... those of them that change into the table, and the blocks that stood there given back.
__device__ __forceinline__ void br_kv_put4(const BrKvTables &t, const BrKvNext &x, int w, int r, int j, int step, int had, int blocks, int end, unsigned changes) {
  const long long at = (long long)r * t.max_blocks;
  int stood[4], next[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int e = min(j + k * step, end - 1);
    stood[k] = t.table[at + e], next[k] = x.table[at + e];  // (both are memory, whatever they hold)
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int e = j + k * step;
    if (e >= end || !(changes >> k & 1) || (e < blocks && next[k] == INT32_MIN)) continue;
    t.table[at + e] = e < blocks ? next[k] : -1;
    const int was = e < had ? stood[k] : -1;
    if ((unsigned)was < (unsigned)t.n_blocks && atomicSub(&t.holders[(long long)w * t.n_blocks + was], 1) == 1)
      atomicAnd(&t.used[(long long)w * t.words + (was >> 5)], ~(1u << (was & 31)));
  }
}

// What each row is to hold, beside the tables: its entries, and one holder more of each block that the row does not hold in that place.  Bound by a launch and its
// chain (lengths and whose, entries, counts), 80 % waiting: one worker of 96 rows, up to 250 entries each, 3.6 us, and 3.4 for the second half below.
template <int G>
__global__ __launch_bounds__(256) void br_kv_k_fork_take(BrKvTables t, BrKvNext x, const int *from, const int *len, int slices) {
  br_kv_rows<G>(t, slices, [&](int r, int w, int first) {
    const int b1 = (1 << t.shift) - 1, f = from[r], held = br_kv_len(t, r), n = br_kv_forked(t, w, r, f, len);
    if (first == 0) x.lens[r] = make_int2(held, n);
    const long long src = ((long long)w * t.B + f) * t.max_blocks;
    const int blocks = (n + b1) >> t.shift, had = (held + b1) >> t.shift;
    const int step = slices * G;
    for (int j = first; j < blocks; j += 4 * step) {
      BrKvFour four;
      four.ask(t, r, src, j, step, blocks);
      const unsigned changes = four.take(t, x, w, r, j, step, had, blocks);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (!(changes >> k & 1) && j + k * step < blocks) x.table[(long long)r * t.max_blocks + j + k * step] = INT32_MIN;  // (no block's id: stays)
    }
  });
}

// ... into the tables, and the blocks that stood there given back (behind br_kv_k_fork_take: none of them loses a holder that it is about to get).
template <int G>
__global__ __launch_bounds__(256) void br_kv_k_fork_put(BrKvTables t, BrKvNext x, int slices) {
  br_kv_rows<G>(t, slices, [&](int r, int w, int first) {
    const int b1 = (1 << t.shift) - 1;
    const int2 n = x.lens[r];
    if (n.y < 0) return;
    const int blocks = (n.y + b1) >> t.shift, had = (n.x + b1) >> t.shift;
    for (int j = first; j < max(blocks, had); j += 4 * slices * G) br_kv_put4(t, x, w, r, j, slices * G, had, blocks, max(blocks, had), 15u);
    if (first == 0) {
      t.lens[r] = n.y;
      if (blocks == 0) t.tail[r] = -1;
    }
  });
  if (blockIdx.x == 0 && threadIdx.x == 0) *t.planned = 0;
}

// Bound by the way to memory: 512 workers of 144 rows, up to 133 entries each, a tenth of which change, 21.4 us, 58 MB of lines of own and others' rows (2.7 TB/s), a
// launch and four dependent trips.  The next four entries on their way beside these ones' work did not change that.
// Both for one worker by one block, 16 lanes to a row: no row's entries are written before all have been read.  A lane notes which of its first 60 entries
// change: rows of one family differ in a few, and the others are not looked at again.
template <int NT>
__global__ __launch_bounds__(NT) void br_kv_k_fork(BrKvTables t, BrKvNext x, const int *from, const int *len) {
  constexpr int G = 16, ROWS = NT / G;
  __shared__ int2 lens[BR_KV_MAX_ROWS];
  __shared__ int whose[BR_KV_MAX_ROWS];
  const int w = blockIdx.x, B = t.B, b1 = (1 << t.shift) - 1, lane = threadIdx.x & (G - 1), row0 = w * B;
  for (int r = threadIdx.x; r < B; r += NT) {
    const int f = from[row0 + r];
    whose[r] = f;
    lens[r] = make_int2(br_kv_len(t, row0 + r), br_kv_forked(t, w, row0 + r, f, len));
  }
  __syncthreads();
  unsigned long long changes = 0;
  int i = 0;
  for (int r = threadIdx.x / G; r < B; r += ROWS) {
    const int2 n = lens[r];  // (a row that stays has -1 tokens here: no blocks)
    const int blocks = (n.y + b1) >> t.shift, had = (n.x + b1) >> t.shift;
    const long long src = (long long)(row0 + whose[r]) * t.max_blocks;
    for (int j = lane; j < blocks; j += 4 * G, i += 4) {
      BrKvFour four;
      four.ask(t, row0 + r, src, j, G, blocks);
      const unsigned some = four.take(t, x, w, row0 + r, j, G, had, blocks);
      if (i < 60) {
        changes |= (unsigned long long)some << i;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (!(some >> k & 1) && j + k * G < blocks) x.table[(long long)(row0 + r) * t.max_blocks + j + k * G] = INT32_MIN;  // (no block's id: stays)
      }
    }
  }
  __syncthreads();
  i = 0;
  for (int r = threadIdx.x / G; r < B; r += ROWS) {
    const int2 n = lens[r];
    if (n.y < 0) continue;
    const int blocks = (n.y + b1) >> t.shift, had = (n.x + b1) >> t.shift;
    for (int j = lane; j < blocks; j += 4 * G, i += 4) {
      const unsigned four = i < 60 ? (unsigned)(changes >> i) & 15u : 15u;
      if (four) br_kv_put4(t, x, w, row0 + r, j, G, had, blocks, blocks, four);
    }
    for (int j = blocks + lane; j < had; j += 4 * G) br_kv_put4(t, x, w, row0 + r, j, G, had, blocks, had, 15u);
    if (lane == 0) {
      t.lens[row0 + r] = n.y;
      if (blocks == 0) t.tail[row0 + r] = -1;
    }
  }
  if (w == 0 && threadIdx.x == 0) *t.planned = 0;
}

// One block for each worker: which blocks go where, the used bits and the counts.  The used bits are in LDS.  Bound by four scans and the trips between them,
// not by what they move: one worker of 96 rows and 3916 blocks, 856 of which move, 11.0 us, 2.8 if none does; 300 of 31 rows, 56 moves each, 12.1; 83 to 87 % of the
// time waiting.
template <int NT>
__global__ __launch_bounds__(NT) void br_kv_k_compact(BrKvTables t, BrKvNext x, BrKvMoves m) {
  extern __shared__ unsigned used[];
  __shared__ int part[16 * (NT / 64)], least;
  const int w = blockIdx.x, tid = threadIdx.x;
  int turn = 0;
  unsigned *gused = t.used + (long long)w * t.words;
  int *moved = x.moved + (long long)w * t.n_blocks, *holders = t.holders + (long long)w * t.n_blocks;
  int n[1] = {0}, all[1];
  for (int i = tid; i < t.words; i += NT) used[i] = gused[i], n[0] += __popc(used[i]);
  if (tid == 0) least = INT32_MAX;
  br_kv_scan<NT, 1>(n, all, part, turn);
  const int u = all[0];  // ids from u on are to be left
  auto above = [&](int i) { return 32 * i >= u ? ~0u : 32 * i + 32 <= u ? 0u : ~0u << (u & 31); };
  n[0] = 0;
  for (int i = tid; i < t.words; i += NT) n[0] += __popc(used[i] & above(i));
  br_kv_scan<NT, 1>(n, all, part, turn);
  const int moves = all[0], done = min(moves, m.n);  // (as many free ids below u as used ones from there on)
  // free ids below u, in moved[k] for the k-th move: that is below u, where no block that moves has its place there
  int before = 0;
  for (int i0 = 0; i0 < t.words && 32 * i0 < u; i0 += NT) {
    const int i = i0 + tid;
    unsigned bits = i < t.words ? ~used[i] & ~above(i) : 0u;
    n[0] = __popc(bits);
    const int mine = n[0];
    br_kv_scan<NT, 1>(n, all, part, turn);
    int k = before + n[0] - mine;
    for (; bits && k < done; bits &= bits - 1, ++k) moved[k] = 32 * i + __ffs(bits) - 1;
    before += all[0];
  }
  __syncthreads();
  before = 0;
  for (int i0 = u / 32; i0 < t.words; i0 += NT) {
    const int i = i0 + tid;
    unsigned bits = i < t.words ? used[i] & above(i) : 0u;
    n[0] = __popc(bits);
    const int mine = n[0];
    br_kv_scan<NT, 1>(n, all, part, turn);
    int k = moves - 1 - (before + n[0] - mine);  // the highest is move 0
    for (; bits; bits &= bits - 1, --k) {
      if (k >= done) continue;
      const int id = 32 * i + __ffs(bits) - 1, to = moved[k];
      moved[id] = to;
      holders[to] = holders[id], holders[id] = 0;
      atomicAnd(&used[i], ~(bits & -bits));
      atomicOr(&used[to >> 5], 1u << (to & 31));
      m.src[(long long)w * m.n + k] = id, m.dst[(long long)w * m.n + k] = to;
      if (k == done - 1) least = id;
    }
    before += all[0];
  }
  for (int k = done + tid; k < m.n; k += NT) m.src[(long long)w * m.n + k] = m.dst[(long long)w * m.n + k] = -1;
  __syncthreads();
  if (tid == 0) x.least[w] = least;
  if (done > 0)
    for (int i = tid; i < t.words; i += NT) gused[i] = used[i];
}

// The tables' entries, by where the blocks have gone (behind br_kv_k_compact): three dependent trips, 4.4 us of one worker, 5.2 of 300 of 31 rows.
template <int G>
__global__ __launch_bounds__(256) void br_kv_k_compact_tables(BrKvTables t, BrKvNext x, int slices) {
  br_kv_rows<G>(t, slices, [&](int r, int w, int first) {
    const int least = x.least[w], blocks = (br_kv_len(t, r) + (1 << t.shift) - 1) >> t.shift;
    const int *moved = x.moved + (long long)w * t.n_blocks;
    int *table = t.table + (long long)r * t.max_blocks;
    const int step = slices * G;
    for (int j = first; j < blocks; j += 4 * step) {
      int id[4], to[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) id[k] = table[min(j + k * step, blocks - 1)];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        to[k] = -1;
        if (j + k * step < blocks && id[k] >= least && id[k] < t.n_blocks) to[k] = moved[id[k]];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (to[k] < 0) continue;
        table[j + k * step] = to[k];
        if (j + k * step == blocks - 1) t.tail[r] = to[k];
      }
    }
  });
}

// Large blocks: a block of threads has one piece of a pair's keys or values, all of it on its way at once; the scales go with the first.  Bound by memory: requests
// of 64 KB a block, 1.39 GB read and written, 278 us = 5.0 TB/s (a large copy 5.1); 856 such blocks out of 3916 places, 225 MB, 54 us = 4.2.  A place that is no
// pair costs its turns all the same, each a wait for src and dst: 73728 of them 59 us (blocks of 16 KB), 113 (64 KB).
template <int AT_ONCE>
__global__ __launch_bounds__(256) void br_kv_k_copy(BrKvCache c, BrKvMoves m, int W, int chunks, long long units) {
  constexpr int CHUNK = AT_ONCE * 256 * 16;
  typedef unsigned u4 __attribute__((ext_vector_type(4)));
  const long long bytes = ((long long)c.heads * c.dim) << c.shift;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int pair = (int)(u / (2 * chunks)), part = (int)(u - (long long)pair * 2 * chunks), w = pair / m.n;
    const int from = m.src[pair], to = m.dst[pair], sw = m.src_worker ? m.src_worker[pair] : w;
    if ((unsigned)from >= (unsigned)c.n_blocks || (unsigned)to >= (unsigned)c.n_blocks || (unsigned)sw >= (unsigned)W) continue;
    const long long a = (long long)sw * c.n_blocks + from, b = (long long)w * c.n_blocks + to;
    unsigned char *codes = part < chunks ? c.k : c.v;
    const long long in = (long long)(part < chunks ? part : part - chunks) * CHUNK + 16 * threadIdx.x;
    const unsigned char *src = codes + a * bytes + in;
    unsigned char *dst = codes + b * bytes + in;
    u4 x[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k)
      if (in + k * 4096 < bytes) x[k] = *(const u4 *)(src + k * 4096);
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k)
      if (in + k * 4096 < bytes) *(u4 *)(dst + k * 4096) = x[k];
    if (part == 0)
      for (int h = threadIdx.x; h < c.heads; h += 256) c.ks[b * c.heads + h] = c.ks[a * c.heads + h], c.vs[b * c.heads + h] = c.vs[a * c.heads + h];
  }
}

// Pairs' codes in pieces of 1 KB, 16 bytes a lane: a block's keys, its values, then its scales as one piece.  A wave has eight pieces on their way at once.  Bound by
// what a wave does before them, a division and three dependent loads for each piece: 16800 pairs, 69 MB, 26.9 us = 2.6 TB/s, 71 % of the time waiting; 73728 places
// without a pair 28.
__global__ __launch_bounds__(256) void br_kv_k_copy_small(BrKvCache c, BrKvMoves m, int W, int half, long long batches) {
  constexpr int AT_ONCE = 8;
  typedef unsigned u4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63, pieces = 2 * half + 1;
  const long long bytes = ((long long)c.heads * c.dim) << c.shift, pairs = (long long)W * m.n;
  for (long long at = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); at < batches; at += (long long)gridDim.x * 4) {
    long long pair = at * AT_ONCE / pieces;
    int piece = (int)(at * AT_ONCE - pair * pieces);
    long long src[AT_ONCE], dst[AT_ONCE];  // blocks; dst -1: none
    int of[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      dst[k] = -1, of[k] = piece;
      if (pair < pairs) {
        const int p = (int)pair, w = p / m.n, from = m.src[p], to = m.dst[p], sw = m.src_worker ? m.src_worker[p] : w;
        if ((unsigned)from < (unsigned)c.n_blocks && (unsigned)to < (unsigned)c.n_blocks && (unsigned)sw < (unsigned)W)
          src[k] = (long long)sw * c.n_blocks + from, dst[k] = (long long)w * c.n_blocks + to;
      }
      if (++piece == pieces) piece = 0, ++pair;
    }
    u4 x[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const long long in = (long long)(of[k] < half ? of[k] : of[k] - half) * 1024 + 16 * lane;
      if (dst[k] >= 0 && of[k] < 2 * half && in < bytes) x[k] = *(const u4 *)((of[k] < half ? c.k : c.v) + src[k] * bytes + in);
    }
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const long long in = (long long)(of[k] < half ? of[k] : of[k] - half) * 1024 + 16 * lane;
      if (dst[k] >= 0 && of[k] < 2 * half && in < bytes) *(u4 *)((of[k] < half ? c.k : c.v) + dst[k] * bytes + in) = x[k];
    }
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      if (dst[k] < 0 || of[k] != 2 * half) continue;
      for (int h = lane; h < c.heads; h += 64) c.ks[dst[k] * c.heads + h] = c.ks[src[k] * c.heads + h], c.vs[dst[k] * c.heads + h] = c.vs[src[k] * c.heads + h];
    }
  }
}

// Lanes and waves for a row: no more than its entries fill, and no more than fill the card when the rows do.
struct BrKvGrid {
  int lanes, slices;
  unsigned blocks;
  explicit BrKvGrid(const BrKvTables &t) {
    const long long rows = (long long)t.W * t.B;
    lanes = rows >= 32768 || t.max_blocks <= 16 ? 16 : 64;
    const long long want = (8192 + rows - 1) / rows, most = (t.max_blocks + lanes - 1) / lanes;
    slices = (int)(want < most ? want : most);
    const long long n = (rows * slices * lanes + 255) / 256;
    blocks = (unsigned)(n < 1 << 20 ? n : 1 << 20);
  }
};

void br_kv_launch_fork(const BrKvTables &t, const BrKvNext &x, const int *from, const int *len, hipStream_t st) {
  // A block for a worker goes over its rows' entries in rounds of some 1.2 us; two launches spread one worker over the card.  64 rows of up to 2048 tokens in
  // blocks of 64: one worker 5.1 us and 9.7, 512 of them 9.9 and 14.9; 256 rows of up to 8192: 14.4 and 8.4, 256 workers 20 and 29; 64 rows
  // of up to 16384 tokens in blocks of 16, 128 workers 27 and 17, 300 of them 16 and 45.  Workers of a few rows fill no blocks: 16384 of 4 rows 29 and 18.
  const long long rounds = (long long)((t.B + 63) / 64) * ((t.max_blocks + 63) / 64);
  if ((rounds <= 2 && t.W <= 4096) || (rounds <= 16 && t.W >= 256 && t.B > 32)) {
    if (t.B <= 16) br_kv_k_fork<256><<<t.W, 256, 0, st>>>(t, x, from, len);
    else if (t.B <= 32) br_kv_k_fork<512><<<t.W, 512, 0, st>>>(t, x, from, len);
    else br_kv_k_fork<1024><<<t.W, 1024, 0, st>>>(t, x, from, len);
    return;
  }
  const BrKvGrid g(t);
  if (g.lanes == 16) {
    br_kv_k_fork_take<16><<<g.blocks, 256, 0, st>>>(t, x, from, len, g.slices);
    br_kv_k_fork_put<16><<<g.blocks, 256, 0, st>>>(t, x, g.slices);
  } else {
    br_kv_k_fork_take<64><<<g.blocks, 256, 0, st>>>(t, x, from, len, g.slices);
    br_kv_k_fork_put<64><<<g.blocks, 256, 0, st>>>(t, x, g.slices);
  }
}

void br_kv_launch_compact(const BrKvTables &t, const BrKvNext &x, const BrKvMoves &m, hipStream_t st) {
  const BrKvGrid g(t);
  br_kv_k_compact<256><<<t.W, 256, (size_t)t.words * 4, st>>>(t, x, m);
  if (g.lanes == 16) br_kv_k_compact_tables<16><<<g.blocks, 256, 0, st>>>(t, x, g.slices);
  else br_kv_k_compact_tables<64><<<g.blocks, 256, 0, st>>>(t, x, g.slices);
}

template <int AT_ONCE>
static void launch_copy(const BrKvCache &c, const BrKvMoves &m, int W, long long bytes, hipStream_t st) {
  const int chunk = AT_ONCE * 4096, chunks = (int)((bytes + chunk - 1) / chunk);
  const long long units = (long long)W * m.n * 2 * chunks;
  // (more blocks than are on the card at once: 16384 for requests of 64 KB a block 278 us, 4096 289; lists that are mostly empty are passed
  // over faster by fewer, 3916 places with 1000 pairs 51 and 48)
  br_kv_k_copy<AT_ONCE><<<(unsigned)(units < 16384 ? units : 16384), 256, 0, st>>>(c, m, W, chunks, units);
}

void br_kv_launch_copy(const BrKvCache &c, const BrKvMoves &m, int W, hipStream_t st) {
  const long long bytes = ((long long)c.heads * c.dim) << c.shift, pairs = (long long)W * m.n;
  // Many small blocks: 4882 pairs of 2 KB 11.7 us, by the other kernel 13.5, 9765 of 1 KB 13.3 and 23.6; but 96 of them 6.8 and 5.3.
  if (bytes <= 2048 && pairs >= 2048) {
    const int half = (int)((bytes + 1023) / 1024);
    const long long batches = (pairs * (2 * half + 1) + 7) / 8, blocks = (batches + 3) / 4;
    br_kv_k_copy_small<<<(unsigned)(blocks < 2048 ? blocks : 2048), 256, 0, st>>>(c, m, W, half, batches);
  } else if (bytes <= 16384) {
    launch_copy<4>(c, m, W, bytes, st);
  } else {
    launch_copy<8>(c, m, W, bytes, st);
  }
}
