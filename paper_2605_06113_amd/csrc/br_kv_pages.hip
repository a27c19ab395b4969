// Blocks that several rows hold (include/br_kv.h): rows that take over others' (br_kv_fork), blocks that move to the lowest ids
// (br_kv_compact), and their keys and values (br_kv_copy).
#include "br_kv_device.h"

// Rows' entries are dealt to waves, `slices` to a row, 64 at a time in turns: f(row, its worker, the first entry of this lane).
template <class Fn>
__device__ __forceinline__ void br_kv_rows(const BrKvTables &t, int slices, Fn &&f) {
  const int lane = threadIdx.x & 63, rows = t.W * t.B;
  const long long all = (long long)rows * slices, step = (long long)gridDim.x * 4;
  for (long long at = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); at < all; at += step) {
    const int r = (int)(at / slices);
    f(r, r / t.B, (int)(at - (long long)r * slices) * 64 + lane);
  }
}

// What each row is to hold, beside the tables: its entries, and one holder more of each block that the row does not hold in that place.
__global__ __launch_bounds__(256) void br_kv_k_fork_take(BrKvTables t, BrKvNext x, const int *from, const int *len, int slices) {
  br_kv_rows(t, slices, [&](int r, int w, int first) {
    const int b1 = (1 << t.shift) - 1, f = from[r], held = br_kv_len(t, r);
    const bool forked = (unsigned)f < (unsigned)t.B;
    int n = -1;
    if (forked) {
      n = br_kv_len(t, w * t.B + f);
      const int cut = len ? len[r] : -1;
      if (cut >= 0) n = min(n, cut);
    }
    if (first == 0) x.lens[r] = make_int2(held, n);
    const long long at = (long long)r * t.max_blocks, src = ((long long)w * t.B + f) * t.max_blocks;
    const int blocks = (n + b1) >> t.shift, had = (held + b1) >> t.shift;
    if (!forked) return;
    for (int j = first; j < blocks; j += slices * 64) {
      const int id = t.table[src + j];
      x.table[at + j] = id;
      if ((unsigned)id < (unsigned)t.n_blocks && !(j < had && t.table[at + j] == id)) atomicAdd(&t.holders[(long long)w * t.n_blocks + id], 1);
    }
  });
}

// ... into the tables, and the blocks that stood there given back (behind br_kv_k_fork_take: none of them loses a holder that it is about to get).
__global__ __launch_bounds__(256) void br_kv_k_fork_put(BrKvTables t, BrKvNext x, int slices) {
  br_kv_rows(t, slices, [&](int r, int w, int first) {
    const int b1 = (1 << t.shift) - 1;
    const int2 n = x.lens[r];
    if (n.y < 0) return;
    const long long at = (long long)r * t.max_blocks;
    const int blocks = (n.y + b1) >> t.shift, had = (n.x + b1) >> t.shift;
    for (int j = first; j < max(blocks, had); j += slices * 64) {
      const int was = j < had ? t.table[at + j] : -1, id = j < blocks ? x.table[at + j] : -1;
      if (j == blocks - 1) t.tail[r] = id;
      if (was == id) continue;
      t.table[at + j] = id;
      if ((unsigned)was < (unsigned)t.n_blocks && atomicSub(&t.holders[(long long)w * t.n_blocks + was], 1) == 1)
        atomicAnd(&t.used[(long long)w * t.words + (was >> 5)], ~(1u << (was & 31)));
    }
    if (first == 0) {
      t.lens[r] = n.y;
      if (blocks == 0) t.tail[r] = -1;
    }
  });
}

// One block for each worker: which blocks go where, the used bits and the counts.  The used bits are in LDS.
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

// The tables' entries, by where the blocks have gone (behind br_kv_k_compact).
__global__ __launch_bounds__(256) void br_kv_k_compact_tables(BrKvTables t, BrKvNext x, int slices) {
  br_kv_rows(t, slices, [&](int r, int w, int first) {
    const int least = x.least[w], blocks = (br_kv_len(t, r) + (1 << t.shift) - 1) >> t.shift;
    const int *moved = x.moved + (long long)w * t.n_blocks;
    int *table = t.table + (long long)r * t.max_blocks;
    for (int j = first; j < blocks; j += slices * 64) {
      const int id = table[j];
      if (id < least || id >= t.n_blocks) continue;
      const int to = moved[id];
      table[j] = to;
      if (j == blocks - 1) t.tail[r] = to;
    }
  });
}

// A pair's codes of keys and values, `chunk` bytes of one of them to a block at a time, the scales with the first.
__global__ __launch_bounds__(256) void br_kv_k_copy(BrKvCache c, BrKvMoves m, int W, int chunk, int chunks) {
  const long long bytes = ((long long)c.heads * c.dim) << c.shift, units = (long long)W * m.n * 2 * chunks;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int pair = (int)(u / (2 * chunks)), part = (int)(u - (long long)pair * 2 * chunks), w = pair / m.n;
    const int from = m.src[pair], to = m.dst[pair], sw = m.src_worker ? m.src_worker[pair] : w;
    if ((unsigned)from >= (unsigned)c.n_blocks || (unsigned)to >= (unsigned)c.n_blocks || (unsigned)sw >= (unsigned)W) continue;
    const long long a = (long long)sw * c.n_blocks + from, b = (long long)w * c.n_blocks + to;
    unsigned char *codes = part < chunks ? c.k : c.v;
    const long long begin = (long long)(part < chunks ? part : part - chunks) * chunk, end = min(bytes, begin + chunk);
    const unsigned char *src = codes + a * bytes;
    unsigned char *dst = codes + b * bytes;
    for (long long i = begin + 16 * threadIdx.x; i < end; i += 256 * 16) *(uint4 *)(dst + i) = *(const uint4 *)(src + i);
    if (part == 0)
      for (int h = threadIdx.x; h < c.heads; h += 256) c.ks[b * c.heads + h] = c.ks[a * c.heads + h], c.vs[b * c.heads + h] = c.vs[a * c.heads + h];
  }
}

// Waves for a row: no more than its entries fill, and no more than fill the card when the rows do.
static int slices_for(const BrKvTables &t) {
  const long long rows = (long long)t.W * t.B, want = (8192 + rows - 1) / rows, most = (t.max_blocks + 63) / 64;
  return (int)(want < most ? want : most);
}

static unsigned blocks_for(const BrKvTables &t, int slices) {
  const long long blocks = ((long long)t.W * t.B * slices + 3) / 4;
  return (unsigned)(blocks < 1 << 20 ? blocks : 1 << 20);
}

void br_kv_launch_fork(const BrKvTables &t, const BrKvNext &x, const int *from, const int *len, hipStream_t st) {
  const int slices = slices_for(t);
  br_kv_k_fork_take<<<blocks_for(t, slices), 256, 0, st>>>(t, x, from, len, slices);
  br_kv_k_fork_put<<<blocks_for(t, slices), 256, 0, st>>>(t, x, slices);
}

void br_kv_launch_compact(const BrKvTables &t, const BrKvNext &x, const BrKvMoves &m, hipStream_t st) {
  const int slices = slices_for(t);
  br_kv_k_compact<256><<<t.W, 256, (size_t)t.words * 4, st>>>(t, x, m);
  br_kv_k_compact_tables<<<blocks_for(t, slices), 256, 0, st>>>(t, x, slices);
}

void br_kv_launch_copy(const BrKvCache &c, const BrKvMoves &m, int W, hipStream_t st) {
  const long long bytes = ((long long)c.heads * c.dim) << c.shift;
  const int chunk = 16384, chunks = (int)((bytes + chunk - 1) / chunk);
  const long long units = (long long)W * m.n * 2 * chunks;
  br_kv_k_copy<<<(unsigned)(units < 4096 ? units : 4096), 256, 0, st>>>(c, m, W, chunk, chunks);
}
