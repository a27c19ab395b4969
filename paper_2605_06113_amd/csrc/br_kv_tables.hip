// Block tables and slot maps of a step (br_kv_step), and the kernels that set a context up.
#include "br_kv_device.h"

// Every row empty, every block free; nothing begun.
__global__ __launch_bounds__(256) void br_kv_k_clear(BrKvTables t, int *arrived) {
  const long long n = (long long)t.W * t.B * t.max_blocks, rows = (long long)t.W * t.B, words = (long long)t.W * t.words;
  const long long step = (long long)gridDim.x * 256;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    t.table[i] = -1;
    if (i < rows) t.lens[i] = 0;
  }
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < words; i += step) t.used[i] = 0;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < BR_KV_SPLIT_WGS; i += step) arrived[i] = 0;
}

// The rows held at the start (behind br_kv_k_clear).
__global__ __launch_bounds__(256) void br_kv_k_load(BrKvTables t, const int *lens, const int *table) {
  const long long n = (long long)t.W * t.B * t.max_blocks, step = (long long)gridDim.x * 256;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    const long long row = i / t.max_blocks;
    const int j = (int)(i - row * t.max_blocks);
    const int len = min(max(lens[row], 0), t.max_blocks << t.shift);
    if (j == 0) t.lens[row] = len;
    if (j >= (len + (1 << t.shift) - 1) >> t.shift) continue;
    const int id = table[i];
    if (id < 0 || id >= t.n_blocks) continue;
    t.table[i] = id;
    atomicOr(&t.used[row / t.B * t.words + (id >> 5)], 1u << (id & 31));
  }
}

// Inclusive sum over the block's threads; *total: all of them.
template <int NT>
__device__ __forceinline__ int br_kv_scan(int x, int *part, int *total) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(x, d, 64);
    if (lane >= d) x += o;
  }
  __syncthreads();
  if (lane == 63) part[wv] = x;
  __syncthreads();
  int all = 0;
  for (int k = 0; k < NT / 64; ++k) {
    if (k < wv) x += part[k];
    all += part[k];
  }
  *total = all;
  return x;
}

// Largest r in [0, n) with before[r] <= k (before ascending, before[0] = 0).
__device__ __forceinline__ int br_kv_find(const int *before, int n, int k) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (before[mid] <= k) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// One block of NT threads per worker; a thread has the RPT rows from tid * RPT on.  The used bits are in LDS.
template <int NT, int RPT>
__global__ __launch_bounds__(NT) void br_kv_k_step(BrKvTables t, BrKvStep s) {
  extern __shared__ unsigned used[];
  __shared__ int part[NT / 64], give_n, need_before[NT * RPT], tok_before[NT * RPT], row_kp[NT * RPT], give[NT * RPT], ids[NT * 32];
  const int w = blockIdx.x, tid = threadIdx.x, lane = tid & 63, B = t.B, b1 = (1 << t.shift) - 1;
  int *lens = t.lens + (long long)w * B;
  int *table = t.table + (long long)w * B * t.max_blocks;
  unsigned *gused = t.used + (long long)w * t.words;
  if (tid == 0) give_n = 0;
  for (int i = tid; i < t.words; i += NT) used[i] = gused[i];
  __syncthreads();

  int kp[RPT], have[RPT], why[RPT], held[RPT];
  long long want[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i;
    kp[i] = have[i] = why[i] = held[i] = 0, want[i] = 0;
    if (r < B) {
      const int len = lens[r], keep = s.keep[(long long)w * B + r], add = s.add[(long long)w * B + r];
      kp[i] = keep < 0 ? len : min(keep, len);
      want[i] = max(add, 0);
      have[i] = (kp[i] + b1) >> t.shift;
      held[i] = (len + b1) >> t.shift;
      if (held[i] > have[i]) give[atomicAdd(&give_n, 1)] = r;
      if (want[i] > 0 && (kp[i] + want[i] + b1) >> t.shift > t.max_blocks) why[i] = BR_KV_TOO_LONG, want[i] = 0;
      need_before[r] = have[i], tok_before[r] = held[i];
    }
  }
  __syncthreads();
  // blocks given back: a wave per row, in any order
  for (int k = tid >> 6; k < give_n; k += NT / 64) {
    const int r = give[k], from = need_before[r], to = tok_before[r];
    for (int j = from + lane; j < to; j += 64) {
      const int id = table[(long long)r * t.max_blocks + j];
      if (id >= 0) atomicAnd(&used[id >> 5], ~(1u << (id & 31)));
      table[(long long)r * t.max_blocks + j] = -1;
    }
  }
  // tokens that find room in the list
  int x = 0, total = 0;
  long long sum = 0;
#pragma unroll
  for (int i = 0; i < RPT; ++i) sum += want[i];
  x = br_kv_scan<NT>((int)sum, part, &total);
  int run = x - (int)sum;
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    run += (int)want[i];
    if (want[i] > 0 && run > s.cap) why[i] = BR_KV_NO_ROOM, want[i] = 0;
  }
  // (the scans' barriers stand between the blocks given back and here)
  int nfree = 0;
  for (int i = tid; i < t.words; i += NT) nfree += 32 - __popc(used[i]);
  br_kv_scan<NT>(nfree, part, &nfree);
  nfree -= t.words * 32 - t.n_blocks;
  int need[RPT], needs = 0, need_all;
#pragma unroll
  for (int i = 0; i < RPT; ++i) need[i] = (int)((kp[i] + want[i] + b1) >> t.shift) - have[i], needs += need[i];
  x = br_kv_scan<NT>(needs, part, &need_all);
  run = x - needs;
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    run += need[i];
    if (need[i] > 0 && run > nfree) why[i] = BR_KV_NO_BLOCKS, want[i] = 0, need[i] = 0;
  }
  int toks = 0;
  needs = 0;
#pragma unroll
  for (int i = 0; i < RPT; ++i) toks += (int)want[i], needs += need[i];
  x = br_kv_scan<NT>(needs, part, &need_all) - needs;
  int y = br_kv_scan<NT>(toks, part, &total) - toks;
  int sums[5] = {0, 0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i;
    need_before[r] = x, tok_before[r] = y, row_kp[r] = kp[i];
    const int len = kp[i] + (int)want[i];
    if (r < B) {
      const long long at = (long long)w * B + r;
      lens[r] = len;
      if (s.start) s.start[at] = w * s.cap + y;
      if (s.count) s.count[at] = (int)want[i];
      if (s.status) s.status[at] = why[i];
      sums[0] += len, sums[1] += len > 0, sums[2] += why[i] > 0, sums[3] += why[i] == BR_KV_NO_BLOCKS;
    }
    x += need[i], y += (int)want[i];
  }
  // blocks taken, lowest ids first
  int taken = 0;
  for (int i0 = 0; taken < need_all && i0 < t.words; i0 += NT) {
    const int i = i0 + tid;
    unsigned bits = i < t.words ? ~used[i] : 0u;
    if (i == t.words - 1 && (t.n_blocks & 31)) bits &= (1u << (t.n_blocks & 31)) - 1;
    int here;
    int k = br_kv_scan<NT>(__popc(bits), part, &here) - __popc(bits);
    unsigned got = 0;
    for (; bits && taken + k < need_all; ++k, bits &= bits - 1) {
      ids[k] = 32 * i + __ffs(bits) - 1;
      got |= bits & -bits;
    }
    if (got) used[i] |= got;
    __syncthreads();
    here = min(here, need_all - taken);
    for (int j = tid; j < here; j += NT) {
      const int r = br_kv_find(need_before, NT * RPT, taken + j);
      const int first = (row_kp[r] + b1) >> t.shift;
      table[(long long)r * t.max_blocks + first + taken + j - need_before[r]] = ids[j];
    }
    taken += here;
  }
  __syncthreads();
  for (int i = tid; i < t.words; i += NT) gused[i] = used[i];
  if (s.slot || s.pos) {
    for (int j = tid; j < s.cap; j += NT) {
      int pos = -1, slot = -1;
      if (j < total) {
        const int r = br_kv_find(tok_before, NT * RPT, j);
        pos = row_kp[r] + j - tok_before[r];
        const int id = table[(long long)r * t.max_blocks + (pos >> t.shift)];
        slot = id < 0 ? -1 : (id << t.shift) + (pos & b1);
      }
      if (s.slot) s.slot[(long long)w * s.cap + j] = slot;
      if (s.pos) s.pos[(long long)w * s.cap + j] = pos;
    }
  }
  if (s.stats) {
    int n_used = 0;
    for (int i = tid; i < t.words; i += NT) n_used += __popc(used[i]);
    int all[5];
    sums[4] = n_used;
#pragma unroll
    for (int k = 0; k < 5; ++k) br_kv_scan<NT>(sums[k], part, &all[k]);
    if (tid == 0) {
      long long *o = s.stats + (long long)w * BR_KV_NSTATS;
      o[BR_KV_ST_TOKENS] = all[0], o[BR_KV_ST_USED] = all[4], o[BR_KV_ST_FREE] = t.n_blocks - all[4], o[BR_KV_ST_ROWS] = all[1];
      o[BR_KV_ST_ADDED] = total, o[BR_KV_ST_REFUSED] = all[2], o[BR_KV_ST_NO_BLOCKS] = all[3], o[BR_KV_ST_TAKEN] = need_all;
    }
  }
}

static int grid_for(long long n) { return (int)(n < 1 ? 1 : n > 4096ll * 256 ? 4096 : (n + 255) / 256); }

void br_kv_launch_clear(const BrKvTables &t, int *arrived, hipStream_t st) {
  br_kv_k_clear<<<grid_for((long long)t.W * t.B * t.max_blocks), 256, 0, st>>>(t, arrived);
}

void br_kv_launch_load(const BrKvTables &t, const int *lens, const int *table, hipStream_t st) {
  br_kv_k_load<<<grid_for((long long)t.W * t.B * t.max_blocks), 256, 0, st>>>(t, lens, table);
}

void br_kv_launch_step(const BrKvTables &t, const BrKvStep &s, hipStream_t st) {
  const size_t lds = (size_t)t.words * 4;
  if (t.B <= 256) br_kv_k_step<256, 1><<<t.W, 256, lds, st>>>(t, s);
  else br_kv_k_step<256, 4><<<t.W, 256, lds, st>>>(t, s);
}
