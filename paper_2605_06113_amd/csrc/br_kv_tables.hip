// Block tables and slot maps of a step (br_kv_step), and the kernels that set a context up.
#include <type_traits>

#include "br_kv_device.h"

// Every row empty, every block free; nothing begun.
__global__ __launch_bounds__(256) void br_kv_k_clear(BrKvTables t, int4 *companies) {
  const long long n = (long long)t.W * t.B * t.max_blocks, rows = (long long)t.W * t.B, words = (long long)t.W * t.words;
  const long long step = (long long)gridDim.x * 256;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    t.table[i] = -1;
    if (i < rows) t.lens[i] = 0, t.tail[i] = -1;
  }
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < words; i += step) t.used[i] = 0;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < BR_KV_SPLIT_WGS; i += step) t.arrived[i] = 0;
  if (t.holders)
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < (long long)t.W * t.n_blocks; i += step) t.holders[i] = 0;
  if (companies) {  // (a plan that was captured and not run yet has planned nothing)
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < 2ll * t.W * t.B; i += step) companies[i] = make_int4(0, 0, 0, 0);
    if (blockIdx.x == 0 && threadIdx.x == 0) *t.planned = 0;
  }
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
    if (j == (len - 1) >> t.shift) t.tail[row] = id;
    atomicOr(&t.used[row / t.B * t.words + (id >> 5)], 1u << (id & 31));
    if (t.holders) atomicAdd(&t.holders[row / t.B * t.n_blocks + id], 1);
  }
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

// Fours of places begin where 16 bytes of the workers' lists side by side do, as many places before a worker's first one (by its own
// places, four stores of 4 bytes where the lists' length is odd: 1350 lists of 5159 places 38 us).
__device__ __forceinline__ int br_kv_lead(int w, int cap) { return (int)((unsigned)w * (unsigned)cap & 3u); }
__host__ __device__ __forceinline__ int br_kv_list_parts(int cap) { return (cap + 3 + BR_KV_LIST - 1) / BR_KV_LIST; }

// Places j0 .. j0 + 3 of a worker's token list, those that it has (j0 may be below 0): rows' tokens from before[r] on, at positions from kp[r] on.  tail: the block of the last
// position before those (a decode step then reads no table: a line for each row would be more than all the rest, 16384 workers
// of 144 rows 99 us), or null.
__device__ __forceinline__ void br_kv_list4(const BrKvTables &t, const BrKvStep &s, long long list, const int *table, const int *before, const int *kp, const int *tail, int rows,
                                            int total, int j0, int cap) {
  int slot[4] = {-1, -1, -1, -1}, pos[4] = {-1, -1, -1, -1};
  if (j0 < total) {
    int r = br_kv_find(before, rows, max(j0, 0));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (j0 + k >= total) break;
      if (j0 + k < 0) continue;
      while (r + 1 < rows && before[r + 1] <= j0 + k) ++r;
      pos[k] = kp[r] + j0 + k - before[r];
      const int id = tail && pos[k] >> t.shift == (kp[r] - 1) >> t.shift ? tail[r] : table[(long long)r * t.max_blocks + (pos[k] >> t.shift)];
      slot[k] = id < 0 ? -1 : (id << t.shift) + (pos[k] & ((1 << t.shift) - 1));
    }
  }
  if (s.wide && j0 >= 0 && j0 + 4 <= cap) {
    typedef int i4 __attribute__((ext_vector_type(4)));
    if (s.slot) __builtin_nontemporal_store(i4{slot[0], slot[1], slot[2], slot[3]}, (i4 *)(s.slot + list + j0));
    if (s.pos) __builtin_nontemporal_store(i4{pos[0], pos[1], pos[2], pos[3]}, (i4 *)(s.pos + list + j0));
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (j0 + k >= cap) break;
      if (j0 + k < 0) continue;
      if (s.slot) s.slot[list + j0 + k] = slot[k];
      if (s.pos) s.pos[list + j0 + k] = pos[k];
    }
  }
}

// One block of NT threads per worker; a thread has the RPT rows from tid * RPT on.  The used bits are in LDS.  LIST: writes the
// token list as well; else leaves each row's first place in it and first position to br_kv_k_list.
// A chain of dependent steps (rows, blocks given back, sums, free ids, lists), so its time is their latencies: barriers are few (the
// sums of a step in which nothing is refused take one), scans stay in registers.  One worker of 96 rows 4.8 us (a launch that does
// nothing: 4); 16384 workers of 144 rows, a token each, 259 MB, most of them stores of the outputs: 58 us = 4.5 TB/s where the 256 MB cache has part
// of them from the call before, 76 us = 3.4 TB/s where three such states take turns.
// SHARED: blocks may have several holders, whose counts are in global memory (a worker's may be 1 MB): a block that is given back is free when
// the last one gives it, and a row that would write into one that others hold gets another in its place.  One worker of 96 rows 7.2 us: the counts are two trips to
// memory more in the chain.
template <int NT, int RPT, bool LIST, bool SHARED>
__global__ __launch_bounds__(NT) void br_kv_k_step(BrKvTables t, BrKvStep s) {
  constexpr int ROWS = NT * RPT, IDS = NT * 8, AT_ONCE = 8;
  extern __shared__ unsigned used[];
  __shared__ int part[16 * (NT / 64)], give_n, need_before[ROWS], tok_before[ROWS], row_kp[ROWS], give[ROWS], row_tail[ROWS], ids[IDS];
  __shared__ int dropped;
  int *const row_in = give;  // 1: the row's first block comes in the place of its last one (whose blocks are given back is done with by then)
  const int w = blockIdx.x, tid = threadIdx.x, B = t.B, b1 = (1 << t.shift) - 1;
  int turn = 0;
  int *lens = t.lens + (long long)w * B;
  int *table = t.table + (long long)w * B * t.max_blocks;
  int *tails = t.tail + (long long)w * B;
  unsigned *gused = t.used + (long long)w * t.words;
  int *holders = SHARED ? t.holders + (long long)w * t.n_blocks : nullptr;
  // (the count's change comes back: whoever takes it to 0 is the last)
  auto give_back = [&](int id) {
    if (!SHARED || atomicSub(&holders[id], 1) == 1) atomicAnd(&used[id >> 5], ~(1u << (id & 31)));
  };
  if (tid == 0) give_n = 0;
  if (SHARED && tid == 0) dropped = 0;
  if (w == 0)  // (nothing of an attention that went wrong outlives the step behind it)
    for (int i = tid; i < BR_KV_SPLIT_WGS; i += NT) t.arrived[i] = 0;
  int kp[RPT], have[RPT], why[RPT], held[RPT], want[RPT], tail[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i;
    int keep = 0;
    kp[i] = want[i] = 0, tail[i] = -1;
    if (r < B) kp[i] = lens[r], tail[i] = tails[r], keep = s.keep[(long long)w * B + r], want[i] = s.add[(long long)w * B + r];
    held[i] = (kp[i] + b1) >> t.shift;
    kp[i] = keep < 0 ? kp[i] : min(keep, kp[i]);
    want[i] = max(want[i], 0);
  }
  for (int i = tid; i < t.words; i += NT) used[i] = gused[i];
  __syncthreads();
  int long_ones = 0;
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i;
    why[i] = 0;
    have[i] = (kp[i] + b1) >> t.shift;
    if (held[i] != have[i]) tail[i] = have[i] > 0 ? table[(long long)r * t.max_blocks + have[i] - 1] : -1;
    // blocks given back: one here, of a longer run by 16 threads below
    if (held[i] == have[i] + 1) {
      int *at = table + (long long)r * t.max_blocks + have[i];
      const int id = *at;
      if (id >= 0) give_back(id);
      *at = -1;
    } else if (held[i] > have[i]) {
      give[atomicAdd(&give_n, 1)] = r, need_before[r] = have[i], tok_before[r] = held[i];
    }
    if ((long long)kp[i] + want[i] > (long long)t.max_blocks << t.shift) {
      if (want[i] > 0) why[i] = BR_KV_TOO_LONG;
      want[i] = 0;
    }
  }
  __syncthreads();
  if (give_n > 0) {
    for (int k = tid >> 4; k < give_n; k += NT / 16) {
      const int r = give[k], from = need_before[r], to = tok_before[r];
      int *row = table + (long long)r * t.max_blocks;
      for (int j = from + (tid & 15); j < to; j += 16 * AT_ONCE) {
        int id[AT_ONCE];
#pragma unroll
        for (int m = 0; m < AT_ONCE; ++m) id[m] = row[min(j + 16 * m, to - 1)];
#pragma unroll
        for (int m = 0; m < AT_ONCE; ++m) {
          if (j + 16 * m >= to) continue;
          if (id[m] >= 0) give_back(id[m]);
          row[j + 16 * m] = -1;
        }
      }
    }
    __syncthreads();
  }

  int in[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i)
    in[i] = SHARED && want[i] > 0 && (kp[i] & b1) && tail[i] >= 0 && __hip_atomic_load(&holders[max(tail[i], 0)], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) > 1;

  // sums, as if nothing were refused: tokens, blocks, and what is counted of them
  int need[RPT], sum[6], all[6], nfree = 0;
  auto count = [&]() {
#pragma unroll
    for (int k = 0; k < 6; ++k) sum[k] = 0;
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      need[i] = ((kp[i] + want[i] + b1) >> t.shift) - have[i];
      if (SHARED && want[i] > 0) need[i] += in[i];
      sum[0] += want[i], sum[1] += need[i], sum[2] += kp[i] + want[i];
      sum[3] += kp[i] + want[i] > 0, sum[5] += (why[i] > 0) + (why[i] == BR_KV_NO_BLOCKS ? 1 << 16 : 0);
    }
    sum[4] = nfree;
  };
  for (int i = tid; i < t.words; i += NT) nfree += 32 - __popc(used[i]);
  count();
  br_kv_scan<NT, 6>(sum, all, part, turn);
  const int free_blocks = all[4] - (t.words * 32 - t.n_blocks);
  if (all[0] > s.cap || all[1] > free_blocks) {
    int run[1] = {sum[0]}, ignore[1];
#pragma unroll
    for (int i = 0; i < RPT; ++i) run[0] -= want[i];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      run[0] += want[i];
      if (want[i] > 0 && run[0] > s.cap) why[i] = BR_KV_NO_ROOM, want[i] = 0;
    }
    count();
    run[0] = sum[1];
    br_kv_scan<NT, 1>(run, ignore, part, turn);
    run[0] -= sum[1];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      run[0] += need[i];
      if (need[i] > 0 && run[0] > free_blocks) why[i] = BR_KV_NO_BLOCKS, want[i] = 0;
    }
    count();
    br_kv_scan<NT, 6>(sum, all, part, turn);
  }
  const int total = all[0], need_all = all[1];
  int x = sum[1], y = sum[0];
#pragma unroll
  for (int i = 0; i < RPT; ++i) x -= need[i], y -= want[i];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i;
    need_before[r] = x, tok_before[r] = y, row_kp[r] = kp[i], row_tail[r] = tail[i];
    if (r < B) {
      const long long at = (long long)w * B + r;
      lens[r] = kp[i] + want[i];
      if (held[i] != have[i] && need[i] == 0) tails[r] = tail[i];
      if (s.start) s.start[at] = w * s.cap + y;
      if (s.count) s.count[at] = want[i];
      if (s.status) s.status[at] = why[i];
      if (!LIST) s.runs[at] = make_int2(y, kp[i]);
      if (SHARED) s.copy_src[at] = want[i] > 0 && in[i] ? tail[i] : -1;
      if (SHARED && !(want[i] > 0 && in[i])) s.copy_dst[at] = -1;
    }
    if (SHARED) row_in[r] = want[i] > 0 ? in[i] : 0;
    x += need[i], y += want[i];
  }
  auto say = [&](int free_again) {
    long long *o = s.stats + (long long)w * BR_KV_NSTATS;
    const int n_used = t.n_blocks - free_blocks + need_all - free_again;
    o[BR_KV_ST_TOKENS] = all[2], o[BR_KV_ST_USED] = n_used, o[BR_KV_ST_FREE] = t.n_blocks - n_used, o[BR_KV_ST_ROWS] = all[3];
    o[BR_KV_ST_ADDED] = total, o[BR_KV_ST_REFUSED] = all[5] & 0xffff, o[BR_KV_ST_NO_BLOCKS] = all[5] >> 16, o[BR_KV_ST_TAKEN] = need_all;
  };
  if (!SHARED && tid == 0 && s.stats) say(0);
  // ids of blocks first .. first + n - 1 of those taken, to their rows
  auto hand_out = [&](auto many, int first, int n) {
    constexpr int MINE = decltype(many)::value;
    int r[MINE];
#pragma unroll
    for (int m = 0; m < MINE; ++m) r[m] = 0;
    for (int half = ROWS / 2; half; half >>= 1)
#pragma unroll
      for (int m = 0; m < MINE; ++m)
        if (need_before[r[m] + half] <= first + tid + m * NT) r[m] += half;
#pragma unroll
    for (int m = 0; m < MINE; ++m) {
      const int j = tid + m * NT, q = first + j;
      if (j >= n) continue;
      int entry = ((row_kp[r[m]] + b1) >> t.shift) + q - need_before[r[m]];
      if (SHARED) {
        holders[ids[j]] = 1;
        entry -= row_in[r[m]];
        if (row_in[r[m]] && q == need_before[r[m]]) row_tail[r[m]] = ids[j], s.copy_dst[(long long)w * B + r[m]] = ids[j];
      }
      table[(long long)r[m] * t.max_blocks + entry] = ids[j];
      if (q + 1 == (r[m] + 1 < ROWS ? need_before[r[m] + 1] : need_all)) tails[r[m]] = ids[j];
    }
  };
  // blocks taken, lowest ids first: NT words of used bits at a time, IDS ids at a time
  int taken = 0;
  for (int i0 = 0; taken < need_all && i0 < t.words; i0 += NT) {
    const int i = i0 + tid;
    unsigned bits = i < t.words ? ~used[i] : 0u;
    if (i == t.words - 1 && (t.n_blocks & 31)) bits &= (1u << (t.n_blocks & 31)) - 1;
    int k[1] = {(int)__popc(bits)}, here[1];
    const int mine = k[0];
    br_kv_scan<NT, 1>(k, here, part, turn);
    int at = k[0] - mine;
    const int n = min(here[0], need_all - taken);
    unsigned got = 0;
    for (int from = 0; from < n; from += IDS) {
      for (; bits && at < min(n, from + IDS); ++at, bits &= bits - 1) {
        ids[at - from] = 32 * i + __ffs(bits) - 1;
        got |= bits & -bits;
      }
      __syncthreads();
      // (searches side by side, if there are many: one after the other they were half of a step in which 80 prompts of a worker
      // begin, 22 us; eight where one would do, 16384 workers of 144 rows 79 us, not 62)
      if (n - from > NT) hand_out(std::integral_constant<int, IDS / NT>(), taken + from, n - from);
      else hand_out(std::integral_constant<int, 1>(), taken + from, n - from);
      __syncthreads();
    }
    if (got) used[i] |= got;
    taken += n;
  }
  __syncthreads();
  if (SHARED) {
    // (those in whose place others came: none of them was free for this step)
#pragma unroll
    for (int i = 0; i < RPT; ++i)
      if (want[i] > 0 && in[i] && atomicSub(&holders[tail[i]], 1) == 1) atomicAnd(&used[tail[i] >> 5], ~(1u << (tail[i] & 31))), atomicAdd(&dropped, 1);
    __syncthreads();
    if (tid == 0 && s.stats) say(dropped);
    if (w == 0 && tid == 0) *t.planned = 0;
  }
  for (int i = tid; i < t.words; i += NT) gused[i] = used[i];
  if (LIST && (s.slot || s.pos))
    for (int j = 4 * tid - br_kv_lead(w, s.cap); j < s.cap; j += 4 * NT) br_kv_list4(t, s, (long long)w * s.cap, table, tok_before, row_kp, row_tail, ROWS, total, j, s.cap);
}

// The token lists of a step, BR_KV_LIST places of a worker's for each block (behind br_kv_k_step).  Bound by the search for each place's
// row and the trip to its table: 37 workers, 7 M places, 16 us, 61 MB = 3.7 TB/s.
__global__ __launch_bounds__(256) void br_kv_k_list(BrKvTables t, BrKvStep s) {
  __shared__ int before[BR_KV_MAX_ROWS], kp[BR_KV_MAX_ROWS], total;
  const int parts = br_kv_list_parts(s.cap), w = blockIdx.x / parts, j0 = (blockIdx.x - w * parts) * BR_KV_LIST - br_kv_lead(w, s.cap), B = t.B;
  for (int r = threadIdx.x; r < B; r += 256) {
    const int2 x = s.runs[(long long)w * B + r];
    before[r] = x.x, kp[r] = x.y;
    if (r == B - 1) total = x.x + t.lens[(long long)w * B + r] - x.y;
  }
  __syncthreads();
  const int *table = t.table + (long long)w * B * t.max_blocks;
  for (int j = j0 + 4 * threadIdx.x; j < min(s.cap, j0 + BR_KV_LIST); j += 1024) br_kv_list4(t, s, (long long)w * s.cap, table, before, kp, nullptr, B, total, j, s.cap);
}

static int grid_for(long long n) { return (int)(n < 1 ? 1 : n > 4096ll * 256 ? 4096 : (n + 255) / 256); }

void br_kv_launch_clear(const BrKvTables &t, int4 *companies, hipStream_t st) {
  br_kv_k_clear<<<grid_for((long long)t.W * t.B * t.max_blocks), 256, 0, st>>>(t, companies);
}

void br_kv_launch_load(const BrKvTables &t, const int *lens, const int *table, hipStream_t st) {
  br_kv_k_load<<<grid_for((long long)t.W * t.B * t.max_blocks), 256, 0, st>>>(t, lens, table);
}

template <bool LIST, bool SHARED>
static void launch_step(const BrKvTables &t, const BrKvStep &s, hipStream_t st) {
  const size_t lds = (size_t)t.words * 4;
  // (as few rows to a thread as will do: its arrays in LDS go by it, and with them the blocks on a compute unit)
  if (t.B <= 256) br_kv_k_step<256, 1, LIST, SHARED><<<t.W, 256, lds, st>>>(t, s);
  else if (t.B <= 512) br_kv_k_step<256, 2, LIST, SHARED><<<t.W, 256, lds, st>>>(t, s);
  else br_kv_k_step<256, 4, LIST, SHARED><<<t.W, 256, lds, st>>>(t, s);
}

void br_kv_launch_step(const BrKvTables &t, const BrKvStep &s, hipStream_t st) {
  const bool list = s.slot || s.pos;
  if (!list || s.cap <= BR_KV_LIST) return t.holders ? launch_step<true, true>(t, s, st) : launch_step<true, false>(t, s, st);
  if (t.holders) launch_step<false, true>(t, s, st);
  else launch_step<false, false>(t, s, st);
  br_kv_k_list<<<t.W * br_kv_list_parts(s.cap), 256, 0, st>>>(t, s);
}
