// Which rows are read together (br_kv_plan): companies of rows whose tables begin with the same blocks.
#include "br_kv_device.h"

// How many of its tokens row r of worker w holds in the same blocks as the row that leads it: by a wave, 256 entries at a time.
__device__ __forceinline__ int br_kv_common(const BrKvTables &t, const BrKvPlan &x, int w, int r) {
  const int lane = threadIdx.x & 63, f = br_kv_leader(t, x, w, r), row0 = w * t.B;
  int same = br_kv_len(t, row0 + r);
  if (f == r) return same;
  same = min(same, br_kv_len(t, row0 + f));
  const int *a = t.table + (long long)(row0 + r) * t.max_blocks, *b = t.table + (long long)(row0 + f) * t.max_blocks;
  const int blocks = (same + (1 << t.shift) - 1) >> t.shift;
  for (int j = 0; j < blocks; j += 256) {
    int u[4], v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = min(j + 64 * k + lane, blocks - 1);
      u[k] = a[at], v[k] = b[at];
    }
    int first = INT32_MAX;
#pragma unroll
    for (int k = 3; k >= 0; --k) {
      const unsigned long long other = __ballot(u[k] != v[k]);
      if (other) first = j + 64 * k + __ffsll(other) - 1;
    }
    if (first != INT32_MAX) return min(same, min(first, blocks - 1) << t.shift);
  }
  return same;
}

__global__ __launch_bounds__(256) void br_kv_k_plan_common(BrKvTables t, BrKvPlan x) {
  const int rows = t.W * t.B;
  for (int at = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); at < rows; at += gridDim.x * 4) {
    if (x.count && x.count[at] != 1) continue;
    const int w = at / t.B, same = br_kv_common(t, x, w, at - w * t.B);
    if ((threadIdx.x & 63) == 0) x.common[at] = same;
  }
}

// One block for each worker: a family's rows in companies of at most `most`, evenly, in the order of the rows.
// ALONE: what rows have in common is found here too (else by br_kv_k_plan_common, before).
template <int NT, int RPT, bool ALONE>
__global__ __launch_bounds__(NT) void br_kv_k_plan(BrKvTables t, BrKvPlan x) {
  constexpr int ROWS = NT * RPT;
  __shared__ __attribute__((aligned(16))) int family[ROWS];
  __shared__ int part[16 * (NT / 64)], common[ALONE ? ROWS : 1], size[ROWS], before[ROWS], first_of[ROWS], least[ROWS], tiles[ROWS], n_of[ROWS], begin_of[ROWS], by16[4 * ROWS], by32[2 * ROWS];
  const int w = blockIdx.x, tid = threadIdx.x, B = t.B;
  int turn = 0;
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i;
    family[r] = r < B && (!x.count || x.count[(long long)w * B + r] == 1) ? br_kv_leader(t, x, w, r) : -1;
    size[r] = n_of[r] = begin_of[r] = tiles[r] = 0, least[r] = INT32_MAX;
    by16[4 * r] = by16[4 * r + 1] = by16[4 * r + 2] = by16[4 * r + 3] = by32[2 * r] = by32[2 * r + 1] = 0;
  }
  __syncthreads();
  if (ALONE)
    for (int r = __builtin_amdgcn_readfirstlane(tid >> 6); r < B; r += NT / 64) {
      if (family[r] < 0) continue;
      const int same = br_kv_common(t, x, w, r);
      if ((tid & 63) == 0) common[r] = same;
    }
  int rank[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i, f = family[r];
    rank[i] = 0;
    if (f < 0) continue;
    for (int k = 0; k < r; k += 4) {  // (up to three rows from r on are looked at and not counted)
      const int4 x4 = *(const int4 *)(family + k);
      rank[i] += (x4.x == f) + (x4.y == f && k + 1 < r) + (x4.z == f && k + 2 < r) + (x4.w == f && k + 3 < r);
    }
    atomicAdd(&size[f], 1);
  }
  __syncthreads();
  int sum[2] = {0, 0}, all[2];
#pragma unroll
  for (int i = 0; i < RPT; ++i) sum[0] += size[tid * RPT + i], sum[1] += (size[tid * RPT + i] + x.most - 1) / x.most;
  const int mine[2] = {sum[0], sum[1]};
  br_kv_scan<NT, 2>(sum, all, part, turn);
  int a = sum[0] - mine[0], b = sum[1] - mine[1];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i;
    before[r] = a, first_of[r] = b;
    a += size[r], b += (size[r] + x.most - 1) / x.most;
  }
  __syncthreads();
  int company[RPT], tokens[RPT], place[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i, f = family[r];
    company[i] = -1;
    if (f < 0) continue;
    const long long at = (long long)w * B + r;
    const int companies = (size[f] + x.most - 1) / x.most, per = (size[f] + companies - 1) / companies, k = rank[i] / per;
    company[i] = first_of[f] + k, place[i] = rank[i] - k * per;
    tokens[i] = br_kv_len(t, (int)at);
    atomicMin(&least[company[i]], ALONE ? common[r] : x.common[at]);
    if (rank[i] == k * per) n_of[company[i]] = min(per, size[f] - k * per), begin_of[company[i]] = before[f] + k * per;
    x.members[(long long)w * B + before[f] + rank[i]] = make_int4((int)at, x.start ? x.start[at] : (int)at, tokens[i], 0);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    if (company[i] < 0) continue;
    const int together = n_of[company[i]] > 1 ? least[company[i]] / BR_KV_TILE : 0, own = (tokens[i] + BR_KV_TILE - 1) / BR_KV_TILE - together;
    atomicAdd(&tiles[company[i]], own);
    // (of one member all waves have the same; several have 64 query rows at most)
    const int first = place[i] * x.group, last = n_of[company[i]] > 1 ? first + x.group - 1 : first;
    for (int k = first / 16; k <= min(last / 16, 3); ++k) atomicAdd(&by16[4 * company[i] + k], own);
    for (int k = first / 32; k <= min(last / 32, 1); ++k) atomicAdd(&by32[2 * company[i] + k], own);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int c = tid * RPT + i;
    if (c >= B) continue;
    const int together = n_of[c] > 1 ? least[c] / BR_KV_TILE : 0;
    int4 *to = x.companies + 2 * ((long long)w * B + c);
    to[0] = make_int4(n_of[c], w * B + begin_of[c], together, together + tiles[c]);
    to[1] = make_int4(together + max(max(by16[4 * c], by16[4 * c + 1]), max(by16[4 * c + 2], by16[4 * c + 3])), together + max(by32[2 * c], by32[2 * c + 1]), 0, 0);
  }
}

void br_kv_launch_plan(const BrKvTables &t, const BrKvPlan &x, hipStream_t st) {
  // A wave takes some 1.2 us for what a row has in common with its leader.  One worker's rows by its one block, in one launch, or by the card, in two: 16 rows
  // 5.3 us and 8.9, 64 rows (a block of 16 waves) 6.7 and 8.6, 96 rows with tables out of memory 11.6 and 9.6, 256 rows 16 and 10.  Many workers fill the card by themselves, with blocks of four waves if
  // they are very many: 512 of 144 rows 18 us and 27, 4096 of 32 rows 25, 43 with 16 waves each, and 45.
  if (t.B <= 16 || (t.W >= 1024 && t.B <= 256)) {
    br_kv_k_plan<256, 1, true><<<t.W, 256, 0, st>>>(t, x);
    return;
  }
  if (t.B <= 64 || (t.W >= 128 && t.B <= 256)) {
    br_kv_k_plan<1024, 1, true><<<t.W, 1024, 0, st>>>(t, x);
    return;
  }
  const long long blocks = ((long long)t.W * t.B + 3) / 4;
  br_kv_k_plan_common<<<(unsigned)(blocks < 1 << 20 ? blocks : 1 << 20), 256, 0, st>>>(t, x);
  if (t.B <= 256) br_kv_k_plan<256, 1, false><<<t.W, 256, 0, st>>>(t, x);
  else br_kv_k_plan<1024, 1, false><<<t.W, 1024, 0, st>>>(t, x);
}
