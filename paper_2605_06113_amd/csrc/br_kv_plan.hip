// Which rows are read together (br_kv_plan): companies of rows whose tables begin with the same blocks.
#include "br_kv_device.h"

// The row that those of r's family are compared with: the one that leads them, if it is one of them and holds tokens, or the first of them that does (what leads
// a family may have left, or go with another one).  By a wave; r itself if it holds none.
__device__ __forceinline__ int br_kv_compared(const BrKvTables &t, const BrKvPlan &x, int w, int r) {
  const int lane = threadIdx.x & 63, row0 = w * t.B, f = br_kv_leader(t, x, w, r);
  const int len = br_kv_len(t, row0 + r);
  auto one_of_them = [&](int k) {  // (asked for at once)
    const int lead = br_kv_leader(t, x, w, k), count = x.count ? x.count[row0 + k] : 1, len = br_kv_len(t, row0 + k);
    return (lead == f) & (count == 1) & (len > 0);
  };
  if (one_of_them(f)) return len == 0 ? r : f;
  if (len == 0) return r;
  for (int k = 0; k < r; k += 64) {
    const unsigned long long some = __ballot(k + lane < r && one_of_them(min(k + lane, r)));
    if (some) return k + __ffsll(some) - 1;
  }
  return r;
}

// How many of its tokens row r of worker w holds in the same blocks as row f: by a wave, 256 entries at a time.
__device__ __forceinline__ int br_kv_common(const BrKvTables &t, int w, int r, int f) {
  const int lane = threadIdx.x & 63, row0 = w * t.B;
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
    const int w = at / t.B, r = at - w * t.B, same = br_kv_common(t, w, r, br_kv_compared(t, x, w, r));
    if ((threadIdx.x & 63) == 0) x.common[at] = same;
  }
}

// One block for each worker, a thread for each row: a family's rows in companies of at most `most`, evenly, in the order of the rows.  Rows without tokens
// are families of their own: they have nothing in common with any other.
// ALONE: what rows have in common is found here too (else by br_kv_k_plan_common, before).  Bound by its chain of loads and barriers: four rows of one worker
// 3.9 us; 96 rows in two launches 4.8 and 5.5.
template <int NT, bool ALONE>
__global__ __launch_bounds__(NT) void br_kv_k_plan(BrKvTables t, BrKvPlan x) {
  __shared__ __attribute__((aligned(16))) int family[NT];
  __shared__ int part[16 * (NT / 64)], common[ALONE ? NT : 1], size[NT], before[NT], first_of[NT], least[NT], tiles[NT], n_of[NT], begin_of[NT], by16[4 * NT], by32[2 * NT];
  const int w = blockIdx.x, r = threadIdx.x, B = t.B;
  const long long at = (long long)w * B + r;
  int turn = 0;
  const int lead = r < B && (!x.count || x.count[at] == 1) ? br_kv_leader(t, x, w, r) : -1, tokens = lead >= 0 ? br_kv_len(t, (int)at) : 0;
  size[r] = n_of[r] = begin_of[r] = tiles[r] = 0, least[r] = INT32_MAX;
  by16[4 * r] = by16[4 * r + 1] = by16[4 * r + 2] = by16[4 * r + 3] = by32[2 * r] = by32[2 * r + 1] = 0;
  __syncthreads();
  if (tokens > 0) atomicMin(&least[lead], r == lead ? -1 : r);
  __syncthreads();
  const int first = tokens > 0 ? least[lead] : r, f = lead < 0 ? -1 : first < 0 ? lead : first;  // (br_kv_compared)
  family[r] = f;
  __syncthreads();
  least[r] = INT32_MAX;
  if (ALONE)
    for (int k = __builtin_amdgcn_readfirstlane(r >> 6); k < B; k += NT / 64) {
      if (family[k] < 0) continue;
      const int same = br_kv_common(t, w, k, __builtin_amdgcn_readfirstlane(family[k]));
      if ((r & 63) == 0) common[k] = same;
    }
  int rank = 0;
  if (f >= 0) {
    for (int k = 0; k < r; k += 4) {  // (up to three rows from r on are looked at and not counted)
      const int4 x4 = *(const int4 *)(family + k);
      rank += (x4.x == f) + (x4.y == f && k + 1 < r) + (x4.z == f && k + 2 < r) + (x4.w == f && k + 3 < r);
    }
    atomicAdd(&size[f], 1);
  }
  __syncthreads();
  const int mine[2] = {size[r], (size[r] + x.most - 1) / x.most};
  int sum[2] = {mine[0], mine[1]}, all[2];
  br_kv_scan<NT, 2>(sum, all, part, turn);
  before[r] = sum[0] - mine[0], first_of[r] = sum[1] - mine[1];
  __syncthreads();
  int company = -1, place = 0;
  if (f >= 0) {
    const int companies = (size[f] + x.most - 1) / x.most, per = (size[f] + companies - 1) / companies, k = rank / per;
    company = first_of[f] + k, place = rank - k * per;
    atomicMin(&least[company], ALONE ? common[r] : x.common[at]);
    if (place == 0) n_of[company] = min(per, size[f] - k * per), begin_of[company] = before[f] + k * per;
    x.members[(long long)w * B + before[f] + rank] = make_int4((int)at, x.start ? x.start[at] : (int)at, tokens, 0);
  }
  __syncthreads();
  if (company >= 0) {
    const int together = n_of[company] > 1 ? least[company] / BR_KV_TILE : 0, own = (tokens + BR_KV_TILE - 1) / BR_KV_TILE - together;
    atomicAdd(&tiles[company], own);
    // (of one member all waves have the same; several have 64 query rows at most)
    const int first = place * x.group, last = n_of[company] > 1 ? first + x.group - 1 : first;
    for (int k = first / 16; k <= min(last / 16, 3); ++k) atomicAdd(&by16[4 * company + k], own);
    for (int k = first / 32; k <= min(last / 32, 1); ++k) atomicAdd(&by32[2 * company + k], own);
  }
  __syncthreads();
  if (r >= B) return;
  if (at == 0) *t.planned = 1;  // (a store before the loads would keep them from being what they are: 4096 workers of 96 rows 61 us and 76)
  const int together = n_of[r] > 1 ? least[r] / BR_KV_TILE : 0;
  int4 *to = x.companies + 2 * at;
  to[0] = make_int4(n_of[r], w * B + begin_of[r], together, together + tiles[r]);
  to[1] = make_int4(together + max(max(by16[4 * r], by16[4 * r + 1]), max(by16[4 * r + 2], by16[4 * r + 3])), together + max(by32[2 * r], by32[2 * r + 1]), 0, 0);
}

void br_kv_launch_plan(const BrKvTables &t, const BrKvPlan &x, hipStream_t st) {
  // A wave takes some 1.2 us for what a row has in common with its leader.  One worker's rows by its one block, in one launch, or by the card, in two: 16 rows
  // 5.3 us and 9.0, 64 rows (a block of 16 waves) 6.5 and 8.6, 96 rows behind an attention, plan and attention together, 81.3 and 79.4, 256 rows 15.4 and 11.5.  Many workers
  // fill the card by themselves, with blocks of four waves if they are very many: 512 of 144 rows 17.5 us and 32, 4096 of 32 rows 24.5, 45 with 16 waves each, and 54.
  if (t.B <= 16 || (t.W >= 1024 && t.B <= 256)) {
    br_kv_k_plan<256, true><<<t.W, 256, 0, st>>>(t, x);
    return;
  }
  if (t.B <= 64 || (t.W >= 128 && t.B <= 256)) {
    br_kv_k_plan<1024, true><<<t.W, 1024, 0, st>>>(t, x);
    return;
  }
  const long long blocks = ((long long)t.W * t.B + 3) / 4;
  br_kv_k_plan_common<<<(unsigned)(blocks < 1 << 20 ? blocks : 1 << 20), 256, 0, st>>>(t, x);
  if (t.B <= 256) br_kv_k_plan<256, false><<<t.W, 256, 0, st>>>(t, x);
  else br_kv_k_plan<1024, false><<<t.W, 1024, 0, st>>>(t, x);
}
