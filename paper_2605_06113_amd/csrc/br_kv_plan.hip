// Which rows are read together (br_kv_plan): companies of rows whose tables begin with the same blocks.
#include "br_kv_device.h"

// How many of its tokens each row holds in the same blocks as the row that leads it: a wave a row, 256 entries at a time.
__global__ __launch_bounds__(256) void br_kv_k_plan_common(BrKvTables t, BrKvPlan x) {
  const int lane = threadIdx.x & 63, rows = t.W * t.B;
  for (int r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); r < rows; r += gridDim.x * 4) {
    const int w = r / t.B, f = br_kv_leader(t, x, w, r - w * t.B), len = br_kv_len(t, r);
    if (x.count && x.count[r] != 1) continue;
    int same = len;
    if (w * t.B + f != r) {
      same = min(len, br_kv_len(t, w * t.B + f));
      const int *a = t.table + (long long)r * t.max_blocks, *b = t.table + (long long)(w * t.B + f) * t.max_blocks;
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
        if (first != INT32_MAX) {
          same = min(same, min(first, blocks - 1) << t.shift);
          break;
        }
      }
    }
    if (lane == 0) x.common[r] = same;
  }
}

// One block for each worker: a family's rows in companies of at most `most`, evenly, in the order of the rows.
template <int RPT>
__global__ __launch_bounds__(256) void br_kv_k_plan(BrKvTables t, BrKvPlan x) {
  constexpr int ROWS = 256 * RPT;
  __shared__ int part[16 * 4], family[ROWS], size[ROWS], before[ROWS], first_of[ROWS], least[ROWS], tiles[ROWS], n_of[ROWS], begin_of[ROWS];
  const int w = blockIdx.x, tid = threadIdx.x, B = t.B;
  int turn = 0;
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i;
    family[r] = r < B && (!x.count || x.count[(long long)w * B + r] == 1) ? br_kv_leader(t, x, w, r) : -1;
    size[r] = n_of[r] = begin_of[r] = tiles[r] = 0, least[r] = INT32_MAX;
  }
  __syncthreads();
  int rank[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i, f = family[r];
    rank[i] = 0;
    if (f < 0) continue;
    for (int k = 0; k < r; ++k) rank[i] += family[k] == f;
    atomicAdd(&size[f], 1);
  }
  __syncthreads();
  int sum[2] = {0, 0}, all[2];
#pragma unroll
  for (int i = 0; i < RPT; ++i) sum[0] += size[tid * RPT + i], sum[1] += (size[tid * RPT + i] + x.most - 1) / x.most;
  const int mine[2] = {sum[0], sum[1]};
  br_kv_scan<256, 2>(sum, all, part, turn);
  int a = sum[0] - mine[0], b = sum[1] - mine[1];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i;
    before[r] = a, first_of[r] = b;
    a += size[r], b += (size[r] + x.most - 1) / x.most;
  }
  __syncthreads();
  int company[RPT], tokens[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int r = tid * RPT + i, f = family[r];
    company[i] = -1;
    if (f < 0) continue;
    const long long at = (long long)w * B + r;
    const int companies = (size[f] + x.most - 1) / x.most, per = (size[f] + companies - 1) / companies, k = rank[i] / per;
    company[i] = first_of[f] + k;
    tokens[i] = br_kv_len(t, (int)at);
    atomicMin(&least[company[i]], x.common[at]);
    if (rank[i] == k * per) n_of[company[i]] = min(per, size[f] - k * per), begin_of[company[i]] = before[f] + k * per;
    x.members[(long long)w * B + before[f] + rank[i]] = make_int4((int)at, x.start ? x.start[at] : (int)at, tokens[i], 0);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    if (company[i] < 0) continue;
    const int together = n_of[company[i]] > 1 ? least[company[i]] / BR_KV_TILE : 0;
    atomicAdd(&tiles[company[i]], (tokens[i] + BR_KV_TILE - 1) / BR_KV_TILE - together);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int c = tid * RPT + i;
    if (c >= B) continue;
    const int together = n_of[c] > 1 ? least[c] / BR_KV_TILE : 0;
    x.companies[(long long)w * B + c] = make_int4(n_of[c], w * B + begin_of[c], together, together + tiles[c]);
  }
}

void br_kv_launch_plan(const BrKvTables &t, const BrKvPlan &x, hipStream_t st) {
  const long long blocks = ((long long)t.W * t.B + 3) / 4;
  br_kv_k_plan_common<<<(unsigned)(blocks < 1 << 20 ? blocks : 1 << 20), 256, 0, st>>>(t, x);
  if (t.B <= 256) br_kv_k_plan<1><<<t.W, 256, 0, st>>>(t, x);
  else br_kv_k_plan<4><<<t.W, 256, 0, st>>>(t, x);
}
