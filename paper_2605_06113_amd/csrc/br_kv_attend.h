// Attention over the 8-bit block cache (br_kv_attend).
//
// o = sum_j e^(s_j - m) vs_j v_j / sum_j e^(s_j - m),  s_j = scale ks_j (q . k_j), over the visible cached tokens j; k_j, v_j are
// codes, ks_j, vs_j the scales of j's block and head.  One pass over the tokens with a running m.
//
// Work: a tile is 64 cached tokens of one row and key head against TQ query rows (query tokens x heads of the group).  All tiles
// of the call, in the order (row, key head, query tile, token tile), are dealt to the blocks in equal runs, whatever the lengths: a
// block's run may end inside a row and head, whose pieces are then joined by br_kv_k_join in the order of their tokens.
//
// A wave's tile on the matrix units, 16x16x32 in f16 (codes are exact there; the queries are scaled to 1..2 by a power of two per
// row, so they are too unless they span more than f16's exponents):
//   S^T [token][query] = K Q^T: row i of the t-th of four products is token 16 (i / 4) + 4 t + i % 4, so that lane (query n, g)
//     holds tokens 16 g .. 16 g + 15 of the tile, which one block covers: one ks and one vs per lane;
//   O^T [channel][query] += V^T P^T: the weights of lane (n, g) are this product's operand as they stand, and the values come as
//     16 bytes of 16 consecutive tokens of a channel (the cache keeps them that way round).
// Nothing passes between lanes but the maxima.  Weights go to f16 as 256 e^(s - m) vs / c, c a power of two above the largest vs so
// far, so that they use f16's range whatever the scales are: 11 bits, where the codes have 4 or 8; sums stay in 32 bits.
// m and c only move when a weight would pass 2^4 and a ratio 2^3: the sums are rescaled a few times a row.
#ifndef BR_KV_ATTEND_H
#define BR_KV_ATTEND_H

#include "br_kv_device.h"

#define BR_KV_NEG (-__builtin_inff())

struct BrKvRow {
  int n, len, start;  // query tokens, cached tokens, first token
};

__device__ __forceinline__ BrKvRow br_kv_row(const BrKvAttend &p, int r) {
  BrKvRow w;
  w.n = p.count ? min(max(p.count[r], 0), p.n_tokens) : 1;
  w.start = p.start ? p.start[r] : r;
  w.len = min(max(p.lens[r], 0), p.max_blocks << p.shift);
  return w;
}

// First token tile of a query tile, one past the last, and what it counts in the division of the work: a tile that sees nothing still has
// zeros to write.
template <int TQ>
__device__ __forceinline__ int br_kv_span(const BrKvAttend &p, const BrKvRow &w, int qi, int &t0, int &t1) {
  const int i0 = qi * TQ / p.group, i1 = min(w.n - 1, (qi * TQ + TQ - 1) / p.group), at = w.len - w.n;
  const int hi = max(0, at + i1 + 1), lo = p.window > 0 ? max(0, at + i0 - p.window + 1) : 0;
  t0 = lo / BR_KV_TILE;
  t1 = max(t0, (hi + BR_KV_TILE - 1) / BR_KV_TILE);
  return max(1, t1 - t0);
}

// Tiles of one row and key head.
template <int TQ>
__device__ __forceinline__ long long br_kv_row_tiles(const BrKvAttend &p, const BrKvRow &w) {
  const int nq = (int)(((long long)w.n * p.group + TQ - 1) / TQ);
  long long s = 0;
  for (int qi = 0; qi < nq; ++qi) {
    int t0, t1;
    s += br_kv_span<TQ>(p, w, qi, t0, t1);
  }
  return s;
}

__device__ __forceinline__ unsigned br_kv_pack(float a, float b, int bf16) {
  return bf16 ? (unsigned)br_kv_to_bf16(a) | (unsigned)br_kv_to_bf16(b) << 16 : (unsigned)br_kv_to_f16(a) | (unsigned)br_kv_to_f16(b) << 16;
}

// 4 channels of one query row, final
__device__ __forceinline__ void br_kv_store4(const BrKvAttend &p, const BrKvRow &w, int h, int ri, int d, br_f4 x) {
  const int i = ri / p.group, t = w.start + i;
  if (i >= w.n || t < 0 || t >= p.n_tokens) return;
  unsigned short *at = p.out + (long long)t * p.out_token + (long long)(h * p.group + ri - i * p.group) * p.out_head + d;
  const unsigned a = br_kv_pack(x[0], x[1], p.bf16), b = br_kv_pack(x[2], x[3], p.bf16);
  if (p.out_wide) {
    *(uint2 *)at = make_uint2(a, b);
  } else {
    at[0] = (unsigned short)a, at[1] = (unsigned short)(a >> 16), at[2] = (unsigned short)b, at[3] = (unsigned short)(b >> 16);
  }
}

__device__ __forceinline__ void br_kv_store_lse(const BrKvAttend &p, const BrKvRow &w, int h, int ri, float m, float l) {
  const int i = ri / p.group, t = w.start + i;
  if (!p.lse || i >= w.n || t < 0 || t >= p.n_tokens) return;
  p.lse[(long long)t * p.kv_heads * p.group + h * p.group + ri - i * p.group] = l == 0.0f ? BR_KV_NEG : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

// D channels, NQ groups of 16 query rows a wave; the block's four waves share the query rows and deal the token tiles (WQ = 1) or
// have query rows of their own (WQ = 4).
template <int D, int NQ, int WQ, bool FP8>
__global__ __launch_bounds__(256, 2) void br_kv_k_attend(BrKvAttend p) {
  constexpr int TQ = 16 * NQ * WQ, WT = 4 / WQ, NI = D / 64, REST = D % 64 / 32, NK = 2 * NI + REST, ND = D / 16;
  __shared__ long long before[257], wave_sum[4];
  __shared__ br_f4 red[WQ == 1 ? 4 * ND * 64 : 1];
  __shared__ float red_m[4][16], red_l[4][16], red_c[4];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, n = lane & 15, g = lane >> 4;
  const int wq = WQ == 1 ? 0 : wv, wt = WQ == 1 ? wv : 0;

  // the division of the work: tiles before each thread's rows
  const int per = (p.n_rows + 255) / 256;
  long long mine = 0;
  for (int r = tid * per; r < min(p.n_rows, (tid + 1) * per); ++r) {
    const BrKvRow w = br_kv_row(p, r);
    if (w.n > 0) mine += br_kv_row_tiles<TQ>(p, w) * p.kv_heads;
  }
  long long sum = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const long long o = __shfl_up(sum, d, 64);
    if (lane >= d) sum += o;
  }
  if (lane == 63) wave_sum[wv] = sum;
  __syncthreads();
  for (int k = 0; k < wv; ++k) sum += wave_sum[k];
  before[tid + 1] = sum;
  if (tid == 0) before[0] = 0;
  __syncthreads();
  const long long all = before[256];
  const long long G = max(1ll, min((long long)gridDim.x, all / WT));
  const int wg = blockIdx.x;
  if (wg >= G) {
    if (tid == 0) p.desc[4 * wg + 3] = 0;
    return;
  }
  long long u = all * wg / G;
  const long long end = all * (wg + 1) / G;
  int split_r = 0, split_h = 0, split_q = 0, split_n = 0;  // the piece that begins here and ends in another block

  if (u < end) {
    int lo = 0, hi = 255;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (before[mid] <= u) lo = mid;
      else hi = mid - 1;
    }
    int r = lo * per;
    long long base = before[lo], tiles = 0;
    BrKvRow w;
    for (; r < p.n_rows; ++r) {
      w = br_kv_row(p, r);
      tiles = w.n > 0 ? br_kv_row_tiles<TQ>(p, w) : 0;
      if (u < base + tiles * p.kv_heads) break;
      base += tiles * p.kv_heads;
    }
    if (r >= p.n_rows) return;  // (only if lengths were changed under the launch)
    int h = (int)((u - base) / tiles), qi = 0, t0, t1;
    long long seg = base + h * tiles;  // first tile of the query tile
    int size = br_kv_span<TQ>(p, w, 0, t0, t1);
    while (u >= seg + size) seg += size, size = br_kv_span<TQ>(p, w, ++qi, t0, t1);

    for (;;) {
      const int a = (int)(u - seg), b = (int)min((long long)size, end - seg);
      const bool whole = a == 0 && b == size;
      const int first_pos = w.len - w.n + qi * TQ / p.group, last_pos = w.len - w.n + min(w.n - 1, (qi * TQ + TQ - 1) / p.group);

      // queries: channels 64 i + 16 g .. + 15 of its row for each lane, then 8 g .. + 7 of the last 32
      br_h8 qf[NQ][NK];
      float qs[NQ];
      int pos[NQ];
#pragma unroll
      for (int x = 0; x < NQ; ++x) {
        const int ri = qi * TQ + (wq * NQ + x) * 16 + n, i = ri / p.group, t = w.start + i;
        const bool in = i < w.n && t >= 0 && t < p.n_tokens;
        pos[x] = in ? w.len - w.n + i : -1;
        const unsigned short *at = p.q + (in ? (long long)t * p.q_token + (long long)(h * p.group + ri - i * p.group) * p.q_head : 0);
        float f[NK * 8], top = 0.0f;
#pragma unroll
        for (int c = 0; c < NK; ++c) {
          const int d = c < 2 * NI ? (c / 2) * 64 + g * 16 + (c & 1) * 8 : NI * 64 + g * 8;
          unsigned short e[8];
          if (p.q_wide) {
            *(uint4 *)e = *(const uint4 *)(at + d);
          } else {
            for (int j = 0; j < 8; ++j) e[j] = at[d + j];
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float y = in ? (p.bf16 ? br_kv_bf16(e[j]) : br_kv_f16(e[j])) : 0.0f;
            f[8 * c + j] = y;
            top = fmaxf(top, fabsf(y));
          }
        }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        // the power of two at or below `top`; not below 2^-100, where its inverse would leave the range
        const int ex = max((int)(__float_as_uint(top) >> 23), 27);
        const float inv = __uint_as_float((unsigned)(254 - min(ex, 253)) << 23);
        qs[x] = top > 3.0e38f && top * 0.0f != 0.0f ? __builtin_nanf("") : __uint_as_float((unsigned)min(ex, 253) << 23) * p.scale2;
#pragma unroll
        for (int c = 0; c < NK; ++c)
#pragma unroll
          for (int j = 0; j < 8; ++j) qf[x][c][j] = (_Float16)(f[8 * c + j] * inv);
      }

      br_f4 o[NQ][ND];
      float m[NQ], l[NQ], cmax = 0.0f, cinv = 0.0f;  // c and its inverse
#pragma unroll
      for (int x = 0; x < NQ; ++x) {
        m[x] = BR_KV_NEG, l[x] = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[x][d] = br_f4{0.0f, 0.0f, 0.0f, 0.0f};
      }

      const int worker = r / p.rows;
      const int *table = p.table + (long long)r * p.max_blocks;
      const int last_block = max(0, (w.len - 1) >> p.shift);
      const long long cache0 = (long long)worker * p.n_blocks;
      const int mask = (1 << p.shift) - 1;
      const int kg = n >> 2, kr = n & 3;  // the token group, and the place in fours, of the lane's row of K

      uint4 kc[4][NI + (NI == 0)];
      uint2 kx[4];
      uint4 vc[ND];
      const int rows_q = (int)min((long long)TQ, (long long)w.n * p.group - (long long)qi * TQ);  // query rows of the tile
      const int stop = wq * NQ * 16 < rows_q ? min(t0 + b, t1) : 0;
      // block of a lane's 16 tokens, -1: none
      auto block_of = [&](int token) {
        const int id = table[min(token >> p.shift, last_block)];
        return id >= 0 && id < p.n_blocks ? id : -1;
      };
      auto load_k = [&](int t, int id) {
        const unsigned char *at = p.k + ((((cache0 + max(id, 0)) * p.kv_heads + h) << p.shift) + ((t * BR_KV_TILE + 16 * kg) & mask) + kr) * D;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
          for (int i = 0; i < NI; ++i) kc[s][i] = *(const uint4 *)(at + 4 * s * D + 64 * i + 16 * g);
          if (REST) kx[s] = *(const uint2 *)(at + 4 * s * D + 64 * NI + 8 * g);
        }
      };

      int t = t0 + a + wt;
      int kid = 0, vid = 0, kid1 = 0, vid1 = 0;
      if (t < stop) {
        kid = block_of(t * BR_KV_TILE + 16 * kg), vid = block_of(t * BR_KV_TILE + 16 * g);
        if (t + WT < stop) kid1 = block_of((t + WT) * BR_KV_TILE + 16 * kg), vid1 = block_of((t + WT) * BR_KV_TILE + 16 * g);
        load_k(t, kid);
      }
      for (; t < stop; t += WT) {
        const int token = t * BR_KV_TILE + 16 * g;  // of the lane's first weight
        const long long vb = (cache0 + max(vid, 0)) * p.kv_heads + h;
        {
          const unsigned char *at = p.v + (((vb * D + n) << p.shift) + (token & mask));
#pragma unroll
          for (int d = 0; d < ND; ++d) vc[d] = *(const uint4 *)(at + ((16 * d) << p.shift));
        }
        const float ks = vid < 0 ? 0.0f : p.ks[vb], vs = vid < 0 ? 0.0f : p.vs[vb];
        const int have = vid < 0 ? 0 : min(max(w.len - token, 0), 16);  // of the lane's tokens, those that exist
        int kid2 = 0, vid2 = 0;
        if (t + 2 * WT < stop) kid2 = block_of((t + 2 * WT) * BR_KV_TILE + 16 * kg), vid2 = block_of((t + 2 * WT) * BR_KV_TILE + 16 * g);

        br_f4 s[NQ][4];
#pragma unroll
        for (int x = 0; x < NQ; ++x)
#pragma unroll
          for (int y = 0; y < 4; ++y) s[x][y] = br_f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
#pragma unroll
          for (int c = 0; c < NK; ++c) {
            br_h8 kf;
            if (c < 2 * NI) kf = c & 1 ? br_kv_decode8<FP8>(kc[y][c / 2].z, kc[y][c / 2].w) : br_kv_decode8<FP8>(kc[y][c / 2].x, kc[y][c / 2].y);
            else kf = br_kv_decode8<FP8>(kx[y].x, kx[y].y);
#pragma unroll
            for (int x = 0; x < NQ; ++x) s[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[x][c], s[x][y], 0, 0, 0);
          }
        }
        if (t + WT < stop) load_k(t + WT, kid1);

        // (a block that no query of the tile sees has no say in c)
        float top = have > 0 && token <= last_pos && (p.window == 0 || token + 15 > first_pos - p.window) ? fabsf(vs) : 0.0f;
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        float cf = 1.0f;
        if (top > 8.0f * cmax) {
          const unsigned e = min(max(__float_as_uint(top) >> 23, 20u), 252u) + 1;
          cinv = __uint_as_float((254u - e) << 23);
          cf = cmax * cinv;
          cmax = __uint_as_float(e << 23);
        }
        const float wgt = vs * (256.0f * cinv);
        // inside: every query of the tile sees all of its tokens, and all exist
        const bool inside = t * BR_KV_TILE + BR_KV_TILE - 1 <= first_pos && (p.window == 0 || t * BR_KV_TILE > last_pos - p.window) && !__any(vid < 0);
        br_h8 pf[NQ][2];
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
          const float f = qs[x] * ks;
          float z[16], mx = BR_KV_NEG;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            z[j] = s[x][j >> 2][j & 3] * f;
            if (!inside && !(j < have && token + j <= pos[x] && (p.window == 0 || token + j > pos[x] - p.window))) z[j] = BR_KV_NEG;
            mx = fmaxf(mx, z[j]);
          }
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
          const bool up = mx > m[x] + 4.0f;
          if (__any(up || cf != 1.0f)) {
            const float to = up ? mx : m[x];
            const float al = m[x] == BR_KV_NEG ? (l[x] != 0.0f ? 1.0f : 0.0f) : __builtin_amdgcn_exp2f(m[x] - to), ao = al * cf;
            m[x] = to;
            l[x] *= al;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
              for (int j = 0; j < 4; ++j) o[x][d][j] *= ao;
          }
          const float ref = m[x] == BR_KV_NEG ? 0.0f : m[x];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float e = __builtin_amdgcn_exp2f(z[j] - ref);
            l[x] += e;
            // (a token that is not seen has no weight, whatever its block's scale)
            pf[x][j >> 3][j & 7] = (_Float16)(!inside && z[j] == BR_KV_NEG ? 0.0f : e * wgt);
          }
        }
        // bytes behind the row's end are whatever memory held: an 8-bit float may be a NaN there
        if (FP8 && __any(have < 16)) {
          const unsigned long long full = ~0ull;
          const unsigned long long m0 = have >= 8 ? full : ~(full << (8 * have));
          const unsigned long long m1 = have >= 16 ? full : have <= 8 ? 0ull : ~(full << (8 * (have - 8)));
#pragma unroll
          for (int d = 0; d < ND; ++d) vc[d].x &= (unsigned)m0, vc[d].y &= (unsigned)(m0 >> 32), vc[d].z &= (unsigned)m1, vc[d].w &= (unsigned)(m1 >> 32);
        }
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const br_h8 v0 = br_kv_decode8<FP8>(vc[d].x, vc[d].y), v1 = br_kv_decode8<FP8>(vc[d].z, vc[d].w);
#pragma unroll
          for (int x = 0; x < NQ; ++x) {
            o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pf[x][0], o[x][d], 0, 0, 0);
            o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pf[x][1], o[x][d], 0, 0, 0);
          }
        }
        vid = vid1;
        kid1 = kid2, vid1 = vid2;
      }
      cmax *= 1.0f / 256.0f;
#pragma unroll
      for (int x = 0; x < NQ; ++x) {
        l[x] += __shfl_xor(l[x], 16, 64);
        l[x] += __shfl_xor(l[x], 32, 64);
        if (m[x] == BR_KV_NEG) m[x] = 0.0f;
      }

      // the pieces of a split row: the one that begins in this block in the second place, others in the first
      const int piece = 2 * wg + (a == 0 ? 1 : 0);
      auto put = [&](int row, int d, br_f4 x, float inv) {  // row: of the query tile
        if (row >= rows_q) return;
        if (whole) br_kv_store4(p, w, h, qi * TQ + row, d, br_f4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv});
        else *(br_f4 *)(p.part + ((long long)piece * TQ + row) * D + d) = x;
      };
      auto put_ml = [&](int row, float mm, float ll) {
        if (row >= rows_q) return;
        if (whole) br_kv_store_lse(p, w, h, qi * TQ + row, mm, ll);
        else *(float2 *)(p.ml + ((long long)piece * TQ + row) * 2) = make_float2(mm, ll);
      };
      if constexpr (WQ == 1) {
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
          __syncthreads();
#pragma unroll
          for (int d = 0; d < ND; ++d) red[(wv * ND + d) * 64 + lane] = o[x][d];
          if (g == 0) red_m[wv][n] = m[x], red_l[wv][n] = l[x];
          if (lane == 0) red_c[wv] = cmax;
          __syncthreads();
          float mm = BR_KV_NEG, ll = 0.0f, f[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (red_l[k][n] != 0.0f) mm = fmaxf(mm, red_m[k][n]);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float e = red_l[k][n] != 0.0f ? __builtin_amdgcn_exp2f(red_m[k][n] - mm) : 0.0f;
            ll += red_l[k][n] * e;
            f[k] = e * red_c[k];
          }
          const float inv = ll != 0.0f ? 1.0f / ll : 0.0f;
          for (int d = wv; d < ND; d += 4) {
            br_f4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const br_f4 v = red[(k * ND + d) * 64 + lane];
#pragma unroll
              for (int j = 0; j < 4; ++j) y[j] += v[j] * f[k];
            }
            put(16 * x + n, 16 * d + 4 * g, y, inv);
          }
          if (wv == 0 && g == 0) put_ml(16 * x + n, ll != 0.0f ? mm : 0.0f, ll);
        }
      } else {
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
          const int row = (wq * NQ + x) * 16 + n;
          const float inv = l[x] != 0.0f ? 1.0f / l[x] : 0.0f;
#pragma unroll
          for (int d = 0; d < ND; ++d) put(row, 16 * d + 4 * g, br_f4{o[x][d][0] * cmax, o[x][d][1] * cmax, o[x][d][2] * cmax, o[x][d][3] * cmax}, inv);
          if (g == 0) put_ml(row, m[x], l[x]);
        }
      }

      if (a == 0 && b < size) {
        const long long last = ((seg + size) * G - 1) / all;  // the block of the piece's last tile
        split_r = r, split_h = h, split_q = qi, split_n = (int)(last - wg + 1);
      }
      u = seg + b;
      if (u >= end) break;
      seg += size;
      if (seg < base + (h + 1) * tiles) {
        ++qi;
      } else {
        qi = 0;
        if (++h == p.kv_heads) {
          h = 0;
          base += tiles * p.kv_heads;
          while (++r < p.n_rows) {
            w = br_kv_row(p, r);
            tiles = w.n > 0 ? br_kv_row_tiles<TQ>(p, w) : 0;
            if (tiles > 0) break;
          }
          if (r >= p.n_rows) break;
        }
      }
      size = br_kv_span<TQ>(p, w, qi, t0, t1);
    }
  }
  if (tid == 0) *(int4 *)(p.desc + 4 * wg) = make_int4(split_r, split_h, split_q, split_n);
}

// Joins the pieces of the query tile that block `blockIdx.x` of the attention has begun and others have gone on with.
template <int D, int TQ>
__global__ __launch_bounds__(256) void br_kv_k_join(BrKvAttend p) {
  const int wg = blockIdx.x, parts = p.desc[4 * wg + 3];
  if (parts < 2) return;
  const int r = p.desc[4 * wg], h = p.desc[4 * wg + 1], qi = p.desc[4 * wg + 2];
  const BrKvRow w = br_kv_row(p, r);
  const int rows_q = (int)min((long long)TQ, (long long)w.n * p.group - (long long)qi * TQ);
  for (int at = threadIdx.x; at < rows_q * (D / 4); at += 256) {
    const int row = at / (D / 4), d = at % (D / 4) * 4;
    float m = BR_KV_NEG, l = 0.0f;
    for (int k = 0; k < parts; ++k) {
      const float2 x = *(const float2 *)(p.ml + ((long long)(k ? 2 * (wg + k) : 2 * wg + 1) * TQ + row) * 2);
      if (x.y != 0.0f) m = fmaxf(m, x.x);
    }
    br_f4 y = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < parts; ++k) {
      const long long piece = (long long)(k ? 2 * (wg + k) : 2 * wg + 1) * TQ + row;
      const float2 x = *(const float2 *)(p.ml + piece * 2);
      const br_f4 v = *(const br_f4 *)(p.part + piece * D + d);
      if (x.y == 0.0f) continue;
      const float e = __builtin_amdgcn_exp2f(x.x - m);
      l += x.y * e;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] += v[j] * e;
    }
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
    br_kv_store4(p, w, h, qi * TQ + row, d, br_f4{y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv});
    if (d == 0) br_kv_store_lse(p, w, h, qi * TQ + row, l != 0.0f ? m : 0.0f, l);
  }
}

template <int D, int NQ, int WQ>
void br_kv_attend_tile(const BrKvAttend &p, bool fp8, int blocks, hipStream_t st) {
  if (fp8) br_kv_k_attend<D, NQ, WQ, true><<<blocks, 256, 0, st>>>(p);
  else br_kv_k_attend<D, NQ, WQ, false><<<blocks, 256, 0, st>>>(p);
  br_kv_k_join<D, 16 * NQ * WQ><<<blocks, 256, 0, st>>>(p);
}

template <int D>
void br_kv_attend_dim(const BrKvAttend &p, int tile, bool fp8, int cus, hipStream_t st) {
  const int blocks = 2 * cus < BR_KV_SPLIT_WGS ? 2 * cus : BR_KV_SPLIT_WGS;
  if (tile == BR_KV_TILE_16) br_kv_attend_tile<D, 1, 1>(p, fp8, blocks, st);
  else if (tile == BR_KV_TILE_32) br_kv_attend_tile<D, 2, 1>(p, fp8, blocks, st);
  else br_kv_attend_tile<D, 2, 4>(p, fp8, blocks, st);
}

#endif
