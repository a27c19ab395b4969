// Attention over the 8-bit block cache (br_kv_attend).
//
// o = sum_j e^(s_j - m) vs_j v_j / sum_j e^(s_j - m),  s_j = scale ks_j (q . k_j), over the visible cached tokens j; k_j, v_j are
// codes, ks_j, vs_j the scales of j's block and head.  One pass over the tokens with a running m.
//
// Work: a tile is 64 cached tokens of one row and key head against TQ query rows (query tokens x heads of the group).  All tiles
// of the call, in the order (row, key head, query tile, token tile), are dealt to the waves in equal runs, whatever the lengths.  A
// run may end inside a query tile's tokens: pieces of a block's waves are joined in LDS at its end, pieces of several blocks go to
// memory, where the last block to arrive joins them in the order of their tokens, so that the result does not depend on who that was.
//
// A wave's tile on the matrix units, 16x16x32 in f16 (codes are exact there; the queries are scaled to 1..2 by a power of two per
// row, so they are too unless they span more than f16's exponents):
//   S^T [token][query] = K Q^T: row i of the t-th of four products is token 16 (i / 4) + 4 t + i % 4, so that lane (query n, g)
//     holds tokens 16 g .. 16 g + 15 of the tile, which one block covers: one ks and one vs per lane;
//   O^T [channel][query] += V^T P^T: the weights of lane (n, g) are this product's operand as they stand, and the values come as
//     16 bytes of 16 consecutive tokens of a channel (the cache keeps them that way round).
// Nothing passes between lanes but the maxima.  Weights go to f16 as 512 e^(s - m) vs / c, where c is a power of two about the largest product
// e^(s - m) vs that the query has seen so far: 11 bits, where the codes have 4 or 8, of every weight down to 2^-22 of the largest, and none is
// off by more than 2^-33 of it, whatever the scales are; sums stay in 32 bits.  m and c are the query's own (what another query of
// the tile sees has no say in them) and only move when e^(s - m) would pass 2^4 or a product 2^5 c: the sums are rescaled a few times a row.
#ifndef BR_KV_ATTEND_H
#define BR_KV_ATTEND_H

#include "br_kv_device.h"

#define BR_KV_NEG (-__builtin_inff())
#define BR_KV_LEAST_TILES 8  // of a block with many query rows: its pieces are large

struct BrKvRow {
  int n, len, start;  // query tokens, cached tokens, first token
};

// (a row that is not this launch's has no queries here)
__device__ __forceinline__ BrKvRow br_kv_row(const BrKvAttend &p, int r) {
  BrKvRow w;
  w.n = p.count ? min(max(p.count[r], 0), p.n_tokens) : 1;
  if (w.n < p.least || w.n > p.most) w.n = 0;
  w.start = p.start ? p.start[r] : r;
  w.len = min(max(p.lens[r], 0), p.max_blocks << p.shift);
  return w;
}

// Query token of a query row: row / group, by a multiplication.
__device__ __forceinline__ int br_kv_token(const BrKvAttend &p, int row) { return (int)((__umulhi(p.group_mul, (unsigned)row) + (unsigned)row) >> p.group_shift); }

// First token tile of a query tile, one past the last, and what it counts in the division of the work: a tile that sees nothing still has
// zeros to write.
template <int TQ>
__device__ __forceinline__ int br_kv_span(const BrKvAttend &p, const BrKvRow &w, int qi, int &t0, int &t1) {
  const int i0 = br_kv_token(p, qi * TQ), i1 = min(w.n - 1, br_kv_token(p, qi * TQ + TQ - 1)), at = w.len - w.n;
  const int hi = max(0, at + i1 + 1), lo = p.window > 0 ? max(0, max(at + i0, 0) - p.window + 1) : 0;
  t0 = lo / BR_KV_TILE;
  t1 = max(t0, (hi + BR_KV_TILE - 1) / BR_KV_TILE);
  return max(1, t1 - t0);
}

// Query tiles of one row and key head; the token tiles of every `step`-th from `first` on, and the most that one of them has.
template <int TQ>
__device__ __forceinline__ int br_kv_row_tiles(const BrKvAttend &p, const BrKvRow &w, long long &tiles, int &most, int first = 0, int step = 1) {
  const int nq = (int)(((long long)w.n * p.group + TQ - 1) / TQ);
  tiles = 0, most = 0;
  for (int qi = first; qi < nq; qi += step) {
    int t0, t1;
    const int size = br_kv_span<TQ>(p, w, qi, t0, t1);
    tiles += size, most = max(most, size);
  }
  return nq;
}

// 16 codes; ONCE: that nobody else of the launch reads
template <bool ONCE>
__device__ __forceinline__ uint4 br_kv_load16(const unsigned char *at) {
  typedef unsigned u4 __attribute__((ext_vector_type(4)));
  const u4 x = ONCE ? __builtin_nontemporal_load((const u4 *)at) : *(const u4 *)at;
  return make_uint4(x[0], x[1], x[2], x[3]);
}

// One query row's place in the output: its 4 N channels d, d + 16, ..., of the lane, times inv.
template <int N>
__device__ __forceinline__ void br_kv_store(const BrKvAttend &p, const BrKvRow &w, int h, int ri, int d, const br_f4 (&x)[N], float inv) {
  const int i = br_kv_token(p, ri), t = w.start + i;
  if (i >= w.n || t < 0 || t >= p.n_tokens) return;
  unsigned short *at = p.out + (long long)t * p.out_token + (long long)(h * p.group + ri - i * p.group) * p.out_head + d;
  uint2 y[N];
  if (p.bf16) {
#pragma unroll
    for (int k = 0; k < N; ++k) y[k] = make_uint2(br_kv_pair<__bf16>(x[k][0] * inv, x[k][1] * inv), br_kv_pair<__bf16>(x[k][2] * inv, x[k][3] * inv));
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) y[k] = make_uint2(br_kv_pair<_Float16>(x[k][0] * inv, x[k][1] * inv), br_kv_pair<_Float16>(x[k][2] * inv, x[k][3] * inv));
  }
  if (p.out_wide) {
#pragma unroll
    for (int k = 0; k < N; ++k) *(uint2 *)(at + 16 * k) = y[k];
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      at[16 * k] = (unsigned short)y[k].x, at[16 * k + 1] = (unsigned short)(y[k].x >> 16), at[16 * k + 2] = (unsigned short)y[k].y, at[16 * k + 3] = (unsigned short)(y[k].y >> 16);
  }
}

__device__ __forceinline__ void br_kv_store_lse(const BrKvAttend &p, const BrKvRow &w, int h, int ri, float m, float l) {
  const int i = br_kv_token(p, ri), t = w.start + i;
  if (!p.lse || i >= w.n || t < 0 || t >= p.n_tokens) return;
  p.lse[(long long)t * p.kv_heads * p.group + h * p.group + ri - i * p.group] = l == 0.0f ? BR_KV_NEG : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

// Pieces go from block to block past the L2s that the XCDs do not share; the writer waits for its stores before it says that it has
// delivered.  (Plain stores between fences of the device cost more than the attention: the fences empty whole L2s, 144 rows 390 us.)
// Sums go 16 bytes a lane, in the order in which the lanes have them: piece after piece of TQ rows, 16 rows' channels 16 d + 4 g
// .. + 3 side by side; of a query tile of fewer rows, so many.  (8 bytes at a time, row after row, every store is half of each of
// 16 lines: 48 rows of 80 queries and 7 key heads of 256 channels 112 us.)
template <int D, int TQ>
struct BrKvPieces {
  typedef unsigned u4 __attribute__((ext_vector_type(4)));
  static constexpr int PAST_L2 = 16;  // (sc1)
  __amdgpu_buffer_rsrc_t all;
  int rows, n16;  // rows side by side
  __device__ __forceinline__ BrKvPieces(const BrKvAttend &p, int rows_q)
      : all(__builtin_amdgcn_make_buffer_rsrc(p.part, 0, 2 * BR_KV_SPLIT_WGS_OF(D) * TQ * D * 4, 0x00020000)), rows(min(rows_q, 16)), n16((rows_q + 15) / 16) {}
  __device__ __forceinline__ int items() const { return n16 * (D / 4) * rows; }
  __device__ __forceinline__ int item(int x, int d, int g, int n) const { return ((x * (D / 16) + d) * 4 + g) * rows + n; }
  // row and first channel of an item
  __device__ __forceinline__ void place(int item, int &row, int &channel) const {
    const int c = rows == 16 ? item >> 4 : (int)((unsigned)item / (unsigned)rows), x = c / (D / 4);
    row = 16 * x + item - c * rows, channel = 4 * (c - x * (D / 4));
  }
  __device__ __forceinline__ void put(int piece, int item, br_f4 y) const {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, y), all, (piece * (TQ * D / 4) + item) * 16, 0, PAST_L2);
  }
  __device__ __forceinline__ br_f4 get(int piece, int item) const {
    return __builtin_bit_cast(br_f4, __builtin_amdgcn_raw_buffer_load_b128(all, (piece * (TQ * D / 4) + item) * 16, 0, PAST_L2));
  }
};

__device__ __forceinline__ void br_kv_put2(float *at, float x, float y) {
  __hip_atomic_store((unsigned long long *)at, (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ float2 br_kv_get2(const float *at) {
  const unsigned long long x = __hip_atomic_load((const unsigned long long *)at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((unsigned)x), __uint_as_float((unsigned)(x >> 32)));
}

__device__ __forceinline__ void br_kv_stores_done() {
  __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Sums of one wave over some tokens of 16 NQ query rows: o [channel 16 d + 4 g + j][row 16 x + n] (to be multiplied by c), l the sum of
// weights, both of e^(s - m), m in powers of two (0 where nothing was seen).
template <int D, int NQ>
struct BrKvSums {
  // m is kept ROOM below the largest score, so that weights of 2^-126 and a scale of 2^126 meet in range; UNIT: a weight of 1 there is 1 / UNIT
  static constexpr float ROOM = 13.0f, UNIT = 0x1p-13f;
  static constexpr float ONE = 512.0f;  // what a product of c is in f16; products of 2^6 c are below its end
  br_f4 o[NQ][D / 16];
  float m[NQ], l[NQ], c[NQ];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      m[x] = BR_KV_NEG, l[x] = 0.0f, c[x] = 0x1p-106f;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) o[x][d] = br_f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
  }
  // behind the last tile: l of all the row's lanes, in weights of m; what o is to be multiplied by
  __device__ __forceinline__ void close();
};

__device__ __forceinline__ float br_kv_sum4(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <int D, int NQ>
__device__ __forceinline__ void BrKvSums<D, NQ>::close() {
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    l[x] = br_kv_sum4(l[x]) * UNIT;
    c[x] *= 1.0f / ONE;
    m[x] = m[x] == BR_KV_NEG ? 0.0f : m[x] + ROOM;
  }
}

// The queries of 16 NQ rows from row0 on in f16, one row's to four lanes: channels 64 i + 16 g .. + 15 of its row for each lane, then
// 8 g .. + 7 of the last 32; what their scores are multiplied by (in powers of two; never below zero), and their positions.
template <int D, int NQ>
struct BrKvQueries {
  static constexpr int NI = D / 64, NK = D / 32;
  br_h8 qf[NQ][NK];
  float qs[NQ];
  int pos[NQ];

  template <class Fn>
  __device__ __forceinline__ void load(const BrKvAttend &p, const BrKvRow &w, int h, int row0, Fn &&meanwhile) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      const int ri = row0 + 16 * x + n, i = br_kv_token(p, ri), t = w.start + i;
      const bool in = i < w.n && t >= 0 && t < p.n_tokens;
      pos[x] = in ? max(w.len - w.n + i, -1) : -1;
      const unsigned short *at = p.q + (in ? (long long)t * p.q_token + (long long)(h * p.group + ri - i * p.group) * p.q_head : 0);
      uint4 e[NK];
      auto channel = [&](int c) { return c < 2 * NI ? (c / 2) * 64 + g * 16 + (c & 1) * 8 : NI * 64 + g * 8; };
      if (p.q_wide) {
#pragma unroll
        for (int c = 0; c < NK; ++c) e[c] = *(const uint4 *)(at + channel(c));
      } else {
#pragma unroll
        for (int c = 0; c < NK; ++c) {
          const unsigned short *y = at + channel(c);
          e[c] = make_uint4(y[0] | (unsigned)y[1] << 16, y[2] | (unsigned)y[3] << 16, y[4] | (unsigned)y[5] << 16, y[6] | (unsigned)y[7] << 16);
        }
      }
      if (x == 0) meanwhile();
      float f[NK * 8], top = 0.0f;
      auto half = [&](int c) {
        const uint4 y = e[c / 8];
        const unsigned z = c % 8 < 2 ? y.x : c % 8 < 4 ? y.y : c % 8 < 6 ? y.z : y.w;
        return (unsigned short)(c & 1 ? z >> 16 : z);
      };
      if (p.bf16) {
#pragma unroll
        for (int c = 0; c < 8 * NK; ++c) f[c] = br_kv_bf16(half(c));
      } else {
#pragma unroll
        for (int c = 0; c < 8 * NK; ++c) f[c] = br_kv_f16(half(c));
      }
      // (a row of the tile that is none takes the first one's values: its results go nowhere)
#pragma unroll
      for (int c = 0; c < 8 * NK; ++c) top = fmaxf(top, fabsf(f[c]));
      top = br_kv_max4(top);
      // the power of two at or below `top`; not below 2^-100, where its inverse would leave the range
      const int ex = max((int)(__float_as_uint(top) >> 23), 27);
      const float inv = __builtin_copysignf(__uint_as_float((unsigned)(254 - min(ex, 253)) << 23), p.scale2);
      qs[x] = top > 3.0e38f && top * 0.0f != 0.0f ? __builtin_nanf("") : __uint_as_float((unsigned)min(ex, 253) << 23) * fabsf(p.scale2);
#pragma unroll
      for (int c = 0; c < 8 * NK; ++c) qf[x][c / 8][c % 8] = (_Float16)(f[c] * inv);
    }
  }
};

// Weights of a tile from its scores: s [16 tokens 4 y + i of the lane's group][query n of group x]; ks, vs the scales of the lane's tokens,
// `have` of them; exist: all of the tile's blocks do.  Moves m and c, and the sums with them.
template <int D, int NQ>
__device__ __forceinline__ void br_kv_weights(const BrKvAttend &p, const BrKvQueries<D, NQ> &q, const br_f4 (&s)[NQ][4], float ks, float vs, int have, int t, int first_pos,
                                              int last_pos, bool exist, BrKvSums<D, NQ> &sums, br_h8 (&pf)[NQ][2]) {
  constexpr int ND = D / 16;
  constexpr float ROOM = BrKvSums<D, NQ>::ROOM, UNIT = BrKvSums<D, NQ>::UNIT;
  const int token = t * BR_KV_TILE + 16 * ((threadIdx.x & 63) >> 4);
  auto &o = sums.o;
  auto &m = sums.m;
  auto &l = sums.l;
  auto &c = sums.c;
  const float vmax = br_kv_max4(have > 0 ? vs : 0.0f);  // (of who sees what is asked below, where it matters)
  // inside: every query of the tile sees all of its tokens, and all exist
  const bool inside = t * BR_KV_TILE + BR_KV_TILE - 1 <= first_pos && (p.window == 0 || t * BR_KV_TILE > last_pos - p.window) && exist;
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    float f = q.qs[x] * ks;  // (not below zero: the sign of the caller's scale is in the queries)
    float z[16], mx = BR_KV_NEG, vx = vs;
#pragma unroll
    for (int j = 0; j < 16; ++j) z[j] = s[x][j >> 2][j & 3];
    if (!inside) {  // of the lane's tokens, those from `lo` on, `seen` of them
      const int lo = p.window > 0 ? max(q.pos[x] - p.window + 1 - token, 0) : 0, seen = max(min(have, q.pos[x] + 1 - token) - lo, 0);
#pragma unroll
      for (int j = 0; j < 16; ++j) z[j] = (unsigned)(j - lo) < (unsigned)seen ? z[j] * f : BR_KV_NEG;
      f = 1.0f;
      vx = seen > 0 ? vs : 0.0f;  // (a block that is not seen has no weight, whatever its scale)
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) mx = fmaxf(mx, z[j]);
    const float all = br_kv_max4(mx * f);
    const bool up = all > m[x] + (ROOM + 4.0f);
    const bool large = fabsf(all) > 0x1p22f;
    // (without any of these no product passes 2^6 c, whatever the tile's scores)
    if (__any(up | (vmax > 4.0f * c[x]) | large)) {
      // (where rounding moves a score by more than those 4, the rounded ones go against m, which is one of them)
      const float g = large ? f : 1.0f;
      f = large ? 1.0f : f;
      mx *= g;
#pragma unroll
      for (int j = 0; j < 16; ++j) z[j] *= g;
      const float to = up ? all - ROOM : m[x], al = m[x] == BR_KV_NEG ? (l[x] != 0.0f ? 1.0f : 0.0f) : __builtin_amdgcn_exp2f(m[x] - to), was = c[x] * al;
      const float top = br_kv_max4(__builtin_amdgcn_exp2f(__builtin_fmaf(mx, f, to == BR_KV_NEG ? 0.0f : -to)) * UNIT * vx);  // the tile's largest product
      // c falls as the sums do (to a power of two below: what is larger than c already is in 32 bits), so that it is the largest product's still
      const unsigned e = min(max(max(__float_as_uint(was) >> 23 & 255u, (__float_as_uint(top) >> 23 & 255u) + 1), 21u), 253u);
      c[x] = __uint_as_float(up | top > 32.0f * c[x] ? e << 23 : __float_as_uint(c[x]));
      const float ao = was * __uint_as_float(0x7f000000u - __float_as_uint(c[x]));
      m[x] = to;
      l[x] *= al;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[x][d][j] *= ao;
    }
    __asm__("" : "+v"(m[x]), "+v"(c[x]));  // (or what follows is partly done on both ways here, and all sums are moved for the shorter one)
    const float ref = m[x] == BR_KV_NEG ? 0.0f : m[x];
    // (a scale far above c has weights that are next to nothing: their product stays in range, and a scale of NaN one)
    float wx = vx * (BrKvSums<D, NQ>::ONE * UNIT * __uint_as_float(0x7f000000u - __float_as_uint(c[x])));
    wx = wx > 3.0e38f ? 3.0e38f : wx;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j], f, -ref));
      l[x] += e;
      pf[x][j >> 3][j & 7] = (_Float16)(e * wx);
    }
  }
}

// ONCE: nobody else reads these codes; ONCE_V: nor these values' lines (blocks of 128 tokens have two tiles' in one).
// Token tiles t .. stop - 1 of row r and key head h for the query rows from row0 on, whose positions lie in first_pos .. last_pos.
template <int D, int NQ, bool FP8, bool ONCE_V, bool ONCE>
__device__ __forceinline__ void br_kv_tiles(const BrKvAttend &p, BrKvRow w0, int r, int h, int row0, int first_pos, int last_pos, int t, int stop,
                                            BrKvSums<D, NQ> &sums) {
  constexpr int NI = D / 64, REST = D % 64 / 32, NK = 2 * NI + REST, ND = D / 16;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  // (what is the same for the wave, in scalar registers)
  auto scalar = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  w0.n = scalar(w0.n), w0.len = scalar(w0.len), w0.start = scalar(w0.start);
  r = scalar(r), h = scalar(h), row0 = scalar(row0), first_pos = scalar(first_pos), last_pos = scalar(last_pos), t = scalar(t), stop = scalar(stop);
  const BrKvRow &w = w0;
  auto &o = sums.o;
  sums.clear();

  const int worker = r / p.rows;
  const int *table = p.table + (long long)r * p.max_blocks;
  const int last_block = max(0, (w.len - 1) >> p.shift);
  const long long cache0 = (long long)worker * p.n_blocks;
  const int mask = (1 << p.shift) - 1;
  const int kg = n >> 2, kr = n & 3;  // the token group, and the place in fours, of the lane's row of K

  uint4 kc[4][NI + (NI == 0)];
  uint2 kx[4];
  uint4 vc[ND];
  // block of a lane's 16 tokens, as the table has it; where it is read, one that does not exist is block 0
  auto id_of = [&](int token) { return table[min(token >> p.shift, last_block)]; };
  auto there = [&](int id) { return (unsigned)id < (unsigned)p.n_blocks; };
  auto load_k = [&](int t, int id, bool live) {
    const unsigned char *at =
        live ? p.k + ((((cache0 + (there(id) ? id : 0)) * p.kv_heads + h) << p.shift) + ((t * BR_KV_TILE + 16 * kg) & mask) + kr) * D : p.k;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
#pragma unroll
      for (int i = 0; i < NI; ++i) kc[s][i] = br_kv_load16<ONCE>(at + 4 * s * D + 64 * i + 16 * g);
      if (REST) kx[s] = *(const uint2 *)(at + 4 * s * D + 64 * NI + 8 * g);
    }
  };

  // Codes of K are asked for a tile ahead, scales too, ids two ahead, always, behind a wave's last tile for the cache's first
  // lines: loads under a branch would make every wait one for all of them (144 rows of 8 key heads, 666 MB: 195 us).
  int kid1 = 0, vid = 0, vid1 = 0;
  float ks1 = 0.0f, vs1 = 0.0f;
  auto load_scales = [&](int id) {
    const long long at = (cache0 + (there(id) ? id : 0)) * p.kv_heads + h;
    ks1 = p.ks[at], vs1 = p.vs[at];
  };
  const bool t_any = t < stop;
  int kid = 0;
  if (t_any) {
    const int next = t + 1 < stop ? t + 1 : t;
    kid = id_of(t * BR_KV_TILE + 16 * kg), vid = id_of(t * BR_KV_TILE + 16 * g);
    kid1 = id_of(next * BR_KV_TILE + 16 * kg), vid1 = id_of(next * BR_KV_TILE + 16 * g);
  }
  auto load_first = [&]() {
    load_k(t, kid, true);
    load_scales(vid);
  };
  BrKvQueries<D, NQ> q;
  q.load(p, w, h, row0, [&] {
    if (t_any) load_first();  // (while the queries are on their way)
  });

  for (; t < stop; ++t) {
    const int token = t * BR_KV_TILE + 16 * g;  // of the lane's first weight
    {
      const unsigned char *at = p.v + ((((cache0 + (there(vid) ? vid : 0)) * p.kv_heads + h) * D + n) << p.shift) + (token & mask);
#pragma unroll
      for (int d = 0; d < ND; ++d) vc[d] = br_kv_load16<ONCE_V>(at + ((16 * d) << p.shift));
    }
    const float ks = there(vid) ? br_kv_sound(ks1) : 0.0f, vs = there(vid) ? br_kv_sound(vs1) : 0.0f;
    const int have = there(vid) ? min(max(w.len - token, 0), 16) : 0;  // of the lane's tokens, those that exist

    br_f4 s[NQ][4];
#pragma unroll
    for (int x = 0; x < NQ; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y) s[x][y] = br_f4{0.0f, 0.0f, 0.0f, 0.0f};
    // (products into one sum do not follow each other directly)
#pragma unroll
    for (int c = 0; c < NK; ++c) {
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        br_h8 kf;
        if (c < 2 * NI) kf = c & 1 ? br_kv_decode8<FP8>(kc[y][c / 2].z, kc[y][c / 2].w) : br_kv_decode8<FP8>(kc[y][c / 2].x, kc[y][c / 2].y);
        else kf = br_kv_decode8<FP8>(kx[y].x, kx[y].y);
#pragma unroll
        for (int x = 0; x < NQ; ++x) s[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, q.qf[x][c], s[x][y], 0, 0, 0);
      }
    }
    const int next = t + 1 < stop ? t + 1 : t, after = next + 1 < stop ? next + 1 : next;
    load_k(next, kid1, t + 1 < stop);
    load_scales(vid1);
    kid1 = id_of(after * BR_KV_TILE + 16 * kg);
    const int vid2 = id_of(after * BR_KV_TILE + 16 * g);


    br_h8 pf[NQ][2];
    br_kv_weights<D, NQ>(p, q, s, ks, vs, have, t, first_pos, last_pos, !__any(!there(vid)), sums, pf);
    // bytes behind the row's end are whatever memory held: an 8-bit float may be a NaN there
    if (FP8 && __any(have < 16)) {
      const unsigned long long full = ~0ull;
      const unsigned long long m0 = have >= 8 ? full : ~(full << (8 * have));
      const unsigned long long m1 = have >= 16 ? full : have <= 8 ? 0ull : ~(full << (8 * (have - 8)));
#pragma unroll
      for (int d = 0; d < ND; ++d) vc[d].x &= (unsigned)m0, vc[d].y &= (unsigned)(m0 >> 32), vc[d].z &= (unsigned)m1, vc[d].w &= (unsigned)(m1 >> 32);
    }
#pragma unroll
    for (int d0 = 0; d0 < ND; d0 += 2) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = d0; d < d0 + 2; ++d) {
          const br_h8 v = k ? br_kv_decode8<FP8>(vc[d].z, vc[d].w) : br_kv_decode8<FP8>(vc[d].x, vc[d].y);
#pragma unroll
          for (int x = 0; x < NQ; ++x) o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pf[x][k], o[x][d], 0, 0, 0);
        }
    }
    vid = vid1, vid1 = vid2;
  }
  sums.close();
}

// Joins the pieces of a query tile, of blocks first .. first + parts - 1, into its result (all of the block's threads; sums and ml: NT of
// each in LDS).  A thread has four channels of a row; where those are less than half of the threads the pieces are shared out as
// well.  One way to memory and back: each thread weighs its pieces against the largest maximum among them.
template <int D, int TQ, int NT>
__device__ __forceinline__ void br_kv_join(const BrKvAttend &p, const BrKvRow &w, int h, int qi, int rows_q, int first, int parts, br_f4 *sums, float2 *ml) {
  // few rows have many pieces (up to a block of the launch each), many rows few: places asked for at once are AT_ONCE pieces of ROWS rows
  constexpr int ROWS = TQ > 64 ? 8 : TQ > 32 ? 4 : 1, AT_ONCE = TQ > 32 ? 2 : 8, STEP = NT * ROWS;
  const BrKvPieces<D, TQ> pieces(p, rows_q);
  const int tid = threadIdx.x, items = pieces.items(), S = items < NT ? max(1, NT / items) : 1;
  for (int at0 = tid; at0 < max(items, NT); at0 += STEP) {
    br_f4 ys[ROWS];
    float ms[ROWS], ls[ROWS];
#pragma unroll
    for (int q = 0; q < ROWS; ++q) ys[q] = br_f4{0.0f, 0.0f, 0.0f, 0.0f}, ms[q] = ls[q] = 0.0f;
    const int k0 = at0 / items;
    for (int k = k0; k < (k0 < S ? parts : 0); k += S * AT_ONCE) {
      float2 x[ROWS][AT_ONCE];
      br_f4 v[ROWS][AT_ONCE];
#pragma unroll
      for (int q = 0; q < ROWS; ++q) {
        const int it = S > 1 ? at0 % items : min(at0 + q * NT, items - 1);
        int row, d;
        pieces.place(it, row, d);
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
          const int kk = min(k + j * S, parts - 1);
          const int piece = kk ? 2 * (first + kk) : 2 * first + 1;
          x[q][j] = br_kv_get2(p.ml + (piece * TQ + row) * 2);
          v[q][j] = pieces.get(piece, it);
        }
      }
#pragma unroll
      for (int q = 0; q < ROWS; ++q) {
        br_f4 &y = ys[q];
        float &m = ms[q], &l = ls[q], top = l != 0.0f ? m : BR_KV_NEG;
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
          if (k + j * S >= parts) x[q][j].y = 0.0f;
          if (x[q][j].y != 0.0f) top = fmaxf(top, x[q][j].x);
        }
        const float e0 = l != 0.0f ? __builtin_amdgcn_exp2f(m - top) : 0.0f;
        l *= e0;
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] *= e0;
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
          if (x[q][j].y == 0.0f) continue;
          const float e = __builtin_amdgcn_exp2f(x[q][j].x - top);
          l += x[q][j].y * e;
#pragma unroll
          for (int c = 0; c < 4; ++c) y[c] = __builtin_fmaf(v[q][j][c], e, y[c]);
        }
        m = top == BR_KV_NEG ? 0.0f : top;
      }
    }
    br_f4 y = ys[0];
    float m = ms[0], l = ls[0];
    if (S > 1) {
      sums[tid] = y, ml[tid] = make_float2(m, l);
      __syncthreads();
      if (k0 == 0) {
        float top = BR_KV_NEG;
        for (int k = 0; k < S; ++k)
          if (ml[tid + k * items].y != 0.0f) top = fmaxf(top, ml[tid + k * items].x);
        y = br_f4{0.0f, 0.0f, 0.0f, 0.0f};
        l = 0.0f;
        for (int k = 0; k < S; ++k) {
          const float2 x = ml[tid + k * items];
          if (x.y == 0.0f) continue;
          const float e = __builtin_amdgcn_exp2f(x.x - top);
          const br_f4 v = sums[tid + k * items];
          l += x.y * e;
#pragma unroll
          for (int c = 0; c < 4; ++c) y[c] += v[c] * e;
        }
        m = top;
      }
    }
    ys[0] = y, ms[0] = m, ls[0] = l;
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      const int it = at0 + q * NT;
      if (it >= items) continue;
      int row, d;
      pieces.place(it, row, d);
      if (row >= rows_q) continue;
      const br_f4 one[1] = {ys[q]};
      br_kv_store<1>(p, w, h, qi * TQ + row, d, one, ls[q] != 0.0f ? 1.0f / ls[q] : 0.0f);
      if (d == 0) br_kv_store_lse(p, w, h, qi * TQ + row, ms[q], ls[q]);
    }
  }
}

// What is the same for the wave, in scalar registers
template <class T>
__device__ __forceinline__ T br_kv_scalar(T x) {
  if constexpr (sizeof(T) == 8) return (T)((unsigned long long)br_kv_scalar((unsigned)((unsigned long long)x >> 32)) << 32 | br_kv_scalar((unsigned)x));
  else return (T)__builtin_amdgcn_readfirstlane((int)x);
}

// The division of a call's tiles among `workers` (waves, groups of waves, or blocks: NR to a block).  Where there are few query tiles and
// none is much longer than an equal share, each goes to a block, in NR parts: nothing is left to be joined through memory, which
// takes about as long as SLACK tiles.  Else the workers get runs of tiles that differ by one at most.  What is dealt are units: tiles, or a
// query tile's NR parts.
template <int TQ, int NT, int NR, int SLACK>
struct BrKvRuns {
  static constexpr bool MANY = TQ > 64;  // a row may well have more than one query tile
  struct Shared {
    long long before[NT + 1], wave_sum[NT / 64];
    int wave_parts[NT / 64], wave_most[NT / 64];
    int4 row[NT];
  };
  Shared &s;
  long long all;
  unsigned share, extra;  // a worker has `share` units, and extra / 2^32 of one more
  int per, workers;
  bool parts;  // the units are parts of query tiles
  int log_per_row;  // 2^.. threads count a row's tiles (chunks of thousands of query rows have many: one thread 5 us); the first has the sum

  // (a worker gets at least `least` tiles, if there are as many)
  __device__ __forceinline__ BrKvRuns(const BrKvAttend &p, Shared &sh, int blocks, int least) : s(sh) {
    const int tid = threadIdx.x, lane = tid & 63;
    per = (p.n_rows + NT - 1) / NT;
    log_per_row = MANY && per == 1 ? min(__builtin_ctz(NT) - (p.n_rows > 1 ? 32 - __builtin_clz(p.n_rows - 1) : 0), 6) : 0;
    const int at = tid >> log_per_row, one = tid & ((1 << log_per_row) - 1);
    long long mine = 0;
    int mine_q = 0, most = 0;
    for (int r = at * per; r < min(p.n_rows, (at + 1) * per); ++r) {
      const BrKvRow w = br_kv_row(p, r);
      s.row[at] = make_int4(w.n, w.len, w.start, 0);
      if (w.n <= 0) continue;
      long long tiles;
      int longest;
      mine_q = min(mine_q + br_kv_row_tiles<TQ>(p, w, tiles, longest, one, 1 << log_per_row), 4096);
      mine += tiles, most = max(most, longest);
    }
    if (MANY) {
      for (int d = 1; d < 1 << log_per_row; d <<= 1) mine += __shfl_xor(mine, d, 64);
      if (one) mine = 0, mine_q = 0;
    }
    mine *= p.kv_heads;
    // (query tiles as far as they could go to a block each)
    mine_q *= p.kv_heads * NR;
    long long sum = mine;
    mine_q = min(mine_q, 1 << 20);
    const int sum_lane = br_kv_wave_scan(mine_q);
    most = (int)br_kv_max64((float)most);
    if (!__any(mine >> 24 != 0)) {
      sum = br_kv_wave_scan((int)mine);
    } else {  // (sums beyond 32 bits)
      for (int d = 1; d < 64; d <<= 1) {
        const long long o = __shfl_up(sum, d, 64);
        if (lane >= d) sum += o;
      }
    }
    int sum_q = sum_lane;
    if (lane == 63) s.wave_sum[tid >> 6] = sum, s.wave_parts[tid >> 6] = sum_q, s.wave_most[tid >> 6] = most;
    __syncthreads();
    long long total = 0;
    int total_q = 0;
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) {
      if (k < (tid >> 6)) sum += s.wave_sum[k], sum_q += s.wave_parts[k];
      total += s.wave_sum[k], total_q += s.wave_parts[k], most = max(most, s.wave_most[k]);
    }
    const int workers_most = blocks * NR;
    workers = total >= (long long)workers_most * least ? workers_most : max(1, (int)total / least);
    long long q = (long long)((double)total * (1.0 / workers)), left = total - q * workers;  // (exact behind the step up or down)
    if (left < 0) --q, left += workers;
    if (left >= workers) ++q, left -= workers;
    // (those with one more are spread evenly: one row of 40960 tokens, the first half of the blocks 24 tiles and the others 16, not 20
    // each: 34 us)
    share = (unsigned)q, extra = (unsigned)((double)left * 4294967296.0 * (1.0 / workers) + 0.5);
    all = total;
    parts = total_q <= workers_most && (most + NR - 1) / NR <= (int)min(q, 1ll << 20) + SLACK;
    if (parts) workers = total_q, all = total_q, share = 1, extra = 0, sum = sum_q;
    share = br_kv_scalar(share), extra = br_kv_scalar(extra), workers = br_kv_scalar(workers), all = br_kv_scalar(all);
    s.before[tid + 1] = sum;
    if (tid == 0) s.before[0] = 0;
    __syncthreads();
  }
  // units of one row and key head, and of one query tile of `size` tiles
  __device__ __forceinline__ long long units_of(const BrKvAttend &p, const BrKvRow &w) const {
    if (w.n <= 0) return 0;
    long long tiles;
    int most;
    if (parts) return (int)(((long long)w.n * p.group + TQ - 1) / TQ) * NR;
    if (MANY) {
      br_kv_row_tiles<TQ>(p, w, tiles, most, threadIdx.x & 63, 64);
      for (int d = 1; d < 64; d <<= 1) tiles += __shfl_xor(tiles, d, 64);
    } else {
      br_kv_row_tiles<TQ>(p, w, tiles, most);
    }
    return tiles;
  }
  __device__ __forceinline__ int units_of(int size) const { return parts ? NR : size; }
  __device__ __forceinline__ long long begin_of(int k) const {
    const long long at = (long long)((unsigned long long)(unsigned)k * share + __umulhi((unsigned)k, extra));
    return k < workers ? at : all;
  }
  // The thread in whose rows tile u is: every lane looks at NT / 64 threads' ends, then at one of them.
  __device__ __forceinline__ int find(long long u) const {
    constexpr int PER_LANE = NT / 64;
    const int lane = threadIdx.x & 63;
    const int chunk = __popcll(__ballot(s.before[(lane + 1) * PER_LANE] <= u)) * PER_LANE;
    return chunk + __popcll(__ballot(lane < PER_LANE && s.before[min(chunk + lane + 1, NT)] <= u));
  }
  // The last worker that begins at x or before (within one of what 24 bits say)
  __device__ __forceinline__ int owner_of(long long x) const {
    int k = min(max((int)((float)x * ((float)workers * __builtin_amdgcn_rcpf((float)all))), 0), workers - 1);
    while (k > 0 && begin_of(k) > x) --k;
    while (k + 1 < workers && begin_of(k + 1) <= x) ++k;
    return k;
  }
  __device__ __forceinline__ BrKvRow row_of(const BrKvAttend &p, int r) const {
    if (per > 1) return br_kv_row(p, r);
    const int4 x = s.row[r];
    return BrKvRow{x.x, x.y, x.z};
  }
};

// Where a run stands: query tile qi of row r and key head h, tiles t0 .. t1 - 1 of its tokens, the first of which is tile `seg` of the call.
template <int TQ, int NT, class Runs>
struct BrKvPlace {
  BrKvRow w;
  long long base, seg, tiles;
  int r, h, qi, size, t0, t1;  // size: units of the query tile

  __device__ __forceinline__ bool find(const BrKvAttend &p, const Runs &runs, long long u) {
    const int lo = runs.find(u);
    r = (lo >> runs.log_per_row) * runs.per;
    base = runs.s.before[lo];
    for (; r < p.n_rows; ++r) {
      w = runs.row_of(p, r);
      tiles = runs.units_of(p, w);
      if (u < base + tiles * p.kv_heads) break;
      base += tiles * p.kv_heads;
    }
    if (r >= p.n_rows) return false;  // (only if lengths were changed under the launch)
    h = (int)((float)(u - base) * __builtin_amdgcn_rcpf((float)tiles));
    while (h > 0 && u - base < h * tiles) --h;
    while (u - base >= (h + 1) * tiles) ++h;
    qi = 0;
    seg = base + h * tiles;
    if (Runs::MANY) {  // 64 query tiles at a time
      const int last = (int)(((long long)w.n * p.group + TQ - 1) / TQ) - 1;
      for (int k = 64; k == 64; qi += k) {
        const int sum = br_kv_wave_scan(runs.units_of(br_kv_span<TQ>(p, w, min(qi + (int)(threadIdx.x & 63), last), t0, t1)));
        k = __popcll(__ballot(seg + sum <= u));
        if (k > 0) seg += __shfl(sum, k - 1, 64);
      }
      size = runs.units_of(br_kv_span<TQ>(p, w, qi, t0, t1));
    } else {
      size = runs.units_of(br_kv_span<TQ>(p, w, 0, t0, t1));
      while (u >= seg + size) seg += size, size = runs.units_of(br_kv_span<TQ>(p, w, ++qi, t0, t1));
    }
    return true;
  }
  __device__ __forceinline__ bool next(const BrKvAttend &p, const Runs &runs) {
    seg += size;
    if (seg < base + (h + 1) * tiles) {
      ++qi;
    } else {
      qi = 0;
      if (++h == p.kv_heads) {
        h = 0;
        base += tiles * p.kv_heads;
        while (++r < p.n_rows) {
          w = runs.row_of(p, r);
          tiles = runs.units_of(p, w);
          if (tiles > 0) break;
        }
        if (r >= p.n_rows) return false;
      }
    }
    size = runs.units_of(br_kv_span<TQ>(p, w, qi, t0, t1));
    return true;
  }
  // the first tile of its unit k (one past the last, for k = size)
  __device__ __forceinline__ int tile_of(const Runs &runs, int k) const { return runs.parts ? t0 + (int)((long long)(t1 - t0) * k / size) : min(t0 + k, t1); }
  __device__ __forceinline__ int rows_q(const BrKvAttend &p) const { return (int)min((long long)TQ, (long long)w.n * p.group - (long long)qi * TQ); }
  // position of the query of that row of the tile, or of the last one; -1 of any before the row's first token
  __device__ __forceinline__ int pos_of(const BrKvAttend &p, int row) const { return max(w.len - w.n + min(w.n - 1, br_kv_token(p, qi * TQ + row)), -1); }
};

// A wave's result of query rows row.. of the tile, to its place, or as piece `piece` to memory
template <int D, int NQ, int TQ>
__device__ __forceinline__ void br_kv_result(const BrKvAttend &p, const BrKvRow &w, int h, int qi, int row, int rows_q, const BrKvSums<D, NQ> &s) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    const int at = row + 16 * x + n;
    if (at >= rows_q) continue;
    const float inv = s.l[x] != 0.0f ? s.c[x] / s.l[x] : 0.0f;
    br_kv_store<D / 16>(p, w, h, qi * TQ + at, 4 * g, s.o[x], inv);
    if (g == 0) br_kv_store_lse(p, w, h, qi * TQ + at, s.m[x], s.l[x]);
  }
}

template <int D, int NQ, int TQ>
__device__ __forceinline__ void br_kv_piece(const BrKvAttend &p, int piece, int row, int rows_q, const BrKvSums<D, NQ> &s) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const BrKvPieces<D, TQ> pieces(p, rows_q);
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    const int at = row + 16 * x + n;
    if (at >= rows_q) continue;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
      br_f4 y = s.o[x][d];
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] *= s.c[x];
      pieces.put(piece, pieces.item(row / 16 + x, d, g, n), y);
    }
    if (g == 0) br_kv_put2(p.ml + (piece * TQ + at) * 2, s.m[x], s.l[x]);
  }
}

// A query tile that several of a block's waves have pieces of: whose it is, and the blocks that have (`parts` 1: this one alone).
struct BrKvShare {
  int on, first, parts, r, h, qi;
};

// Few query rows: a run for each SHARE waves, which have 16 query rows each, NW waves to a block.  Pieces of a run (of a query tile that it
// takes up in the middle, and of one that goes on in the next run) wait in LDS until the block's end, where all waves join them,
// each its share of the channels.  Bound by memory: each code comes once from there (waves of one run find it in the caches).  144 rows
// of 256 to 8192 tokens, 8 key heads of 128 channels, groups of 8: 128 us, 691 MB = 5.4 TB/s (a large copy: 5.1).  One row of 40 thousand
// tokens: 26 us, 87 MB, of them some 6 us for the pieces' way through LDS and memory; one of 500 13 us, a launch and a chain
// of loads (lengths, ids, codes, the join).
template <int D, int SHARE, bool FP8, bool HALF, int NW, int WAVES>
__global__ __launch_bounds__(64 * NW, WAVES) void br_kv_k_attend(BrKvAttend p) {
  constexpr int TQ = 16 * SHARE, NT = 64 * NW, ND = D / 16, NR = NW / SHARE;  // NR: runs of a block
  using Runs = BrKvRuns<TQ, NT, NR, 6>;
  __shared__ typename Runs::Shared shared;
  __shared__ br_f4 kept[2 * NW * ND * 64];  // piece 2 k: taken up by run k, 2 k + 1: begun by it
  __shared__ float2 kept_ml[2 * NW * 16];
  __shared__ int goes_on[NR], arrived[2];
  __shared__ BrKvShare chains[NR + 1];  // of the query tile that run k has begun; the last: of one that an earlier block has
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), rn = wv / SHARE, row = 16 * (wv % SHARE);  // the wave's run, its first query row of the tile
  Runs runs(p, shared, gridDim.x, 1);
  // runs that follow each other go to one XCD (blocks go round them), which has what they share in its L2
  const int blocks = (runs.workers + NR - 1) / NR, b8 = blockIdx.x, wg = b8 < (blocks & ~7) ? (b8 & 7) * (blocks >> 3) + (b8 >> 3) : b8;
  if (wg >= blocks) return;
  if (tid <= NR) chains[tid].on = 0;
  __syncthreads();
  const int me = wg * NR + rn;
  long long u = runs.begin_of(me);
  const long long end = runs.begin_of(me + 1);

  bool open = false;  // the query tile that was taken up goes on in the next wave
  {
    BrKvPlace<TQ, NT, Runs> at;
    BrKvSums<D, 1> s;
    if (u < end && at.find(p, runs, u)) {
      for (;;) {
        const int a = (int)(u - at.seg), b = (int)min((long long)at.size, end - at.seg);
        const int rows_q = at.rows_q(p);
        br_kv_tiles<D, 1, FP8, SHARE == 1 && !HALF, SHARE == 1>(p, at.w, at.r, at.h, at.qi * TQ + row, at.pos_of(p, row), at.pos_of(p, row + 15), at.tile_of(runs, a),
                                                               row < rows_q ? at.tile_of(runs, b) : 0, s);
        if (a == 0 && b == at.size) {
          br_kv_result<D, 1, TQ>(p, at.w, at.h, at.qi, row, rows_q, s);
        } else {
          const int piece = (2 * rn + (a == 0)) * SHARE + wv % SHARE;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            br_f4 y = s.o[0][d];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] *= s.c[0];
            kept[(piece * ND + d) * 64 + lane] = y;
          }
          if (g == 0) kept_ml[piece * 16 + n] = make_float2(s.m[0], s.l[0]);
          open = a > 0 && b < at.size;
          if (row == 0 && (a == 0 || rn == 0)) {
            BrKvShare c = {1, wg, 1, at.r, at.h, at.qi};
            if (a > 0 || at.seg + at.size > runs.begin_of((wg + 1) * NR)) c.first = runs.owner_of(at.seg) / NR, c.parts = runs.owner_of(at.seg + at.size - 1) / NR - c.first + 1;
            if (lane == 0) chains[a == 0 ? rn : NR] = c;
          }
        }
        u = at.seg + b;
        if (u >= end || !at.next(p, runs)) break;
      }
    }
  }
  if (lane == 0 && row == 0) goes_on[rn] = open;
  __syncthreads();

  const unsigned on = (unsigned)__ballot(lane <= NR && chains[min(lane, NR)].on), going_on = (unsigned)__ballot(lane < NR && goes_on[min(lane, NR - 1)]);
#pragma unroll 1
  for (unsigned left = on; left; left &= left - 1) {
    const int c = __ffs(left) - 1;
    const BrKvShare chain = chains[c];
    const int k0 = c < NR ? c + 1 : 0;  // the chain: piece 2 c + 1 (c < NR), then the pieces taken up by runs k0 .. k1
    const int k1 = min(k0 + __ffs(~(going_on >> k0)) - 1, NR - 1);
    auto member = [&](int k) { return k < k0 ? 2 * c + 1 : 2 * k; };
    const int begin = c < NR ? k0 - 1 : k0;
    const BrKvRow w = runs.row_of(p, chain.r);
    const int rows_q = (int)min((long long)TQ, (long long)w.n * p.group - (long long)chain.qi * TQ);
    for (int it = wv; it < SHARE * ND; it += NW) {
      const int x = it / ND, d = it - x * ND, row = 16 * x + n;
      // (all asked for at once, the last one again for those that a chain may have and this one has not)
      float2 mls[NR + 1];
      br_f4 vs[NR + 1];
#pragma unroll
      for (int i = 0; i <= NR; ++i) {
        const int at = member(min(begin + i, k1)) * SHARE + x;
        mls[i] = kept_ml[at * 16 + n], vs[i] = kept[(at * ND + d) * 64 + lane];
      }
      float top = BR_KV_NEG, l = 0.0f;
#pragma unroll
      for (int i = 0; i <= NR; ++i)
        if (mls[i].y != 0.0f) top = fmaxf(top, mls[i].x);
      br_f4 y[1] = {{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
      for (int i = 0; i <= NR; ++i) {
        const float e = mls[i].y != 0.0f && begin + i <= k1 ? __builtin_amdgcn_exp2f(mls[i].x - top) : 0.0f;
        l += mls[i].y * e;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[0][j] = __builtin_fmaf(vs[i][j], e, y[0][j]);
      }
      if (row >= rows_q) continue;
      if (top == BR_KV_NEG) top = 0.0f;
      if (chain.parts == 1) {
        br_kv_store<1>(p, w, chain.h, chain.qi * TQ + row, 16 * d + 4 * g, y, l != 0.0f ? 1.0f / l : 0.0f);
        if (d == 0 && g == 0) br_kv_store_lse(p, w, chain.h, chain.qi * TQ + row, top, l);
      } else {
        const int piece = 2 * wg + (c < NR);
        const BrKvPieces<D, TQ> pieces(p, rows_q);
        pieces.put(piece, pieces.item(x, d, g, n), y[0]);
        if (d == 0 && g == 0) br_kv_put2(p.ml + (piece * TQ + row) * 2, top, l);
      }
    }
  }
  br_kv_stores_done();
  __syncthreads();
  // the query tiles that other blocks have pieces of: at most one of an earlier block, and one that goes on in a later one
  const unsigned going = (unsigned)__ballot(lane < NR && chains[min(lane, NR - 1)].on && chains[min(lane, NR - 1)].parts > 1);
  const bool goes = going != 0, came = on >> NR & 1;
  const int which = goes ? __ffs(going) - 1 : 0;
  if (!goes && !came) return;
  if (tid == 0 && came) arrived[0] = __hip_atomic_fetch_add(&p.arrived[chains[NR].first], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (tid == 1 && goes) arrived[1] = __hip_atomic_fetch_add(&p.arrived[chains[which].first], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    const BrKvShare c = chains[k ? which : NR];
    if ((k ? !goes : !came) || arrived[k] != c.parts - 1) continue;
    const BrKvRow w = runs.row_of(p, c.r);
    br_kv_join<D, TQ, NT>(p, w, c.h, c.qi, (int)min((long long)TQ, (long long)w.n * p.group - (long long)c.qi * TQ), c.first, c.parts, kept, (float2 *)(kept + NT));
    if (tid == 0) p.arrived[c.first] = 0;  // (for the next launch)
    __syncthreads();
  }
}

// Steps 0 .. N - 1 with four operands from LDS each, asked for AHEAD steps before.
template <int N, int AHEAD, class Get, class Use>
__device__ __forceinline__ void br_kv_ahead(Get &&get, Use &&use) {
  br_h8 f[AHEAD + 1][4];
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) get(k, f[k]);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (k + AHEAD < N) get(k + AHEAD, f[(k + AHEAD) % (AHEAD + 1)]);
    __builtin_amdgcn_sched_barrier(0);
    use(k, f[k % (AHEAD + 1)]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Many query rows: the block's four waves have 16 NQ each and go over the same tokens.  Each wave brings a quarter of a tile's codes to f16 and
// puts them into LDS as the matrix products take them (1 KB for each operand, 16 bytes a lane); two tiles there, one barrier a
// tile.  Bound by the issue of vector instructions between the products (310 a tile and wave, 32 of them exponentials, to 64 products): chunks
// of 512 tokens of two rows, groups of 4, 8 key heads of 128 channels behind up to 8192 tokens 207 us, 0.61 PFLOP/s; a wave issues in 44 %
// of its time and waits for its turn, beside the other wave of its SIMD, in 30 %; the matrix units are busy a third.
template <int D, int NQ, bool FP8, int WAVES>
__global__ __launch_bounds__(256, WAVES) void br_kv_k_attend_rows(BrKvAttend p) {
  constexpr int TQ = 64 * NQ, NT = 256, NI = D / 64, REST = D % 64 / 32, NK = D / 32, ND = D / 16, VG = (ND + 3) / 4, AHEAD = WAVES == 1 ? 2 : 1;  // VG: groups of 16 channels of values that a wave brings
  using Runs = BrKvRuns<TQ, NT, 1, 8>;
  __shared__ typename Runs::Shared shared;
  __shared__ br_h8 tile[2][(4 * NK + 2 * ND) * 64];
  __shared__ int arrived;
  const int tid = threadIdx.x, wv = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 15, g = lane >> 4;
  Runs runs(p, shared, gridDim.x, BR_KV_LEAST_TILES);
  const int blocks = runs.workers, b8 = blockIdx.x, wg = b8 < (blocks & ~7) ? (b8 & 7) * (blocks >> 3) + (b8 >> 3) : b8;
  if (wg >= blocks) return;
  long long u = runs.begin_of(wg);
  const long long end = runs.begin_of(wg + 1);
  BrKvPlace<TQ, NT, Runs> at;
  if (u >= end || !at.find(p, runs, u)) return;
  const int kg = n >> 2, kr = n & 3, mask = (1 << p.shift) - 1;
  // Of two blocks on a compute unit the one that came first would have its way, and be done long before the other: they go first in turns.
  const int turn = 2 * blockIdx.x >= gridDim.x;
  auto scalar = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  auto there = [&](int id) { return (unsigned)id < (unsigned)p.n_blocks; };
  for (;;) {
    const int a = (int)(u - at.seg), b = (int)min((long long)at.size, end - at.seg), rows_q = at.rows_q(p), row = 16 * NQ * wv;
    const bool whole = a == 0 && b == at.size;
    const int first_pos = scalar(at.pos_of(p, row)), last_pos = scalar(at.pos_of(p, row + 16 * NQ - 1)), h = scalar(at.h), r = scalar(at.r), len = scalar(at.w.len);
    const int first = scalar(at.tile_of(runs, a)), stop = scalar(at.tile_of(runs, b));
    const bool busy = row < rows_q;
    BrKvSums<D, NQ> s;
    s.clear();
    const int *table = p.table + (long long)r * p.max_blocks;
    const int last_block = max(0, (len - 1) >> p.shift);
    auto id_of = [&](int token) { return table[min(token >> p.shift, last_block)]; };

    // this wave's quarter of a tile: rows 4 wv + kr of each token group of K, channels 16 (wv + 4 i) + n of V; from a lane's place in the
    // worker's block 0 to that in block id: one multiplication
    const long long block0 = (long long)(r / p.rows) * p.n_blocks * p.kv_heads + h;
    const unsigned char *k0 = p.k + ((block0 << p.shift) + ((16 * kg) & mask) + 4 * wv + kr) * D + 16 * g;
    const unsigned char *v0 = p.v + ((block0 * D + 16 * wv + n) << p.shift) + ((16 * g) & mask);
    const float *ks0 = p.ks + block0, *vs0 = p.vs + block0;
    const unsigned step = (unsigned)(p.kv_heads * D) << p.shift;
    uint4 kc[NI + (NI == 0)], vc[VG];
    uint2 kx;
    float ks1 = 0.0f, vs1 = 0.0f;
    auto fetch = [&](int t, int kid, int vid) {
      const int in = (t * BR_KV_TILE) & mask;
      const unsigned char *k = k0 + (unsigned long long)(there(kid) ? (unsigned)kid : 0u) * step + in * D;
#pragma unroll
      for (int i = 0; i < NI; ++i) kc[i] = *(const uint4 *)(k + 64 * i);
      if (REST) kx = *(const uint2 *)(k + 64 * NI - 8 * g);
      const unsigned vb = there(vid) ? (unsigned)vid : 0u;
      const unsigned char *v = v0 + (unsigned long long)vb * step + in;
#pragma unroll
      for (int i = 0; i < VG; ++i)
        if (ND % 4 == 0 || wv + 4 * i < ND) vc[i] = *(const uint4 *)(v + ((64 * i) << p.shift));
      ks1 = ks0[(unsigned long long)vb * (unsigned)p.kv_heads], vs1 = vs0[(unsigned long long)vb * (unsigned)p.kv_heads];
    };
    auto bring = [&](int t, int vid, br_h8 *to) {
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        br_h8 y;
        if (c < 2 * NI) y = c & 1 ? br_kv_decode8<FP8>(kc[c / 2].z, kc[c / 2].w) : br_kv_decode8<FP8>(kc[c / 2].x, kc[c / 2].y);
        else y = br_kv_decode8<FP8>(kx.x, kx.y);
        to[(wv * NK + c) * 64 + lane] = y;
      }
      // (bytes behind the row's end are whatever memory held: an 8-bit float may be a NaN there)
      if (FP8 && (t * BR_KV_TILE + BR_KV_TILE > len || __any(!there(vid)))) {
        const int have = there(vid) ? min(max(len - t * BR_KV_TILE - 16 * g, 0), 16) : 0;
        __asm__ volatile("");  // (a branch: taken at a row's end)
        const unsigned long long full = ~0ull;
        const unsigned long long m0 = have >= 8 ? full : ~(full << (8 * have)), m1 = have >= 16 ? full : have <= 8 ? 0ull : ~(full << (8 * (have - 8)));
#pragma unroll
        for (int i = 0; i < VG; ++i) vc[i].x &= (unsigned)m0, vc[i].y &= (unsigned)(m0 >> 32), vc[i].z &= (unsigned)m1, vc[i].w &= (unsigned)(m1 >> 32);
      }
#pragma unroll
      for (int i = 0; i < VG; ++i) {
        if (ND % 4 != 0 && wv + 4 * i >= ND) continue;
        to[(4 * NK + 2 * (wv + 4 * i)) * 64 + lane] = br_kv_decode8<FP8>(vc[i].x, vc[i].y);
        to[(4 * NK + 2 * (wv + 4 * i) + 1) * 64 + lane] = br_kv_decode8<FP8>(vc[i].z, vc[i].w);
      }
    };
    int kid2 = 0, vid = 0, vid1 = 0, vid2 = 0;  // of this tile, of the next, of the one behind it
    float ks = 0.0f, vs = 0.0f;
    int kid1 = 0;
    if (first < stop) {
      const int next = min(first + 1, stop - 1), after = min(first + 2, stop - 1);
      const int kid = id_of(first * BR_KV_TILE + 16 * kg);
      vid = id_of(first * BR_KV_TILE + 16 * g);
      kid1 = id_of(next * BR_KV_TILE + 16 * kg), vid1 = id_of(next * BR_KV_TILE + 16 * g);
      kid2 = id_of(after * BR_KV_TILE + 16 * kg), vid2 = id_of(after * BR_KV_TILE + 16 * g);
      fetch(first, kid, vid);
    }
    BrKvQueries<D, NQ> q;
    q.load(p, at.w, h, at.qi * TQ + row, [] {});
    if (first < stop) {
      ks = ks1, vs = vs1;
      bring(first, vid, tile[0]);
      fetch(min(first + 1, stop - 1), kid1, vid1);
    }
    __syncthreads();
    for (int t = first; t < stop; ++t) {
      const br_h8 *now = tile[(t - first) & 1];
      if (turn ^ ((t - first) & 1)) __builtin_amdgcn_s_setprio(1);
      else __builtin_amdgcn_s_setprio(0);
      // the next tile to the other half, the one behind it on its way, the ids of the third
      const int after = min(t + 2, stop - 1), third = min(t + 3, stop - 1);
      const int kid3 = id_of(third * BR_KV_TILE + 16 * kg), vid3 = id_of(third * BR_KV_TILE + 16 * g);
      const float ks_next = ks1, vs_next = vs1;
      if (t + 1 < stop) bring(t + 1, vid1, tile[(t + 1 - first) & 1]);
      fetch(after, kid2, vid2);
      // (tiles behind a wave's last query, or before its first one's window, have nothing for it)
      if (busy && t * BR_KV_TILE <= last_pos && (p.window == 0 || t * BR_KV_TILE + BR_KV_TILE - 1 > first_pos - p.window)) {
        br_f4 z[NQ][4];
#pragma unroll
        for (int x = 0; x < NQ; ++x)
#pragma unroll
          for (int y = 0; y < 4; ++y) z[x][y] = br_f4{0.0f, 0.0f, 0.0f, 0.0f};
        br_kv_ahead<NK, AHEAD>(
            [&](int c, br_h8 (&f)[4]) {
#pragma unroll
              for (int y = 0; y < 4; ++y) f[y] = now[(y * NK + c) * 64 + lane];
            },
            [&](int c, const br_h8 (&f)[4]) {
#pragma unroll
              for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int x = 0; x < NQ; ++x) z[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[y], q.qf[x][c], z[x][y], 0, 0, 0);
            });
        const int have = there(vid) ? min(max(len - t * BR_KV_TILE - 16 * g, 0), 16) : 0;
        br_h8 pf[NQ][2];
        br_kv_weights<D, NQ>(p, q, z, there(vid) ? br_kv_sound(ks) : 0.0f, there(vid) ? br_kv_sound(vs) : 0.0f, have, t, first_pos, last_pos, !__any(!there(vid)), s, pf);
        br_kv_ahead<ND / 2, AHEAD>(
            [&](int d, br_h8 (&f)[4]) {
#pragma unroll
              for (int y = 0; y < 4; ++y) f[y] = now[(4 * NK + 4 * d + y) * 64 + lane];
            },
            [&](int d, const br_h8 (&f)[4]) {
#pragma unroll
              for (int y = 0; y < 4; ++y)  // (products into one sum do not follow each other directly)
#pragma unroll
                for (int x = 0; x < NQ; ++x) {
                  const int v = y % 2 * 2 + y / 2, ch = 2 * d + v / 2;
                  s.o[x][ch] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[v], pf[x][v % 2], s.o[x][ch], 0, 0, 0);
                }
            });
      }
      ks = ks_next, vs = vs_next;
      vid = vid1, vid1 = vid2, vid2 = vid3, kid2 = kid3;
      __syncthreads();
    }
    s.close();
    if (whole) {
      br_kv_result<D, NQ, TQ>(p, at.w, at.h, at.qi, row, rows_q, s);
    } else {
      const int from = runs.owner_of(at.seg), parts = runs.owner_of(at.seg + at.size - 1) - from + 1;
      br_kv_piece<D, NQ, TQ>(p, 2 * wg + (a == 0 ? 1 : 0), row, rows_q, s);
      br_kv_stores_done();
      __syncthreads();
      if (tid == 0) arrived = __hip_atomic_fetch_add(&p.arrived[from], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      if (arrived == parts - 1) {
        br_kv_join<D, TQ, NT>(p, at.w, at.h, at.qi, rows_q, from, parts, (br_f4 *)tile[0], (float2 *)tile[1]);
        if (tid == 0) p.arrived[from] = 0;  // (for the next launch)
      }
      __syncthreads();
    }
    u = at.seg + b;
    if (u >= end || !at.next(p, runs)) break;
  }
}

// WAVES on a SIMD, by the registers that the tile needs; PER blocks of NW waves on a compute unit
template <int D, int SHARE, int NW, int WAVES>
void br_kv_attend_few(const BrKvAttend &p, bool fp8, int cus, hipStream_t st) {
  constexpr int PER = 4 * WAVES / NW;
  const int blocks = PER * cus < BR_KV_SPLIT_WGS_OF(D) ? PER * cus : BR_KV_SPLIT_WGS_OF(D);
  const bool half = SHARE == 1 && p.shift == 7;
  if constexpr (SHARE == 1) {
    if (half) {
      if (fp8) br_kv_k_attend<D, SHARE, true, true, NW, WAVES><<<blocks, 64 * NW, 0, st>>>(p);
      else br_kv_k_attend<D, SHARE, false, true, NW, WAVES><<<blocks, 64 * NW, 0, st>>>(p);
      return;
    }
  }
  if (fp8) br_kv_k_attend<D, SHARE, true, false, NW, WAVES><<<blocks, 64 * NW, 0, st>>>(p);
  else br_kv_k_attend<D, SHARE, false, false, NW, WAVES><<<blocks, 64 * NW, 0, st>>>(p);
}

template <int D, int NQ, int WAVES>
void br_kv_attend_rows(const BrKvAttend &p, bool fp8, int cus, hipStream_t st) {
  const int blocks = WAVES * cus < BR_KV_SPLIT_WGS_OF(D) ? WAVES * cus : BR_KV_SPLIT_WGS_OF(D);
  if (fp8) br_kv_k_attend_rows<D, NQ, true, WAVES><<<blocks, 256, 0, st>>>(p);
  else br_kv_k_attend_rows<D, NQ, false, WAVES><<<blocks, 256, 0, st>>>(p);
}

template <int D>
void br_kv_attend_dim(const BrKvAttend &p, int tile, bool fp8, int cus, hipStream_t st) {
  constexpr int NW = D <= 64 ? 12 : D <= 128 ? 8 : 4, WAVES = D <= 64 ? 3 : D <= 128 ? 2 : 1;
  if (tile == BR_KV_TILE_16) br_kv_attend_few<D, 1, NW, WAVES>(p, fp8, cus, st);
  else if (tile == BR_KV_TILE_32) br_kv_attend_few<D, 2, NW, WAVES>(p, fp8, cus, st);
  else if (tile == BR_KV_TILE_64) br_kv_attend_few<D, 4, NW, WAVES>(p, fp8, cus, st);
  else br_kv_attend_rows<D, 2, D <= 128 ? 2 : 1>(p, fp8, cus, st);
}

#endif
