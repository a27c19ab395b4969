// Device-side parameters and helpers of the worker's part (include/br_kv.h): tables, 8-bit cache, attention over it.
#ifndef BR_KV_DEVICE_H
#define BR_KV_DEVICE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "br_kv.h"

// Most blocks of an attention launch that split rows' tokens among them: two for each of 256 compute units where two waves fit on a SIMD
#define BR_KV_SPLIT_WGS 512
#define BR_KV_SPLIT_WGS_OF(dim) ((dim) <= 128 ? BR_KV_SPLIT_WGS : BR_KV_SPLIT_WGS / 2)
#define BR_KV_LIST 4096      // places of a token list that are written with the tables; longer lists have a launch of their own
#define BR_KV_TILE 64        // cached tokens of an attention tile

// The tables of all workers, inside the context's workspace.
struct BrKvTables {
  int W, B, shift, n_blocks, max_blocks, words;  // words: 32-bit words of a worker's used bits
  int *lens;                                     // [W][B]
  int *table;                                    // [W][B][max_blocks]
  int *tail;                                     // [W][B] each row's last block
  unsigned *used;                                // [W][words]
  int *arrived;                                  // BrKvAttend's
};

struct BrKvStep {
  const int *keep, *add;
  int *slot, *pos, *start, *count, *status;
  long long *stats;
  int2 *runs;     // [W][B] workspace: each row's first place in the token list and first position there
  int cap, wide;  // wide: the lists begin at 16 bytes
};

// One layer's cache and what indexes it.
struct BrKvCache {
  unsigned char *k, *v;
  float *ks, *vs;
  int shift, n_blocks, heads, dim;
};

struct BrKvTokens {
  void *k, *v;
  const int *slot;
  long long k_token, k_head, v_token, v_head;
  int n, W, dtype, wide;  // wide: 8 neighbouring channels can be moved at once
};

struct BrKvAttend {
  const unsigned short *q;
  unsigned short *out;
  float *lse;
  const int *start, *count, *lens, *table;
  const unsigned char *k, *v;
  const float *ks, *vs;
  float *part;  // sums of the pieces of split rows, see br_kv_attend.h
  float *ml;    // their maxima and sums of weights
  int *arrived; // per block: blocks that have delivered a piece of the query tile that is split and begins in it; 0 between launches (a
                // call whose lengths are changed under it may leave others, until the next step)
  long long q_token, q_head, out_token, out_head;
  int least, most;  // query tokens of the rows that this launch takes
  int n_rows, rows, n_tokens, window, group, kv_heads, shift, n_blocks, max_blocks;
  int bf16, q_wide, out_wide;  // wide: rows of q (out) can be read (written) 16 (8) bytes at a time
  unsigned group_mul, group_shift;  // x / group = (high word of group_mul x + x) >> group_shift for 0 <= x < 2^31
  float scale2;                // scale * log2(e)
};

void br_kv_launch_clear(const BrKvTables &t, hipStream_t st);
void br_kv_launch_load(const BrKvTables &t, const int *lens, const int *table, hipStream_t st);
void br_kv_launch_step(const BrKvTables &t, const BrKvStep &s, hipStream_t st);
void br_kv_launch_append(const BrKvCache &c, const BrKvTokens &t, int rows, bool fp8, hipStream_t st);
void br_kv_launch_read(const BrKvCache &c, const BrKvTokens &t, int rows, bool fp8, hipStream_t st);

// br_kv_attend_*.hip, one per head width
enum { BR_KV_TILE_16 = 0, BR_KV_TILE_32 = 1, BR_KV_TILE_64 = 2, BR_KV_TILE_128 = 3 };  // rows of queries of a block's tile
void br_kv_launch_attend_64(const BrKvAttend &p, int tile, bool fp8, int cus, hipStream_t st);
void br_kv_launch_attend_96(const BrKvAttend &p, int tile, bool fp8, int cus, hipStream_t st);
void br_kv_launch_attend_128(const BrKvAttend &p, int tile, bool fp8, int cus, hipStream_t st);
void br_kv_launch_attend_192(const BrKvAttend &p, int tile, bool fp8, int cus, hipStream_t st);
void br_kv_launch_attend_256(const BrKvAttend &p, int tile, bool fp8, int cus, hipStream_t st);

#ifdef __HIPCC__
typedef _Float16 br_h2 __attribute__((ext_vector_type(2)));
typedef _Float16 br_h8 __attribute__((ext_vector_type(8)));
typedef float br_f4 __attribute__((ext_vector_type(4)));

// 4 codes to f16, exactly (e4m3 has 4 significant bits, int8 has 8, f16 has 11).  int8: a code plus 128 is put into the mantissa of
// 1024, 1152 is taken off.
template <bool FP8>
__device__ __forceinline__ void br_kv_decode4(unsigned c, br_h2 &lo, br_h2 &hi) {
  if constexpr (FP8) {
    lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.0f, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.0f, true);
  } else {
    c ^= 0x80808080u;
    const unsigned a = __builtin_amdgcn_perm(0x64646464u, c, 0x04010400u), b = __builtin_amdgcn_perm(0x64646464u, c, 0x04030402u);
    const br_h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
    lo = __builtin_bit_cast(br_h2, a) - off;
    hi = __builtin_bit_cast(br_h2, b) - off;
  }
}

template <bool FP8>
__device__ __forceinline__ br_h8 br_kv_decode8(unsigned c0, unsigned c1) {
  br_h2 a, b, c, d;
  br_kv_decode4<FP8>(c0, a, b);
  br_kv_decode4<FP8>(c1, c, d);
  return br_h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float br_kv_bf16(unsigned short u) { return __uint_as_float((unsigned)u << 16); }
__device__ __forceinline__ float br_kv_f16(unsigned short u) { return (float)__builtin_bit_cast(_Float16, u); }

// Over lanes n, n + 16, n + 32, n + 48: the exchanges of 16 and 32 lanes stay in the vector registers.
__device__ __forceinline__ float br_kv_max4(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Over the wave: within rows of 16 lanes by their neighbours and mirrors, between rows by exchanges
__device__ __forceinline__ float br_kv_max64(float x) {
#define BR_KV_STEP(CTRL) x = fmaxf(x, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), CTRL, 0xf, 0xf, true)))
  BR_KV_STEP(0xB1);   // lane ^ 1
  BR_KV_STEP(0x4E);   // lane ^ 2
  BR_KV_STEP(0x141);  // mirrored in 8
  BR_KV_STEP(0x140);  // mirrored in 16
#undef BR_KV_STEP
  return br_kv_max4(x);
}

// Inclusive sum over the wave, in the vector registers: within rows of 16 lanes, then the rows' last ones handed on
__device__ __forceinline__ int br_kv_wave_scan(int x) {
#define BR_KV_STEP(CTRL, ROWS) x += __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false)
  BR_KV_STEP(0x111, 0xf);  // from 1 lane below
  BR_KV_STEP(0x112, 0xf);
  BR_KV_STEP(0x114, 0xf);
  BR_KV_STEP(0x118, 0xf);
  BR_KV_STEP(0x142, 0xa);  // rows 1 and 3: the last of the row below
  BR_KV_STEP(0x143, 0xc);  // rows 2 and 3: the last of row 1
#undef BR_KV_STEP
  return x;
}

// A block's scale; one that is none (below zero or not finite) makes NaN of what is read with it.
__device__ __forceinline__ float br_kv_sound(float s) { return s >= 0.0f && s < __builtin_inff() ? s : __builtin_nanf(""); }

// Two values in 16 bits each
template <class T>
__device__ __forceinline__ unsigned br_kv_pair(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef T t2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector((f2{a, b}), t2));
}
#endif

#endif
