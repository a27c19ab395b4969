// Tokens into the 8-bit cache and out of it (br_kv_append, br_kv_read).
//
// A run: tokens that stand together in the call's list and in one block.  A wave takes a run and a head: nobody else writes that
// block's codes or scales.
#include "br_kv_device.h"

#define BR_KV_LEAST 27u  // biased exponent of 2^-100, the smallest scale

__device__ __forceinline__ float br_kv_get(const void *x, long long at, int dtype) {
  if (dtype == BR_KV_F32) return ((const float *)x)[at];
  const unsigned short u = ((const unsigned short *)x)[at];
  return dtype == BR_KV_BF16 ? br_kv_bf16(u) : br_kv_f16(u);
}

__device__ __forceinline__ void br_kv_set(void *x, long long at, int dtype, float y) {
  if (dtype == BR_KV_F32) ((float *)x)[at] = y;
  else ((unsigned short *)x)[at] = dtype == BR_KV_BF16 ? br_kv_to_bf16(y) : br_kv_to_f16(y);
}

template <bool FP8>
__device__ __forceinline__ float br_kv_value(unsigned char c) {
  if constexpr (FP8) return __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
  else return (float)(signed char)c;
}

// x of magnitude at most the format's top
template <bool FP8>
__device__ __forceinline__ unsigned char br_kv_code(float x) {
  if constexpr (FP8) return (unsigned char)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false);
  else return (unsigned char)(int)__builtin_rintf(x);
}

// a * r rounded to odd: what is rounded to 8 bits next comes out as if from the exact product (a ratio of scales that is no power
// of two can fall on a tie).
__device__ __forceinline__ float br_kv_times(float a, float r) {
  const float y = a * r, err = __builtin_fmaf(a, r, -y);
  const unsigned u = __float_as_uint(y);
  if (err == 0.0f || (u & 1u)) return y;
  return __uint_as_float((err > 0.0f) == (y > 0.0f) ? u + 1 : u - 1);
}

// Biased exponent of the least power of two s with top <= TOP s: TOP is 1.984375 2^6 or 1.75 2^8.
template <bool FP8>
__device__ __forceinline__ unsigned br_kv_scale_exp(float top) {
  const unsigned u = __float_as_uint(top), e = u >> 23, over = (u & 0x7fffffu) > (FP8 ? 0x600000u : 0x7e0000u);
  const int x = (int)e - (FP8 ? 8 : 6) + (int)over;
  return (unsigned)max(x, (int)BR_KV_LEAST);
}

// 2^-(e - 127) of a biased exponent e in 27..253
__device__ __forceinline__ float br_kv_inverse(unsigned e) { return __uint_as_float((254u - e) << 23); }

// The run that begins with token t of a list of n: its tokens, or 0 if t begins none.
__device__ __forceinline__ int br_kv_run(const int *slot, int t, int n, int slots, int b1) {
  const int s = slot[t];
  if (s < 0 || s >= slots) return 0;
  if (t > 0 && (s & b1) != 0 && slot[t - 1] == s - 1) return 0;
  int k = 1;
  while (t + k < n && ((s + k) & b1) != 0 && slot[t + k] == s + k) ++k;
  return k;
}

template <bool FP8, bool VALUES>
__device__ __forceinline__ void br_kv_append_run(const BrKvCache &c, const void *x, long long x_token, long long x_head, int dtype, long long t, int run,
                                                 int h, long long block, int off) {
  const int lane = threadIdx.x & 63, D = c.dim, b = 1 << c.shift, n = run * D;
  unsigned char *codes = (VALUES ? c.v : c.k) + ((block * D) << c.shift);
  float *scale = (VALUES ? c.vs : c.ks) + block;
  float top = 0.0f;
  bool bad = false;
  for (int i = lane; i < n; i += 64) {
    const float y = fabsf(br_kv_get(x, (t + i / D) * x_token + (long long)h * x_head + i % D, dtype));
    bad |= !(y < __builtin_inff());
    top = fmaxf(top, y);
  }
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  bad = __any(bad);
  unsigned e = br_kv_scale_exp<FP8>(bad ? 0.0f : top);
  if (off > 0) {
    // (a scale that is no power of two, in a cache that was written elsewhere, moves up to one)
    const float old = *scale;
    bad |= !(old >= 0.0f && old < 8.5e37f);
    const unsigned u = bad ? 0u : __float_as_uint(old);
    e = max(e, (u >> 23) + ((u & 0x7fffffu) != 0));
    const float r = old * br_kv_inverse(e);
    if (!bad && r != 1.0f) {
      for (int i = lane; i < off * D; i += 64) {
        unsigned char *at = codes + (VALUES ? (i % D) * b + i / D : i);
        *at = br_kv_code<FP8>(br_kv_times(br_kv_value<FP8>(*at), r));
      }
    }
  }
  const float inv = br_kv_inverse(e);
  for (int i = lane; i < n; i += 64) {
    const int j = i / D, d = i % D;
    const float y = br_kv_get(x, (t + j) * x_token + (long long)h * x_head + d, dtype);
    codes[VALUES ? d * b + off + j : (off + j) * D + d] = bad ? 0 : br_kv_code<FP8>(y * inv);
  }
  if (lane == 0) *scale = bad ? __builtin_nanf("") : __uint_as_float(e << 23);
}

template <bool FP8>
__global__ __launch_bounds__(256) void br_kv_k_append(BrKvCache c, BrKvTokens a) {
  const int b1 = (1 << c.shift) - 1;
  for (long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); id < (long long)a.W * a.n * c.heads; id += (long long)gridDim.x * 4) {
    const long long t = id / c.heads;
    const int h = (int)(id - t * c.heads), w = (int)(t / a.n);
    const int run = br_kv_run(a.slot + (long long)w * a.n, (int)(t - (long long)w * a.n), a.n, c.n_blocks << c.shift, b1);
    if (run == 0) continue;
    const int s = a.slot[t];
    const long long block = ((long long)w * c.n_blocks + (s >> c.shift)) * c.heads + h;
    br_kv_append_run<FP8, false>(c, a.k, a.k_token, a.k_head, a.dtype, t, run, h, block, s & b1);
    br_kv_append_run<FP8, true>(c, a.v, a.v_token, a.v_head, a.dtype, t, run, h, block, s & b1);
  }
}

template <bool FP8>
__global__ __launch_bounds__(256) void br_kv_k_read(BrKvCache c, BrKvTokens a) {
  const int b = 1 << c.shift, D = c.dim, lane = threadIdx.x & 63;
  for (long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); id < (long long)a.W * a.n * c.heads; id += (long long)gridDim.x * 4) {
    const long long t = id / c.heads;
    const int h = (int)(id - t * c.heads), w = (int)(t / a.n), s = a.slot[t];
    const bool in = s >= 0 && s < c.n_blocks << c.shift;
    const long long block = ((long long)w * c.n_blocks + (in ? s >> c.shift : 0)) * c.heads + h;
    const int off = s & (b - 1);
    const float ks = c.ks[block], vs = c.vs[block];
    for (int d = lane; d < D; d += 64) {
      const float k = br_kv_value<FP8>(c.k[((block << c.shift) + off) * D + d]) * ks, v = br_kv_value<FP8>(c.v[((block * D + d) << c.shift) + off]) * vs;
      br_kv_set(a.k, t * a.k_token + h * a.k_head + d, a.dtype, in ? k : 0.0f);
      br_kv_set(a.v, t * a.v_token + h * a.v_head + d, a.dtype, in ? v : 0.0f);
    }
  }
}

void br_kv_launch_append(const BrKvCache &c, const BrKvTokens &t, bool fp8, hipStream_t st) {
  const long long waves = (long long)t.W * t.n * c.heads;
  const unsigned blocks = (unsigned)(waves + 3 < 4ll << 20 ? (waves + 3) / 4 : 1 << 20);
  if (fp8) br_kv_k_append<true><<<blocks, 256, 0, st>>>(c, t);
  else br_kv_k_append<false><<<blocks, 256, 0, st>>>(c, t);
}

void br_kv_launch_read(const BrKvCache &c, const BrKvTokens &t, bool fp8, hipStream_t st) {
  const long long waves = (long long)t.W * t.n * c.heads;
  const unsigned blocks = (unsigned)(waves + 3 < 4ll << 20 ? (waves + 3) / 4 : 1 << 20);
  if (fp8) br_kv_k_read<true><<<blocks, 256, 0, st>>>(c, t);
  else br_kv_k_read<false><<<blocks, 256, 0, st>>>(c, t);
}
