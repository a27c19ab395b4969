// Tokens into the 8-bit cache and out of it (br_kv_append, br_kv_read).
//
// Bound by memory: values are read once (append: twice, the second time from a cache) and written once.  The unit of work is a run, tokens
// that stand together in the call's list and in one block, with a key head: nobody else writes that block's codes or scales, so there
// are no atomics.  A block has 4 to 64 tokens of the list and a head; its four waves share a run or take runs of their own.  Values
// lie with their tokens side by side: a thread turns 8 channels of 4 tokens, 16 bytes of a token on one side and 4 of a channel on
// the other, its neighbours the tokens beside.  Prompts of 57 thousand tokens, 8 heads of 128 channels in f16: append 94 us, 351 MB =
// 3.7 TB/s, read 79 us, 354 MB = 4.5 TB/s; a decode step of 144 rows 7 us, a launch and the chain slot, scale, codes.
#include "br_kv_device.h"

#define BR_KV_LEAST 27u  // biased exponent of 2^-100, the smallest scale

#define BR_KV_FEW 4      // tokens of a run that a wave takes one by one

typedef unsigned br_u4 __attribute__((ext_vector_type(4)));

template <bool FP8>
__device__ __forceinline__ float br_kv_value(unsigned c) {  // of the lowest byte
  if constexpr (FP8) return __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
  else return (float)(signed char)c;
}

// ... of byte m (the 8-bit float's conversion takes any byte, by a constant)
template <bool FP8>
__device__ __forceinline__ float br_kv_value_at(unsigned c, int m) {
  if constexpr (FP8) {
    switch (m) {
      case 0: return __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
      case 1: return __builtin_amdgcn_cvt_f32_fp8((int)c, 1);
      case 2: return __builtin_amdgcn_cvt_f32_fp8((int)c, 2);
      default: return __builtin_amdgcn_cvt_f32_fp8((int)c, 3);
    }
  } else {
    return br_kv_value<FP8>(c >> (8 * m));
  }
}

// Codes of four values of magnitude at most the format's top
template <bool FP8>
__device__ __forceinline__ unsigned br_kv_code4(float a, float b, float c, float d) {
  if constexpr (FP8) {
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
  } else {
    auto q = [](float x) { return (unsigned)(int)__builtin_rintf(x) & 255u; };
    return q(a) | q(b) << 8 | q(c) << 16 | q(d) << 24;
  }
}

// a * r rounded to odd: what is rounded to 8 bits next comes out as if from the exact product (a ratio of scales that is no power
// of two can fall on a tie).
__device__ __forceinline__ float br_kv_times(float a, float r) {
  const float y = a * r, err = __builtin_fmaf(a, r, -y);
  const unsigned u = __float_as_uint(y);
  if (err == 0.0f || (u & 1u)) return y;
  return __uint_as_float((err > 0.0f) == (y > 0.0f) ? u + 1 : u - 1);
}

template <bool FP8>
__device__ __forceinline__ unsigned br_kv_recode4(unsigned c, float r) {
  return br_kv_code4<FP8>(br_kv_times(br_kv_value<FP8>(c), r), br_kv_times(br_kv_value<FP8>(c >> 8), r), br_kv_times(br_kv_value<FP8>(c >> 16), r),
                          br_kv_times(br_kv_value<FP8>(c >> 24), r));
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

template <int DT>
__device__ __forceinline__ float br_kv_to_float(unsigned short u) {
  return DT == BR_KV_BF16 ? br_kv_bf16(u) : br_kv_f16(u);
}

// The largest magnitude so far.  Without their signs the types' bits are ordered as whole numbers, what is not finite above the rest: two
// instructions a word, two values where they have 16 bits.
template <int DT>
struct BrKvTop {
  typedef unsigned short us2 __attribute__((ext_vector_type(2)));
  unsigned top = 0;
  __device__ __forceinline__ void add(unsigned u) {
    if constexpr (DT == BR_KV_F32) top = max(top, u & 0x7fffffffu);
    else top = __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(us2, top), __builtin_bit_cast(us2, u & 0x7fff7fffu)));
  }
  // (infinite if one was not finite)
  __device__ __forceinline__ float get() const {
    if constexpr (DT == BR_KV_F32) return __uint_as_float(min(top, 0x7f800000u));
    else return br_kv_to_float<DT>((unsigned short)min(max(top & 0xffffu, top >> 16), DT == BR_KV_BF16 ? 0x7f80u : 0x7c00u));
  }
};

// N = 8 or 2 neighbours of the caller's array as they lie there, and as floats; WIDE: they are aligned to their size
template <int DT, int N, bool WIDE>
struct BrKvRaw {
  static constexpr int WORDS = DT == BR_KV_F32 ? N : N / 2;
  unsigned u[WORDS];

  __device__ __forceinline__ void fetch(const void *x, unsigned at) {
    if constexpr (WIDE) {
      const unsigned *p = DT == BR_KV_F32 ? (const unsigned *)x + at : (const unsigned *)((const unsigned short *)x + at);
      if constexpr (WORDS >= 4) {
#pragma unroll
        for (int k = 0; k < WORDS; k += 4) {
          const uint4 y = *(const uint4 *)(p + k);
          u[k] = y.x, u[k + 1] = y.y, u[k + 2] = y.z, u[k + 3] = y.w;
        }
      } else if constexpr (WORDS == 2) {
        const uint2 y = *(const uint2 *)p;
        u[0] = y.x, u[1] = y.y;
      } else {
        u[0] = *p;
      }
    } else if constexpr (DT == BR_KV_F32) {
#pragma unroll
      for (int k = 0; k < N; ++k) u[k] = ((const unsigned *)x)[at + k];
    } else {
#pragma unroll
      for (int k = 0; k < WORDS; ++k) u[k] = ((const unsigned short *)x)[at + 2 * k] | (unsigned)((const unsigned short *)x)[at + 2 * k + 1] << 16;
    }
  }
  __device__ __forceinline__ float get(int j) const {
    if constexpr (DT == BR_KV_F32) return __uint_as_float(u[j]);
    else return br_kv_to_float<DT>((unsigned short)(j & 1 ? u[j / 2] >> 16 : u[j / 2]));
  }
  // (keeps the compiler from keeping the floats of the first look at them, twice the registers, for the second)
  __device__ __forceinline__ void keep_raw() {
#pragma unroll
    for (int k = 0; k < WORDS; ++k) __asm__ volatile("" : "+v"(u[k]));
  }
  __device__ __forceinline__ void look(BrKvTop<DT> &top) const {
#pragma unroll
    for (int j = 0; j < WORDS; ++j) top.add(u[j]);
  }
};

template <int DT, int N, bool WIDE>
__device__ __forceinline__ void br_kv_store_out(void *x, unsigned at, const float (&y)[N]) {
  if constexpr (DT == BR_KV_F32) {
    float *p = (float *)x + at;
    if constexpr (WIDE) {
      if constexpr (N == 8) {
        *(float4 *)p = *(const float4 *)y;
        *(float4 *)(p + 4) = *(const float4 *)(y + 4);
      } else {
        *(float2 *)p = *(const float2 *)y;
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) p[j] = y[j];
    }
  } else {
    unsigned short *p = (unsigned short *)x + at;
    unsigned u[N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j) u[j] = DT == BR_KV_BF16 ? br_kv_pair<__bf16>(y[2 * j], y[2 * j + 1]) : br_kv_pair<_Float16>(y[2 * j], y[2 * j + 1]);
    if constexpr (WIDE) {
      if constexpr (N == 8) *(uint4 *)p = *(const uint4 *)u;
      else *(unsigned *)p = u[0];
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) p[j] = (unsigned short)(j & 1 ? u[j / 2] >> 16 : u[j / 2]);
    }
  }
}

// A block's place for one key head, and what a run of n tokens from offset off on does there; t: the run's first token in the list.
struct BrKvRun {
  long long block, t;
  int h, off, n;
};

// The scale of the new tokens' block: `top` of them, infinite if one is not finite.  r: what earlier codes are multiplied by.
struct BrKvScale {
  float inv, s, r;
  bool bad;
};

template <bool FP8>
__device__ __forceinline__ BrKvScale br_kv_scale(float top, int off, float old) {
  const bool bad = !(top < __builtin_inff());
  unsigned e = br_kv_scale_exp<FP8>(bad ? 0.0f : top);
  BrKvScale z = {0.0f, 0.0f, 1.0f, bad};
  if (off > 0) {
    // (a scale that is no power of two, in a cache that was written elsewhere, moves up to one: 2^126 at most, whose inverse is the least normal number)
    z.bad = z.bad || !(old >= 0.0f && old <= 0x1p126f);
    const unsigned u = z.bad ? 0u : __float_as_uint(old);
    e = max(e, (u >> 23) + ((u & 0x7fffffu) != 0));
    z.r = z.bad ? 1.0f : old * br_kv_inverse(e);
  }
  z.inv = br_kv_inverse(e);
  z.s = z.bad ? __builtin_nanf("") : __uint_as_float(e << 23);
  return z;
}

// nt threads (64, a wave, or 256, a block that is all here) write a run.  red: 10 floats of LDS.  Earlier scales are read once for all threads: where a
// list has the run's block in another place too they may be changed beside this, and what threads do behind them has to agree.  The first AT_ONCE rows of keys and 4 x 8 values
// of a thread (all, up to 64 tokens of 128 channels for a block) stay in registers between the maximum and the codes.
template <bool FP8, int DT, bool WIDE>
__device__ __forceinline__ void br_kv_append_run(const BrKvCache &c, const BrKvTokens &a, const BrKvRun &u, int nt, int tid, float *red) {
  constexpr int AT_ONCE = 4, SIZE = DT == BR_KV_F32 ? 4 : 2;
  const int D = c.dim, b = 1 << c.shift, chunks = D >> 3, pairs = D >> 1;
  unsigned char *kc = c.k + ((u.block * D) << c.shift), *vc = c.v + ((u.block * D) << c.shift);
  float old_k = u.off ? c.ks[u.block] : 0.0f, old_v = u.off ? c.vs[u.block] : 0.0f;
  // keys: 8 channels from kd on of tokens kj, kj + kstep, ...
  const int kj = tid / chunks, kd = (tid - kj * chunks) * 8, kstep = nt / chunks, kn = kj < kstep ? u.n : 0;
  const char *xk = (const char *)a.k + (u.t * a.k_token + (long long)u.h * a.k_head) * SIZE, *xv = (const char *)a.v + (u.t * a.v_token + (long long)u.h * a.v_head) * SIZE;
  const int k_token = (int)a.k_token, v_token = (int)a.v_token;
  // values: 8 channels of the block's tokens 4 q .. 4 q + 3
  const int vq0 = u.off >> 2, vqs = ((u.off + u.n - 1) >> 2) - vq0 + 1, vitems = vqs * chunks;
  BrKvTop<DT> most_k, most_v;
  BrKvRaw<DT, 8, WIDE> rk[AT_ONCE];
  BrKvRaw<DT, 8, WIDE> rv[4];
  BrKvRaw<DT, 2, WIDE> rf;
  auto fetch_v = [&](int i) {
    const int oct = i / vqs, q = vq0 + i - oct * vqs, lo = u.off - 4 * q, hi = u.off + u.n - 4 * q;
    const int at = (4 * q - u.off) * v_token + 8 * oct;
    // (places that get no new token take a neighbour's: no branches between the loads, nothing for the maximum)
#pragma unroll
    for (int j = 0; j < 4; ++j) rv[j].fetch(xv, at + min(max(j, lo), hi - 1) * v_token);
  };
#pragma unroll
  for (int m = 0; m < AT_ONCE; ++m) rk[m].fetch(xk, min(kj + m * kstep, u.n - 1) * k_token + kd);
  // a decode step's few tokens: two channels of one token at a time
  const bool few = nt == 64 && u.n <= BR_KV_FEW;
  if (few) {
    for (int i = tid; i < u.n * pairs; i += nt) {
      const int j = i / pairs;
      rf.fetch(xv, j * v_token + (i - j * pairs) * 2);
      rf.look(most_v);
    }
  } else {
    for (int i = tid; i < vitems; i += nt) {
      fetch_v(i);
#pragma unroll
      for (int j = 0; j < 4; ++j) rv[j].look(most_v);
    }
  }
#pragma unroll
  for (int m = 0; m < AT_ONCE; ++m) rk[m].look(most_k);
  for (int j = kj + AT_ONCE * kstep; j < kn; j += AT_ONCE * kstep) {
    BrKvRaw<DT, 8, WIDE> x[AT_ONCE];
#pragma unroll
    for (int m = 0; m < AT_ONCE; ++m) x[m].fetch(xk, min(j + m * kstep, u.n - 1) * k_token + kd);
#pragma unroll
    for (int m = 0; m < AT_ONCE; ++m) x[m].look(most_k);
  }
#pragma unroll
  for (int m = 0; m < AT_ONCE; ++m) rk[m].keep_raw();
#pragma unroll
  for (int j = 0; j < 4; ++j) rv[j].keep_raw();
  float top_k = br_kv_max64(most_k.get()), top_v = br_kv_max64(most_v.get());
  if (nt > 64) {
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = top_k, red[4 + (tid >> 6)] = top_v;
    if (tid == 0) red[8] = old_k, red[9] = old_v;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) top_k = fmaxf(top_k, red[k]), top_v = fmaxf(top_v, red[4 + k]);
    old_k = red[8], old_v = red[9];
  }
  const BrKvScale zk = br_kv_scale<FP8>(top_k, u.off, old_k), zv = br_kv_scale<FP8>(top_v, u.off, old_v);

  if (zk.r != 1.0f) {  // earlier keys
    for (int j = kj; j < (kj < kstep ? u.off : 0); j += kstep) {
      uint2 *at = (uint2 *)(kc + (long long)j * D + kd);
      *at = make_uint2(br_kv_recode4<FP8>(at->x, zk.r), br_kv_recode4<FP8>(at->y, zk.r));
    }
  }
  auto put_k = [&](int j, const BrKvRaw<DT, 8, WIDE> &x) {
    auto q = [&](int m) { return x.get(m) * zk.inv; };
    const unsigned lo = br_kv_code4<FP8>(q(0), q(1), q(2), q(3)), hi = br_kv_code4<FP8>(q(4), q(5), q(6), q(7));
    *(uint2 *)(kc + (long long)(u.off + j) * D + kd) = make_uint2(zk.bad ? 0u : lo, zk.bad ? 0u : hi);
  };
#pragma unroll
  for (int m = 0; m < AT_ONCE; ++m)
    if (kj + m * kstep < kn) put_k(kj + m * kstep, rk[m]);
  for (int j = kj + AT_ONCE * kstep; j < kn; j += AT_ONCE * kstep) {
    BrKvRaw<DT, 8, WIDE> x[AT_ONCE];
#pragma unroll
    for (int m = 0; m < AT_ONCE; ++m) x[m].fetch(xk, min(j + m * kstep, u.n - 1) * k_token + kd);
#pragma unroll
    for (int m = 0; m < AT_ONCE; ++m)
      if (j + m * kstep < kn) put_k(j + m * kstep, x[m]);
  }

  if (zv.r != 1.0f) {  // earlier values
    for (int i = tid; i < ((u.off + 15) >> 4) * D; i += nt) {
      const int g = i / D, n = min(u.off - 16 * g, 16);
      br_u4 *at = (br_u4 *)(vc + ((long long)(i - g * D) << c.shift) + 16 * g);
      br_u4 x = *at;
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const unsigned before = n >= 4 * m + 4 ? ~0u : n <= 4 * m ? 0u : ~(~0u << (8 * (n - 4 * m)));
        x[m] = (br_kv_recode4<FP8>(x[m], zv.r) & before) | (x[m] & ~before);
      }
      if (n > 0) *at = x;
    }
    if (nt > 64) __syncthreads();  // (other threads put new values beside them)
    else __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  }
  if (few) {
    for (int i = tid; i < u.n * pairs; i += nt) {
      const int j = i / pairs, d = (i - j * pairs) * 2;
      if (u.n * pairs > nt) rf.fetch(xv, j * v_token + d);
      const unsigned q = br_kv_code4<FP8>(zv.bad ? 0.0f : rf.get(0) * zv.inv, zv.bad ? 0.0f : rf.get(1) * zv.inv, 0.0f, 0.0f);
      unsigned char *at = vc + ((long long)d << c.shift) + u.off + j;
      at[0] = (unsigned char)q, at[b] = (unsigned char)(q >> 8);
    }
  }
  const bool again = vitems > nt;
  for (int i = tid; i < (few ? 0 : vitems); i += nt) {
    if (again) fetch_v(i);
    const int oct = i / vqs, q = vq0 + i - oct * vqs, lo = max(u.off - 4 * q, 0), hi = min(u.off + u.n - 4 * q, 4);  // new ones: lo .. hi - 1
    unsigned char *at = vc + ((long long)(8 * oct) << c.shift) + 4 * q;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      auto x = [&](int j) { return rv[j].get(k) * zv.inv; };
      const unsigned code = br_kv_code4<FP8>(x(0), x(1), x(2), x(3)), y = zv.bad ? 0u : code;
      if (hi - lo == 4) {
        *(unsigned *)(at + k * b) = y;
      } else {
        for (int j = lo; j < hi; ++j) at[k * b + j] = (unsigned char)(y >> (8 * j));
      }
    }
  }
  if (tid == 0) c.ks[u.block] = zk.s, c.vs[u.block] = zv.s;
}

template <bool FP8, int DT, bool WIDE>
__device__ __forceinline__ void br_kv_read_run(const BrKvCache &c, const BrKvTokens &a, const BrKvRun &u, bool in, int nt, int tid) {
  constexpr int SIZE = DT == BR_KV_F32 ? 4 : 2;
  const int D = c.dim, b = 1 << c.shift, chunks = D >> 3, pairs = D >> 1;
  const unsigned char *kc = c.k + ((u.block * D) << c.shift), *vc = c.v + ((u.block * D) << c.shift);
  // (a slot that is none reads as codes of zero)
  const float ks = in ? br_kv_sound(c.ks[u.block]) : 0.0f, vs = in ? br_kv_sound(c.vs[u.block]) : 0.0f;
  const unsigned there = in ? ~0u : 0u;
  const int kj = tid / chunks, kd = (tid - kj * chunks) * 8, kstep = nt / chunks, kn = kj < kstep ? u.n : 0;
  char *xk = (char *)a.k + (u.t * a.k_token + (long long)u.h * a.k_head) * SIZE, *xv = (char *)a.v + (u.t * a.v_token + (long long)u.h * a.v_head) * SIZE;
  const int k_token = (int)a.k_token, v_token = (int)a.v_token;
  // values: 8 channels of the block's tokens 4 q .. 4 q + 3
  const int vq0 = u.off >> 2, vqs = ((u.off + u.n - 1) >> 2) - vq0 + 1, vitems = vqs * chunks;
  unsigned x[8];
  auto fetch_v = [&](int i) {
    const int oct = i / vqs, q = vq0 + i - oct * vqs;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = *(const unsigned *)(vc + ((long long)(8 * oct + k) << c.shift) + 4 * q) & there;
  };
  const bool few = nt == 64 && u.n <= BR_KV_FEW;
  if (few) {
    for (int i = tid; i < u.n * pairs; i += nt) {
      const int j = i / pairs, d = (i - j * pairs) * 2;
      const unsigned char *at = vc + ((long long)d << c.shift) + u.off + j;
      const float y[2] = {in ? br_kv_value<FP8>(at[0]) * vs : 0.0f, in ? br_kv_value<FP8>(at[b]) * vs : 0.0f};
      br_kv_store_out<DT, 2, WIDE>(xv, j * v_token + d, y);
    }
  } else if (tid < vitems) {
    fetch_v(tid);
  }
#pragma unroll 4
  for (int j = kj; j < kn; j += kstep) {
    const uint2 x = *(const uint2 *)(kc + (long long)(u.off + j) * D + kd);
    float y[8];
#pragma unroll
    for (int m = 0; m < 8; ++m) y[m] = br_kv_value_at<FP8>(m < 4 ? x.x & there : x.y & there, m & 3) * ks;
    br_kv_store_out<DT, 8, WIDE>(xk, j * k_token + kd, y);
  }
  for (int i = tid; i < (few ? 0 : vitems); i += nt) {
    if (i != tid) fetch_v(i);
    const int oct = i / vqs, q = vq0 + i - oct * vqs, lo = u.off - 4 * q, hi = u.off + u.n - 4 * q, at = (4 * q - u.off) * v_token + 8 * oct;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j < lo || j >= hi) continue;
      float y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = br_kv_value_at<FP8>(x[k], j) * vs;
      br_kv_store_out<DT, 8, WIDE>(xv, at + j * v_token, y);
    }
  }
}

// Which tokens of t .. t + 63 of a list of n begin a run (also those behind the list's end; bit k: token t + k).  s: the lane's token's slot.
__device__ __forceinline__ unsigned long long br_kv_heads(const int *slot, int t, int n, int slots, int b1, int &s) {
  const int at = t + (threadIdx.x & 63);
  bool head = true;
  s = -1;
  if (at < n) {
    s = slot[at];
    const int before = at > 0 ? slot[at - 1] : -1;
    head = s < 0 || s >= slots || (s & b1) == 0 || before != s - 1;
  }
  return __ballot(head);
}

// `span` tokens of a list (at most 64) and a key head for a block, or one for a wave (WAVE).  `grain`: tokens that a run may have, less one (append: a block's).
template <bool FP8, int DT, bool READ, bool WIDE, bool WAVE>
__global__ __launch_bounds__(256) void br_kv_k_tokens(BrKvCache c, BrKvTokens a, int span, int grain) {
  __shared__ float red[10];
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, b1 = (1 << c.shift) - 1, slots = c.n_blocks << c.shift;
  if (WAVE) span = 1;
  const int spans = (a.n + span - 1) / span;
  const long long units = (long long)a.W * spans * c.heads, step = WAVE ? (long long)gridDim.x * 4 : gridDim.x;
  for (long long id = WAVE ? (long long)blockIdx.x * 4 + wv : blockIdx.x; id < units; id += step) {
    const long long part = id / c.heads;
    BrKvRun u;
    u.h = (int)(id - part * c.heads);
    const int w = (int)(part / spans), t0 = (int)(part - (long long)w * spans) * span;
    const int *slot = a.slot + (long long)w * a.n;
    // heads of the span's tokens, and of those that its last run may reach (a grain more)
    int own, other;
    unsigned long long heads[3] = {br_kv_heads(slot, t0, a.n, slots, grain, own), ~0ull, ~0ull};
    if (span + grain + 1 > 64) heads[1] = br_kv_heads(slot, t0 + 64, a.n, slots, grain, other);
    if (span + grain + 1 > 128) heads[2] = br_kv_heads(slot, t0 + 128, a.n, slots, grain, other);
    unsigned long long left = heads[0] & (~0ull >> (64 - min(span, a.n - t0)));
    const bool apart = !WAVE && __popcll(left) > 2;  // several short runs: one for each wave
    int turn = 0;
    for (; left; left &= left - 1, ++turn) {
      if (apart && (turn & 3) != wv) continue;
      const int k = __ffsll(left) - 1;
      const unsigned long long rest = k < 63 ? heads[0] >> (k + 1) << (k + 1) : 0;
      const int end = rest ? __ffsll(rest) - 1 : heads[1] ? 63 + __ffsll(heads[1]) : heads[2] ? 127 + __ffsll(heads[2]) : 192;
      const int s = __builtin_amdgcn_readlane(own, k);
      const bool in = s >= 0 && s < slots;
      if (!READ && !in) continue;
      u.t = (long long)w * a.n + t0 + k;
      u.n = in ? min(end - k, grain + 1) : 1;
      u.off = in ? s & b1 : 0;
      u.block = ((long long)w * c.n_blocks + (in ? s >> c.shift : 0)) * c.heads + u.h;
      const int nt = WAVE || apart ? 64 : 256, tid = WAVE || apart ? lane : threadIdx.x;
      if constexpr (READ) br_kv_read_run<FP8, DT, WIDE>(c, a, u, in, nt, tid);
      else br_kv_append_run<FP8, DT, WIDE>(c, a, u, nt, tid, red);
    }
  }
}

template <bool FP8, int DT, bool READ, bool WIDE>
static void launch_wide(const BrKvCache &c, const BrKvTokens &t, int rows, hipStream_t st) {
  // A block's span: at least four tokens, so that a decode step's have a wave each and a prompt's runs a block each, and as many as leave
  // some blocks for each compute unit (7250 tokens, 2 heads of 64 channels in blocks of 16, four tokens each: 22.6 us), up to 16
  // where there are at most a few tokens to a row, and 64 of longer runs, which are four runs of 16, one for each wave, or at
  // most two longer ones.  Reads with short spans are cut every 16 tokens; short lists of fewer tokens a row have a wave for each such
  // piece (144 rows of 9 tokens, 8 heads of 128 channels: 9.9 us, by blocks 11.7; 5 rows of 600 tokens, 4 heads of 256
  // channels: 29 us, by blocks 15.5).
  const long long tokens = (long long)t.W * t.n * c.heads;
  const int block = 1 << c.shift;
  auto grid = [](long long blocks) { return (unsigned)(blocks > 1 << 20 ? 1 << 20 : blocks); };
  if constexpr (READ) {
    if (tokens <= 16384 && t.n <= 16 * rows) {
      br_kv_k_tokens<FP8, DT, READ, WIDE, true><<<grid((tokens + 3) / 4), 256, 0, st>>>(c, t, 1, 15);
      return;
    }
  }
  const int most = t.n > 4 * rows ? (c.shift == 5 ? 32 : 64) : 16;
  int span = 4;
  while (span < most && tokens > 1024ll * span) span *= 2;
  br_kv_k_tokens<FP8, DT, READ, WIDE, false><<<grid((long long)t.W * ((t.n + span - 1) / span) * c.heads), 256, 0, st>>>(c, t, span, READ && span <= 16 ? 15 : block - 1);
}

template <bool FP8, int DT, bool READ>
static void launch(const BrKvCache &c, const BrKvTokens &t, int rows, hipStream_t st) {
  t.wide ? launch_wide<FP8, DT, READ, true>(c, t, rows, st) : launch_wide<FP8, DT, READ, false>(c, t, rows, st);
}

template <bool READ>
static void launch_type(const BrKvCache &c, const BrKvTokens &t, int rows, bool fp8, hipStream_t st) {
  if (t.dtype == BR_KV_F32) fp8 ? launch<true, BR_KV_F32, READ>(c, t, rows, st) : launch<false, BR_KV_F32, READ>(c, t, rows, st);
  else if (t.dtype == BR_KV_BF16) fp8 ? launch<true, BR_KV_BF16, READ>(c, t, rows, st) : launch<false, BR_KV_BF16, READ>(c, t, rows, st);
  else fp8 ? launch<true, BR_KV_F16, READ>(c, t, rows, st) : launch<false, BR_KV_F16, READ>(c, t, rows, st);
}

void br_kv_launch_append(const BrKvCache &c, const BrKvTokens &t, int rows, bool fp8, hipStream_t st) { launch_type<false>(c, t, rows, fp8, st); }

void br_kv_launch_read(const BrKvCache &c, const BrKvTokens &t, int rows, bool fp8, hipStream_t st) { launch_type<true>(c, t, rows, fp8, st); }
