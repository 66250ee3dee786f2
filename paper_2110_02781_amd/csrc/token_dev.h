// Device functions the token kernels share: activations and their derivatives, the 8-bit form of activations, accesses to
// four consecutive columns of a row of any alignment.
#pragma once
#include "dev_common.h"
#include "token.h"

namespace ftp {

// 16 or 8 bytes at any element-aligned address as one access
typedef uint32_t u4v_t __attribute__((ext_vector_type(4)));
typedef uint32_t u2v_t __attribute__((ext_vector_type(2)));
template <int A> struct TkAt;
template <> struct TkAt<1> { typedef u2v_t v8 __attribute__((aligned(1))); };
template <> struct TkAt<2> { typedef u4v_t v16 __attribute__((aligned(2))); typedef u2v_t v8 __attribute__((aligned(2))); };
template <> struct TkAt<4> { typedef u4v_t v16 __attribute__((aligned(4))); };
template <typename E> __device__ __forceinline__ u4v_t tk_ld16(const E* p) { return *reinterpret_cast<const typename TkAt<sizeof(E)>::v16*>(p); }
template <typename E> __device__ __forceinline__ void tk_st16(E* p, u4v_t v) { *reinterpret_cast<typename TkAt<sizeof(E)>::v16*>(p) = v; }

// 1 / (1 + e^-t): the exponential is the hardware's, 2^x; t = -inf .. inf give 0 .. 1
__device__ __forceinline__ float sigmoid_f(float t) { return __builtin_amdgcn_rcpf(1.f + __expf(-t)); }
// GELU in its tanh form: (1 + tanh(s)) / 2 = sigmoid(2 s), s = sqrt(2/pi) (z + 0.044715 z^3).  The square is capped so that
// 0 * inf cannot come up: beyond |z| = 1000 the sigmoid is 0 or 1 exactly.
#define FTP_GELU_2K 1.5957691216057308f
#define FTP_GELU_C 0.044715f

// K values at a time: which activation it is costs a chain of branches, 20 cycles a value if asked for every four
template <int K>
__device__ __forceinline__ void tactn(float* v, int act) {
  if (act == TACT_SILU) {
#pragma unroll
    for (int e = 0; e < K; ++e) v[e] *= sigmoid_f(v[e]);
  } else if (act == TACT_GELU) {
#pragma unroll
    for (int e = 0; e < K; ++e) {
      const float z = v[e], z2 = fminf(z * z, 1e6f);
      v[e] = z * sigmoid_f(FTP_GELU_2K * z * fmaf(FTP_GELU_C, z2, 1.f));
    }
  } else if (act != TACT_NONE) {                 // comparisons, so that NaN stays NaN
    const float top = act == TACT_RELU6 ? 6.f : __uint_as_float(0x7f800000u);
#pragma unroll
    for (int e = 0; e < K; ++e) {
      v[e] = v[e] < 0.f ? 0.f : v[e];
      v[e] = v[e] > top ? top : v[e];
    }
  }
}
__device__ __forceinline__ void tact4(float v[4], int act) { tactn<4>(v, act); }
// a <- act(z), d <- act'(z)
template <int K>
__device__ __forceinline__ void tact_gradn(const float* z, float* a, float* d, int act) {
  if (act == TACT_SILU) {
#pragma unroll
    for (int e = 0; e < K; ++e) {
      const float p = sigmoid_f(z[e]);
      a[e] = z[e] * p;
      d[e] = fmaf(a[e], 1.f - p, p);
    }
  } else if (act == TACT_GELU) {
#pragma unroll
    for (int e = 0; e < K; ++e) {
      const float z2 = fminf(z[e] * z[e], 1e6f);
      const float p = sigmoid_f(FTP_GELU_2K * z[e] * fmaf(FTP_GELU_C, z2, 1.f));
      a[e] = z[e] * p;
      d[e] = fmaf(a[e] * (1.f - p), FTP_GELU_2K * fmaf(3.f * FTP_GELU_C, z2, 1.f), p);
    }
  } else {
#pragma unroll
    for (int e = 0; e < K; ++e) {
      a[e] = z[e];
      d[e] = 1.f;
      if (act != TACT_NONE) {
        const bool over = act == TACT_RELU6 && z[e] >= 6.f;
        a[e] = z[e] < 0.f ? 0.f : over ? 6.f : z[e];
        d[e] = z[e] > 0.f && !over ? 1.f : 0.f;
      }
    }
  }
}
__device__ __forceinline__ void tact_grad4(const float z[4], float a[4], float d[4], int act) { tact_gradn<4>(z, a, d, act); }

// ---- four consecutive columns n .. n+3 of a row of N; `vec`: the row's fours are aligned; F: known to be, and inside ----
template <typename E, bool F = false>
__device__ __forceinline__ void get4(const void* base, int64_t ld, int64_t m, int n, int N, bool vec, float v[4]) {
  const E* p = (const E*)base + m * ld + n;
  if (F || (vec && n + 3 < N)) {
    const float4 t = load4(p);
    v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = n + e < N ? to_f32(p[e]) : 0.f;
  }
}
template <typename E, bool F = false>
__device__ __forceinline__ void put4(void* base, int64_t ld, int64_t m, int n, int N, bool vec, const float v[4]) {
  E* p = (E*)base + m * ld + n;
  if (F || (vec && n + 3 < N)) {
    store4(p, make_float4(v[0], v[1], v[2], v[3]));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < N) p[e] = from_f32<E>(v[e]);
  }
}

// ---- the 8-bit form: groups of 32 columns share 2^(byte - 127); values are e4m3 (largest finite 448 = 1.75 * 2^8) ----
// largest finite magnitude of a group -> the byte.  The exponent field says top = m * 2^E, m in [1, 2): 2^(E-8) holds m <= 1.75.
__device__ __forceinline__ uint32_t act8_scale(float top) {
  const uint32_t b = __float_as_uint(top), E = b >> 23, over = (b & 0x7fffffu) > 0x600000u ? 1u : 0u;
  const int s = (int)E - 8 + (int)over;
  return s < 0 ? 0u : (uint32_t)s;
}
__device__ __forceinline__ float act8_mul(uint32_t s) { return __uint_as_float(s ? s << 23 : 0x00400000u); }         // 2^(s-127)
__device__ __forceinline__ float act8_inv(uint32_t s) { return __uint_as_float(s < 254 ? (254u - s) << 23 : 0x00400000u); }
__device__ __forceinline__ float act8_mag(float v) {                        // magnitude that counts for the scale
  const float a = fabsf(v);
  return a <= 3.402823466e38f ? a : 0.f;                                    // an infinity or NaN does not
}
__device__ __forceinline__ uint32_t act8_pack4(const float v[4], float inv) {
  float t[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = fabsf(v[e]) <= 3.402823466e38f ? v[e] * inv : __uint_as_float(0x7fc00000u);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], r, true);
  return (uint32_t)r;
}
__device__ __forceinline__ void act8_unpack4(uint32_t q, float mul, float v[4]) {
  const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
  v[0] = lo.x * mul; v[1] = lo.y * mul; v[2] = hi.x * mul; v[3] = hi.y * mul;
}
template <bool F = false>
__device__ __forceinline__ uint32_t get_q4(const void* base, int64_t ld, int64_t m, int n, int N, bool vec) {
  const uint8_t* p = (const uint8_t*)base + m * ld + n;
  if (F || (vec && n + 3 < N)) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t r = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < N) r |= (uint32_t)p[e] << (8 * e);
  return r;
}
template <bool F = false>
__device__ __forceinline__ void put_q4(void* base, int64_t ld, int64_t m, int n, int N, bool vec, uint32_t q) {
  uint8_t* p = (uint8_t*)base + m * ld + n;
  if (F || (vec && n + 3 < N)) {
    *reinterpret_cast<uint32_t*>(p) = q;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < N) p[e] = (uint8_t)(q >> (8 * e));
}

// ---- results of four columns, the same code behind a tile and behind the joining of split reductions.  In two parts: `request` loads what the
// results need from memory (rows past the last: the last one's), `finish` computes and stores. ----
template <typename E> struct Tg4;
template <> struct Tg4<bf16_t> { typedef uint2 raw; };
template <> struct Tg4<float> { typedef float4 raw; };
// four columns as stored; where they do not go as one, element by element
template <typename E, bool F = false>
__device__ __forceinline__ typename Tg4<E>::raw get_raw4(const void* base, int64_t ld, int64_t m, int n, int N, bool vec) {
  const E* p = (const E*)base + m * ld + n;
  if (F || (vec && n + 3 < N)) return *reinterpret_cast<const typename Tg4<E>::raw*>(p);
  E t[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = n + e < N ? p[e] : (E)0;
  typename Tg4<E>::raw r;
  __builtin_memcpy(&r, t, sizeof(r));
  return r;
}
template <typename E>
__device__ __forceinline__ void open4(const typename Tg4<E>::raw& r, float v[4]) {
  const float4 t = load4(reinterpret_cast<const E*>(&r));
  v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
}

// Columns from N on only pad a row to a multiple of 16 bytes, and the products that follow read them against zeros: written as zeros, because
// what the sums hold there need not be one (an infinity times the zeros that arrive from outside is NaN; few rows multiply the last weight row again)
__device__ __forceinline__ void tg_no_pad(float* v, int n, int N) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = n + e < N ? v[e] : 0.f;
}

template <typename E, int EPI, bool F = false> struct TgSide;

template <typename E, bool F> struct TgSide<E, TG_LINEAR, F> {
  typename Tg4<E>::raw res;
  __device__ __forceinline__ void request(const TgJob& p, int64_t m, int n) {
    if (p.res) res = get_raw4<E, F>(p.res, p.ldr, m < p.M ? m : p.M - 1, n, p.N, p.flags & TG_VEC_RES);
  }
  __device__ __forceinline__ void finish(const TgJob& p, int64_t m, int n, float v[4]) const {
    if (p.bias) {
      float b[4];
      get4<float, F>(p.bias, 0, 0, n, p.N, p.flags & TG_VEC_BIAS, b);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += b[e];
    }
    if (p.z) put4<E, F>(p.z, p.ldz, m, n, p.N, p.flags & TG_VEC_Z, v);
    tact4(v, p.act);                             // of the sum itself, not of the z that is kept: one rounding less
    if (p.res) {
      float r[4];
      open4<E>(res, r);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += r[e];
    }
    put4<E, F>(p.out, p.ldo, m, n, p.N, p.flags & TG_VEC_OUT, v);
  }
};

template <typename E, bool F> struct TgSide<E, TG_GLUBWD, F> {
  typename Tg4<E>::raw g, u;                     // in 8 bits: x the values, y the scale
  __device__ __forceinline__ void request(const TgJob& p, int64_t m, int n) {
    const bool vec = p.flags & TG_VEC_Z;
    const int64_t r = m < p.M ? m : p.M - 1;
    if (p.save == 2) {
      const bool in = F || n < p.N;
      const int64_t s = r * p.lds + (in ? n : 0) / kAct8Group;
      uint32_t q[4] = {get_q4<F>(p.z, p.ldz, r, n, p.N, vec), in ? p.zs[s] : 0u, get_q4<F>(p.up, p.ldu, r, n, p.N, vec), in ? p.us[s] : 0u};
      __builtin_memcpy(&g, q, 8);
      __builtin_memcpy(&u, q + 2, 8);
    } else {
      g = get_raw4<E, F>(p.z, p.ldz, r, n, p.N, vec);
      u = get_raw4<E, F>(p.up, p.ldu, r, n, p.N, vec);
    }
  }
  __device__ __forceinline__ void finish(const TgJob& p, int64_t m, int n, const float dh[4]) const { finish_rows<1>(this, p, m, n, dh); }
  // K rows, two apart
  template <int K>
  static __device__ __forceinline__ void finish_rows(const TgSide* side, const TgJob& p, int64_t m, int n, const float* dh) {
    float gv[4 * K], uv[4 * K];
    if (p.save == 2) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        uint32_t q[4];
        __builtin_memcpy(q, &side[k].g, 8);
        __builtin_memcpy(q + 2, &side[k].u, 8);
        act8_unpack4(q[0], act8_mul(q[1]), gv + 4 * k);
        act8_unpack4(q[2], act8_mul(q[3]), uv + 4 * k);
      }
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        open4<E>(side[k].g, gv + 4 * k);
        open4<E>(side[k].u, uv + 4 * k);
      }
    }
    float a[4 * K], d[4 * K], dg[4 * K], du[4 * K];
    tact_gradn<4 * K>(gv, a, d, p.act);
#pragma unroll
    for (int e = 0; e < 4 * K; ++e) {
      dg[e] = dh[e] * uv[e] * d[e];
      du[e] = dh[e] * a[e];
      a[e] *= uv[e];
    }
    if (!F && n + 3 >= p.N) {
#pragma unroll
      for (int k = 0; k < K; ++k) { tg_no_pad(dg + 4 * k, n, p.N); tg_no_pad(du + 4 * k, n, p.N); tg_no_pad(a + 4 * k, n, p.N); }
    }
    // rounded to the type of the products that follow, as their operands
#pragma unroll
    for (int k = 0; k < K; ++k) {
      put4<E, F>(p.dgate, p.ldd, m + 2 * k, n, (int)p.ldd, true, dg + 4 * k);
      put4<E, F>(p.dup, p.ldd, m + 2 * k, n, (int)p.ldd, true, du + 4 * k);
      put4<E, F>(p.out, p.ldo, m + 2 * k, n, (int)p.ldo, true, a + 4 * k);
    }
  }
};

template <typename E, bool F> struct TgSide<E, TG_GRAD, F> {
  __device__ __forceinline__ void request(const TgJob&, int64_t, int) {}
  __device__ __forceinline__ void finish(const TgJob& p, int64_t m, int n, float v[4]) const {
    if (p.out_f32) {
      if (p.accumulate) {
        float o[4];
        get4<float, F>(p.out, p.ldo, m, n, p.N, p.flags & TG_VEC_OUT, o);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += o[e];
      }
      put4<float, F>(p.out, p.ldo, m, n, p.N, p.flags & TG_VEC_OUT, v);
    } else {
      put4<E, F>(p.out, p.ldo, m, n, p.N, p.flags & TG_VEC_OUT, v);
    }
  }
};
template <typename E, int EPI>
__device__ __forceinline__ void tg_finish4(const TgJob& p, int64_t m, int n, float v[4]) {
  TgSide<E, EPI> s;
  s.request(p, m, n);
  s.finish(p, m, n, v);
}

// largest of the eight lanes that share 32 columns of a row (lanes 8 i .. 8 i + 7): inside fours, then a half row mirrored
__device__ __forceinline__ float tg_max8(float x) {
  x = fmaxf(x, dpp_move<0xB1>(x));
  x = fmaxf(x, dpp_move<0x4E>(x));
  return fmaxf(x, dpp_move<0x141>(x));
}

// act(g) * u into the hidden rows, whose pad columns (up to a multiple of 16 bytes) become zero.  Kept in the call's type (save 1), gate and up are rounded once
// more than the sums hold: what a stash takes is what bounds the batches in flight, and one in single precision would take twice the bytes
template <typename E, bool F = false>
__device__ __forceinline__ void tg_glu4(const TgJob& p, int64_t m, int n, const float g[4], const float u[4]) {
  if (p.save == 1) {
    put4<E, F>(p.z, p.ldz, m, n, p.N, p.flags & TG_VEC_Z, g);
    put4<E, F>(p.up, p.ldu, m, n, p.N, p.flags & TG_VEC_Z, u);
  }
  float h[4] = {g[0], g[1], g[2], g[3]};
  tact4(h, p.act);
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] *= u[e];
  if (!F && n + 3 >= p.N) tg_no_pad(h, n, p.N);
  put4<E, F>(p.out, p.ldo, m, n, (int)p.ldo, true, h);
}
template <bool F = false>
__device__ __forceinline__ void tg_keep8(void* q, int64_t ldq, uint8_t* s, int64_t lds, int64_t m, int n, int N, bool vec, bool lead,
                                         float top, const float v[4]) {
  const uint32_t b = act8_scale(top);
  if (F || n < N) put_q4<F>(q, ldq, m, n, N, vec, act8_pack4(v, act8_inv(b)));
  if (lead && (F || n < N)) s[m * lds + n / kAct8Group] = (uint8_t)b;
}

}  // namespace ftp
