// Log probabilities of tokens, entropy and the likeliest tokens from rows of logits; the gradient of the first two.
//
// With m the row's largest logit and t = scale (z - m):  s1 = sum e^t, s2 = sum t e^t, and
//   lse = scale m + log s1,   logp = t[id] - log s1,   entropy = log s1 - s2 / s1.
// m and log s1 go to the backward, not their sum: where m is large (a row of the type's lowest value) it would hold nothing of log s1.
// A row is cut into segments where there are few of them; what a block found out about its segment (m, s1, s2 and its likeliest tokens) is joined by a second launch.
#include "between.h"
#include "token_dev.h"

namespace ftp {

enum { kLogpT = 256 };
#define FTP_LOG2E 1.4426950408889634f
#define FTP_LN2 0.6931471805599453f
#define FTP_LEAST -3.402823466e38f

struct LogpPlan {
  int segs, seg;               // segments of a row, columns of each (a multiple of 8)
  float* part;                 // [rows][segs][4]: m, s1, s2
  unsigned long long* tops;    // [rows][segs][top]
};

// the order of the likeliest: larger logits first, of equal ones the lower token; 0: none.  -0 and 0 are equal.
__device__ __forceinline__ unsigned long long logp_key(float v, int col) {
  if (!(v > -__builtin_inff())) return 0;                        // -inf and NaN are no alternatives
  const uint32_t b = __float_as_uint(v + 0.f), s = b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
  return ((unsigned long long)s << 32) | (uint32_t)~col;
}
__device__ __forceinline__ int logp_col(unsigned long long key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float logp_value(unsigned long long key) {
  const uint32_t s = (uint32_t)(key >> 32);
  return __uint_as_float(s ^ (s >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ unsigned long long wave_max64(unsigned long long v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const unsigned long long o = __shfl_xor(v, d);
    v = o > v ? o : v;
  }
  return v;
}

__device__ __forceinline__ float logp_exp(float t) { return __builtin_amdgcn_exp2f(t * FTP_LOG2E); }
// t e^t without 0 * inf (e^-200 is 0)
__device__ __forceinline__ float logp_floor(float t) { return fmaxf(t, -200.f); }

struct LogpSum { float m, s1, s2; };
// two parts of a row as one
__device__ __forceinline__ LogpSum logp_join(LogpSum a, LogpSum b, float scale) {
  const float m = fmaxf(a.m, b.m);                               // NaN does not come up here: a NaN logit makes s1 one
  const float ta = (a.m - m) * scale, tb = (b.m - m) * scale, ea = logp_exp(ta), eb = logp_exp(tb);
  return LogpSum{m, fmaf(a.s1, ea, b.s1 * eb), ea * fmaf(logp_floor(ta), a.s1, a.s2) + eb * fmaf(logp_floor(tb), b.s1, b.s2)};
}

template <typename E>
__device__ __forceinline__ float logp_logit(const ftp_logp_args& a, int64_t row, int64_t id) { return to_f32(((const E*)a.logits)[row * a.ldl + id]); }

// a row's results but the likeliest; one thread
template <typename E>
__device__ __forceinline__ void logp_finish(const ftp_logp_args& a, int64_t row, LogpSum s) {
  const float l = __builtin_amdgcn_logf(s.s1) * FTP_LN2;         // nothing but -inf: -inf
  const bool none = s.s1 == 0.f;
  if (a.lse) a.lse[row] = none ? l : fmaf(s.m, a.scale, l);
  if (a.stats) { a.stats[2 * row] = s.m; a.stats[2 * row + 1] = l; }
  if (a.entropy) a.entropy[row] = none ? 0.f : l - s.s2 / s.s1;
  if (a.logp) {
    const int64_t id = a.ids64 ? ((const int64_t*)a.ids)[row] : (int64_t)((const int32_t*)a.ids)[row];
    float v = __uint_as_float(0x7fc00000u);
    if (id == a.pad_id) v = 0.f;
    else if (id >= 0 && id < a.vocab) v = none ? l : (logp_logit<E>(a, row, id) - s.m) * a.scale - l;
    a.logp[row] = v;
  }
}
// place t of the likeliest
__device__ __forceinline__ void logp_place(const ftp_logp_args& a, int64_t row, int t, unsigned long long key, LogpSum s) {
  const bool nan = s.s1 != s.s1;
  a.top_ids[row * a.top + t] = key ? logp_col(key) : -1;
  a.top_logp[row * a.top + t] = nan ? s.s1 : key ? (logp_value(key) - s.m) * a.scale - __builtin_amdgcn_logf(s.s1) * FTP_LN2 : -__builtin_inff();
}

template <typename E>
__global__ __launch_bounds__(kLogpT) void logp_k(ftp_logp_args a, LogpPlan p) {
  __shared__ LogpSum sums[kLogpT / 64];
  __shared__ unsigned long long best[2][kLogpT / 64];
  const int64_t jobs = a.rows * p.segs;
  for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int64_t row = job / p.segs;
    const int seg = (int)(job - row * p.segs), c0 = seg * p.seg, c1 = c0 + p.seg < a.vocab ? c0 + p.seg : a.vocab;
    const E* const z = (const E*)a.logits + row * a.ldl;
    LogpSum s{FTP_LEAST, 0.f, 0.f};
    for (int c = c0 + threadIdx.x * 8; c < c1; c += kLogpT * 8) {
      float v[8];
      tk_load8<E>(z + c, c1 - c, v);
      float m = s.m;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (c + e >= c1) v[e] = -__builtin_inff();
        m = fmaxf(m, v[e]);
      }
      const float t0 = (s.m - m) * a.scale, e0 = logp_exp(t0);
      s.s2 = e0 * fmaf(logp_floor(t0), s.s1, s.s2);
      s.s1 *= e0;
      s.m = m;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float t = (v[e] - m) * a.scale, x = logp_exp(t);
        s.s1 += x;
        s.s2 = fmaf(x, logp_floor(t), s.s2);
      }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) s = logp_join(s, LogpSum{__shfl_xor(s.m, d), __shfl_xor(s.s1, d), __shfl_xor(s.s2, d)}, a.scale);
    __syncthreads();                     // the last job's readers are done
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    s = sums[0];
#pragma unroll
    for (int i = 1; i < kLogpT / 64; ++i) s = logp_join(s, sums[i], a.scale);
    if (p.segs == 1) {
      if (threadIdx.x == 0) logp_finish<E>(a, row, s);
    } else if (threadIdx.x == 0) {
      float* const o = p.part + job * 4;
      o[0] = s.m; o[1] = s.s1; o[2] = s.s2;
    }
    // the likeliest, one after another: the largest below the last one
    unsigned long long below = ~0ull;
    for (int t = 0; t < a.top; ++t) {
      unsigned long long b = 0;
      if (below)
        for (int c = c0 + (int)threadIdx.x; c < c1; c += kLogpT) {
          const unsigned long long q = logp_key(to_f32(z[c]), c);
          if (q < below && q > b) b = q;
        }
      b = wave_max64(b);
      unsigned long long* const w = best[t & 1];
      if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = b;
      __syncthreads();
      b = w[0];
#pragma unroll
      for (int i = 1; i < kLogpT / 64; ++i) b = w[i] > b ? w[i] : b;
      below = b;
      if (threadIdx.x) continue;
      if (p.segs > 1) p.tops[job * a.top + t] = b;
      else logp_place(a, row, t, b, s);
    }
  }
}

// one wavefront a row: its segments' sums in a fixed order, then the likeliest of their lists
template <typename E>
__global__ __launch_bounds__(64) void logp_join_k(ftp_logp_args a, LogpPlan p) {
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    LogpSum s{FTP_LEAST, 0.f, 0.f};
    for (int i = threadIdx.x; i < p.segs; i += 64) {
      const float* const o = p.part + (row * p.segs + i) * 4;
      s = logp_join(s, LogpSum{o[0], o[1], o[2]}, a.scale);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) s = logp_join(s, LogpSum{__shfl_xor(s.m, d), __shfl_xor(s.s1, d), __shfl_xor(s.s2, d)}, a.scale);
    if (threadIdx.x == 0) logp_finish<E>(a, row, s);
    const unsigned long long* const t0 = p.tops + row * p.segs * a.top;
    unsigned long long below = ~0ull;
    for (int t = 0; t < a.top; ++t) {
      unsigned long long b = 0;
      for (int i = threadIdx.x; i < p.segs * a.top; i += 64) {
        const unsigned long long q = t0[i];
        if (q < below && q > b) b = q;
      }
      b = wave_max64(b);
      below = b;
      if (threadIdx.x == 0) logp_place(a, row, t, b, s);
    }
  }
}

// segments: enough blocks for the card, of 2048 columns at least
static LogpPlan logp_plan(const ftp_logp_args& a) {
  LogpPlan p{};
  const int64_t most = (a.vocab + 2047) / 2048, want = a.rows > 0 ? (1024 + a.rows - 1) / a.rows : 1;
  p.segs = (int)std::max<int64_t>(1, std::min(most, want));
  p.seg = ((a.vocab + p.segs - 1) / p.segs + 7) / 8 * 8;
  p.segs = (a.vocab + p.seg - 1) / p.seg;
  return p;
}
static size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
size_t bt_logp_bytes(const ftp_logp_args& a) {
  const LogpPlan p = logp_plan(a);
  return p.segs == 1 ? 0 : up256((size_t)a.rows * p.segs * 16) + up256((size_t)a.rows * p.segs * a.top * 8);
}
void bt_logp(hipStream_t st, const ftp_logp_args& a) {
  KScope ks(st, "tok_logp", (double)a.rows * a.vocab * (a.dtype == 1 ? 2 : 4), 8.0 * a.rows * a.vocab, a.rows, a.vocab, a.top);
  LogpPlan p = logp_plan(a);
  p.part = (float*)a.ws;
  p.tops = (unsigned long long*)((char*)a.ws + up256((size_t)a.rows * p.segs * 16));
  const dim3 g((unsigned)std::min<int64_t>(a.rows * p.segs, 1 << 20)), j((unsigned)std::min<int64_t>(a.rows, 1 << 20));
  if (a.dtype == FTP_BF16) hipLaunchKernelGGL(logp_k<bf16_t>, g, dim3(kLogpT), 0, st, a, p);
  else hipLaunchKernelGGL(logp_k<float>, g, dim3(kLogpT), 0, st, a, p);
  if (p.segs == 1) return;
  if (a.dtype == FTP_BF16) hipLaunchKernelGGL(logp_join_k<bf16_t>, j, dim3(64), 0, st, a, p);
  else hipLaunchKernelGGL(logp_join_k<float>, j, dim3(64), 0, st, a, p);
}

// dlogits = scale * (dlogp ([v = id] - p) - dentropy p (log p + entropy))
template <typename E>
__global__ __launch_bounds__(256) void logp_bwd_k(ftp_logp_args a, int64_t t0, int rows) {
  const uint32_t per = (a.vocab + 7) / 8, all = (uint32_t)rows * per;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) {
    const uint32_t r = i / per;
    const int64_t t = t0 + r;
    const int c = (int)(i - r * per) * 8, left = a.vocab - c;
    const float m = a.stats[2 * t], ls = a.stats[2 * t + 1];
    const bool none = ls == -__builtin_inff();
    int64_t id = -1;
    float w = 0.f, h = 0.f, ent = 0.f;
    if (a.dlogp) {
      id = a.ids64 ? ((const int64_t*)a.ids)[t] : (int64_t)((const int32_t*)a.ids)[t];
      if (id == a.pad_id || id < 0 || id >= a.vocab) id = -1;
      else w = a.dlogp[t];
    }
    if (a.dentropy) { h = a.dentropy[t]; ent = a.entropy[t]; }
    float v[8];
    tk_load8<E>((const E*)a.logits + t * a.ldl + c, left, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float lp = (v[e] - m) * a.scale - ls, p = logp_exp(lp);
      float o = -p * fmaf(h, logp_floor(lp) + ent, w);
      if (id == c + e) o += w;
      v[e] = none ? 0.f : o * a.scale;
    }
    tk_store8<E>((E*)a.dlogits + t * a.lddl + c, left, v);
  }
}
void bt_logp_bwd(hipStream_t st, const ftp_logp_args& a) {
  KScope ks(st, "tok_logp_bwd", 2.0 * a.rows * a.vocab * (a.dtype == 1 ? 2 : 4), 8.0 * a.rows * a.vocab, a.rows, a.vocab);
  const int64_t per = (a.vocab + 7) / 8;
  by_rows(a.rows, per, [&](int64_t t0, int n) {
    const dim3 g(blocks_of(n * per, 1 << 20));
    if (a.dtype == FTP_BF16) hipLaunchKernelGGL(logp_bwd_k<bf16_t>, g, dim3(256), 0, st, a, t0, n);
    else hipLaunchKernelGGL(logp_bwd_k<float>, g, dim3(256), 0, st, a, t0, n);
  });
}

}  // namespace ftp
