// Log probabilities of tokens, entropy and the likeliest tokens from rows of logits; the gradient of the first two.
//
// With m the row's largest logit and t = scale (z - m):  s1 = sum e^t, s2 = sum t e^t, and
//   lse = scale m + log s1,   logp = t[id] - log s1,   entropy = log s1 - s2 / s1.
// m and log s1 go to the backward, not their sum: where m is large (a row of the type's lowest value) it would hold nothing of log s1.
// A block of T threads has a segment of a row in registers, read once: its largest, then the sums, then (with `top`) its likeliest tokens.  One segment is a row where there are rows enough; a
// second launch joins several.
#include <type_traits>

#include "between.h"
#include "token_dev.h"

namespace ftp {

enum { kLogpHeld = 512 };             // candidates for the likeliest that a block keeps
#define FTP_LOG2E 1.4426950408889634f
#define FTP_LN2 0.6931471805599453f
#define FTP_LEAST -3.402823466e38f

struct LogpPlan {
  int segs, seg;               // segments of a row, columns of each (a multiple of 8)
  int threads, vectors;        // of a block; eights of columns a thread
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

// the given token's logit, asked for early; NaN for an id that is no token's
struct LogpGiven { float z; bool pad; };
template <typename E>
__device__ __forceinline__ LogpGiven logp_given(const ftp_logp_args& a, int64_t row) {
  LogpGiven g{__uint_as_float(0x7fc00000u), false};
  if (!a.logp) return g;
  const int64_t id = a.ids64 ? ((const int64_t*)a.ids)[row] : (int64_t)((const int32_t*)a.ids)[row];
  g.pad = id == a.pad_id;
  if (id >= 0 && id < a.vocab) g.z = to_f32(((const E*)a.logits)[row * a.ldl + id]);
  return g;
}
// scale (z - m) by halves: the difference itself may be past the type's range where the scale brings it back
__device__ __forceinline__ float logp_t(float z, float m, float scale) {
  const float h = fmaf(z, 0.5f, -0.5f * m) * scale;
  return h + h;
}
// a row's results but the likeliest; one thread
__device__ __forceinline__ void logp_finish(const ftp_logp_args& a, int64_t row, LogpSum s, LogpGiven g) {
  const float l = __builtin_amdgcn_logf(s.s1) * FTP_LN2;         // nothing but -inf: -inf
  const bool none = s.s1 == 0.f;
  if (a.lse) a.lse[row] = none ? l : fmaf(s.m, a.scale, l);
  if (a.stats) { a.stats[2 * row] = s.m; a.stats[2 * row + 1] = l; }
  if (a.entropy) a.entropy[row] = none ? 0.f : l - s.s2 / s.s1;
  if (a.logp) a.logp[row] = g.pad ? 0.f : g.z != g.z ? g.z : none ? l : logp_t(g.z, s.m, a.scale) - l;
}
// place t of the likeliest
__device__ __forceinline__ void logp_place(const ftp_logp_args& a, int64_t row, int t, unsigned long long key, LogpSum s) {
  const bool nan = s.s1 != s.s1;
  a.top_ids[row * a.top + t] = key ? logp_col(key) : -1;
  a.top_logp[row * a.top + t] = nan ? s.s1 : key ? logp_t(logp_value(key), s.m, a.scale) - __builtin_amdgcn_logf(s.s1) * FTP_LN2 : -__builtin_inff();
}

__device__ __forceinline__ float wave_max_last(float x) {        // in the last lane
  x = fmaxf(x, dpp_move<0xB1>(x));
  x = fmaxf(x, dpp_move<0x4E>(x));
  x = fmaxf(x, dpp_move<0x141>(x));
  x = fmaxf(x, dpp_move<0x140>(x));
  // row_bcast 15 and 31; lanes that receive nothing keep theirs
  x = fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), 0x142, 0xA, 0xF, false)));
  return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), 0x143, 0xC, 0xF, false)));
}
__device__ __forceinline__ uint32_t logp_order(float v) {        // larger values, larger numbers; -0 as 0
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}

// The k largest keys of a block, in their order, at put(place, key).  s.group holds the largest of each of 64 groups of T / 64 lanes beside one another (a barrier has passed).  Of these the
// k-th, without its last sixteen bits, is a bound that at least k keys reach (fewer groups than k with a key: any); those that do, some more than k as a rule, are shown by some(bound, f) and kept in LDS, where each
// counts the larger ones.  Too many that are alike: one after another, each the largest below the last of those that all(f) shows.
struct LogpTop {
  uint32_t group[64];
  uint32_t bound, count;
  unsigned long long kept[kLogpHeld];
  unsigned long long best[2][16];
};
template <int T, typename S, typename A, typename P>
__device__ __forceinline__ void block_top(LogpTop& s, int k, S some, A all, P put) {
  if (threadIdx.x < 64) {
    const uint32_t g = s.group[threadIdx.x];
    uint32_t b = 0;
#pragma unroll 1
    for (int bit = 30; bit >= 16; bit -= 2) {                    // two bits at a time: three counts that do not wait for one another
      const uint32_t c1 = b | 1u << bit, c2 = b | 2u << bit, c3 = b | 3u << bit;
      const int n1 = __popcll(__ballot(g >= c1)), n2 = __popcll(__ballot(g >= c2)), n3 = __popcll(__ballot(g >= c3));
      b = n3 >= k ? c3 : n2 >= k ? c2 : n1 >= k ? c1 : b;
    }
    if (threadIdx.x == 0) { s.bound = b ? b : 1; s.count = 0; }
  }
  __syncthreads();
  some(s.bound, [&](unsigned long long key) {
    const uint32_t at = atomicAdd(&s.count, 1u);                 // the order does not matter: places go by the keys
    if (at < kLogpHeld) s.kept[at] = key;
  });
  __syncthreads();
  const int n = (int)s.count;
  if (n <= kLogpHeld) {
    for (int i = threadIdx.x; i < n; i += T) {
      const unsigned long long key = s.kept[i];
      int larger = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) larger += s.kept[j] > key;
      if (larger < k) put(larger, key);
    }
    for (int i = n + threadIdx.x; i < k; i += T) put(i, 0);
  } else {
    unsigned long long below = ~0ull;
    for (int t = 0; t < k; ++t) {
      unsigned long long b = 0;
      all([&](unsigned long long key) { if (key < below && key > b) b = key; });
      b = wave_max64(b);
      unsigned long long* const w = s.best[t & 1];
      if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = b;
      __syncthreads();
      b = w[0];
#pragma unroll
      for (int i = 1; i < T / 64; ++i) b = w[i] > b ? w[i] : b;
      below = b;
      if (threadIdx.x == 0) put(t, b);
    }
  }
}

// eight columns as stored; what is not there: -inf
template <typename E> struct LogpRaw { uint32_t w[2 * sizeof(E)]; };
template <typename E, bool ONCE>
__device__ __forceinline__ LogpRaw<E> logp_load(const E* p, int left) {
  if (left >= 8) {
    LogpRaw<E> r;
    if constexpr (ONCE) {
      u4v_t t[sizeof(E) / 2];
#pragma unroll
      for (int i = 0; i < (int)sizeof(E) / 2; ++i) t[i] = tk_ld16_once<E>(p + 4 * i);
      __builtin_memcpy(&r, t, sizeof(r));
    } else {
      struct __attribute__((packed, aligned(sizeof(E)))) At { uint32_t w[2 * sizeof(E)]; };
      const At t = *reinterpret_cast<const At*>(p);
      __builtin_memcpy(&r, &t, sizeof(r));
    }
    return r;
  }
  E t[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t none = sizeof(E) == 2 ? 0xff80u : 0xff800000u;
    __builtin_memcpy(&t[e], &none, sizeof(E));
    if (e < left) t[e] = p[e];
  }
  LogpRaw<E> r;
  __builtin_memcpy(&r, t, sizeof(r));
  return r;
}
template <typename E>
__device__ __forceinline__ float logp_at(const LogpRaw<E>& r, int e) {
  if constexpr (sizeof(E) == 4) return __uint_as_float(r.w[e]);
  else return __uint_as_float(e & 1 ? r.w[e / 2] & 0xffff0000u : r.w[e / 2] << 16);
}
// the next pass opens them again: opened, they would take twice the registers
template <typename E>
__device__ __forceinline__ void logp_anew(LogpRaw<E>& r) {
#pragma unroll
  for (int i = 0; i < (int)(2 * sizeof(E)); ++i) asm volatile("" : "+v"(r.w[i]));
}

// TOP: with likeliest tokens; ONCE: logits past the caches
template <typename E, int T, int NV, bool TOP, bool ONCE>
__global__ __launch_bounds__(T, 1) void logp_k(ftp_logp_args a, LogpPlan p) {
  __shared__ float most[T / 64];
  __shared__ float2 sums[T / 64];
  __shared__ typename std::conditional<TOP, LogpTop, int>::type top;
  const int64_t jobs = a.rows * p.segs;
  for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int64_t row = p.segs == 1 ? job : job / p.segs;
    const int seg = (int)(job - row * p.segs), c0 = seg * p.seg, n = p.seg < a.vocab - c0 ? p.seg : a.vocab - c0;
    const E* const z = (const E*)a.logits + row * a.ldl + c0;
    LogpGiven given{};
    if (p.segs == 1 && threadIdx.x < 64) given = logp_given<E>(a, row);
    LogpRaw<E> r[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * T + (int)threadIdx.x) * 8;
      r[v] = logp_load<E, ONCE>(z + c, n - c);
    }
    float m = FTP_LEAST;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, logp_at<E>(r[v], e));
    if constexpr (TOP && NV == 1) {
      // A short segment: columns are dealt to the groups one by one, so that no group is empty while another has two (by lanes, 1240 columns with 50 wanted would fill 39 groups, and
      // every logit be a candidate: 5 x 2478 took 73 us)
      if (threadIdx.x < 64) top.group[threadIdx.x] = 0;
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = logp_at<E>(r[0], e);
        if (v > FTP_LEAST) atomicMax(&top.group[(threadIdx.x * 8 + e) & 63], logp_order(v));
      }
    } else if constexpr (TOP) {
      // the groups' largest (nothing above the least: no key, 0)
      float g = m;
      if (T > 64) g = fmaxf(g, dpp_move<0xB1>(g));
      if (T > 128) g = fmaxf(g, dpp_move<0x4E>(g));
      if (T > 256) g = fmaxf(g, dpp_move<0x141>(g));
      if (T > 512) g = fmaxf(g, dpp_move<0x140>(g));
      if ((threadIdx.x & (T / 64 - 1)) == 0) top.group[threadIdx.x / (T / 64)] = g > FTP_LEAST ? logp_order(g) : 0;
    }
    const float wm = wave_max_last(m);
    if ((threadIdx.x & 63) == 63) most[threadIdx.x >> 6] = wm;
    __syncthreads();
    m = most[0];
#pragma unroll
    for (int i = 1; i < T / 64; ++i) m = fmaxf(m, most[i]);
    // e^t = 2^d, d = k z - k m with one rounding, which leaves the rounding of k m, `off`, in all of them: taken off the sums below to first order.  |off| is at most half a step of k m, below
    // 4096 at most 2^-13, and what is left out, (off ln 2)^2 / 2, 2^-28 of a sum.  From there on (at 1e9 off is 18), or where k m is no number, d = log2 e (scale (z - m)): two
    // operations a value more, no error that grows with m, and no k, which is infinite for a scale of 2.4e38
    const float k = a.scale * FTP_LOG2E, km = m * k;
    const bool plain = fabsf(km) < 4096.f;
    float s1 = 0.f, s2 = 0.f;
    const auto add = [&](auto fused) __attribute__((always_inline)) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        logp_anew<E>(r[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = logp_at<E>(r[v], e), d = fused.value ? fmaf(z, k, -km) : (z - m) * a.scale * FTP_LOG2E, x = __builtin_amdgcn_exp2f(d);
          s1 += x;
          s2 = fmaf(x, fmaxf(d, -300.f), s2);
        }
      }
    };
    if (plain) add(std::true_type());
    else add(std::false_type());
    const float off = plain ? fmaf(m, k, -km) : 0.f;             // of every d
    s1 = wave_sum_last(s1);
    s2 = wave_sum_last(s2);
    if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = make_float2(s1, s2);
    if (!TOP) __syncthreads();           // block_top has some
    const auto total = [&]() {
      LogpSum s{m, sums[0].x, sums[0].y};
#pragma unroll
      for (int i = 1; i < T / 64; ++i) { s.s1 += sums[i].x; s.s2 += sums[i].y; }
      // 2^(d + off): sums off by that factor, the second by off times the first as well
      s.s2 = fmaf(-off, s.s1, s.s2) * FTP_LN2;
      const float f = fmaf(-off, FTP_LN2, 1.f);
      s.s1 *= f;
      s.s2 *= f;
      return s;
    };
    if constexpr (TOP) {
      block_top<T>(top, a.top, [&](uint32_t bound, auto f) {
        // as a float: what is at least this has a key at least the bound (1: any logit above -inf)
        const float lo = bound == 1 ? FTP_LEAST : logp_value((unsigned long long)bound << 32);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          logp_anew<E>(r[v]);
          float big = logp_at<E>(r[v], 0);
#pragma unroll
          for (int e = 1; e < 8; ++e) big = fmaxf(big, logp_at<E>(r[v], e));
          if (!(big >= lo)) continue;    // few eights have one
#pragma unroll 1
          for (int e = 0; e < 8; ++e) {
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) x = e == i ? logp_at<E>(r[v], i) : x;
            if (x >= lo) f(logp_key(x, c0 + (v * T + (int)threadIdx.x) * 8 + e));
          }
        }
      }, [&](auto f) {
        for (int c = threadIdx.x; c < n; c += T) f(logp_key(to_f32(z[c]), c0 + c));
      }, [&](int t, unsigned long long key) {
        if (p.segs > 1) p.tops[job * a.top + t] = key;
        else logp_place(a, row, t, key, total());
      });
    }
    if (threadIdx.x == 0) {
      const LogpSum s = total();
      if (p.segs == 1) logp_finish(a, row, s, given);
      else {
        float* const o = p.part + job * 4;
        o[0] = s.m; o[1] = s.s1; o[2] = s.s2;
      }
    }
    if (job + gridDim.x < jobs) __syncthreads();                 // LDS is read to the end
  }
}

// one block a row: its segments' sums in a fixed order, then the likeliest of their lists
template <typename E>
__global__ __launch_bounds__(256) void logp_join_k(ftp_logp_args a, LogpPlan p) {
  __shared__ LogpSum whole;
  __shared__ LogpTop top;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const unsigned long long* const t0 = p.tops + row * p.segs * a.top;
    const int n = p.segs * a.top;
    // the largest of a thread's keys, then of its group's four
    uint32_t g = 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += 256) {
      const uint32_t q = (uint32_t)(t0[i] >> 32);
      g = q > g ? q : g;
    }
    if (threadIdx.x < 64) {
      const LogpGiven given = logp_given<E>(a, row);
      LogpSum s{FTP_LEAST, 0.f, 0.f};
      for (int i = threadIdx.x; i < p.segs; i += 64) {
        const float* const o = p.part + (row * p.segs + i) * 4;
        s = logp_join(s, LogpSum{o[0], o[1], o[2]}, a.scale);
      }
#pragma unroll
      for (int d = 32; d; d >>= 1) s = logp_join(s, LogpSum{__shfl_xor(s.m, d), __shfl_xor(s.s1, d), __shfl_xor(s.s2, d)}, a.scale);
      if (threadIdx.x == 0) {
        logp_finish(a, row, s, given);
        whole = s;
      }
    }
    if (a.top) {
      uint32_t o = __shfl_xor(g, 1);
      g = o > g ? o : g;
      o = __shfl_xor(g, 2);
      g = o > g ? o : g;
      if ((threadIdx.x & 3) == 0) top.group[threadIdx.x >> 2] = g;
      __syncthreads();
      block_top<256>(top, a.top, [&](uint32_t bound, auto f) {
        for (int i = threadIdx.x; i < n; i += 256)
          if ((uint32_t)(t0[i] >> 32) >= bound) f(t0[i]);
      }, [&](auto f) {
        for (int i = threadIdx.x; i < n; i += 256) f(t0[i]);
      }, [&](int t, unsigned long long key) { logp_place(a, row, t, key, whole); });
    }
    __syncthreads();
  }
}

// Segments and blocks: a row by one block where there are rows for all CUs, otherwise as many segments as make 256 blocks, but no more than leave them
// over 1024 columns (2049 of one row: two segments, of 1032 and 1017).  Blocks of 256 threads, of which several share a CU and wait at different times, until their registers are full.
static LogpPlan logp_plan(const ftp_logp_args& a) {
  LogpPlan p{};
  // with the likeliest, half as many columns a thread: twice would leave two wavefronts to a SIMD (2048 x 32000 bfloat16 with 5 alternatives 50 us, so 44)
  const int most = (a.dtype == FTP_BF16 ? 65536 : 32768) / (a.top ? 2 : 1);
  const int64_t want = a.rows > 0 ? (256 + a.rows - 1) / a.rows : 1;
  p.segs = (int)std::max<int64_t>((a.vocab + most - 1) / most, std::min<int64_t>((a.vocab + 2047) / 2048, want));
  p.seg = ((a.vocab + p.segs - 1) / p.segs + 7) / 8 * 8;
  p.segs = (a.vocab + p.seg - 1) / p.seg;
  const int eights = p.seg / 8;
  p.threads = eights <= 64 ? 64 : eights <= most / 16 ? 256 : 512;
  p.vectors = 1;
  while (p.threads * p.vectors < eights) p.vectors *= 2;
  return p;
}
template <typename E, int T, int NV>
static void logp_go(hipStream_t st, const ftp_logp_args& a, const LogpPlan& p) {
  const dim3 g((unsigned)std::min<int64_t>(a.rows * p.segs, 1 << 22));
  // kept for a backward, what the caches hold of the logits is read again (8192 x 32000 bfloat16, forward and backward: 285 us, past them 303; forward alone 113 and 91)
  const bool once = !a.stats && past_the_caches((double)a.rows * a.vocab * sizeof(E));
  const auto go = [&](auto k) { hipLaunchKernelGGL(k, g, dim3(T), 0, st, a, p); };
  constexpr int HELD = NV * (int)sizeof(E) / 2;                  // a quarter of a thread's registers for its columns: 16 at most, 8 with the likeliest
  if (a.top) {
    if constexpr (T == 512 ? HELD == 8 : HELD <= 8) once ? go(logp_k<E, T, NV, true, true>) : go(logp_k<E, T, NV, true, false>);
  } else {
    if constexpr (T == 512 ? HELD == 16 : HELD <= 16) once ? go(logp_k<E, T, NV, false, true>) : go(logp_k<E, T, NV, false, false>);
  }
}
template <typename E>
static void logp_by(hipStream_t st, const ftp_logp_args& a, const LogpPlan& p) {
  if (p.threads == 64) logp_go<E, 64, 1>(st, a, p);
  else if (p.threads == 256 && p.vectors == 1) logp_go<E, 256, 1>(st, a, p);
  else if (p.threads == 256 && p.vectors == 2) logp_go<E, 256, 2>(st, a, p);
  else if (p.threads == 256 && p.vectors == 4) logp_go<E, 256, 4>(st, a, p);
  else if (p.threads == 256 && p.vectors == 8) logp_go<E, 256, 8>(st, a, p);
  else if (p.threads == 256) logp_go<E, 256, 16>(st, a, p);
  else if (p.vectors == 4) logp_go<E, 512, 4>(st, a, p);
  else if (p.vectors == 8) logp_go<E, 512, 8>(st, a, p);
  else logp_go<E, 512, 16>(st, a, p);
  if (p.segs > 1) hipLaunchKernelGGL(logp_join_k<E>, dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(256), 0, st, a, p);
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
  if (a.dtype == FTP_BF16) logp_by<bf16_t>(st, a, p);
  else logp_by<float>(st, a, p);
}

// dlogits = scale * (dlogp ([v = id] - p) - dentropy p (log p + entropy))
template <typename E, bool ONCE>
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
    const E* const z = (const E*)a.logits + t * a.ldl + c;
    ONCE ? tk_load8_once<E>(z, left, v) : tk_load8<E>(z, left, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float lp = (v[e] - m) * a.scale - ls, p = logp_exp(lp);
      float d = -p * fmaf(h, logp_floor(lp) + ent, w);
      if (id == c + e) d += w;
      v[e] = none ? 0.f : d * a.scale;
    }
    E* const o = (E*)a.dlogits + t * a.lddl + c;
    ONCE ? tk_store8_once<E>(o, left, v) : tk_store8<E>(o, left, v);
  }
}
void bt_logp_bwd(hipStream_t st, const ftp_logp_args& a) {
  const double bytes = 2.0 * a.rows * a.vocab * (a.dtype == 1 ? 2 : 4);
  const bool once = past_the_caches(bytes);
  KScope ks(st, "tok_logp_bwd", bytes, 8.0 * a.rows * a.vocab, a.rows, a.vocab);
  const int64_t per = (a.vocab + 7) / 8;
  by_rows(a.rows, per, [&](int64_t t0, int n) {
    const auto go = [&](auto k) { hipLaunchKernelGGL(k, dim3(blocks_of(n * per, 2048)), dim3(256), 0, st, a, t0, n); };
    if (a.dtype == FTP_BF16) once ? go(logp_bwd_k<bf16_t, true>) : go(logp_bwd_k<bf16_t, false>);
    else once ? go(logp_bwd_k<float, true>) : go(logp_bwd_k<float, false>);
  });
}

}  // namespace ftp
