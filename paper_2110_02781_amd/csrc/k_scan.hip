// Gated linear recurrence along packed sequences, forward and backward.
//
// Rows are cut into chunks of kScanT.  A state goes through a chunk as A h + B, so that chunks are walked at the same time: one launch finds A and B of each,
// one follows the states from chunk to chunk, one walks the chunks again, each from its own state, and writes the results.  The gradient of a state,
// lambda[t] = dy[t] act(g[t]) + a[t+1] lambda[t+1], goes the other way by the same factors: what a chunk hands to the one in front, a[first] lambda[first], is
// A m + C of what it is handed.  A wavefront has 64 lanes of V columns of one chunk; where sequences begin and end is the same for all its lanes.
#include <type_traits>

#include "between.h"
#include "token_dev.h"

namespace ftp {

enum { kScanT = 32, kScanR = 4 };     // rows of a chunk; rows that are asked for together (eight: 89 us instead of 83 for a forward of 16384 x 2048)
// What the kernels need of a call's record, in few scalar registers: row distances of the matrices in bytes, questions as bits that are tested where they are asked (SK_...)
struct ScanArgs {
  const char *f, *x, *g, *dy;
  char *y, *df, *dx, *dg;
  int ldf, ldx, ldg, lddy, ldy, lddf, lddx, lddg;
  const float *h0, *dh_end;
  float *h_end, *dh0;
  int ldh0, lddhe, ldhe, lddh0;
  int64_t rows, length;
  const int32_t* starts;
  int width, seqs, act, flags;
  int chunks, per;             // rows of a chunk: per <= kScanT
  float *A, *B, *C, *seed, *state, *back;     // [chunks][width] each
};
// SK_WHOLE: no sequence goes on from one chunk to the next
enum { SK_G = 1, SK_Y = 2, SK_DF = 4, SK_DX = 8, SK_DG = 16, SK_HEND = 32, SK_DHEND = 64, SK_DH0 = 128, SK_WHOLE = 256 };
__device__ __forceinline__ int scan_flags(int f) {
  asm volatile("" : "+s"(f));
  return f;
}

typedef uint32_t sc_word __attribute__((aligned(2)));
// V consecutive columns of a row as stored; of the last ones `left` are there (WHOLE: all)
template <typename E, int V> struct ScanRaw { uint32_t w[V * sizeof(E) / 4]; };
template <typename E, int V, bool WHOLE, bool ONCE = false>
__device__ __forceinline__ ScanRaw<E, V> sc_ask(const E* p, int left) {
  ScanRaw<E, V> r;
  if constexpr (ONCE && sizeof(E) * V == 4) {
    r.w[0] = __builtin_nontemporal_load(reinterpret_cast<const sc_word*>(p));
    return r;
  }
  if (WHOLE || left >= V) {
    struct __attribute__((packed, aligned(sizeof(E)))) At { uint32_t w[V * sizeof(E) / 4]; };
    const At t = *reinterpret_cast<const At*>(p);
    __builtin_memcpy(&r, &t, sizeof(r));
    return r;
  }
  E t[V];
#pragma unroll
  for (int e = 0; e < V; ++e) t[e] = e < left ? p[e] : (E)0;
  __builtin_memcpy(&r, t, sizeof(r));
  return r;
}
template <typename E, int V>
__device__ __forceinline__ void sc_open(const ScanRaw<E, V>& r, float v[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e)
    v[e] = sizeof(E) == 4 ? __uint_as_float(r.w[e]) : __uint_as_float(e & 1 ? r.w[e / 2] & 0xffff0000u : r.w[e / 2] << 16);
}
template <typename E, int V, bool WHOLE>
__device__ __forceinline__ void sc_load(const E* p, int left, float v[V]) { sc_open<E, V>(sc_ask<E, V, WHOLE>(p, left), v); }
template <typename E, int V, bool WHOLE, bool ONCE = false>
__device__ __forceinline__ void sc_store(E* p, int left, const float v[V]) {
  if constexpr (ONCE && sizeof(E) * V == 4) {
    __builtin_nontemporal_store(sizeof(E) == 4 ? __float_as_uint(v[0]) : f32x2_to_bf16x2(v[0], v[V - 1]), reinterpret_cast<sc_word*>(p));
    return;
  }
  if (WHOLE || left >= V) {
    struct __attribute__((packed, aligned(sizeof(E)))) At { uint32_t w[V * sizeof(E) / 4]; } t;
#pragma unroll
    for (int i = 0; i < (int)(V * sizeof(E) / 4); ++i) t.w[i] = sizeof(E) == 4 ? __float_as_uint(v[i]) : f32x2_to_bf16x2(v[2 * i % V], v[(2 * i + 1) % V]);
    *reinterpret_cast<At*>(p) = t;
    return;
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < left) p[e] = from_f32<E>(v[e]);
}
template <int V>
__device__ __forceinline__ void sc_zero(float v[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = 0.f;
}

// where the chunk's sequences begin and end: bit t for the row r0 + t; a lane holds its row's sequence
struct ScanRows {
  uint64_t in, first, last;
  int seq;
  __device__ __forceinline__ int of(int t) const { return __builtin_amdgcn_readlane(seq, t); }
  // rows that are not in the middle of a sequence
  __device__ __forceinline__ uint64_t events() const { return ~in | first | last; }
};
__device__ __forceinline__ ScanRows scan_rows(const ScanArgs& k, int64_t r0, int n) {
  ScanRows s;
  const int lane = threadIdx.x & 63;
  const int r = (int)r0 + lane;          // 2^30 rows at most
  bool in = lane < n, first = false, last = false;
  if (!k.starts) {
    const uint32_t len = (uint32_t)k.length, u = (uint32_t)r, q = len == 1 ? u : u / len, m = u - q * len;
    s.seq = (int)q;
    first = m == 0;
    last = m == len - 1;
  } else {
    // how many starts are at r0 or in front, 64 places at a time (by halves, each lane its row's, it is a load behind another for each halving)
    const int all = k.seqs + 1, row0 = (int)r0;
    int from = 0, span = all;            // the first start behind r0 is in from .. from + span
    while (span > 0) {
      const int step = (span + 63) >> 6, i = from + lane * step;
      const int ahead = (int)__popcll(__ballot(i < from + span && k.starts[i < all ? i : 0] <= row0));       // of the places looked at, those not behind r0
      if (ahead == 0) break;
      const int to = from + (ahead - 1) * step + 1;              // one behind the last of them
      span = step == 1 ? 0 : (to - 1 + step < from + span ? to - 1 + step : from + span) - to;
      from = to;
    }
    // the starts behind r0, one a lane; of a row's, those at it or in front count
    const int next = from + lane < all ? k.starts[from + lane] : 0x7fffffff, in_front = from > 0 ? k.starts[from - 1] : -1;
    if (__ballot(next > row0 + 63) || from + 64 >= all) {
      int c = 0;
      for (int t = 0; t < n; ++t) {
        const int m = (int)__popcll(__ballot(next <= row0 + t));
        c = lane == t ? m : c;
      }
      const int begin = __shfl(next, c > 0 ? c - 1 : 0), end = __shfl(next, c < 63 ? c : 63), q = from + c - 1;
      in = in && q >= 0 && q < k.seqs;
      first = (c > 0 ? begin : in_front) == r;
      last = end == r + 1;
      s.seq = q < 0 ? 0 : q < k.seqs ? q : k.seqs - 1;
    } else {                             // more than 64 empty sequences here: the last one that begins at r or in front
      int lo = 0, hi = k.seqs;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (k.starts[mid] <= r) lo = mid;
        else hi = mid - 1;
      }
      s.seq = lo < k.seqs ? lo : k.seqs - 1;
      in = in && lo < k.seqs && k.starts[lo] <= r;
      first = in && k.starts[s.seq] == r;
      last = in && k.starts[s.seq + 1] == r + 1;
    }
  }
  s.in = __ballot(in);
  s.first = __ballot(in && first);
  s.last = __ballot(in && last);
  return s;
}

// a = sigmoid(f), 1 - a and c(a).  With e = e^-|f| the smaller of the first two is q = e / (1 + e), which loses none of its places, and the other 1 - q, rounded once: a
// long product of factors next to 1 is as exact as they are (1 / (1 + e) by the hardware's reciprocal is off by a place more, and so were the states' gradients).
// e = 2^t, t = -|f| log2 e, whose rounding makes e off by some |f| roundings.  FINE (calls in fp32): what t lacks, -|f| - t ln 2, is multiplied in, e (1 + it), which leaves 0.05 |f| of
// them; 128 stands for all beyond, where e is 0, and an infinity's difference would be NaN.  It costs 1 % of 8192 x 1024 both ways (129.2 -> 130.5 us); bfloat16 results, rounded to 2^-9, do without.
struct ScanGate { float a, rest, c; };
template <int FORM, bool FINE>
__device__ __forceinline__ ScanGate scan_gate(float f) {
  float e;
  if constexpr (FINE) {
    const float m = __builtin_elementwise_minimum(fabsf(f), 128.f), t = m * -1.44269504f, w = __builtin_amdgcn_exp2f(t);
    e = fmaf(w, fmaf(t, -0.693147181f, -m), w);
  } else {
    e = __builtin_amdgcn_exp2f(fabsf(f) * -1.44269504f);
  }
  const float q = e * __builtin_amdgcn_rcpf(1.f + e), p = 1.f - q;
  const bool up = f >= 0.f;
  ScanGate s;
  s.a = up ? p : q;
  s.rest = up ? q : p;
  s.c = FORM == FTP_SCAN_MIX ? s.rest : FORM == FTP_SCAN_UNIT ? __builtin_amdgcn_sqrtf(fmaf(s.rest, s.a, s.rest)) : 1.f;
  return s;
}
// lambda's factor in the gradient of f: da/df h + dc/df x, of which da/df = a (1 - a)
template <int FORM>
__device__ __forceinline__ float scan_slope(const ScanGate& g, float h, float x) {
  const float d = g.a * g.rest;
  if (FORM == FTP_SCAN_MIX) return d * (h - x);
  if (FORM == FTP_SCAN_UNIT) return fmaf(d, h, -g.a * g.a * x * g.c * __builtin_amdgcn_rcpf(1.f + g.a));
  return d * h;
}

// a wavefront's place: column groups beside one another
struct ScanAt { int64_t r0; int c, n, left, chunk; };
// a lane's columns of the group `group`.  WHOLE: where the last lane's are fewer than V they begin further in front, and some are computed in two lanes alike (a lane for a column
// alone, 16384 x 2047 both ways: 492 us instead of 302)
template <int V, bool WHOLE>
__device__ __forceinline__ void scan_place(const ScanArgs& k, int group, ScanAt& p) {
  p.c = (group * 64 + (int)(threadIdx.x & 63)) * V;
  p.left = k.width - p.c;
  if (WHOLE && V > 1 && p.left > 0 && p.left < V) {
    p.c = k.width - V;
    p.left = V;
  }
}
template <int V, bool WHOLE>
__device__ __forceinline__ ScanAt scan_at(const ScanArgs& k, int64_t wave) {
  const uint32_t groups = (uint32_t)(k.width + 64 * V - 1) / (64 * V), w = (uint32_t)wave;
  ScanAt p;
  p.chunk = (int)(w / groups);
  scan_place<V, WHOLE>(k, (int)(w - (uint32_t)p.chunk * groups), p);
  p.r0 = (int64_t)p.chunk * k.per;
  const int64_t n = k.rows - p.r0;
  p.n = (int)(n < k.per ? n : k.per);
  return p;
}
// R rows of a matrix, q its rows of the chunk, from the row t on (behind its last row: that one again)
template <typename E, int V, bool WHOLE, int R, bool ONCE = false>
__device__ __forceinline__ void scan_ask(const char* q, int ld, const ScanAt& p, int t, ScanRaw<E, V> r[R]) {
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int u = t + i < p.n ? t + i : p.n - 1;
    r[i] = sc_ask<E, V, WHOLE, ONCE>((const E*)(q + u * ld) + (uint32_t)p.c, p.left);
  }
}
// a sequence's row of states, or zeros
template <int V, bool WHOLE>
__device__ __forceinline__ void scan_state(const float* m, int ld, int seq, const ScanAt& p, float h[V]) {
  if (m) sc_load<float, V, WHOLE>(m + (int64_t)seq * ld + p.c, p.left, h);
  else sc_zero<V>(h);
}

// Past a chunk: what comes out of it for h that goes in; and two factors as one.  Of a chunk where a sequence begins or ends A is kScanCut, and what goes in does not count, whatever it
// is: a factor 0 would make NaN of an infinity or NaN, and one spoiled sequence spoil all others of its batch.  Other factors are products of sigmoids, 0 .. 1; where one is NaN, so are B and C.
#define kScanCut -1.f
__device__ __forceinline__ float scan_past(float A, float h, float B) { return A < 0.f ? B : fmaf(A, h, B); }
__device__ __forceinline__ float scan_both(float a, float b) { return a < 0.f || b < 0.f ? kScanCut : a * b; }

// A and B of a chunk; backward: C too.  `seed` (true is returned where there is one): the state in front of the last sequence that begins here, or what arrives at the end of one from a
// chunk in front, read before another chunk writes its result into the same memory.
template <typename E, int V, bool WHOLE, int FORM, bool BWD, int R>
__device__ __forceinline__ bool scan_sums(const ScanArgs& k, const ScanAt& p, ScanRows& rows, float A[V], float B[V], float C[V], float seed[V]) {
  bool seeded = false, open = true;      // open: no sequence has begun or ended yet
  float own[V];                          // C up to there
#pragma unroll
  for (int e = 0; e < V; ++e) { A[e] = 1.f; B[e] = C[e] = own[e] = 0.f; }
  const auto close = [&]() __attribute__((always_inline)) {
    if (BWD && open) {
#pragma unroll
      for (int e = 0; e < V; ++e) own[e] = C[e];
    }
    open = false;
  };
  ScanRaw<E, V> f[R], x[R], g[R], dy[R];
  const char *const qf = k.f + p.r0 * k.ldf, *const qx = k.x + p.r0 * k.ldx, *const qg = k.g + p.r0 * k.ldg, *const qdy = k.dy + p.r0 * k.lddy;
  int flags = k.flags;
  const auto ask = [&](int t) __attribute__((always_inline)) {
    scan_ask<E, V, WHOLE, R>(qf, k.ldf, p, t, f);
    scan_ask<E, V, WHOLE, R>(qx, k.ldx, p, t, x);
    if (BWD) {
      scan_ask<E, V, WHOLE, R>(qdy, k.lddy, p, t, dy);
      if (flags & SK_G) scan_ask<E, V, WHOLE, R>(qg, k.ldg, p, t, g);
    }
  };
  if (p.left > 0) ask(0);              // before the search for the sequences
  rows = scan_rows(k, p.r0, p.n);
  if (p.left <= 0) return false;
  const uint64_t events = rows.events();
  for (int t0 = 0; t0 < p.n; t0 += R) {
    flags = scan_flags(k.flags);
    float fv[R][V], xv[R][V], into[R][V], gv[R * V];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      sc_open<E, V>(f[i], fv[i]);
      sc_open<E, V>(x[i], xv[i]);
      if (BWD) {
        sc_open<E, V>(dy[i], into[i]);
        if (flags & SK_G) sc_open<E, V>(g[i], gv + i * V);
      }
    }
    if (t0 + R < p.n) ask(t0 + R);
    if (BWD && (flags & SK_G)) {
      tactn<R * V>(gv, k.act);
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) into[i][e] *= gv[i * V + e];
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int t = t0 + i;
      const bool event = events >> t & 1;
      bool last = false;
      if (event) {
        if (!(rows.in >> t & 1)) {     // of no sequence, or behind the chunk: nothing goes through
          if (t < p.n) close();
          continue;
        }
        if (rows.first >> t & 1) {
          scan_state<V, WHOLE>(k.h0, k.ldh0, rows.of(t), p, B);
          close();
          if (!BWD) {
            seeded = true;
#pragma unroll
            for (int e = 0; e < V; ++e) seed[e] = B[e];
          }
        }
        last = rows.last >> t & 1;
        if (BWD && last && (flags & SK_DHEND)) {
          float d[V];
          scan_state<V, WHOLE>(k.dh_end, k.lddhe, rows.of(t), p, d);
#pragma unroll
          for (int e = 0; e < V; ++e) into[i][e] += d[e];
          if (!(rows.first << (63 - t))) {
            seeded = true;
#pragma unroll
            for (int e = 0; e < V; ++e) seed[e] = d[e];
          }
        }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const ScanGate s = scan_gate<FORM, sizeof(E) == 4>(fv[i][e]);
        B[e] = fmaf(s.a, B[e], s.c * xv[i][e]);
        A[e] *= s.a;
        if (BWD) C[e] = fmaf(A[e], into[i][e], C[e]);
      }
      if (BWD && last) close();
    }
  }
  if (!open) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      A[e] = kScanCut;
      if (BWD) C[e] = own[e];
    }
  }
  return seeded;
}
template <typename E, int V, bool WHOLE, int FORM, bool BWD, int R>
__global__ __launch_bounds__(256) void scan_sums_k(ScanArgs k) {
  const int64_t waves = (int64_t)k.chunks * ((k.width + 64 * V - 1) / (64 * V));
  const int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave >= waves) return;
  const ScanAt p = scan_at<V, WHOLE>(k, wave);
  const int64_t mine = (int64_t)p.chunk * k.width + p.c;
  float A[V], B[V], C[V], seed[V];
  ScanRows rows;
  const bool seeded = scan_sums<E, V, WHOLE, FORM, BWD, R>(k, p, rows, A, B, C, seed);
  if (p.left <= 0) return;
  if (seeded) sc_store<float, V, WHOLE>(k.seed + mine, p.left, seed);
  sc_store<float, V, WHOLE>(k.A + mine, p.left, A);
  sc_store<float, V, WHOLE>(k.B + mine, p.left, B);
  if (BWD) sc_store<float, V, WHOLE>(k.C + mine, p.left, C);
}

// From chunk to chunk: state[i] = the state in front of chunk i; the other way (blockIdx.y 1) back[i] = what chunk i + 1 hands back.  32 columns a block, 32
// threads to a column, each with its share of the chunks one behind the other: first their product and sum, then the states.
__global__ __launch_bounds__(1024) void scan_follow_k(ScanArgs k) {
  __shared__ float sa[32][33], sb[32][33];
  const int lane = threadIdx.x & 31, ty = threadIdx.x >> 5, W = k.width, c = blockIdx.x * 32 + lane;
  const bool rev = blockIdx.y == 1;
  const float *const A = k.A, *const B = rev ? k.C : k.B;
  float* const out = rev ? k.back : k.state;
  const int share = (k.chunks + 31) / 32, i0 = ty * share, i1 = i0 + share < k.chunks ? i0 + share : k.chunks;
  const auto at = [&](int i) { return (int64_t)(rev ? k.chunks - 1 - i : i) * W + c; };
  float a = 1.f, b = 0.f, u[8], v[8];
  const bool few = share <= 8;           // kept for the second time
  if (c < W) {
    if (few) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const bool in = i0 + q < i1;
        u[q] = in ? A[at(in ? i0 + q : 0)] : 1.f;
        v[q] = in ? B[at(in ? i0 + q : 0)] : 0.f;
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        b = scan_past(u[q], b, v[q]);
        a = scan_both(a, u[q]);
      }
    } else {
#pragma unroll 8
      for (int i = i0; i < i1; ++i) {
        const float p = A[at(i)], q = B[at(i)];
        b = scan_past(p, b, q);
        a = scan_both(a, p);
      }
    }
  }
  // each share's product and sum with those of the 1, 2, 4, ... shares in front
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    sa[ty][lane] = a;
    sb[ty][lane] = b;
    __syncthreads();
    if (ty >= d) {
      b = scan_past(a, sb[ty - d][lane], b);
      a = scan_both(a, sa[ty - d][lane]);
    }
    __syncthreads();
  }
  sb[ty][lane] = b;
  __syncthreads();
  if (c >= W) return;
  float h = ty ? sb[ty - 1][lane] : 0.f;
  if (few) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      if (i0 + q >= i1) break;
      out[at(i0 + q)] = h;
      h = scan_past(u[q], h, v[q]);
    }
  } else {
#pragma unroll 8
    for (int i = i0; i < i1; ++i) {
      const float p = A[at(i)], q = B[at(i)];
      out[at(i)] = h;
      h = scan_past(p, h, q);
    }
  }
}

// states of empty sequences stay: those of the 64 from `seq0` on
template <int V, bool WHOLE>
__device__ __forceinline__ void scan_empty(const ScanArgs& k, int64_t block, const float* from, int64_t ldf, float* to, int64_t ldt) {
  if (!to || from == to) return;
  const int groups = (k.width + 64 * V - 1) / (64 * V);
  const int64_t seq0 = block / groups * 64, s = seq0 + (threadIdx.x & 63);
  ScanAt p{};
  scan_place<V, WHOLE>(k, (int)(block % groups), p);
  uint64_t todo = __ballot(s < k.seqs && (k.starts ? k.starts[s < k.seqs ? s : 0] >= k.starts[s < k.seqs ? s + 1 : 0] : k.length == 0));
  if (p.left <= 0) return;
  while (todo) {
    const int q = (int)seq0 + __builtin_ctzll(todo);
    todo &= todo - 1;
    float h[V];
    scan_state<V, WHOLE>(from, ldf, q, p, h);
    sc_store<float, V, WHOLE>(to + q * ldt + p.c, p.left, h);
  }
}

// Few rows: a block has all chunks of its 64 V columns, a wavefront each, and the states go from one to the next through LDS: one launch instead of three (57 x 496 float 8.0 us
// instead of 13.5, with the gradients 17.6 instead of 28).  Sixteen wavefronts forward; backward eight, which have the registers it needs.  Past 128 rows a wavefront waits more
// often for its rows than the launches cost (250 x 1024: 17.4 us and 34.3, with three launches 14.3 and 30.9).
constexpr int scan_few_waves(bool backward) { return backward ? 8 : 16; }
enum { kScanFew = 128, kScanFewR = 8 };        // rows at most; rows that are asked for together: nothing else hides what a load takes
// the number that the wavefront has where chunks are dealt to blocks of any: of chunk `me`, -1 where there is none; blocks behind the groups' have the empty sequences
__device__ __forceinline__ int64_t scan_few_wave(const ScanArgs& k, int n, int groups, int me) {
  const int b = (int)blockIdx.x;
  if (b >= groups) return (int64_t)k.chunks * groups + (int64_t)(b - groups) * n + me;
  return me < k.chunks ? (int64_t)me * groups + b : -1;
}
// h and (backward) mu of the wavefront's chunk; false where it has none
template <typename E, int V, bool WHOLE, int FORM, bool BWD, int R, int N>
__device__ __forceinline__ bool scan_pass(const ScanArgs& k, const ScanAt& p, ScanRows& rows, int64_t wave, int me, float h[V], float mu[V], float seed[V]) {
  __shared__ float sA[N][64 * V], sB[N][64 * V], sC[BWD ? N : 1][64 * V];
  const int at = (threadIdx.x & 63) * V;
  if (wave >= 0) {
    float A[V], B[V], C[V];
    scan_sums<E, V, WHOLE, FORM, BWD, R>(k, p, rows, A, B, C, seed);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sA[me][at + e] = A[e];
      sB[me][at + e] = B[e];
      if (BWD) sC[me][at + e] = C[e];
    }
  }
  __syncthreads();
  if (wave < 0) return false;
  for (int j = 0; j < me; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = scan_past(sA[j][at + e], h[e], sB[j][at + e]);
  if (BWD)
    for (int j = k.chunks - 1; j > me; --j)
#pragma unroll
      for (int e = 0; e < V; ++e) mu[e] = scan_past(sA[j][at + e], mu[e], sC[j][at + e]);
  return true;
}

// FEW: the states in front by scan_pass, otherwise from memory
template <typename E, int V, bool WHOLE, int FORM, int R, bool ONCE, bool FEW>
__global__ __launch_bounds__(64 * (FEW ? scan_few_waves(false) : 4)) void scan_walk_k(ScanArgs k) {
  constexpr int N = FEW ? scan_few_waves(false) : 4;
  const int groups = (k.width + 64 * V - 1) / (64 * V);
  const int64_t waves = (int64_t)k.chunks * groups, all = waves + (k.starts || k.length == 0 ? (int64_t)((k.seqs + 63) / 64) * groups : 0);
  const int me = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t wave = FEW ? scan_few_wave(k, N, groups, me) : (int64_t)blockIdx.x * 4 + me;
  if (!FEW && wave >= all) return;
  if (wave >= waves) {
    if (wave < all) scan_empty<V, WHOLE>(k, wave - waves, k.h0, k.ldh0, k.h_end, k.ldhe);
    return;
  }
  const ScanAt p = scan_at<V, WHOLE>(k, wave < 0 ? 0 : wave);
  const int64_t mine = (int64_t)p.chunk * k.width + p.c;
  float h[V], seed[FEW ? V : 1];
  ScanRows rows;
  sc_zero<V>(h);
  if constexpr (FEW) {
    if (!scan_pass<E, V, WHOLE, FORM, false, R, N>(k, p, rows, wave, me, h, h, seed)) return;
  }
  ScanRaw<E, V> f[R], x[R], g[R];
  const char *const qf = k.f + p.r0 * k.ldf, *const qx = k.x + p.r0 * k.ldx, *const qg = k.g + p.r0 * k.ldg;
  char* const qy = k.y + p.r0 * k.ldy;
  int flags = k.flags;
  const auto ask = [&](int t) __attribute__((always_inline)) {
    scan_ask<E, V, WHOLE, R, ONCE>(qf, k.ldf, p, t, f);
    scan_ask<E, V, WHOLE, R, ONCE>(qx, k.ldx, p, t, x);
    if (flags & SK_G) scan_ask<E, V, WHOLE, R, ONCE>(qg, k.ldg, p, t, g);
  };
  if (p.left > 0) {
    if (!FEW && !(flags & SK_WHOLE)) sc_load<float, V, WHOLE>(k.state + mine, p.left, h);
    ask(0);
  }
  if constexpr (!FEW) rows = scan_rows(k, p.r0, p.n);
  if (p.left <= 0) return;
  const uint64_t events = rows.events();
  for (int t0 = 0; t0 < p.n; t0 += R) {
    flags = scan_flags(k.flags);
    float fv[R][V], xv[R][V], gv[R * V];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      sc_open<E, V>(f[i], fv[i]);
      sc_open<E, V>(x[i], xv[i]);
      if (flags & SK_G) sc_open<E, V>(g[i], gv + i * V);
    }
    if (t0 + R < p.n) ask(t0 + R);
    if (flags & SK_G) tactn<R * V>(gv, k.act);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int t = t0 + i;
      bool last = false;
      if (events >> t & 1) {
        if (!(rows.in >> t & 1)) continue;
        if (rows.first >> t & 1) {
          // one that goes on behind the chunk: its state from the copy
          if (!(flags & SK_WHOLE) && !(rows.last >> t)) {
            if constexpr (FEW)
#pragma unroll
              for (int e = 0; e < V; ++e) h[e] = seed[e];
            else sc_load<float, V, WHOLE>(k.seed + mine, p.left, h);
          } else scan_state<V, WHOLE>(k.h0, k.ldh0, rows.of(t), p, h);
        }
        last = rows.last >> t & 1;
      }
      float y[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const ScanGate s = scan_gate<FORM, sizeof(E) == 4>(fv[i][e]);
        h[e] = fmaf(s.a, h[e], s.c * xv[i][e]);
        y[e] = flags & SK_G ? h[e] * gv[i * V + e] : h[e];
      }
      if (flags & SK_Y) sc_store<E, V, WHOLE, ONCE>((E*)(qy + t * k.ldy) + (uint32_t)p.c, p.left, y);
      if (last && (flags & SK_HEND)) sc_store<float, V, WHOLE>(k.h_end + (int64_t)rows.of(t) * k.ldhe + p.c, p.left, h);
    }
  }
}

// A chunk's states from the first row on, of which those in front of every R rows are kept in LDS; then its gradients from the last row to the first, the states of
// R rows at a time made again.
template <typename E, int V, bool WHOLE, int FORM, int R, bool ONCE, bool FEW>
__global__ __launch_bounds__(64 * (FEW ? scan_few_waves(true) : 4)) void scan_back_k(ScanArgs k) {
  constexpr int N = FEW ? scan_few_waves(true) : 4;
  __shared__ float held[N][(FEW ? kScanFew / N : kScanT) / R][64 * V];
  const int groups = (k.width + 64 * V - 1) / (64 * V);
  const int64_t waves = (int64_t)k.chunks * groups, all = waves + (k.starts || k.length == 0 ? (int64_t)((k.seqs + 63) / 64) * groups : 0);
  const int me = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t wave = FEW ? scan_few_wave(k, N, groups, me) : (int64_t)blockIdx.x * 4 + me;
  if (!FEW && wave >= all) return;
  if (wave >= waves) {
    if (wave < all) scan_empty<V, WHOLE>(k, wave - waves, k.dh_end, k.lddhe, k.dh0, k.lddh0);
    return;
  }
  const ScanAt p = scan_at<V, WHOLE>(k, wave < 0 ? 0 : wave);
  const int64_t mine = (int64_t)p.chunk * k.width + p.c;
  float* const keep = held[me][0] + (threadIdx.x & 63) * V;          // a lane's own: nothing to wait for
  float h[V], mu[V], seed[FEW ? V : 1];
  ScanRows rows;
  sc_zero<V>(h);
  sc_zero<V>(mu);
  if constexpr (FEW) {
    if (!scan_pass<E, V, WHOLE, FORM, true, R, N>(k, p, rows, wave, me, h, mu, seed)) return;
  }
  ScanRaw<E, V> f[R], x[R], g[R], dy[R];
  const char *const qf = k.f + p.r0 * k.ldf, *const qx = k.x + p.r0 * k.ldx, *const qg = k.g + p.r0 * k.ldg, *const qdy = k.dy + p.r0 * k.lddy;
  char *const qdf = k.df + p.r0 * k.lddf, *const qdx = k.dx + p.r0 * k.lddx, *const qdg = k.dg + p.r0 * k.lddg;
  int flags = k.flags;
  if (p.left > 0) {
    if (!FEW && !(flags & SK_WHOLE)) {
      sc_load<float, V, WHOLE>(k.state + mine, p.left, h);
      sc_load<float, V, WHOLE>(k.back + mine, p.left, mu);
    }
    scan_ask<E, V, WHOLE, R>(qf, k.ldf, p, 0, f);
    scan_ask<E, V, WHOLE, R>(qx, k.ldx, p, 0, x);
  }
  if constexpr (!FEW) rows = scan_rows(k, p.r0, p.n);
  if (p.left <= 0) return;
  const uint64_t events = rows.events();
  const int t_end = (p.n - 1) / R * R;
  const auto ask_back = [&](int t) __attribute__((always_inline)) {
    scan_ask<E, V, WHOLE, R, ONCE>(qdy, k.lddy, p, t, dy);
    if (flags & SK_G) scan_ask<E, V, WHOLE, R, ONCE>(qg, k.ldg, p, t, g);
  };
  for (int t0 = 0;; t0 += R) {
#pragma unroll
    for (int e = 0; e < V; ++e) keep[t0 / R * 64 * V + e] = h[e];
    if (t0 == t_end) break;
    float fv[R][V], xv[R][V];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      sc_open<E, V>(f[i], fv[i]);
      sc_open<E, V>(x[i], xv[i]);
    }
    scan_ask<E, V, WHOLE, R>(qf, k.ldf, p, t0 + R, f);
    scan_ask<E, V, WHOLE, R>(qx, k.ldx, p, t0 + R, x);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int t = t0 + i;
      if (events >> t & 1) {
        if (!(rows.in >> t & 1)) continue;
        if (rows.first >> t & 1) scan_state<V, WHOLE>(k.h0, k.ldh0, rows.of(t), p, h);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const ScanGate s = scan_gate<FORM, sizeof(E) == 4>(fv[i][e]);
        h[e] = fmaf(s.a, h[e], s.c * xv[i][e]);
      }
    }
  }
  ask_back(t_end);
  for (int t0 = t_end; t0 >= 0; t0 -= R) {
    flags = scan_flags(k.flags);
    float fv[R][V], xv[R][V], lam[R][V], act[R * V], dact[R * V], before[R][V], after[R][V];
    ScanGate s[R][V];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      sc_open<E, V>(f[i], fv[i]);
      sc_open<E, V>(x[i], xv[i]);
      sc_open<E, V>(dy[i], lam[i]);
      if (flags & SK_G) sc_open<E, V>(g[i], act + i * V);
    }
    if (t0 > 0) {
      scan_ask<E, V, WHOLE, R>(qf, k.ldf, p, t0 - R, f);
      scan_ask<E, V, WHOLE, R>(qx, k.ldx, p, t0 - R, x);
      ask_back(t0 - R);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = keep[t0 / R * 64 * V + e];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int t = t0 + i;
#pragma unroll
      for (int e = 0; e < V; ++e) s[i][e] = scan_gate<FORM, sizeof(E) == 4>(fv[i][e]);
      if ((events >> t & 1) && (rows.first >> t & 1)) scan_state<V, WHOLE>(k.h0, k.ldh0, rows.of(t), p, h);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        before[i][e] = h[e];
        after[i][e] = h[e] = fmaf(s[i][e].a, h[e], s[i][e].c * xv[i][e]);
      }
    }
    if (flags & SK_G) tact_gradn<R * V>(act, act, dact, k.act);
#pragma unroll
    for (int i = R - 1; i >= 0; --i) {
      const int t = t0 + i;
      bool first = false;
      if (events >> t & 1) {
        if (!(rows.in >> t & 1)) continue;
        if (rows.last >> t & 1) {
          // of a sequence from a chunk in front: the copy of what arrives at its end
          if ((flags & SK_DHEND) && !(flags & SK_WHOLE) && !(rows.first << (63 - t))) {
            if constexpr (FEW)
#pragma unroll
              for (int e = 0; e < V; ++e) mu[e] = seed[e];
            else sc_load<float, V, WHOLE>(k.seed + mine, p.left, mu);
          }
          else scan_state<V, WHOLE>(k.dh_end, k.lddhe, rows.of(t), p, mu);
        }
        first = rows.first >> t & 1;
      }
      float dg[V], df[V], dx[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const ScanGate& q = s[i][e];
        if (flags & SK_G) {
          dg[e] = lam[i][e] * after[i][e] * dact[i * V + e];
          lam[i][e] *= act[i * V + e];
        }
        const float l = lam[i][e] + mu[e];
        dx[e] = l * q.c;
        df[e] = l * scan_slope<FORM>(q, before[i][e], xv[i][e]);
        mu[e] = l * q.a;
      }
      if (flags & SK_DG) sc_store<E, V, WHOLE, ONCE>((E*)(qdg + t * k.lddg) + (uint32_t)p.c, p.left, dg);
      if (flags & SK_DF) sc_store<E, V, WHOLE, ONCE>((E*)(qdf + t * k.lddf) + (uint32_t)p.c, p.left, df);
      if (flags & SK_DX) sc_store<E, V, WHOLE, ONCE>((E*)(qdx + t * k.lddx) + (uint32_t)p.c, p.left, dx);
      if (first && (flags & SK_DH0)) sc_store<float, V, WHOLE>(k.dh0 + (int64_t)rows.of(t) * k.lddh0 + p.c, p.left, mu);
    }
  }
}

static int scan_per(const ftp_scan_args& a, int V, bool backward, bool& whole) {
  const int64_t groups = (a.width + 64 * V - 1) / (64 * V), slots = backward ? 4096 : 8192;
  whole = a.starts ? a.rows <= kScanT : a.length <= kScanT;
  if (!a.starts && a.length > 0 && whole) return (int)(std::max<int64_t>(1, std::min<int64_t>(kScanT / a.length, a.seqs * groups / 4096)) * a.length);
  if (whole) return kScanT;
  const int few = scan_few_waves(backward);
  if (a.rows <= kScanFew) return (int)((a.rows + few * kScanR - 1) / (few * kScanR) * kScanR);
  int per = kScanT;
  int64_t least = INT64_MAX;
  for (int p = kScanT; p >= 8; p -= kScanR) {
    const int64_t chunks = (a.rows + p - 1) / p, cost = (chunks * groups + slots - 1) / slots * (p + 6) * 64 + chunks;
    if (cost < least) { least = cost; per = p; }
  }
  return per;
}
static int scan_columns(const ftp_scan_args& a) { return a.dtype == FTP_BF16 ? 2 : 1; }
static ScanArgs scan_plan(const ftp_scan_args& a, bool backward, size_t& bytes) {
  ScanArgs k{};
  const int es = a.dtype == FTP_BF16 ? 2 : 4;
  const auto in = [&](const char*& p, int& ld, const void* m, int64_t l, int bit) { p = (const char*)m; ld = (int)(l * es); k.flags |= m ? bit : 0; };
  const auto to = [&](char*& p, int& ld, void* m, int64_t l, int bit) { p = (char*)m; ld = (int)(l * es); k.flags |= m ? bit : 0; };
  in(k.f, k.ldf, a.f, a.ldf, 0);
  in(k.x, k.ldx, a.x, a.ldx, 0);
  in(k.g, k.ldg, a.g, a.ldg, SK_G);
  k.h0 = a.h0; k.ldh0 = (int)a.ldh0;
  if (backward) {
    in(k.dy, k.lddy, a.dy, a.lddy, 0);
    to(k.df, k.lddf, a.df, a.lddf, SK_DF);
    to(k.dx, k.lddx, a.dx, a.lddx, SK_DX);
    if (a.g) to(k.dg, k.lddg, a.dg, a.lddg, SK_DG);
    k.dh_end = a.dh_end; k.lddhe = (int)a.lddhe;
    k.dh0 = a.dh0; k.lddh0 = (int)a.lddh0;
    k.flags |= (a.dh_end ? SK_DHEND : 0) | (a.dh0 ? SK_DH0 : 0);
  } else {
    to(k.y, k.ldy, a.y, a.ldy, SK_Y);
    k.h_end = a.h_end; k.ldhe = (int)a.ldhe;
    k.flags |= a.h_end ? SK_HEND : 0;
  }
  k.rows = a.rows; k.length = a.length; k.starts = a.starts;
  k.width = a.width; k.seqs = a.seqs; k.act = a.act;
  bool whole;
  k.per = scan_per(a, scan_columns(a), backward, whole);
  k.flags |= whole ? SK_WHOLE : 0;
  k.chunks = (int)((a.rows + k.per - 1) / k.per);
  bytes = 0;
  if (whole || a.rows <= kScanFew) return k;
  const size_t one = ((size_t)k.chunks * a.width * 4 + 255) & ~(size_t)255;
  const auto take = [&]() { float* p = (float*)((char*)a.ws + bytes); bytes += one; return p; };
  k.A = take();
  k.B = take();
  k.state = take();
  k.seed = take();             // copies of the states in front (backward: of the gradients behind), which the results may overwrite
  if (backward) { k.C = take(); k.back = take(); }
  return k;
}
size_t bt_scan_bytes(const ftp_scan_args& a, bool backward) {
  size_t n;
  scan_plan(a, backward, n);
  return n;
}
static unsigned scan_blocks(const ScanArgs& k, int V, bool walk) {
  const int64_t groups = (k.width + 64 * V - 1) / (64 * V);
  const int64_t waves = groups * (k.chunks + (walk && (k.starts || k.length == 0) ? (k.seqs + 63) / 64 : 0));
  return (unsigned)std::max<int64_t>(1, (waves + 3) / 4);
}
template <bool BWD, typename E, int V, bool WHOLE, int FORM>
static void scan_launch(hipStream_t st, const ScanArgs& k) {
  // what is read and written for the last time goes past the caches (16384 x 2048 bfloat16 forward 90 -> 82 us, both ways 281 -> 266)
  const bool once = past_the_caches((double)k.rows * k.width * sizeof(E) * (BWD ? 6 : 4));
  if (scan_blocks(k, V, true) >= 1u << 24) return launch_plan_failed("scan: more than 2^32 threads");
  if (!(k.flags & SK_WHOLE) && k.rows <= kScanFew) {
    constexpr int N = scan_few_waves(BWD);
    const int groups = (k.width + 64 * V - 1) / (64 * V);
    const int64_t blocks = groups + (k.starts ? ((int64_t)((k.seqs + 63) / 64) * groups + N - 1) / N : 0);
    if (BWD) hipLaunchKernelGGL((scan_back_k<E, V, WHOLE, FORM, kScanFewR, false, true>), dim3((unsigned)blocks), dim3(64 * N), 0, st, k);
    else hipLaunchKernelGGL((scan_walk_k<E, V, WHOLE, FORM, kScanFewR, false, true>), dim3((unsigned)blocks), dim3(64 * N), 0, st, k);
    return;
  }
  if (!(k.flags & SK_WHOLE)) {
    hipLaunchKernelGGL((scan_sums_k<E, V, WHOLE, FORM, BWD, kScanR>), dim3(scan_blocks(k, V, false)), dim3(256), 0, st, k);
    hipLaunchKernelGGL(scan_follow_k, dim3((k.width + 31) / 32, BWD ? 2 : 1), dim3(1024), 0, st, k);
  }
  const auto go = [&](auto f) { hipLaunchKernelGGL(f, dim3(scan_blocks(k, V, true)), dim3(256), 0, st, k); };
  constexpr bool ONCE = WHOLE && sizeof(E) * V == 4;
  if (BWD) once ? go(scan_back_k<E, V, WHOLE, FORM, kScanR, ONCE, false>) : go(scan_back_k<E, V, WHOLE, FORM, kScanR, false, false>);
  else once ? go(scan_walk_k<E, V, WHOLE, FORM, kScanR, ONCE, false>) : go(scan_walk_k<E, V, WHOLE, FORM, kScanR, false, false>);
}
template <bool BWD, typename E, int V, bool WHOLE>
static void scan_form(hipStream_t st, const ScanArgs& k, int form) {
  if (form == FTP_SCAN_ADD) scan_launch<BWD, E, V, WHOLE, FTP_SCAN_ADD>(st, k);
  else if (form == FTP_SCAN_MIX) scan_launch<BWD, E, V, WHOLE, FTP_SCAN_MIX>(st, k);
  else scan_launch<BWD, E, V, WHOLE, FTP_SCAN_UNIT>(st, k);
}
template <bool BWD>
static void scan_go(hipStream_t st, const ftp_scan_args& a) {
  size_t bytes;
  const ScanArgs k = scan_plan(a, BWD, bytes);
  if (a.dtype == FTP_F32) scan_form<BWD, float, 1, true>(st, k, a.form);
  // pairs of columns; of an odd width all but those whose last column would be alone in its wavefront (a state that is written where it was read must not be another's, too)
  else if (a.width % 128 != 1) scan_form<BWD, bf16_t, 2, true>(st, k, a.form);
  else scan_form<BWD, bf16_t, 2, false>(st, k, a.form);
}
void bt_scan(hipStream_t st, const ftp_scan_args& a) {
  const double n = (double)a.rows * a.width;
  KScope ks(st, "tok_scan", n * (a.dtype == 1 ? 2 : 4) * (3 + (a.g != nullptr)), 12 * n, a.rows, a.width, a.seqs);
  scan_go<false>(st, a);
}
void bt_scan_bwd(hipStream_t st, const ftp_scan_args& a) {
  const double n = (double)a.rows * a.width;
  KScope ks(st, "tok_scan_bwd", n * (a.dtype == 1 ? 2 : 4) * (3 + (a.df != nullptr) + (a.dx != nullptr) + (a.g ? 1 + (a.dg != nullptr) : 0)), 40 * n, a.rows, a.width, a.seqs);
  scan_go<true>(st, a);
}

}  // namespace ftp
