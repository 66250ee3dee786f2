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

enum { kScanT = 32 };
struct ScanArgs {
  ftp_scan_args a;
  int chunks, per;             // rows of a chunk: per <= kScanT
  int whole;                   // no sequence goes on from one chunk to the next
  float *A, *B, *C, *seed, *state, *back;     // [chunks][width] each
};

// V consecutive columns, of which `left` are there
template <typename E, int V>
__device__ __forceinline__ void sc_load(const E* p, int left, float v[V]) {
  if constexpr (sizeof(E) * V == 4) {
    if (left >= V) {
      uint32_t t;
      __builtin_memcpy(&t, p, 4);
      if constexpr (V == 1) v[0] = __uint_as_float(t);
      else { v[0] = __uint_as_float(t << 16); v[1] = __uint_as_float(t & 0xffff0000u); }
      return;
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = e < left ? to_f32(p[e]) : 0.f;
}
template <typename E, int V>
__device__ __forceinline__ void sc_store(E* p, int left, const float v[V]) {
  if constexpr (sizeof(E) * V == 4 && V == 2) {
    if (left >= V) {
      const uint32_t t = f32x2_to_bf16x2(v[0], v[1]);
      __builtin_memcpy(p, &t, 4);
      return;
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < left) p[e] = from_f32<E>(v[e]);
}

// where the chunk's sequences begin and end: bit t for the row r0 + t; a lane holds its row's sequence
struct ScanRows {
  uint64_t in, first, last;
  int seq;
  __device__ __forceinline__ int of(int t) const { return __builtin_amdgcn_readlane(seq, t); }
};
__device__ __forceinline__ ScanRows scan_rows(const ftp_scan_args& a, int64_t r0, int n) {
  ScanRows s;
  const int lane = threadIdx.x & 63;
  const int64_t r = r0 + lane;
  bool in = lane < n, first = false, last = false;
  if (!a.starts) {
    const int64_t q = r / a.length, at = r - q * a.length;
    s.seq = (int)q;
    first = at == 0;
    last = at == a.length - 1;
  } else {
    int lo = 0, hi = a.seqs;             // the last sequence that begins at r or in front (of several, all but one are empty)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((int64_t)a.starts[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    s.seq = lo < a.seqs ? lo : a.seqs - 1;
    in = in && lo < a.seqs && (int64_t)a.starts[lo] <= r;
    first = in && (int64_t)a.starts[s.seq] == r;
    last = in && (int64_t)a.starts[s.seq + 1] == r + 1;
  }
  s.in = __ballot(in);
  s.first = __ballot(in && first);
  s.last = __ballot(in && last);
  return s;
}

// a, 1 - a, c(a) and the derivative of c by f
struct ScanGate { float a, rest, c; };
__device__ __forceinline__ ScanGate scan_gate(float f, int form) {
  const float e = __expf(-fabsf(f)), r = __builtin_amdgcn_rcpf(1.f + e), s = e * r;      // of sigmoid(|f|) and sigmoid(-|f|) none loses its places
  ScanGate g;
  g.a = f >= 0.f ? r : s;
  g.rest = f >= 0.f ? s : r;
  if (!(f == f)) g.a = g.rest = f;
  g.c = form == FTP_SCAN_MIX ? g.rest : form == FTP_SCAN_UNIT ? sqrtf(g.rest * (1.f + g.a)) : 1.f;
  return g;
}
__device__ __forceinline__ float scan_gate_slope(const ScanGate& g, int form) {
  return form == FTP_SCAN_MIX ? -g.a * g.rest : form == FTP_SCAN_UNIT ? -g.a * g.a * sqrtf(g.rest * __builtin_amdgcn_rcpf(1.f + g.a)) : 0.f;
}

struct ScanAt { int64_t r0; int c, n, left; int chunk; };
// the wavefront's place: column groups beside one another
template <int V>
__device__ __forceinline__ bool scan_at(const ScanArgs& k, int wave, ScanAt& p) {
  const int groups = (k.a.width + 64 * V - 1) / (64 * V);
  p.chunk = wave / groups;
  p.c = (wave - p.chunk * groups) * 64 * V + (int)(threadIdx.x & 63) * V;
  p.left = k.a.width - p.c;
  p.r0 = (int64_t)p.chunk * k.per;
  const int64_t n = k.a.rows - p.r0;
  p.n = (int)(n < k.per ? n : k.per);
  return p.left > 0;
}

// A and B of a chunk; backward: C too
template <typename E, int V, bool BWD>
__global__ __launch_bounds__(256) void scan_sums_k(ScanArgs k) {
  const ftp_scan_args& a = k.a;
  const int groups = (a.width + 64 * V - 1) / (64 * V);
  const int64_t waves = (int64_t)k.chunks * groups;
  for (int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); wave < waves; wave += (int64_t)gridDim.x * 4) {
    ScanAt p;
    const bool there = scan_at<V>(k, (int)wave, p);
    const ScanRows rows = scan_rows(a, p.r0, p.n);
    if (!there) continue;
    float A[V], B[V], C[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { A[e] = 1.f; B[e] = C[e] = 0.f; }
    for (int t = 0; t < p.n; ++t) {
      const uint64_t bit = 1ull << t;
      if (!(rows.in & bit)) {            // of no sequence: nothing goes through
#pragma unroll
        for (int e = 0; e < V; ++e) A[e] = 0.f;
        continue;
      }
      const int64_t r = p.r0 + t;
      float f[V], x[V];
      sc_load<E, V>((const E*)a.f + r * a.ldf + p.c, p.left, f);
      sc_load<E, V>((const E*)a.x + r * a.ldx + p.c, p.left, x);
      if (rows.first & bit) {
        if (a.h0) sc_load<float, V>(a.h0 + (int64_t)rows.of(t) * a.ldh0 + p.c, p.left, B);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          A[e] = 0.f;
          if (!a.h0) B[e] = 0.f;
        }
        // the state in front of a sequence that goes on behind this chunk, before another chunk writes the one behind it into the same memory
        if (!BWD && k.seed) sc_store<float, V>(k.seed + (int64_t)p.chunk * a.width + p.c, p.left, B);
      }
      float dy[V], g[V], d[V];
      if (BWD) {
        sc_load<E, V>((const E*)a.dy + r * a.lddy + p.c, p.left, dy);
        if (a.g) {
          sc_load<E, V>((const E*)a.g + r * a.ldg + p.c, p.left, g);
          tactn<V>(g, a.act);
#pragma unroll
          for (int e = 0; e < V; ++e) dy[e] *= g[e];
        }
        if ((rows.last & bit) && a.dh_end) {
          sc_load<float, V>(a.dh_end + (int64_t)rows.of(t) * a.lddhe + p.c, p.left, d);
#pragma unroll
          for (int e = 0; e < V; ++e) dy[e] += d[e];
          // what arrives at the end of a sequence from a chunk in front, before another chunk writes dh0 into the same memory
          if (k.seed && !(rows.first << (63 - t))) sc_store<float, V>(k.seed + (int64_t)p.chunk * a.width + p.c, p.left, d);
        }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const ScanGate s = scan_gate(f[e], a.form);
        B[e] = fmaf(s.a, B[e], s.c * x[e]);
        A[e] *= s.a;
        if (BWD) {
          C[e] = fmaf(A[e], dy[e], C[e]);
          if (rows.last & bit) A[e] = 0.f;
        }
      }
    }
    const int64_t to = (int64_t)p.chunk * a.width + p.c;
    sc_store<float, V>(k.A + to, p.left, A);
    sc_store<float, V>(k.B + to, p.left, B);
    if (BWD) sc_store<float, V>(k.C + to, p.left, C);
  }
}

// From chunk to chunk: state[i] = the state in front of chunk i; the other way (blockIdx.y 1) back[i] = what chunk i + 1 hands back.  64 columns a block, sixteen
// threads to a column, each with its share of the chunks one behind the other: first their product and sum, then the states.
__global__ __launch_bounds__(1024) void scan_follow_k(ScanArgs k) {
  __shared__ float sa[16][64], sb[16][64];
  const int lane = threadIdx.x & 63, ty = threadIdx.x >> 6, W = k.a.width, c = blockIdx.x * 64 + lane;
  const bool rev = blockIdx.y == 1;
  const float *const A = k.A, *const B = rev ? k.C : k.B;
  float* const out = rev ? k.back : k.state;
  const int share = (k.chunks + 15) / 16, i0 = ty * share, i1 = i0 + share < k.chunks ? i0 + share : k.chunks;
  const auto at = [&](int i) { return (int64_t)(rev ? k.chunks - 1 - i : i) * W + c; };
  float a = 1.f, b = 0.f;
  if (c < W) {
#pragma unroll 8
    for (int i = i0; i < i1; ++i) {
      const float u = A[at(i)], v = B[at(i)];
      b = fmaf(u, b, v);
      a *= u;
    }
  }
  sa[ty][lane] = a;
  sb[ty][lane] = b;
  __syncthreads();
  if (c >= W) return;
  float h = 0.f;
  for (int j = 0; j < ty; ++j) h = fmaf(sa[j][lane], h, sb[j][lane]);
#pragma unroll 8
  for (int i = i0; i < i1; ++i) {
    const float u = A[at(i)], v = B[at(i)];
    out[at(i)] = h;
    h = fmaf(u, h, v);
  }
}

// states of empty sequences stay: those of the 64 from `seq0` on
template <int V>
__device__ __forceinline__ void scan_empty(const ScanArgs& k, int64_t seq0, int c, int left, const float* from, int64_t ldf, float* to, int64_t ldt) {
  if (!to || (from == to && ldf == ldt)) return;
  const ftp_scan_args& a = k.a;
  const int64_t s = seq0 + (threadIdx.x & 63);
  uint64_t todo = __ballot(s < a.seqs && (a.starts ? a.starts[s < a.seqs ? s : 0] >= a.starts[s < a.seqs ? s + 1 : 0] : a.length == 0));
  if (left <= 0) return;
  while (todo) {
    const int64_t q = seq0 + __builtin_ctzll(todo);
    todo &= todo - 1;
    float h[V];
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = 0.f;
    if (from) sc_load<float, V>(from + q * ldf + c, left, h);
    sc_store<float, V>(to + q * ldt + c, left, h);
  }
}

template <typename E, int V>
__global__ __launch_bounds__(256) void scan_walk_k(ScanArgs k) {
  const ftp_scan_args& a = k.a;
  const int groups = (a.width + 64 * V - 1) / (64 * V);
  const int64_t waves = (int64_t)k.chunks * groups, all = waves + (a.starts || a.length == 0 ? (int64_t)((a.seqs + 63) / 64) * groups : 0);
  for (int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); wave < all; wave += (int64_t)gridDim.x * 4) {
    ScanAt p;
    if (wave >= waves) {
      const int64_t w = wave - waves, block = w / groups;
      const int c = (int)(w - block * groups) * 64 * V + (int)(threadIdx.x & 63) * V;
      scan_empty<V>(k, block * 64, c, a.width - c, a.h0, a.ldh0, a.h_end, a.ldhe);
      continue;
    }
    const bool there = scan_at<V>(k, (int)wave, p);
    const ScanRows rows = scan_rows(a, p.r0, p.n);
    if (!there) continue;
    const int64_t mine = (int64_t)p.chunk * a.width + p.c;
    float h[V];
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = 0.f;
    if (!k.whole) sc_load<float, V>(k.state + mine, p.left, h);
    for (int t = 0; t < p.n; ++t) {
      const uint64_t bit = 1ull << t;
      if (!(rows.in & bit)) continue;
      const int64_t r = p.r0 + t;
      float f[V], x[V], g[V];
      sc_load<E, V>((const E*)a.f + r * a.ldf + p.c, p.left, f);
      sc_load<E, V>((const E*)a.x + r * a.ldx + p.c, p.left, x);
      if (rows.first & bit) {
        // one that goes on behind the chunk: its state from the copy
        if (!k.whole && !(rows.last >> t)) sc_load<float, V>(k.seed + mine, p.left, h);
        else if (a.h0) sc_load<float, V>(a.h0 + (int64_t)rows.of(t) * a.ldh0 + p.c, p.left, h);
        else
#pragma unroll
          for (int e = 0; e < V; ++e) h[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const ScanGate s = scan_gate(f[e], a.form);
        h[e] = fmaf(s.a, h[e], s.c * x[e]);
      }
      if (a.y) {
        float y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = h[e];
        if (a.g) {
          sc_load<E, V>((const E*)a.g + r * a.ldg + p.c, p.left, g);
          tactn<V>(g, a.act);
#pragma unroll
          for (int e = 0; e < V; ++e) y[e] *= g[e];
        }
        sc_store<E, V>((E*)a.y + r * a.ldy + p.c, p.left, y);
      }
      if ((rows.last & bit) && a.h_end) sc_store<float, V>(a.h_end + (int64_t)rows.of(t) * a.ldhe + p.c, p.left, h);
    }
  }
}

// The states of a chunk in front, then its gradients from the last row to the first.
template <typename E, int V>
__global__ __launch_bounds__(256) void scan_back_k(ScanArgs k) {
  const ftp_scan_args& a = k.a;
  const int groups = (a.width + 64 * V - 1) / (64 * V);
  const int64_t waves = (int64_t)k.chunks * groups, all = waves + (a.starts || a.length == 0 ? (int64_t)((a.seqs + 63) / 64) * groups : 0);
  for (int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); wave < all; wave += (int64_t)gridDim.x * 4) {
    ScanAt p;
    if (wave >= waves) {
      const int64_t w = wave - waves, block = w / groups;
      const int c = (int)(w - block * groups) * 64 * V + (int)(threadIdx.x & 63) * V;
      scan_empty<V>(k, block * 64, c, a.width - c, a.dh_end, a.lddhe, a.dh0, a.lddh0);
      continue;
    }
    const bool there = scan_at<V>(k, (int)wave, p);
    const ScanRows rows = scan_rows(a, p.r0, p.n);
    if (!there) continue;
    const int64_t mine = (int64_t)p.chunk * a.width + p.c;
    float before[kScanT][V], h[V], mu[V];
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = mu[e] = 0.f;
    if (!k.whole) {
      sc_load<float, V>(k.state + mine, p.left, h);
      sc_load<float, V>(k.back + mine, p.left, mu);
    }
#pragma unroll
    for (int t = 0; t < kScanT; ++t) {
      const uint64_t bit = 1ull << t;
      if (t < p.n && (rows.in & bit)) {
        const int64_t r = p.r0 + t;
        float f[V], x[V];
        sc_load<E, V>((const E*)a.f + r * a.ldf + p.c, p.left, f);
        sc_load<E, V>((const E*)a.x + r * a.ldx + p.c, p.left, x);
        if (rows.first & bit) {
          if (a.h0) sc_load<float, V>(a.h0 + (int64_t)rows.of(t) * a.ldh0 + p.c, p.left, h);
          else
#pragma unroll
            for (int e = 0; e < V; ++e) h[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
          before[t][e] = h[e];
          const ScanGate s = scan_gate(f[e], a.form);
          h[e] = fmaf(s.a, h[e], s.c * x[e]);
        }
      }
    }
#pragma unroll
    for (int t = kScanT - 1; t >= 0; --t) {
      const uint64_t bit = 1ull << t;
      if (t < p.n && (rows.in & bit)) {
        const int64_t r = p.r0 + t;
        float f[V], x[V], dy[V], df[V], dx[V];
        sc_load<E, V>((const E*)a.f + r * a.ldf + p.c, p.left, f);
        sc_load<E, V>((const E*)a.x + r * a.ldx + p.c, p.left, x);
        sc_load<E, V>((const E*)a.dy + r * a.lddy + p.c, p.left, dy);
        ScanGate s[V];
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] = scan_gate(f[e], a.form);
        if (a.g) {
          float g[V], act[V], dact[V], dg[V];
          sc_load<E, V>((const E*)a.g + r * a.ldg + p.c, p.left, g);
          tact_gradn<V>(g, act, dact, a.act);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            dg[e] = dy[e] * fmaf(s[e].a, before[t][e], s[e].c * x[e]) * dact[e];
            dy[e] *= act[e];
          }
          if (a.dg) sc_store<E, V>((E*)a.dg + r * a.lddg + p.c, p.left, dg);
        }
        if (rows.last & bit) {
          if (!a.dh_end) {
#pragma unroll
            for (int e = 0; e < V; ++e) mu[e] = 0.f;
          } else if (!k.whole && !(rows.first << (63 - t))) {      // a sequence from a chunk in front: the copy of what arrives at its end
            sc_load<float, V>(k.seed + mine, p.left, mu);
          } else {
            sc_load<float, V>(a.dh_end + (int64_t)rows.of(t) * a.lddhe + p.c, p.left, mu);
          }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float lam = dy[e] + mu[e];
          dx[e] = lam * s[e].c;
          df[e] = lam * fmaf(before[t][e], s[e].a * s[e].rest, x[e] * scan_gate_slope(s[e], a.form));
          mu[e] = lam * s[e].a;
        }
        if (a.df) sc_store<E, V>((E*)a.df + r * a.lddf + p.c, p.left, df);
        if (a.dx) sc_store<E, V>((E*)a.dx + r * a.lddx + p.c, p.left, dx);
        if ((rows.first & bit) && a.dh0) sc_store<float, V>(a.dh0 + (int64_t)rows.of(t) * a.lddh0 + p.c, p.left, mu);
      }
    }
  }
}

static int scan_per(const ftp_scan_args& a, bool& whole) {
  whole = a.starts ? a.rows <= kScanT : a.length <= kScanT;
  return !a.starts && a.length > 0 && whole ? (int)(kScanT / a.length * a.length) : kScanT;
}
static ScanArgs scan_plan(const ftp_scan_args& a, bool backward, size_t& bytes) {
  ScanArgs k{};
  k.a = a;
  bool whole;
  k.per = scan_per(a, whole);
  k.whole = whole;
  k.chunks = (int)((a.rows + k.per - 1) / k.per);
  bytes = 0;
  if (whole) return k;
  const size_t one = ((size_t)k.chunks * a.width * 4 + 255) & ~(size_t)255;
  const auto take = [&]() { float* p = (float*)((char*)a.ws + bytes); bytes += one; return p; };
  k.A = take();
  k.B = take();
  k.state = take();
  // a copy of the states in front (backward: of the gradients behind) is needed where the results may overwrite them
  if (backward) { k.C = take(); k.back = take(); }
  const float* const from = backward ? a.dh_end : a.h0;
  k.seed = take();
  if (!from && backward) k.seed = nullptr;
  return k;
}
size_t bt_scan_bytes(const ftp_scan_args& a, bool backward) {
  size_t n;
  scan_plan(a, backward, n);
  return n;
}
// bfloat16: two columns a lane
template <typename F>
static void scan_by_type(int dt, F f) {
  if (dt == FTP_BF16) f((bf16_t*)nullptr, std::integral_constant<int, 2>());
  else f((float*)nullptr, std::integral_constant<int, 1>());
}
static unsigned scan_blocks(const ScanArgs& k, int V, bool walk) {
  const int64_t groups = (k.a.width + 64 * V - 1) / (64 * V);
  const int64_t waves = groups * (k.chunks + (walk && (k.a.starts || k.a.length == 0) ? (k.a.seqs + 63) / 64 : 0));
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>((waves + 3) / 4, 1 << 20));
}
template <bool BWD>
static void scan_go(hipStream_t st, const ftp_scan_args& a) {
  size_t bytes;
  const ScanArgs k = scan_plan(a, BWD, bytes);
  scan_by_type(a.dtype, [&](auto* e, auto v) {
    typedef std::remove_pointer_t<decltype(e)> E;
    constexpr int V = decltype(v)::value;
    if (!k.whole) {
      hipLaunchKernelGGL((scan_sums_k<E, V, BWD>), dim3(scan_blocks(k, V, false)), dim3(256), 0, st, k);
      hipLaunchKernelGGL(scan_follow_k, dim3((a.width + 63) / 64, BWD ? 2 : 1), dim3(1024), 0, st, k);
    }
    if (BWD) hipLaunchKernelGGL((scan_back_k<E, V>), dim3(scan_blocks(k, V, true)), dim3(256), 0, st, k);
    else hipLaunchKernelGGL((scan_walk_k<E, V>), dim3(scan_blocks(k, V, true)), dim3(256), 0, st, k);
  });
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
