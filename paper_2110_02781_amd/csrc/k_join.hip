// Dropout and the join of a block's output with the stream and its norms, forward and backward.
#include <type_traits>

#include "between.h"
#include "token_dev.h"

namespace ftp {

// ---------------------------------------------------------------- the mask
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011): ten rounds, each two products of 32 bits whose high words go crosswise into the other pair.
__device__ __forceinline__ uint4 philox10(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}
struct MaskKey { uint32_t k0, k1; };
__device__ __forceinline__ MaskKey mask_key(const DropMask& m) {
  const uint64_t s = m.seed + (m.seed_dev ? *m.seed_dev : 0);
  return MaskKey{(uint32_t)s, (uint32_t)(s >> 32)};
}
// the columns 8 j .. 8 j + 7 of a row: all ones where a value is kept, zero where it is dropped
__device__ __forceinline__ void mask8(const DropMask& m, MaskKey k, uint64_t row, uint32_t j, uint32_t keep[8]) {
  asm volatile("" : "+s"(k.k0), "+s"(k.k1));             // the rounds' keys are added up by the scalar unit each time; kept, they would take twenty registers
  const uint4 w = philox10(make_uint4(j, m.site, (uint32_t)row, (uint32_t)(row >> 32)), k.k0, k.k1);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w}, under = m.least - 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    keep[2 * i] = (uint32_t)((int32_t)(under - (u[i] & 0xffffu)) >> 31);
    keep[2 * i + 1] = (uint32_t)((int32_t)(under - (u[i] >> 16)) >> 31);
  }
}
// what is dropped is 0, whatever it was
__device__ __forceinline__ float dropped(float v, uint32_t keep) { return __uint_as_float(__float_as_uint(v) & keep); }

// ---------------------------------------------------------------- dropout
template <typename E, bool ONCE>
__global__ __launch_bounds__(256) void dropout_k(DropMask m, int64_t t0, int rows, int cols, const E* x, int64_t ldx, const E* r, int64_t ldr, E* y, int64_t ldy) {
  const uint32_t per = (cols + 7) / 8, all = (uint32_t)rows * per;
  const MaskKey key = mask_key(m);
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) {
    const uint32_t row = i / per, j = i - row * per;
    const int64_t t = t0 + row;
    const int left = cols - (int)(j * 8);
    float v[8], o[8];
    ONCE ? tk_load8_once<E>(x + t * ldx + j * 8, left, v) : tk_load8<E>(x + t * ldx + j * 8, left, v);
    if (r) ONCE ? tk_load8_once<E>(r + t * ldr + j * 8, left, o) : tk_load8<E>(r + t * ldr + j * 8, left, o);
    if (m.least) {
      uint32_t k[8];
      mask8(m, key, (uint64_t)(m.row0 + t), j, k);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = dropped(v[e] * m.up, k[e]);
    }
    if (r) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += o[e];
    }
    ONCE ? tk_store8_once<E>(y + t * ldy + j * 8, left, v) : tk_store8<E>(y + t * ldy + j * 8, left, v);
  }
}
void bt_dropout(hipStream_t st, int dt, int64_t rows, int cols, const DropMask& m, const void* x, int64_t ldx, const void* r, int64_t ldr, void* y, int64_t ldy) {
  KScope ks(st, "tok_dropout", (double)rows * cols * (dt == 1 ? 2 : 4) * (r ? 3 : 2), 2.0 * rows * cols, rows, cols);
  const int64_t per = (cols + 7) / 8;
  const bool once = past_the_caches((double)rows * cols * (dt == 1 ? 2 : 4) * (r ? 3 : 2));
  by_rows(rows, per, [&](int64_t t0, int n) {
    const dim3 b(blocks_of(n * per, 8192));
    const auto go = [&](auto k, auto* e) {
      typedef std::remove_pointer_t<decltype(e)> E;
      hipLaunchKernelGGL(k, b, dim3(256), 0, st, m, t0, n, cols, (const E*)x, ldx, (const E*)r, ldr, (E*)y, ldy);
    };
    if (dt == 1) once ? go(dropout_k<bf16_t, true>, (bf16_t*)nullptr) : go(dropout_k<bf16_t, false>, (bf16_t*)nullptr);
    else once ? go(dropout_k<float, true>, (float*)nullptr) : go(dropout_k<float, false>, (float*)nullptr);
  });
}

// ---------------------------------------------------------------- the join
// Sum over the block's threads of one value or of two, the same in all of them: within a wavefront into its last lane, through LDS into groups of T / 64 lanes of all
// wavefronts, and there once more.  `s` is used in turn by calls that follow one another.
template <int N>
__device__ __forceinline__ float lanes_sum(float v) {            // over N consecutive lanes, 2 .. 32
  v += dpp_move<0xB1>(v);
  if (N > 2) v += dpp_move<0x4E>(v);
  if (N > 4) v += dpp_move<0x141>(v);
  if (N > 8) v += dpp_move<0x140>(v);
  if (N > 16) v += __shfl_xor(v, 16);
  return v;
}
constexpr int join_waves(int T) { return T < 64 ? 1 : T / 64; }
template <int T>
__device__ __forceinline__ float block_sum(float a, float2 (*s)[join_waves(T)], int& turn) {
  if constexpr (T < 64) return lanes_sum<T>(a);
  if constexpr (T == 64) return wave_sum(a);
  a = wave_sum_last(a);
  float2* const p = s[turn ^= 1];
  if ((threadIdx.x & 63) == 63) p[threadIdx.x >> 6].x = a;
  __syncthreads();
  return lanes_sum<join_waves(T)>(p[threadIdx.x & (join_waves(T) - 1)].x);
}
template <int T>
__device__ __forceinline__ float2 block_sum2(float a, float b, float2 (*s)[join_waves(T)], int& turn) {
  if constexpr (T < 64) return make_float2(lanes_sum<T>(a), lanes_sum<T>(b));
  if constexpr (T == 64) return make_float2(wave_sum(a), wave_sum(b));
  a = wave_sum_last(a);
  b = wave_sum_last(b);
  float2* const p = s[turn ^= 1];
  if ((threadIdx.x & 63) == 63) p[threadIdx.x >> 6] = make_float2(a, b);
  __syncthreads();
  const float2 t = p[threadIdx.x & (join_waves(T) - 1)];
  return make_float2(lanes_sum<join_waves(T)>(t.x), lanes_sum<join_waves(T)>(t.y));
}

// one row's operands, eight columns at a time
template <typename E>
struct JoinRow {
  const ftp_join_args& a;
  const DropMask& m;
  MaskKey key;
  int64_t row;
  float mb, rb;                          // mean and inverse deviation of b (with post)
  __device__ __forceinline__ void weight(const float* w, int c, int left, float v[8], float none) const {
    if (w) tk_load8<float>(w + c, left, v);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = none;
  }
  __device__ __forceinline__ void load(const void* p, int64_t ld, int c, int left, float v[8]) const {
    if (p) tk_load8<E>((const E*)p + row * ld + c, left, v);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
  }
  // bh: b normed (or b); cc: what the gate multiplies
  __device__ __forceinline__ void branch(int c, int left, float bh[8], float cc[8]) const {
    load(a.b, a.ldb, c, left, bh);
    if (!a.post) {
#pragma unroll
      for (int e = 0; e < 8; ++e) cc[e] = bh[e];
      return;
    }
    float w[8], o[8];
    weight(a.post_w, c, left, w, 1.f);
    weight(a.post_bias, c, left, o, 0.f);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      bh[e] = e < left ? (bh[e] - mb) * rb : 0.f;
      cc[e] = fmaf(bh[e], w[e], o[e]);
    }
  }
  __device__ __forceinline__ void mask(int c, uint32_t k[8]) const {
    if (m.least) mask8(m, key, (uint64_t)(m.row0 + row), (uint32_t)c / 8, k);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) k[e] = ~0u;
  }
  __device__ __forceinline__ void gate(int c, int left, float v[8]) const {
    if (!a.gate) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 1.f;
      return;
    }
    const int64_t at = row / a.gate_rows * a.ldg + c;
    if (a.gate_dtype == FTP_F32) tk_load8<float>((const float*)a.gate + at, left, v);
    else tk_load8<bf16_t>((const bf16_t*)a.gate + at, left, v);
  }
  // y; where they are wanted, what made it
  __device__ __forceinline__ void stream(int c, int left, float y[8], float bh[8], float cc[8], uint32_t k[8], float g[8]) const {
    load(a.x, a.ldx, c, left, y);
    if (!a.b) return;
    branch(c, left, bh, cc);
    mask(c, k);
    gate(c, left, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fmaf(a.scale * m.up * g[e], dropped(cc[e], k[e]), y[e]);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= left) y[e] = 0.f;
  }
};
__device__ __forceinline__ float inv_dev(float squares, int width, float eps) { return 1.f / sqrtf(squares / (float)width + eps); }

// Rows of any width, each by one block in passes over its columns: what a pass needs is read (and computed) again, from the caches as a rule.  1024 threads: 2048 x 16384 bfloat16 with
// two norms, gate and dropout, both ways, 481 us (385 without gate and dropout); 256 threads 917.
enum { kJoinT = 1024 };
template <typename E>
struct JoinWide {
  JoinRow<E> r;
  int N, turn;
  float2 (*s)[kJoinT / 64];
  template <typename F>
  __device__ __forceinline__ void columns(F f) const {
    for (int c = threadIdx.x * 8; c < N; c += kJoinT * 8) f(c, N - c);
  }
  // mean and inverse deviation of what get(c, left, v) gives
  template <typename G>
  __device__ __forceinline__ void deviation(G get, float& mean, float& rinv) {
    mean = 0.f;
    if (r.a.norm == FTP_NORM_LAYER) {
      float t = 0.f;
      columns([&](int c, int left) {
        float v[8];
        get(c, left, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) t += e < left ? v[e] : 0.f;
      });
      mean = block_sum<kJoinT>(t, s, turn) / (float)N;
    }
    float q = 0.f;
    columns([&](int c, int left) {
      float v[8];
      get(c, left, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = e < left ? v[e] - mean : 0.f;
        q = fmaf(d, d, q);
      }
    });
    rinv = inv_dev(block_sum<kJoinT>(q, s, turn), N, r.a.eps);
  }
  __device__ __forceinline__ void branch_deviation() {
    r.mb = 0.f;
    r.rb = 1.f;
    if (r.a.b && r.a.post) {
      float mean, rinv;
      deviation([&](int c, int left, float v[8]) { r.load(r.a.b, r.a.ldb, c, left, v); }, mean, rinv);
      r.mb = mean;
      r.rb = rinv;
    }
  }
  __device__ __forceinline__ void stream_deviation(float& mean, float& rinv) {
    deviation([&](int c, int left, float v[8]) { float bh[8], cc[8], g[8]; uint32_t k[8]; r.stream(c, left, v, bh, cc, k, g); }, mean, rinv);
  }
};

template <typename E>
__global__ __launch_bounds__(kJoinT) void join_wide_k(ftp_join_args a, DropMask m) {
  __shared__ float2 s[2][kJoinT / 64];
  JoinWide<E> w{JoinRow<E>{a, m, mask_key(m), 0, 0.f, 1.f}, a.width, 0, s};
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    w.r.row = row;
    w.branch_deviation();
    float my = 0.f, ry = 1.f;
    if (a.n) w.stream_deviation(my, ry);
    // y may lie where x or b does: everything has been read but what this thread writes
    w.columns([&](int c, int left) {
      float y[8], bh[8], cc[8], g[8];
      uint32_t k[8];
      w.r.stream(c, left, y, bh, cc, k, g);
      if (a.y) tk_store8<E>((E*)a.y + row * a.ldy + c, left, y);
      if (a.n) {
        float pw[8], pb[8];
        w.r.weight(a.pre_w, c, left, pw, 1.f);
        w.r.weight(a.pre_bias, c, left, pb, 0.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = fmaf((y[e] - my) * ry, pw[e], pb[e]);
        tk_store8<E>((E*)a.n + row * a.ldn + c, left, y);
      }
    });
  }
}
// Rows of up to kJoinHeld columns: a block of T threads has eight columns in each and everything it needs of a row in registers.  What a row costs beside its bytes are
// the meetings of its wavefronts, one for each mean.  ROWS: 1 where they are a
// multiple of eight columns, 2 where besides the call's operands are more than the caches hold, and go past them.
enum { JK_X = 1, JK_B = 2, JK_GATE = 4, JK_DY = 8, JK_DN = 16, JK_Y = 32, JK_N = 64, JK_DX = 128, JK_DB = 256, JK_DGATE = 512, JK_POST = 1024, JK_LAYER = 2048, JK_GATE_F32 = 4096, JK_GATE_ADD = 8192 };
// what the kernels need of a call's record, in as few scalar registers as it goes into: row distances in bytes, questions as bits
struct JoinK {
  const char *x, *b, *gate, *dy, *dn;
  char *y, *n, *dx, *db, *dgate;
  int ldx, ldb, ldg, lddy, lddn, ldy, ldn, lddx, lddb, lddg;
  const float *pre_w, *pre_bias, *post_w, *post_bias;
  int64_t rows, gate_rows;
  int width, flags;
  float eps, scale;            // scale: with the mask's factor
};
static JoinK join_k(const ftp_join_args& a, const DropMask& m, bool backward) {
  JoinK k{};
  const int es = a.dtype == FTP_BF16 ? 2 : 4, gs = a.gate_dtype == FTP_F32 ? 4 : 2;
  const auto put = [&](const char*& p, int& ld, const void* from, int64_t l, int size, int bit) {
    p = (const char*)from;
    ld = (int)(l * size);
    k.flags |= from ? bit : 0;
  };
  const auto put_out = [&](char*& p, int& ld, void* to, int64_t l, int size, int bit) {
    p = (char*)to;
    ld = (int)(l * size);
    k.flags |= to ? bit : 0;
  };
  put(k.x, k.ldx, a.x, a.ldx, es, JK_X);
  put(k.b, k.ldb, a.b, a.ldb, es, JK_B);
  if (a.b) put(k.gate, k.ldg, a.gate, a.ldg, gs, JK_GATE);
  if (backward) {
    put(k.dy, k.lddy, a.dy, a.lddy, es, JK_DY);
    put(k.dn, k.lddn, a.dn, a.lddn, es, JK_DN);
    put_out(k.dx, k.lddx, a.dx, a.lddx, es, JK_DX);
    put_out(k.db, k.lddb, a.db, a.lddb, es, JK_DB);
    put_out(k.dgate, k.lddg, a.dgate, a.lddg, gs, JK_DGATE);
  } else {
    put_out(k.y, k.ldy, a.y, a.ldy, es, JK_Y);
    put_out(k.n, k.ldn, a.n, a.ldn, es, JK_N);
  }
  k.flags |= (a.post ? JK_POST : 0) | (a.norm == FTP_NORM_LAYER ? JK_LAYER : 0) | (gs == 4 ? JK_GATE_F32 : 0) | (a.gate_accumulate ? JK_GATE_ADD : 0);
  k.pre_w = a.pre_w; k.pre_bias = a.pre_bias; k.post_w = a.post_w; k.post_bias = a.post_bias;
  k.rows = a.rows; k.gate_rows = a.gate ? a.gate_rows : INT64_MAX;
  k.width = a.width; k.eps = a.eps; k.scale = a.scale * m.up;
  return k;
}

template <typename E> struct Raw8 { u4v_t a[sizeof(E) / 2]; };
template <typename E, bool WHOLE, bool ONCE = false>
__device__ __forceinline__ Raw8<E> raw8_load(const char* row, int c, int left, int back = 0) {
  const E* const p = (const E*)row + (uint32_t)(c - back);
  Raw8<E> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(E) / 2; ++i) r.a[i] = u4v_t{0, 0, 0, 0};
  if (left >= 8 || back) {
    if (ONCE) {
      r.a[0] = tk_ld16_once<E>(p);
      if constexpr (sizeof(E) == 4) r.a[1] = tk_ld16_once<E>(p + 4);
    } else {
      r.a[0] = tk_ld16<E>(p);
      if constexpr (sizeof(E) == 4) r.a[1] = tk_ld16<E>(p + 4);
    }
  } else if (!WHOLE) {
#pragma unroll
    for (int e = 0; e < 7; ++e) {
      if (e >= left) break;
      if constexpr (sizeof(E) == 4) r.a[e / 4][e & 3] = __float_as_uint(p[e]);
      else r.a[0][e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
    }
  }
  return r;
}
// two-byte columns `back` places down
__device__ __forceinline__ void columns_down(int back, uint32_t w[4]) {
#pragma unroll
  for (int by = 2; by; --by)
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = back & (2 * by) ? (i + by < 4 ? w[i + by] : 0) : w[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = back & 1 ? __builtin_amdgcn_alignbit(i < 3 ? w[i + 1] : 0, w[i], 16) : w[i];
}
template <typename E, bool WHOLE>
__device__ __forceinline__ void raw8_open(const Raw8<E>& r, int back, float v[8]) {
  constexpr int N = 2 * sizeof(E);
  uint32_t w[N];
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = r.a[i / 4][i & 3];
  if (!WHOLE && N == 4) columns_down(back, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(N == 8 ? w[i] : i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
}
// The last columns of a bfloat16 row, where they are fewer than eight, are read with those in front of them and moved down when they are needed: one load, as for all others (column by
// column each load is waited for, to be joined to the one in front: 19759 x 309 both ways 135 us instead of 82).  Columns of four bytes, which are nobody's half, are read one by one
// (moved down, 1000 x 1001 both ways 29.5 us instead of 26.5).
template <typename E, bool WHOLE>
__device__ __forceinline__ int row_back(int c, int left) { return !WHOLE && sizeof(E) == 2 && c > 0 && left > 0 && left < 8 ? 8 - left : 0; }
template <typename E, bool WHOLE, bool ONCE = false>
__device__ __forceinline__ void row_store8(char* row, int c, int left, const float v[8]) {
  if (!(WHOLE ? left >= 8 : left > 0)) return;
  if (ONCE) tk_store8_once<E>((E*)row + (uint32_t)c, WHOLE ? 8 : left, v);
  else tk_store8<E>((E*)row + (uint32_t)c, WHOLE ? 8 : left, v);
}
// the operands of a row: x, b, the gate's row, backward dy and dn as well
template <typename E, bool BWD>
struct JoinIn {
  Raw8<E> x, b, dy, dn;
  u4v_t g, g2;                 // the gate's row: bfloat16 in g
  __device__ __forceinline__ void take(const JoinIn& o) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(E) / 2; ++i) {
      x.a[i] = o.x.a[i];
      b.a[i] = o.b.a[i];
      if (BWD) { dy.a[i] = o.dy.a[i]; dn.a[i] = o.dn.a[i]; }
    }
    g = o.g;
    g2 = o.g2;
  }
};
// The questions of a call as they are asked in the loop over its rows: tested there anew (one scalar instruction each), because as conditions that the compiler keeps they
// take two scalar registers each, more than there are
__device__ __forceinline__ int join_flags(int f) {
  asm volatile("" : "+s"(f));
  return f;
}
// the rows of the operands that are asked for next
struct JoinWalk {
  const char *x, *b, *gate, *dy, *dn;
  int to_next;                 // rows until the gate's next
};
template <bool BWD>
__device__ __forceinline__ JoinWalk join_walk(const JoinK& k, int64_t row) {
  JoinWalk w{k.x + row * k.ldx, k.b + row * k.ldb, k.gate, nullptr, nullptr, 0x7fffffff};
  if (k.flags & JK_GATE) {
    const int64_t q = k.gate_rows == 1 ? row : row / k.gate_rows, rest = k.gate_rows == 1 ? 1 : (q + 1) * k.gate_rows - row;
    w.gate += q * k.ldg;
    if (rest < w.to_next) w.to_next = (int)rest;
  }
  if (BWD) { w.dy = k.dy + row * k.lddy; w.dn = k.dn + row * k.lddn; }
  return w;
}
template <typename E, bool BWD, bool WHOLE, bool ONCE>
__device__ __forceinline__ void join_ask(const JoinK& k, int flags, JoinWalk& w, int c, int left, int back, JoinIn<E, BWD>& in) {
  if (flags & JK_X) in.x = raw8_load<E, WHOLE, ONCE>(w.x, c, left, back);
  w.x += k.ldx;
  if (flags & JK_B) in.b = raw8_load<E, WHOLE, ONCE>(w.b, c, left, back);
  w.b += k.ldb;
  if (flags & JK_GATE) {
    const bool wide = sizeof(E) == 4 || (flags & JK_GATE_F32);
    const int down = wide ? 0 : back;
    const char* const p = w.gate + (uint32_t)(c - down) * (wide ? 4u : 2u);
    u4v_t lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
    if (left >= 8 || down) {
      lo = tk_ld16<bf16_t>((const bf16_t*)p);
      if (wide) hi = tk_ld16<bf16_t>((const bf16_t*)p + 8);
    } else if (!WHOLE) {
#pragma unroll
      for (int e = 0; e < 7; ++e) {
        if (e >= left) break;
        const uint32_t u = wide ? ((const uint32_t*)p)[e] : (uint32_t)((const bf16_t*)p)[e] << (16 * (e & 1));
        const int at = wide ? e : e / 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          lo[i] |= at == i ? u : 0;
          hi[i] |= at == i + 4 ? u : 0;
        }
      }
    }
    in.g = lo;
    in.g2 = hi;
    if (--w.to_next == 0) {
      w.gate += k.ldg;
      w.to_next = k.gate_rows < 0x7fffffff ? (int)k.gate_rows : 0x7fffffff;
    }
  }
  if constexpr (BWD) {
    if (flags & JK_DY) in.dy = raw8_load<E, WHOLE, ONCE>(w.dy, c, left, back);
    w.dy += k.lddy;
    if (flags & JK_DN) in.dn = raw8_load<E, WHOLE, ONCE>(w.dn, c, left, back);
    w.dn += k.lddn;
  }
}
template <typename E, bool WHOLE>
__device__ __forceinline__ void join_open(bool there, const Raw8<E>& r, int back, float v[8]) {
  if (there) raw8_open<E, WHOLE>(r, back, v);
  else
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
}
// scale * gate
template <typename E, bool BWD, bool WHOLE>
__device__ __forceinline__ void join_open_gate(const JoinK& k, int flags, const JoinIn<E, BWD>& in, int back, float g[8]) {
  if (!(flags & JK_GATE)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = k.scale;
    return;
  }
  const bool wide = sizeof(E) == 4 || (flags & JK_GATE_F32);
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = i < 4 ? in.g[i & 3] : in.g2[i & 3];
  if (!WHOLE && !wide) columns_down(back, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] = __uint_as_float(wide ? w[e] : e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] *= k.scale;
}
template <bool WHOLE>
__device__ __forceinline__ void join_weight(const float* w, int c, int left, float none, float v[8]) {
  if (w) {
    raw8_open<float, WHOLE>(raw8_load<float, WHOLE>((const char*)w, c, left), 0, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = none;
  }
}
// v (zeros past the row's end) less its mean (layer), and its inverse deviation
template <int T, bool WHOLE>
__device__ __forceinline__ float join_deviation(const JoinK& k, int flags, float inv, int left, float v[8], float2 (*s)[join_waves(T)], int& turn) {
  if (flags & JK_LAYER) {
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) t += v[e];
    const float mean = block_sum<T>(t, s, turn) * inv;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (WHOLE ? left > 0 : e < left) ? v[e] - mean : 0.f;
  }
  float q = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) q = fmaf(v[e], v[e], q);
  return 1.f / sqrtf(fmaf(block_sum<T>(q, s, turn), inv, k.eps));
}

// Rows of up to 128 columns take 16 lanes and those of up to 256 take 32: a wavefront has four rows or two at a time, each group of lanes its own range
// (a wavefront a row: 65536 x 128 bfloat16, one norm, forward 23 us and both ways 89; so 12 and 46).
template <int T>
__device__ __forceinline__ int join_lane() { return T < 64 ? threadIdx.x & (T - 1) : threadIdx.x; }
template <int T>
__device__ __forceinline__ int64_t join_walker() { return T < 64 ? (int64_t)blockIdx.x * (64 / T) + threadIdx.x / T : blockIdx.x; }
constexpr int join_walkers(int T) { return T < 64 ? 64 / T : 1; }        // of a block

template <typename E, int T, int ROWS>
__global__ __launch_bounds__(64 * join_waves(T)) void join_row_k(JoinK k, DropMask m, int64_t per) {
  constexpr bool WHOLE = ROWS > 0, ONCE = ROWS == 2;
  __shared__ float2 s[2][join_waves(T)];
  const int me = join_lane<T>(), c = me * 8, left = k.width - c, back = row_back<E, WHOLE>(c, left);
  const float inv = 1.f / (float)k.width;
  const MaskKey key = mask_key(m);
  const int64_t r0 = join_walker<T>() * per, r1 = r0 + per < k.rows ? r0 + per : k.rows;
  if (T < 64 && r0 >= k.rows) return;
  int turn = 0, flags = k.flags;
  JoinWalk at = join_walk<false>(k, r0);
  JoinIn<E, false> in, next;
  join_ask<E, false, WHOLE, ONCE>(k, flags, at, c, left, back, in);
  char *py = k.y + r0 * k.ldy, *pn = k.n + r0 * k.ldn;
  float pw[8], pb[8], qw[8], qb[8];
  join_weight<WHOLE>(k.pre_w, c, left, 1.f, pw);
  join_weight<WHOLE>(k.pre_bias, c, left, 0.f, pb);
  join_weight<WHOLE>(k.post_w, c, left, 1.f, qw);
  join_weight<WHOLE>(k.post_bias, c, left, 0.f, qb);
  uint64_t number = (uint64_t)(m.row0 + r0);
  for (int row = (int)(r1 - r0); row > 0; --row, ++number) {
    flags = join_flags(k.flags);
    if (row > 1) join_ask<E, false, WHOLE, ONCE>(k, flags, at, c, left, back, next);
    float y[8];
    join_open<E, WHOLE>(flags & JK_X, in.x, back, y);
    if (flags & JK_B) {
      float v[8], g[8];
      raw8_open<E, WHOLE>(in.b, back, v);
      if (flags & JK_POST) {
        const float r = join_deviation<T, WHOLE>(k, flags, inv, left, v, s, turn);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e] * r, qw[e], qb[e]);
      }
      join_open_gate<E, false, WHOLE>(k, flags, in, back, g);
      if (m.least) {
        uint32_t keep[8];
        mask8(m, key, number, me, keep);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = dropped(v[e], keep[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = (WHOLE ? left > 0 : e < left) ? fmaf(g[e], v[e], y[e]) : 0.f;
    }
    if (flags & JK_Y) row_store8<E, WHOLE, ONCE>(py, c, left, y);
    py += k.ldy;
    if (flags & JK_N) {
      const float r = join_deviation<T, WHOLE>(k, flags, inv, left, y, s, turn);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = fmaf(y[e] * r, pw[e], pb[e]);
      row_store8<E, WHOLE, ONCE>(pn, c, left, y);
    }
    pn += k.ldn;
    in.take(next);
  }
}
enum { kJoinHeld = 8192 };
static int join_threads(int width) {
  int t = 16;
  while (t * 8 < width) t *= 2;
  return t;
}
template <typename F>
static void join_by_threads(int t, F f) {
  if (t == 16) f(std::integral_constant<int, 16>());
  else if (t == 32) f(std::integral_constant<int, 32>());
  else if (t == 64) f(std::integral_constant<int, 64>());
  else if (t == 128) f(std::integral_constant<int, 128>());
  else if (t == 256) f(std::integral_constant<int, 256>());
  else if (t == 512) f(std::integral_constant<int, 512>());
  else f(std::integral_constant<int, 1024>());
}

void bt_join(hipStream_t st, const ftp_join_args& a, const DropMask& m) {
  const double n = (double)a.rows * a.width;
  const double bytes = n * (a.dtype == 1 ? 2 : 4) * ((a.x != nullptr) + (a.b != nullptr) + (a.y != nullptr) + (a.n != nullptr) + (a.gate && a.gate_rows == 1));
  KScope ks(st, "tok_join", bytes, 15 * n, a.rows, a.width);
  const bool once = past_the_caches(bytes);
  if (a.width <= kJoinHeld) {
    const int t = join_threads(a.width);
    // forward there are no blocks' sums: four rounds of the wavefronts that the card holds (16384 x 1024 34 us, one round 37), sixteen where a wavefront has several rows (400000 x 128
    // 72 us, four 85, one 99)
    const int64_t want = std::min<int64_t>(a.rows, (t < 64 ? 1024 : 256) * 4096 / t), per = (a.rows + want - 1) / want;
    const int64_t walkers = (a.rows + per - 1) / per;
    const dim3 g((unsigned)((walkers + join_walkers(t) - 1) / join_walkers(t))), b(64 * join_waves(t));
    join_by_threads(t, [&](auto tc) {
      constexpr int T = decltype(tc)::value;
      const JoinK k = join_k(a, m, false);
      const auto go = [&](auto f) { hipLaunchKernelGGL(f, g, b, 0, st, k, m, per); };
      const auto by = [&](auto* e) {
        typedef std::remove_pointer_t<decltype(e)> E;
        a.width % 8 ? go(join_row_k<E, T, 0>) : once ? go(join_row_k<E, T, 2>) : go(join_row_k<E, T, 1>);
      };
      if (a.dtype == FTP_BF16) by((bf16_t*)nullptr);
      else by((float*)nullptr);
    });
    return;
  }
  const dim3 b((unsigned)std::min<int64_t>(a.rows, 1 << 20));
  if (a.dtype == FTP_BF16) hipLaunchKernelGGL(join_wide_k<bf16_t>, b, dim3(kJoinT), 0, st, a, m);
  else hipLaunchKernelGGL(join_wide_k<float>, b, dim3(kJoinT), 0, st, a, m);
}

// ---------------------------------------------------------------- its backward
// A block has a range of rows one behind the other and adds up what the weights' gradients (and that of a gate that rows share) get from them; the
// blocks' sums are added in their order.  A range never has rows of a gate's group and of only a part of another: whole groups, or a part of one.
struct JoinRanges {
  int64_t per;         // rows of a block; with parts > 1: of a part
  int64_t group;       // rows that share a gate row (all of them where there is none, or one each)
  int parts;           // blocks of a group
  int blocks;
  int sums;            // rows of the weights' sums: one of each block of threads, which may have several ranges
};
static bool join_biased(const ftp_join_args& a) { return a.dpre_bias || a.dpost_bias || (a.post && a.post_bias); }
// Wavefronts that a SIMD holds of the kernel that a call takes.  As many blocks as the card holds go through their rows at once: a second, shorter round leaves most of it idle, and more
// blocks are more sums (bfloat16 forward and backward with four to a SIMD where it holds three: 16384 x 1024 111 us instead of 102, 400000 x 128 271 instead of 234; float where it holds
// two: 8000 x 1024 88 instead of 79)
static int join_resident(const ftp_join_args& a, int t) {
  if (t == 1024) return 4;
  if (t == 512) return a.dtype == FTP_BF16 ? 4 : 2;
  return a.dtype == FTP_BF16 && !join_biased(a) ? 3 : 2;
}
static JoinRanges join_ranges(const ftp_join_args& a) {
  const int t = a.width <= kJoinHeld ? join_threads(a.width) : 1024;
  const int64_t blocks = 256 * 4 * 64 * join_resident(a, t) / t, want = std::max<int64_t>(1, (a.rows + blocks - 1) / blocks);
  JoinRanges r{want, 0, 1, 0, 0};
  r.group = a.gate && a.gate_rows > 1 ? std::min(a.gate_rows, a.rows) : 0;
  if (r.group == 0) {
    r.blocks = (int)((a.rows + want - 1) / want);
  } else if (r.group <= want) {
    r.per = want / r.group * r.group;
    r.blocks = (int)((a.rows + r.per - 1) / r.per);
  } else {
    r.parts = (int)((r.group + want - 1) / want);
    r.per = (r.group + r.parts - 1) / r.parts;
    r.blocks = (int)((a.rows + r.group - 1) / r.group) * r.parts;
  }
  r.sums = (r.blocks + join_walkers(t) - 1) / join_walkers(t);
  return r;
}
enum { JP_PRE_W, JP_PRE_BIAS, JP_POST_W, JP_POST_BIAS, JP_GATE, JP_ALL };
struct JoinParts { float* p[JP_ALL]; };           // [blocks][width] each, or null

__device__ __forceinline__ void join_range(const JoinRanges& g, int64_t walker, int64_t rows, int64_t& r0, int64_t& r1) {
  if (g.parts == 1) {
    r0 = walker * g.per;
    r1 = r0 + g.per;
  } else {
    const int64_t first = (int64_t)((uint32_t)walker / g.parts) * g.group, at = (int64_t)((uint32_t)walker % g.parts) * g.per;
    r0 = first + at;
    r1 = first + (at + g.per < g.group ? at + g.per : g.group);
  }
  if (r1 > rows) r1 = rows;
}

// a row of dgate
template <bool WHOLE>
__device__ __forceinline__ void join_put_gate(int flags, char* row, int c, int left, const float v[8]) {
  if (flags & JK_GATE_F32) {
    if (flags & JK_GATE_ADD) {
      float o[8];
      raw8_open<float, WHOLE>(raw8_load<float, WHOLE>(row, c, left), 0, o);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += v[e];
      row_store8<float, WHOLE>(row, c, left, o);
    } else {
      row_store8<float, WHOLE>(row, c, left, v);
    }
  } else {
    row_store8<bf16_t, WHOLE>(row, c, left, v);
  }
}

template <typename E>
__global__ __launch_bounds__(kJoinT) void join_wide_bwd_k(ftp_join_args a, JoinK jk, DropMask m, JoinRanges g, JoinParts parts) {
  __shared__ float2 s[2][kJoinT / 64];
  JoinWide<E> w{JoinRow<E>{a, m, mask_key(m), 0, 0.f, 1.f}, a.width, 0, s};
  const int N = a.width;
  int64_t r0, r1;
  join_range(g, blockIdx.x, a.rows, r0, r1);
  if (r0 >= r1) {                        // a part behind the last row
    for (int k = 0; k < JP_ALL; ++k)
      if (float* const p = parts.p[k]) w.columns([&](int c, int left) { const float z[8] = {}; tk_store8<float>(p + (int64_t)blockIdx.x * N + c, left, z); });
    return;
  }
  for (int64_t row = r0; row < r1; ++row) {
    w.r.row = row;
    w.branch_deviation();
    float my = 0.f, ry = 0.f, s1 = 0.f, s2 = 0.f;
    if (a.dn) {
      w.stream_deviation(my, ry);
      w.columns([&](int c, int left) {
        float y[8], bh[8], cc[8], gt[8], d[8], pw[8];
        uint32_t k[8];
        w.r.stream(c, left, y, bh, cc, k, gt);
        w.r.load(a.dn, a.lddn, c, left, d);
        w.r.weight(a.pre_w, c, left, pw, 1.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float dv = e < left ? d[e] * pw[e] : 0.f;
          s1 += dv;
          s2 = fmaf(dv, (y[e] - my) * ry, s2);
        }
      });
      const float2 t = block_sum2<kJoinT>(s1, s2, s, w.turn);
      s1 = a.norm == FTP_NORM_LAYER ? t.x / (float)N : 0.f;
      s2 = t.y / (float)N;
    }
    // gradient of y, and of c; with `add` the column sums too
    const auto at = [&](int c, int left, float dY[8], float dc[8], float bh[8], bool add) __attribute__((always_inline)) {
      float y[8], cc[8], gt[8], dn[8], pw[8], yh[8];
      uint32_t f[8];
      w.r.stream(c, left, y, bh, cc, f, gt);
      w.r.load(a.dy, a.lddy, c, left, dY);
      if (a.dn) {
        w.r.load(a.dn, a.lddn, c, left, dn);
        w.r.weight(a.pre_w, c, left, pw, 1.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          yh[e] = (y[e] - my) * ry;
          dY[e] += ry * (dn[e] * pw[e] - fmaf(yh[e], s2, s1));
        }
      }
      if (a.b) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dc[e] = dropped(a.scale * m.up * gt[e] * dY[e], f[e]);
      }
      if (!add) return;
      const auto sum = [&](int k, auto value) __attribute__((always_inline)) {
        float* const p = parts.p[k];
        if (!p) return;
        float* const q = p + (int64_t)blockIdx.x * N + c;
        float o[8];
        const bool fresh = row == r0 || (k == JP_GATE && row % g.group == 0);
        if (!fresh) tk_load8<float>(q, left, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fresh ? value(e) : o[e] + value(e);
        tk_store8<float>(q, left, o);
        if (k == JP_GATE && g.parts == 1 && (row + 1 == r1 || (row + 1) % g.group == 0)) {
          join_put_gate<false>(jk.flags, jk.dgate + row / g.group * jk.lddg, c, left, o);
        }
      };
      if (a.dn) {
        sum(JP_PRE_W, [&](int e) { return dn[e] * yh[e]; });
        sum(JP_PRE_BIAS, [&](int e) { return dn[e]; });
      }
      if (!a.b) return;
      sum(JP_POST_W, [&](int e) { return dc[e] * bh[e]; });
      sum(JP_POST_BIAS, [&](int e) { return dc[e]; });
      const auto dg = [&](int e) { return a.scale * m.up * dropped(cc[e], f[e]) * dY[e]; };
      sum(JP_GATE, dg);
      if (a.dgate && g.group == 0) {     // a gate row for each row
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = dg(e);
        join_put_gate<false>(jk.flags, jk.dgate + row * jk.lddg, c, left, v);
      }
    };
    const bool again = a.db && a.post;
    float t1 = 0.f, t2 = 0.f;
    w.columns([&](int c, int left) {
      float dY[8], dc[8], bh[8];
      at(c, left, dY, dc, bh, true);
      if (a.dx && !again) tk_store8<E>((E*)a.dx + row * a.lddx + c, left, dY);
      if (a.db && !again) tk_store8<E>((E*)a.db + row * a.lddb + c, left, dc);
      if (again) {
        float pw[8];
        w.r.weight(a.post_w, c, left, pw, 1.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float dv = e < left ? dc[e] * pw[e] : 0.f;
          t1 += dv;
          t2 = fmaf(dv, bh[e], t2);
        }
      }
    });
    if (!again) continue;
    const float2 t = block_sum2<kJoinT>(t1, t2, s, w.turn);
    t1 = a.norm == FTP_NORM_LAYER ? t.x / (float)N : 0.f;
    t2 = t.y / (float)N;
    w.columns([&](int c, int left) {     // dx may lie where dy does: it is written when nothing is read any more
      float dY[8], dc[8], bh[8], pw[8];
      at(c, left, dY, dc, bh, false);
      w.r.weight(a.post_w, c, left, pw, 1.f);
#pragma unroll
      for (int e = 0; e < 8; ++e) dc[e] = w.r.rb * (dc[e] * pw[e] - fmaf(bh[e], t2, t1));
      tk_store8<E>((E*)a.db + row * a.lddb + c, left, dc);
      if (a.dx) tk_store8<E>((E*)a.dx + row * a.lddx + c, left, dY);
    });
  }
}

// Eight columns a thread.  Column sums in registers, or (blocks of 1024 threads, which have 128 registers each) in LDS, two fours a thread for each sum that is wanted.
template <int T, bool LDS>
struct JoinSums {
  float r[LDS ? 1 : JP_ALL][8];
  float4* at;                            // [sums][2][T]
  int want;
  // sums that are not wanted have no place in front of others
  __device__ __forceinline__ float4* place(int k) const { return at + 2 * __popc(want & ((1 << k) - 1)) * T; }
  __device__ __forceinline__ void start(int wanted, float4* lds) {
    if constexpr (LDS) {
      at = lds + threadIdx.x;
      want = wanted;
      for (int n = 2 * __popc(wanted) - 1; n >= 0; --n) at[n * T] = make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
#pragma unroll
      for (int k = 0; k < JP_ALL; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) r[k][e] = 0.f;
    }
  }
  template <typename F>
  __device__ __forceinline__ void add(int k, F value) {                  // value(e, old)
    if constexpr (LDS) {
      float4 *const p = place(k), *const q = p + T;
      float4 u = *p, v = *q;
      u.x = value(0, u.x); u.y = value(1, u.y); u.z = value(2, u.z); u.w = value(3, u.w);
      v.x = value(4, v.x); v.y = value(5, v.y); v.z = value(6, v.z); v.w = value(7, v.w);
      *p = u;
      *q = v;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[k][e] = value(e, r[k][e]);
    }
  }
  // the sum, and zero in its place
  __device__ __forceinline__ void take(int k, float v[8]) {
    if constexpr (LDS) {
      float4* const p = place(k);
      const float4 a = p[0], b = p[T];
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
      p[0] = p[T] = make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) { v[e] = r[k][e]; r[k][e] = 0.f; }
    }
  }
};
// BIAS: sums of the biases as well, and a bias behind the block
template <typename E, int T, bool BIAS, int ROWS, bool LDS, bool AHEAD, bool HOLD>
__global__ __launch_bounds__(64 * join_waves(T), T == 512 && sizeof(E) == 2 ? 4 : 1) void join_row_bwd_k(JoinK k, DropMask m, JoinRanges gr, float* parts, int64_t part_size, int wanted) {
  constexpr bool WHOLE = ROWS > 0, ONCE = ROWS == 2;
  __shared__ float2 s[2][join_waves(T)];
  extern __shared__ float4 held[];
  const int me = join_lane<T>(), c = me * 8, left = k.width - c, back = row_back<E, WHOLE>(c, left);
  const int64_t walker = join_walker<T>();
  const float inv = 1.f / (float)k.width;
  const MaskKey key = mask_key(m);
  int64_t r0, r1;
  join_range(gr, walker, k.rows, r0, r1);
  JoinSums<T, LDS> sum;
  sum.start(wanted, held);
  int turn = 0, flags = k.flags, want = wanted;
  if (r0 < r1) {
    JoinWalk at = join_walk<true>(k, r0);
    JoinIn<E, true> in, next;
    join_ask<E, true, WHOLE, ONCE>(k, flags, at, c, left, back, in);
    const int64_t group = want >> JP_GATE & 1 ? r0 / gr.group : r0;               // dgate's row
    char *pdx = k.dx + r0 * k.lddx, *pdb = k.db + r0 * k.lddb, *pdg = k.dgate + group * k.lddg;
    const int64_t rest = want >> JP_GATE & 1 ? (group + 1) * gr.group - r0 : 1;
    int to_end = gr.parts > 1 || rest > 0x7fffffff ? 0x7fffffff : (int)rest;      // rows until the group's sum is whole
    float pw[8], qw[8], qb[8];
    if (HOLD) {
      join_weight<WHOLE>(k.pre_w, c, left, 1.f, pw);
      join_weight<WHOLE>(k.post_w, c, left, 1.f, qw);
      if (BIAS) join_weight<WHOLE>(k.post_bias, c, left, 0.f, qb);
    }
    uint64_t number = (uint64_t)(m.row0 + r0);
    for (int row = (int)(r1 - r0); row > 0; --row, ++number) {
      flags = join_flags(k.flags);
      want = join_flags(wanted);
      if (AHEAD && row > 1) join_ask<E, true, WHOLE, ONCE>(k, flags, at, c, left, back, next);
      float dY[8], bh[8], cc[8], g[8];                   // g: scale * gate; cc: what it multiplies, dropped
      uint32_t keep[8];
      float rb = 1.f;
      join_open<E, WHOLE>(flags & JK_DY, in.dy, back, dY);
      if (flags & JK_B) {
        raw8_open<E, WHOLE>(in.b, back, bh);
        if (flags & JK_POST) {
          rb = join_deviation<T, WHOLE>(k, flags, inv, left, bh, s, turn);
          if (!HOLD) {
            join_weight<WHOLE>(k.post_w, c, left, 1.f, qw);
            if (BIAS) join_weight<WHOLE>(k.post_bias, c, left, 0.f, qb);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            bh[e] *= rb;
            cc[e] = BIAS ? fmaf(bh[e], qw[e], qb[e]) : bh[e] * qw[e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) cc[e] = bh[e];
        }
        join_open_gate<E, true, WHOLE>(k, flags, in, back, g);
        if (m.least) {
          mask8(m, key, number, me, keep);
#pragma unroll
          for (int e = 0; e < 8; ++e) cc[e] = dropped(cc[e], keep[e]);
        }
      }
      if (flags & JK_DN) {
        float y[8], dn[8];
        join_open<E, WHOLE>(flags & JK_X, in.x, back, y);
        raw8_open<E, WHOLE>(in.dn, back, dn);
        if (flags & JK_B) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = (WHOLE ? left > 0 : e < left) ? fmaf(g[e], cc[e], y[e]) : 0.f;
        }
        const float ry = join_deviation<T, WHOLE>(k, flags, inv, left, y, s, turn);
        float s1 = 0.f, s2 = 0.f;
        if (!HOLD) join_weight<WHOLE>(k.pre_w, c, left, 1.f, pw);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= ry;
        if (want >> JP_PRE_W & 1) sum.add(JP_PRE_W, [&](int e, float o) { return fmaf(dn[e], y[e], o); });
        if (BIAS && (want >> JP_PRE_BIAS & 1)) sum.add(JP_PRE_BIAS, [&](int e, float o) { return o + dn[e]; });
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dn[e] *= pw[e];                                // past the row's end dn is 0
          s1 += dn[e];
          s2 = fmaf(dn[e], y[e], s2);
        }
        const float2 t = block_sum2<T>((flags & JK_LAYER) ? s1 : 0.f, s2, s, turn);
        s1 = t.x * inv;
        s2 = t.y * inv;
#pragma unroll
        for (int e = 0; e < 8; ++e) dY[e] += ry * (dn[e] - fmaf(y[e], s2, s1));
      }
      if (flags & JK_DX) row_store8<E, WHOLE, ONCE>(pdx, c, left, dY);
      pdx += k.lddx;
      if (flags & JK_B) {
        if (flags & JK_DGATE) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = k.scale * cc[e] * dY[e];
          const bool shared = want >> JP_GATE & 1;
          if (shared) sum.add(JP_GATE, [&](int e, float o) { return o + v[e]; });
          if (--to_end == 0) {
            if (shared) sum.take(JP_GATE, v);
            join_put_gate<WHOLE>(flags, pdg, c, left, v);
            pdg += k.lddg;
            to_end = shared ? (int)gr.group : 1;         // no more than a block's rows, or it would not be one's
          } else if (row == 1 && gr.parts == 1) {        // the batch ends inside a group
            sum.take(JP_GATE, v);
            join_put_gate<WHOLE>(flags, pdg, c, left, v);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) dY[e] *= g[e];
        if (m.least) {
#pragma unroll
          for (int e = 0; e < 8; ++e) dY[e] = dropped(dY[e], keep[e]);
        }
        if (flags & JK_POST) {
          float t1 = 0.f, t2 = 0.f;
          if (want >> JP_POST_W & 1) sum.add(JP_POST_W, [&](int e, float o) { return fmaf(dY[e], bh[e], o); });
          if (BIAS && (want >> JP_POST_BIAS & 1)) sum.add(JP_POST_BIAS, [&](int e, float o) { return o + dY[e]; });
          if (flags & JK_DB) {
            if (!HOLD) join_weight<WHOLE>(k.post_w, c, left, 1.f, qw);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              dY[e] = (WHOLE ? left > 0 : e < left) ? dY[e] * qw[e] : 0.f;
              t1 += dY[e];
              t2 = fmaf(dY[e], bh[e], t2);
            }
            const float2 t = block_sum2<T>((flags & JK_LAYER) ? t1 : 0.f, t2, s, turn);
            t1 = t.x * inv;
            t2 = t.y * inv;
#pragma unroll
            for (int e = 0; e < 8; ++e) dY[e] = rb * (dY[e] - fmaf(bh[e], t2, t1));
          }
        }
        if (flags & JK_DB) row_store8<E, WHOLE, ONCE>(pdb, c, left, dY);
      }
      pdb += k.lddb;
      if (AHEAD) in.take(next);
      else if (row > 1) join_ask<E, true, WHOLE, ONCE>(k, flags, at, c, left, back, in);
    }
  }
  if (left <= 0) return;
  float* to = parts + c;
#pragma unroll
  for (int j = 0; j < JP_ALL; ++j) {
    if (!(wanted >> j & 1)) continue;
    if ((BIAS || (j != JP_PRE_BIAS && j != JP_POST_BIAS)) && !(j == JP_GATE && gr.parts == 1)) {
      float v[8];
      sum.take(j, v);
      if (T < 64 && j != JP_GATE) {      // the lanes' groups are added up
#pragma unroll
        for (int n = T; n < 64; n *= 2)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += __shfl_xor(v[e], n);
        if (threadIdx.x < T) tk_store8<float>(to + (int64_t)blockIdx.x * k.width, left, v);
      } else if (T >= 64 || walker < gr.blocks) {
        tk_store8<float>(to + walker * k.width, left, v);
      }
    }
    to += part_size;
  }
}

// Sums of the blocks' rows, in their order: 32 columns a block, 32 threads to a column.  Results 0 .. 3 are the weights' gradients, of all blocks; from
// there on a row of dgate each, of its group's blocks.
__global__ __launch_bounds__(1024) void join_sum_k(JoinParts parts, JoinRanges g, int N, float* w0, float* w1, float* w2, float* w3, int accumulate, void* dgate, int64_t lddg,
                                                   int gate_bf16, int gate_accumulate, int first, int64_t jobs) {
  __shared__ float sum[32][33];
  const int lane = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  for (int64_t job = first + blockIdx.y; job < jobs; job += gridDim.y) {
    const bool gate = job >= JP_GATE;
    const float* const p = gate ? parts.p[JP_GATE] + (job - JP_GATE) * g.parts * N : parts.p[job];
    if (!p) continue;                    // the same for all threads
    const int n = gate ? g.parts : g.sums;
    float v = 0.f;
    if (c < N) {
#pragma unroll 16
      for (int i = ty; i < n; i += 32) v += p[(int64_t)i * N + c];
    }
    __syncthreads();
    sum[ty][lane] = v;
    __syncthreads();
    if (ty || c >= N) continue;
#pragma unroll
    for (int i = 1; i < 32; ++i) v += sum[i][lane];
    if (gate) {
      const int64_t to = (job - JP_GATE) * lddg + c;
      if (gate_bf16) ((bf16_t*)dgate)[to] = f32_to_bf16(v);
      else ((float*)dgate)[to] = gate_accumulate ? ((float*)dgate)[to] + v : v;
    } else {
      float* const o = job == 0 ? w0 : job == 1 ? w1 : job == 2 ? w2 : w3;
      o[c] = accumulate ? o[c] + v : v;
    }
  }
}

// which column sums a call needs
static void join_wanted(const ftp_join_args& a, const JoinRanges& r, bool wanted[JP_ALL]) {
  wanted[JP_PRE_W] = a.dpre_w;
  wanted[JP_PRE_BIAS] = a.dpre_bias;
  wanted[JP_POST_W] = a.dpost_w;
  wanted[JP_POST_BIAS] = a.dpost_bias;
  wanted[JP_GATE] = a.dgate && r.group > 0;
}
static size_t join_part_bytes(const ftp_join_args& a, const JoinRanges& r) { return ((size_t)r.blocks * a.width * 4 + 255) & ~(size_t)255; }
size_t bt_join_bwd_bytes(const ftp_join_args& a) {
  const JoinRanges r = join_ranges(a);
  bool wanted[JP_ALL];
  join_wanted(a, r, wanted);
  size_t n = 0;
  for (bool w : wanted) n += w ? join_part_bytes(a, r) : 0;
  return n;
}
void bt_join_bwd(hipStream_t st, const ftp_join_args& a, const DropMask& m) {
  if (a.rows == 0) {
    if (!a.accumulate)
      for (float* p : {a.dpre_w, a.dpre_bias, a.dpost_w, a.dpost_bias})
        if (p) tk_fill(st, p, 1, (int64_t)a.width * 4, (int64_t)a.width * 4);
    return;
  }
  const double n = (double)a.rows * a.width;
  const double bytes = n * (a.dtype == 1 ? 2 : 4) * ((a.x != nullptr) + (a.b != nullptr) + (a.dy != nullptr) + (a.dn != nullptr) + (a.dx != nullptr) + (a.db != nullptr) +
                       (a.gate && a.gate_rows == 1 ? 1 + (a.dgate != nullptr) : 0));
  KScope ks(st, "tok_join_bwd", bytes, 50 * n, a.rows, a.width);
  const bool once = past_the_caches(bytes);
  const JoinRanges r = join_ranges(a);
  bool wanted[JP_ALL];
  join_wanted(a, r, wanted);
  JoinParts parts{};
  char* at = (char*)a.ws;
  bool weights = false;
  int sums = 0, want = 0;
  for (int k = 0; k < JP_ALL; ++k) {
    if (!wanted[k]) continue;
    ++sums;
    want |= 1 << k;
    parts.p[k] = (float*)at;
    at += join_part_bytes(a, r);
    weights |= k < JP_GATE;
  }
  const JoinK k = join_k(a, m, true);
  // five sums of 8192 columns would be all of the LDS
  const bool held = a.width <= kJoinHeld && (sums < JP_ALL || join_threads(a.width) < 1024);
  if (held) {
    const int t = join_threads(a.width);
    const bool bias = join_biased(a);
    join_by_threads(t, [&](auto tc) {
      constexpr int T = decltype(tc)::value;
      constexpr bool L = T >= 512;
      const auto go = [&](auto f) { hipLaunchKernelGGL(f, dim3(r.sums), dim3(64 * join_waves(T)), L ? (size_t)sums * T * 32 : 0, st, k, m, r, (float*)a.ws, (int64_t)(join_part_bytes(a, r) / 4), want); };
      const auto by = [&](auto* e) {
        typedef std::remove_pointer_t<decltype(e)> E;
        if (a.width % 8) bias ? go(join_row_bwd_k<E, T, true, 0, L, !L, !L>) : go(join_row_bwd_k<E, T, false, 0, L, !L, !L>);
        else if (once) bias ? go(join_row_bwd_k<E, T, true, 2, L, !L, !L>) : go(join_row_bwd_k<E, T, false, 2, L, !L, !L>);
        else bias ? go(join_row_bwd_k<E, T, true, 1, L, !L, !L>) : go(join_row_bwd_k<E, T, false, 1, L, !L, !L>);
      };
      if (a.dtype == FTP_BF16) by((bf16_t*)nullptr);
      else by((float*)nullptr);
    });
  } else if (a.dtype == FTP_BF16) hipLaunchKernelGGL(join_wide_bwd_k<bf16_t>, dim3(r.blocks), dim3(kJoinT), 0, st, a, k, m, r, parts);
  else hipLaunchKernelGGL(join_wide_bwd_k<float>, dim3(r.blocks), dim3(kJoinT), 0, st, a, k, m, r, parts);
  const bool gate = wanted[JP_GATE] && r.parts > 1;
  if (!weights && !gate) return;
  const int first = weights ? 0 : JP_GATE;
  const int64_t jobs = JP_GATE + (gate ? (a.rows + r.group - 1) / r.group : 0);
  hipLaunchKernelGGL(join_sum_k, dim3((a.width + 31) / 32, (unsigned)std::min<int64_t>(jobs - first, 256)), dim3(1024), 0, st, parts, r, a.width, a.dpre_w, a.dpre_bias, a.dpost_w,
                     a.dpost_bias, a.accumulate, a.dgate, a.lddg, a.gate_dtype == FTP_BF16, a.gate_accumulate, first, jobs);
}

}  // namespace ftp
