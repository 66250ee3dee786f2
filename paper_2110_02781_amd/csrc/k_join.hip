// Dropout and the join of a block's output with the stream and its norms, forward and backward.
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
// 0 or the factor of what is kept, for the columns 8 j .. 8 j + 7 of a row
__device__ __forceinline__ void mask8(const DropMask& m, MaskKey k, uint64_t row, uint32_t j, float f[8]) {
  const uint4 w = philox10(make_uint4(j, m.site, (uint32_t)row, (uint32_t)(row >> 32)), k.k0, k.k1);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = (u[i] & 0xffffu) >= m.least ? m.up : 0.f;
    f[2 * i + 1] = (u[i] >> 16) >= m.least ? m.up : 0.f;
  }
}
// what is dropped is 0, whatever it was
__device__ __forceinline__ float dropped(float v, float f) { return f == 0.f ? 0.f : v * f; }

// ---------------------------------------------------------------- dropout
template <typename E>
__global__ __launch_bounds__(256) void dropout_k(DropMask m, int64_t t0, int rows, int cols, const E* x, int64_t ldx, const E* r, int64_t ldr, E* y, int64_t ldy) {
  const uint32_t per = (cols + 7) / 8, all = (uint32_t)rows * per;
  const MaskKey key = mask_key(m);
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) {
    const uint32_t row = i / per, j = i - row * per;
    const int64_t t = t0 + row;
    const int left = cols - (int)(j * 8);
    float v[8], f[8], o[8];
    tk_load8<E>(x + t * ldx + j * 8, left, v);
    if (r) tk_load8<E>(r + t * ldr + j * 8, left, o);
    if (m.least) {
      mask8(m, key, (uint64_t)(m.row0 + t), j, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = dropped(v[e], f[e]);
    }
    if (r) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += o[e];
    }
    tk_store8<E>(y + t * ldy + j * 8, left, v);
  }
}
void bt_dropout(hipStream_t st, int dt, int64_t rows, int cols, const DropMask& m, const void* x, int64_t ldx, const void* r, int64_t ldr, void* y, int64_t ldy) {
  KScope ks(st, "tok_dropout", (double)rows * cols * (dt == 1 ? 2 : 4) * (r ? 3 : 2), 2.0 * rows * cols, rows, cols);
  const int64_t per = (cols + 7) / 8;
  by_rows(rows, per, [&](int64_t t0, int n) {
    const dim3 b(blocks_of(n * per, 1 << 20));
    if (dt == 1) hipLaunchKernelGGL(dropout_k<bf16_t>, b, dim3(256), 0, st, m, t0, n, cols, (const bf16_t*)x, ldx, (const bf16_t*)r, ldr, (bf16_t*)y, ldy);
    else hipLaunchKernelGGL(dropout_k<float>, b, dim3(256), 0, st, m, t0, n, cols, (const float*)x, ldx, (const float*)r, ldr, (float*)y, ldy);
  });
}

// ---------------------------------------------------------------- the join
// Sum of two values over the block's threads, the same in all of them; `s` is used in turn by calls that follow one another (sum2[2][.]).
template <int T>
__device__ __forceinline__ float2 block_sum2(float a, float b, float2 (*s)[T / 64], int& turn) {
  a = wave_sum(a);
  b = wave_sum(b);
  if (T == 64) return make_float2(a, b);
  float2* const p = s[turn ^= 1];
  if ((threadIdx.x & 63) == 0) p[threadIdx.x >> 6] = make_float2(a, b);
  __syncthreads();
  float2 t = p[0];
#pragma unroll
  for (int i = 1; i < T / 64; ++i) { t.x += p[i].x; t.y += p[i].y; }
  return t;
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
  // scale * mask (keep: 0 or its factor)
  __device__ __forceinline__ void mask(int c, float f[8]) const {
    if (m.least) mask8(m, key, (uint64_t)(m.row0 + row), (uint32_t)c / 8, f);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = 1.f;
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
  __device__ __forceinline__ void stream(int c, int left, float y[8], float bh[8], float cc[8], float f[8], float g[8]) const {
    load(a.x, a.ldx, c, left, y);
    if (!a.b) return;
    branch(c, left, bh, cc);
    mask(c, f);
    gate(c, left, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fmaf(a.scale * g[e], dropped(cc[e], f[e]), y[e]);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= left) y[e] = 0.f;
  }
};
__device__ __forceinline__ float inv_dev(float squares, int width, float eps) { return 1.f / sqrtf(squares / (float)width + eps); }

// Rows of any width, each by one block in passes over its columns: what a pass needs is read (and computed) again.
enum { kJoinT = 256 };
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
      mean = block_sum2<kJoinT>(t, 0.f, s, turn).x / (float)N;
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
    rinv = inv_dev(block_sum2<kJoinT>(q, 0.f, s, turn).x, N, r.a.eps);
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
    deviation([&](int c, int left, float v[8]) { float bh[8], cc[8], f[8], g[8]; r.stream(c, left, v, bh, cc, f, g); }, mean, rinv);
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
      float y[8], bh[8], cc[8], f[8], g[8];
      w.r.stream(c, left, y, bh, cc, f, g);
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
void bt_join(hipStream_t st, const ftp_join_args& a, const DropMask& m) {
  const double n = (double)a.rows * a.width;
  KScope ks(st, "tok_join", n * (a.dtype == 1 ? 2 : 4) * ((a.x != nullptr) + (a.b != nullptr) + (a.y != nullptr) + (a.n != nullptr) + (a.gate && a.gate_rows == 1)), 15 * n,
            a.rows, a.width);
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
};
static JoinRanges join_ranges(const ftp_join_args& a) {
  const int64_t want = std::max<int64_t>(1, (a.rows + 511) / 512);
  JoinRanges r{want, 0, 1, 0};
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
  return r;
}
enum { JP_PRE_W, JP_PRE_BIAS, JP_POST_W, JP_POST_BIAS, JP_GATE, JP_ALL };
struct JoinParts { float* p[JP_ALL]; };           // [blocks][width] each, or null

__device__ __forceinline__ void join_range(const JoinRanges& g, int64_t rows, int64_t& r0, int64_t& r1) {
  if (g.parts == 1) {
    r0 = blockIdx.x * g.per;
    r1 = r0 + g.per;
  } else {
    const int64_t first = (int64_t)(blockIdx.x / g.parts) * g.group, at = (int64_t)(blockIdx.x % g.parts) * g.per;
    r0 = first + at;
    r1 = first + (at + g.per < g.group ? at + g.per : g.group);
  }
  if (r1 > rows) r1 = rows;
}

template <typename E>
__global__ __launch_bounds__(kJoinT) void join_wide_bwd_k(ftp_join_args a, DropMask m, JoinRanges g, JoinParts parts) {
  __shared__ float2 s[2][kJoinT / 64];
  JoinWide<E> w{JoinRow<E>{a, m, mask_key(m), 0, 0.f, 1.f}, a.width, 0, s};
  const int N = a.width;
  int64_t r0, r1;
  join_range(g, a.rows, r0, r1);
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
        float y[8], bh[8], cc[8], f[8], gt[8], d[8], pw[8];
        w.r.stream(c, left, y, bh, cc, f, gt);
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
      float y[8], cc[8], f[8], gt[8], dn[8], pw[8], yh[8];
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
        for (int e = 0; e < 8; ++e) dc[e] = dropped(a.scale * gt[e] * dY[e], f[e]);
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
          const int64_t to = row / g.group * a.lddg + c;
          if (a.gate_dtype == FTP_F32) {
            float v[8];
            if (a.gate_accumulate) tk_load8<float>((float*)a.dgate + to, left, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = a.gate_accumulate ? v[e] + o[e] : o[e];
            tk_store8<float>((float*)a.dgate + to, left, v);
          } else {
            tk_store8<bf16_t>((bf16_t*)a.dgate + to, left, o);
          }
        }
      };
      if (a.dn) {
        sum(JP_PRE_W, [&](int e) { return dn[e] * yh[e]; });
        sum(JP_PRE_BIAS, [&](int e) { return dn[e]; });
      }
      if (!a.b) return;
      sum(JP_POST_W, [&](int e) { return dc[e] * bh[e]; });
      sum(JP_POST_BIAS, [&](int e) { return dc[e]; });
      const auto dg = [&](int e) { return a.scale * dropped(cc[e], f[e]) * dY[e]; };
      sum(JP_GATE, dg);
      if (a.dgate && g.group == 0) {     // a gate row for each row
        const int64_t to = row * a.lddg + c;
        float v[8];
        if (a.gate_dtype == FTP_F32) {
          if (a.gate_accumulate) tk_load8<float>((float*)a.dgate + to, left, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = a.gate_accumulate ? v[e] + dg(e) : dg(e);
          tk_store8<float>((float*)a.dgate + to, left, v);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = dg(e);
          tk_store8<bf16_t>((bf16_t*)a.dgate + to, left, v);
        }
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

// Sums of the blocks' rows, in their order: 64 columns a block, sixteen threads to a column.  Results 0 .. 3 are the weights' gradients, of all blocks; from
// there on a row of dgate each, of its group's blocks.
__global__ __launch_bounds__(1024) void join_sum_k(JoinParts parts, JoinRanges g, int N, float* w0, float* w1, float* w2, float* w3, int accumulate, void* dgate, int64_t lddg,
                                                   int gate_bf16, int gate_accumulate, int first, int64_t jobs) {
  __shared__ float sum[16][64];
  const int lane = threadIdx.x & 63, ty = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  for (int64_t job = first + blockIdx.y; job < jobs; job += gridDim.y) {
    const bool gate = job >= JP_GATE;
    const float* const p = gate ? parts.p[JP_GATE] + (job - JP_GATE) * g.parts * N : parts.p[job];
    if (!p) continue;                    // the same for all threads
    const int n = gate ? g.parts : g.blocks;
    float v = 0.f;
    if (c < N) {
#pragma unroll 8
      for (int i = ty; i < n; i += 16) v += p[(int64_t)i * N + c];
    }
    __syncthreads();
    sum[ty][lane] = v;
    __syncthreads();
    if (ty || c >= N) continue;
#pragma unroll
    for (int i = 1; i < 16; ++i) v += sum[i][lane];
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
  KScope ks(st, "tok_join_bwd", n * (a.dtype == 1 ? 2 : 4) * ((a.x != nullptr) + (a.b != nullptr) + (a.dy != nullptr) + (a.dn != nullptr) + (a.dx != nullptr) + (a.db != nullptr) +
            (a.gate && a.gate_rows == 1 ? 1 + (a.dgate != nullptr) : 0)), 50 * n, a.rows, a.width);
  const JoinRanges r = join_ranges(a);
  bool wanted[JP_ALL];
  join_wanted(a, r, wanted);
  JoinParts parts{};
  char* at = (char*)a.ws;
  bool weights = false;
  for (int k = 0; k < JP_ALL; ++k) {
    if (!wanted[k]) continue;
    parts.p[k] = (float*)at;
    at += join_part_bytes(a, r);
    weights |= k < JP_GATE;
  }
  if (a.dtype == FTP_BF16) hipLaunchKernelGGL(join_wide_bwd_k<bf16_t>, dim3(r.blocks), dim3(kJoinT), 0, st, a, m, r, parts);
  else hipLaunchKernelGGL(join_wide_bwd_k<float>, dim3(r.blocks), dim3(kJoinT), 0, st, a, m, r, parts);
  const bool gate = wanted[JP_GATE] && r.parts > 1;
  if (!weights && !gate) return;
  const int first = weights ? 0 : JP_GATE;
  const int64_t jobs = JP_GATE + (gate ? (a.rows + r.group - 1) / r.group : 0);
  hipLaunchKernelGGL(join_sum_k, dim3((a.width + 63) / 64, (unsigned)std::min<int64_t>(jobs - first, 256)), dim3(1024), 0, st, parts, r, a.width, a.dpre_w, a.dpre_bias, a.dpost_w,
                     a.dpost_bias, a.accumulate, a.dgate, a.lddg, a.gate_dtype == FTP_BF16, a.gate_accumulate, first, jobs);
}

}  // namespace ftp
