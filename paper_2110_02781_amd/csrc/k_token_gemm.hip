// Matrix products of the token operators: the small tiles, the joining of split reductions, the choice among tiles, few rows against all of the weights.
// How operands reach the matrix cores is told in token_tile.h; the large tile is in k_token_big.hip.
#include <algorithm>

#include "token_tile.h"

namespace ftp {

// ---- a wavefront's results: acc[a][b][e] is row m + 16 a, column n + 16 b + e; with TG_GLU the second half of the b are the up
// projection's, columns from n again.  Two b of 16 columns are a group of the 8-bit form ----
template <typename E, int EPI, int S, int T, bool PART>
__device__ __forceinline__ void tg_results(const TgJob& p, f4v_t (&acc)[S][T], int split, int row, int jb, int G) {
  constexpr bool GLU = EPI == TG_GLU;
  constexpr int H = T / 2;
  const int M = p.M, N = p.N;
  if constexpr (PART) {
    const int64_t np = (N + 3) & ~3, plane = (int64_t)M * np;
    float* const part = p.part + (int64_t)split * (GLU ? 2 : 1) * plane;
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) {
        const int m = row + a * 16, n = jb + (GLU ? b % H : b) * 16;
        if (m < M && n < np)
          *reinterpret_cast<float4*>(part + (GLU && b >= H ? plane : 0) + m * np + n) = make_float4(acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]);
      }
  } else if constexpr (GLU) {
    static_assert(H % 2 == 0, "a wavefront has whole groups of 32 gate columns");
#pragma unroll
    for (int a = 0; a < S; ++a) {
      const int64_t m = row + a * 16;
      if (p.save == 2) {         // before the rows past M leave: the maximum goes across lanes (of one row)
#pragma unroll
        for (int b0 = 0; b0 < H; b0 += 2) {
          float tg = 0.f, tu = 0.f;
#pragma unroll
          for (int b = b0; b < b0 + 2; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              tg = fmaxf(tg, act8_mag(acc[a][b][e]));
              tu = fmaxf(tu, act8_mag(acc[a][b + H][e]));
            }
          tg = fmaxf(tg, __shfl_xor(tg, 16)); tu = fmaxf(tu, __shfl_xor(tu, 16));
          tg = fmaxf(tg, __shfl_xor(tg, 32)); tu = fmaxf(tu, __shfl_xor(tu, 32));
          if (m < M) {
#pragma unroll
            for (int b = b0; b < b0 + 2; ++b) {
              const float g[4] = {acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]};
              const float u[4] = {acc[a][b + H][0], acc[a][b + H][1], acc[a][b + H][2], acc[a][b + H][3]};
              const bool vec = p.flags & TG_VEC_Z;
              tg_keep8(p.z, p.ldz, p.zs, p.lds, m, jb + b * 16, N, vec, b == b0 && G == 0, tg, g);
              tg_keep8(p.up, p.ldu, p.us, p.lds, m, jb + b * 16, N, vec, b == b0 && G == 0, tu, u);
            }
          }
        }
      }
#pragma unroll
      for (int b = 0; b < H; ++b) {
        const int n = jb + b * 16;
        const float g[4] = {acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]};
        const float u[4] = {acc[a][b + H][0], acc[a][b + H][1], acc[a][b + H][2], acc[a][b + H][3]};
        if (m < M && n < p.ldo) tg_glu4<E>(p, m, n, g, u);
      }
    }
  } else if constexpr (EPI == TG_LINEAR) {
    // what comes from memory is under way for all of the results before any is waited for, and which activation it is asked once
    typename Tg4<E>::raw res[S][T];
    float v[S * T * 4];
    if (p.res) {
#pragma unroll
      for (int a = 0; a < S; ++a)
#pragma unroll
        for (int b = 0; b < T; ++b)
          res[a][b] = get_raw4<E>(p.res, p.ldr, row + a * 16 < M ? row + a * 16 : M - 1, jb + b * 16, N, p.flags & TG_VEC_RES);
    }
#pragma unroll
    for (int b = 0; b < T; ++b) {
      float t[4] = {0.f, 0.f, 0.f, 0.f};
      if (p.bias) get4<float>(p.bias, 0, 0, jb + b * 16, N, p.flags & TG_VEC_BIAS, t);
#pragma unroll
      for (int a = 0; a < S; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[(a * T + b) * 4 + e] = acc[a][b][e] + t[e];
    }
    if (p.z) {
#pragma unroll
      for (int a = 0; a < S; ++a)
#pragma unroll
        for (int b = 0; b < T; ++b)
          if (row + a * 16 < M && jb + b * 16 < N) put4<E>(p.z, p.ldz, row + a * 16, jb + b * 16, N, p.flags & TG_VEC_Z, v + (a * T + b) * 4);
    }
    tactn<S * T * 4>(v, p.act);
    if (p.res) {
#pragma unroll
      for (int i = 0; i < S * T; ++i) {
        float r[4];
        open4<E>(res[i / T][i % T], r);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i * 4 + e] += r[e];
      }
    }
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b)
        if (row + a * 16 < M && jb + b * 16 < N) put4<E>(p.out, p.ldo, row + a * 16, jb + b * 16, N, p.flags & TG_VEC_OUT, v + (a * T + b) * 4);
  } else {
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) {
        const int64_t m = row + a * 16;
        const int n = jb + b * 16;
        float v[4] = {acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]};
        if (m < M && n < (EPI == TG_GLUBWD ? (int)p.ldo : N)) {
          tg_finish4<E, EPI>(p, m, n, v);
        }
      }
  }
}

// The small tiles.  KG 2: twice the wavefronts, of which one half takes the first 64 bytes of a step's reduction and the other half the second, and
// which add up at the end: two to a SIMD where one alone waits for every LDS read, every meeting and its own last products (1024 x 1024 x 4096
// bfloat16 in tiles of 64 19.5 us, 23 with one half).  fp32 is bound by its matrix instruction, 150 TFLOP/s at best, beside which no vector instruction
// runs: 517 x 1024 x 5632 in 74 us, 1000 x 777 x 1001 (208 tiles for 256 CUs) in 28.
template <typename E, int LAY, int EPI, int BM, int BN, int WM, int WN, int KG, bool PART>
__global__ __launch_bounds__(64 * WM * WN * KG) void tg_gemm_k(const TgGroup grp) {
  typedef TgBlock<E, LAY, EPI, BM, BN, WM * WN * KG> B;
  constexpr int S = BM / (16 * WM), T = BN / (16 * WN);
  constexpr bool F32 = Tg<E>::F32, GLU = EPI == TG_GLU;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  int lb;
  const TgJob& p = B::job(grp, lb);
  B blk;
  if (!blk.init(p, lb, smem)) return;
  const int kg = blk.wave / (WM * WN), w = blk.wave % (WM * WN);
  const int l16 = blk.lane & 15, G = blk.lane >> 4, wm = w / WN, wn = w % WN;
  const int s0 = blk.s0, s1 = blk.s1, m0 = blk.m0, j0 = blk.j0, split = blk.split;
  const int arow = wm * 16 * S, bsub = wn * T;
  auto brow = [&](int b) __attribute__((always_inline)) {        // first column (row of the LDS tile) of fragment b
    return GLU ? (b < T / 2 ? (bsub / 2 + b) * 16 : BN / 2 + (bsub / 2 + b - T / 2) * 16) : (bsub + b) * 16;
  };

  f4v_t acc[S][T];
#pragma unroll
  for (int a = 0; a < S; ++a)
#pragma unroll
    for (int b = 0; b < T; ++b) acc[a][b] = f4v_t{0.f, 0.f, 0.f, 0.f};
  // fp32: the sums of four steps are a chain of their own, added up outside it: a reduction of 16384 would otherwise be one chain of as many
  // additions.  (Vector instructions and these matrix instructions do not overlap: adding up in every step was a tenth of the time.)
  f4v_t tot[F32 ? S : 1][F32 ? T : 1];
  if constexpr (F32)
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) tot[a][b] = f4v_t{0.f, 0.f, 0.f, 0.f};

  // NB - 1 steps are on their way while one is multiplied; past the last one the requests go on, for nothing (zeros), so that what is waited for
  // is always "all but the youngest"
  constexpr int NB = tg_buffers(BM), L = B::NL;
#pragma unroll
  for (int i = 0; i < NB - 1; ++i) blk.fetch(p, i * B::BUF, i * B::BUF + B::ABYTES);
  uint32_t at = 0, to = (NB - 1) * B::BUF;
  // a wavefront whose rows or columns all lie past the last only loads: 517 rows are eight tiles of 64 and five rows
  const bool idle = m0 + arow >= p.M || j0 + (GLU ? bsub / 2 : bsub) * 16 >= (GLU ? (int)p.ldo : p.N);
  for (int s = s0; s < s1; ++s) {
    tg_meet<(NB - 2) * L>();     // this step's operands are there, and the buffer of the step before is free
    blk.fetch(p, to, to + B::ABYTES);
    const char* ta = smem + at;
    const char* tb = ta + B::ABYTES;
    to = at;
    at = at + B::BUF == NB * B::BUF ? 0 : at + B::BUF;
    if (idle) continue;
    if (F32 && ((s - s0) & 3) == 0) {
#pragma unroll
      for (int a = 0; a < S; ++a)
#pragma unroll
        for (int b = 0; b < T; ++b) {
          tot[F32 ? a : 0][F32 ? b : 0] += acc[a][b];
          acc[a][b] = f4v_t{0.f, 0.f, 0.f, 0.f};
        }
    }
#pragma unroll
    for (int k2 = 0; k2 < 2 / KG; ++k2) {
      const int kk = KG == 2 ? kg : k2;
      uint4 af[S], bf[T];
#pragma unroll
      for (int b = 0; b < T; ++b) bf[b] = tg_frag<E, B::BX, BN>(tb, brow(b), kk, l16, G);
#pragma unroll
      for (int a = 0; a < S; ++a) af[a] = tg_frag<E, B::AX, BM>(ta, arow + a * 16, kk, l16, G);
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int a = 0; a < S; ++a)
#pragma unroll
            for (int b = 0; b < T; ++b)
              acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float((&bf[b].x)[e]), __uint_as_float((&af[a].x)[e]),
                                                               acc[a][b], 0, 0, 0);
      } else {
#pragma unroll
        for (int a = 0; a < S; ++a)
#pragma unroll
          for (int b = 0; b < T; ++b)
            acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, bf[b]), __builtin_bit_cast(bf16x8_t, af[a]), acc[a][b], 0, 0, 0);
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");               // LDS is somebody else's once this block ends
  if constexpr (F32) {
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) acc[a][b] += tot[a][b];
  }

  if constexpr (KG == 2) {
    static_assert(S * T * WM * WN * 1024 <= tg_buffers(BM) * B::BUF, "the sums of one half fit where the operands were");
    __syncthreads();
    f4v_t* const other = reinterpret_cast<f4v_t*>(smem) + w * (S * T * 64) + blk.lane;
    if (kg == 1) {
#pragma unroll
      for (int a = 0; a < S; ++a)
#pragma unroll
        for (int b = 0; b < T; ++b) other[(a * T + b) * 64] = acc[a][b];
    }
    __syncthreads();
    if (kg == 1) return;
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) acc[a][b] += other[(a * T + b) * 64];
  }
  tg_results<E, EPI, S, T, PART>(p, acc, split, m0 + arow + l16, j0 + (GLU ? bsub / 2 : bsub) * 16 + 4 * G, G);
}

// adds the partial sums of a split reduction, split after split, and finishes the results: a thread has four columns of a row,
// the eight threads of 32 columns lie next to one another.  Memory: 1900 x 2040 from three planes of fp32, 50 MB, 13.5 us
template <typename E, int EPI>
__global__ __launch_bounds__(256) void tg_join_k(const TgGroup grp) {
  const TgJob& p = grp.j[EPI == TG_GRAD ? blockIdx.y : 0];
  constexpr bool GLU = EPI == TG_GLU;
  const int np = (p.N + 3) & ~3, n32 = (p.N + 31) / 32 * 8;      // fours of columns to a row, whole groups
  const int64_t plane = (int64_t)p.M * np, all = (int64_t)p.M * n32;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (all + 63) / 64 * 64; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / n32;
    const int n = (int)(i - m * n32) * 4;
    const bool in = m < p.M && n < np;
    float v[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
    if (in) {
      const float* q = p.part + m * np + n;
      for (int s = 0; s < p.splits; ++s, q += (GLU ? 2 : 1) * plane) {
        const float4 t = ld4(q);
        v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
        if (GLU) {
          const float4 w = ld4(q + plane);
          u[0] += w.x; u[1] += w.y; u[2] += w.z; u[3] += w.w;
        }
      }
    }
    if constexpr (GLU) {
      if (p.save == 2) {
        float tg = 0.f, tu = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) { tg = fmaxf(tg, act8_mag(v[e])); tu = fmaxf(tu, act8_mag(u[e])); }
        tg = tg_max8(tg);
        tu = tg_max8(tu);
        if (in) {
          tg_keep8(p.z, p.ldz, p.zs, p.lds, m, n, p.N, p.flags & TG_VEC_Z, (n & 31) == 0, tg, v);
          tg_keep8(p.up, p.ldu, p.us, p.lds, m, n, p.N, p.flags & TG_VEC_Z, (n & 31) == 0, tu, u);
        }
      }
      if (m < p.M && n < p.ldo) tg_glu4<E>(p, m, n, v, u);
    } else if constexpr (EPI == TG_GLUBWD) {
      if (m < p.M && n < p.ldo) tg_finish4<E, EPI>(p, m, n, v);
    } else {
      if (in) tg_finish4<E, EPI>(p, m, n, v);
    }
  }
}

// ------------------------------------------------------------------ host
size_t tg_part_bytes(int epi, int M, int N, int splits) {
  return splits > 1 ? (size_t)splits * (epi == TG_GLU ? 2 : 1) * M * ((N + 3) & ~3) * 4 : 0;
}

// Which tile, and over how many blocks a reduction is split: what a simple model of the time says is least.  A CU works on ceil(blocks / 256) blocks; a block's
// step takes `one` us while it has the CU to itself, and `all` us for each block there once they share what bounds them (the matrix cores; for the large
// tile, alone on its CU, one after the other); `base` + `each` per block are launch, first loads and results; a split adds the partial sums' way
// through memory at 4 TB/s and the joining launch.  The constants were fitted to the measured times of all tiles and splits at 39 products (rows 32 .. 4096, columns
// 512 .. 8192, reductions 512 .. 8192, the three operand orders): what it chooses is 0.3 % (bfloat16) and 0.5 % (fp32) slower than the best on average.
// Either side, bfloat16: 1024 x 1024 x 1024 7.6 us in tiles of 64, 14.7 in 128; 4096 x 4096 x 1024 60 / 42 and 42 in 256; 1900 x 2040 x 5464 57 in 256 split by
// three, 74 in 128.  fp32: 1024 x 1024 x 1024 26 / 74, 4096 x 4096 x 1024 311 / 284.
TgPlan tg_plan(int dt, int epi, int M, int N, int K, size_t max_bytes) {
  struct Cost { int tile; double one, all, base, each; };
  static const Cost costs[2][3] = {{{128, 2.2, 2.0, 6.0, 2.0}, {64, 0.66, 0.55, 5.0, 1.0}, {0, 0, 0, 0, 0}},
                                   {{256, 1.3, 1.3, 0.0, 10.0}, {128, 0.6, 0.52, 5.0, 3.0}, {64, 0.25, 0.17, 4.0, 1.0}}};
  const int ks = dt == 1 ? 64 : 32, steps = std::max(1, (K + ks - 1) / ks);
  TgPlan best{128, 1};
  double best_us = 1e30;
  for (const Cost& c : costs[dt == 1]) {
    if (!c.tile) break;
    const int bn = epi == TG_GLU ? c.tile / 2 : c.tile;
    const double tiles = (double)((M + c.tile - 1) / c.tile) * ((N + bn - 1) / bn);
    // A launch of 2^32 threads or more is cut off without an error: 2^29 rows and more, of a few columns, are too many tiles of 64.  (With 8: the padding of a
    // group's jobs.  Tiles of 128 take 2^31 rows, and more columns than the memory holds.)
    if ((tiles + 8) * (c.tile == 64 ? 512 : 256) >= 4294967296.0) continue;
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      const size_t part = tg_part_bytes(epi, M, N, s);
      if (s > 1 && (steps < 4 * s || part > max_bytes)) break;
      const double n = std::ceil(tiles * s / 256), per = (steps + s - 1) / s;
      const double us = per * std::max(c.one, c.all * n) + c.base + c.each * n + (s > 1 ? 3.0 + part / 4e6 : 0.0);
      if (us < best_us) { best_us = us; best = TgPlan{c.tile, s}; }
    }
  }
  return best;
}

template <typename E, int LAY, int EPI, int BM, int BN, int WM, int WN, int KG = 1>
static void launch_tile(hipStream_t st, TgGroup& g, bool part) {
  constexpr int KS = Tg<E>::KS, LDS = tg_buffers(BM) * (BM + BN) * 128;
  int blocks = 0;
  for (int i = 0; i < g.n; ++i) {
    TgJob& j = g.j[i];
    const int bn = EPI == TG_GLU ? BN / 2 : BN;
    j.tiles_m = (j.M + BM - 1) / BM;
    j.tiles_n = (j.N + bn - 1) / bn;
    const int total = ((j.K + KS - 1) / KS) * j.nseg;
    j.steps = (total + j.splits - 1) / j.splits;
    j.splits = (total + j.steps - 1) / j.steps;                  // none without steps: its requests would be of a reduction that is not there
    g.blk0[i] = blocks;
    blocks += g.n > 1 ? (j.tiles_m * j.tiles_n * j.splits + 7) / 8 * 8 : j.tiles_m * j.tiles_n * j.splits;
  }
  g.blk0[g.n] = blocks;
  if constexpr (BM == 256) {
    tg_big_launch(st, LAY, EPI, g, blocks, part);
  } else {
    if (part) tg_launch_lds<tg_gemm_k<E, LAY, EPI, BM, BN, WM, WN, KG, true>>(st, g, blocks, 64 * WM * WN * KG, LDS);
    else tg_launch_lds<tg_gemm_k<E, LAY, EPI, BM, BN, WM, WN, KG, false>>(st, g, blocks, 64 * WM * WN * KG, LDS);
  }
}

template <typename E, int LAY, int EPI>
static void launch(hipStream_t st, TgGroup& g, TgPlan plan) {
  const bool part = plan.splits > 1;
  if (sizeof(E) == 2 && plan.tile == 256) {
    if constexpr (sizeof(E) == 2) launch_tile<E, LAY, EPI, 256, 256, 2, 2>(st, g, part);
  } else if (plan.tile == 64) {
    // (a wavefront has 32 gate columns, a group of the 8-bit form)
    if constexpr (EPI == TG_GLU) launch_tile<E, LAY, EPI, 64, 64, 4, 1, 2>(st, g, part);
    else launch_tile<E, LAY, EPI, 64, 64, 2, 2, 2>(st, g, part);
  } else {
    launch_tile<E, LAY, EPI, 128, 128, 2, 2>(st, g, part);
  }
  if (part) {
    int64_t most = 0;
    for (int i = 0; i < g.n; ++i) most = std::max<int64_t>(most, (int64_t)g.j[i].M * ((g.j[i].N + 31) / 32 * 8));
    const int64_t blocks = std::min<int64_t>((most + 255) / 256, 4096);
    hipLaunchKernelGGL((tg_join_k<E, EPI>), dim3((unsigned)blocks, g.n), dim3(256), 0, st, g);
  }
}

void tg_launch(int dt, hipStream_t st, int lay, int epi, TgJob* jobs, int n, TgPlan plan) {
  TgGroup g;
  g.n = n;
  double bytes = 0, flops = 0;
  const double es = dt == 1 ? 2 : 4;
  for (int i = 0; i < n; ++i) {
    g.j[i] = jobs[i];
    TgJob& j = g.j[i];
    j.splits = plan.splits;
    const double two = epi == TG_GLU ? 2 : 1;
    flops += 2.0 * two * j.M * j.N * j.K * j.nseg;
    bytes += es * (((double)j.M * j.K + two * j.N * j.K) * j.nseg + (double)j.M * j.N);
  }
  static const char* const names[4] = {"tok_linear", "tok_glu", "tok_glu_bwd", "tok_wgrad"};
  KScope ks(st, names[epi], bytes, flops, g.j[0].M, g.j[0].K, g.j[0].N);
  static const char* const tiles[3][2] = {{"64", "64 split"}, {"128", "128 split"}, {"256", "256 split"}};
  ks.route(tiles[plan.tile / 128][plan.splits > 1]);
  if (dt == 1) {
    if (epi == TG_LINEAR && lay == TG_NT) launch<bf16_t, TG_NT, TG_LINEAR>(st, g, plan);
    else if (epi == TG_LINEAR) launch<bf16_t, TG_NN, TG_LINEAR>(st, g, plan);
    else if (epi == TG_GLU) launch<bf16_t, TG_NT, TG_GLU>(st, g, plan);
    else if (epi == TG_GLUBWD) launch<bf16_t, TG_NN, TG_GLUBWD>(st, g, plan);
    else launch<bf16_t, TG_TN, TG_GRAD>(st, g, plan);
  } else {
    if (epi == TG_LINEAR && lay == TG_NT) launch<float, TG_NT, TG_LINEAR>(st, g, plan);
    else if (epi == TG_LINEAR) launch<float, TG_NN, TG_LINEAR>(st, g, plan);
    else if (epi == TG_GLU) launch<float, TG_NT, TG_GLU>(st, g, plan);
    else if (epi == TG_GLUBWD) launch<float, TG_NN, TG_GLUBWD>(st, g, plan);
    else launch<float, TG_TN, TG_GRAD>(st, g, plan);
  }
}

// ------------------------------------------------------------------ few rows
// Up to 16 rows against all of the weights: the weights' bytes are the time.  A block owns 16 columns (with TG_GLU 16 of both
// matrices) and its wavefronts share the reduction; a turn is four vectors a lane, all in flight, each load 64 consecutive bytes of 16 weight rows,
// as operands of the matrix instruction (16 weight rows by 16 rows of x), which takes reduction elements in any order as
// long as both operands agree.  (64 consecutive bytes a lane, so 16 of every 64 a load: 4096 x 14336 block, 4 rows 96.6 us, so 73.5, 4.8 TB/s.)  The
// wavefronts' sums meet in LDS in a fixed order; four with TG_GLU, eight without: 73.5 us, twice as many 76.7, four times 79.1.
template <typename E, int EPI, int NW>
__global__ __launch_bounds__(64 * NW) void tg_skinny_k(const TgJob p) {
  constexpr int V = Tg<E>::V, U = 4;                              // vectors a lane reads per turn
  constexpr bool F32 = Tg<E>::F32, GLU = EPI == TG_GLU;
  __shared__ float4 meet[GLU ? 2 : 1][NW][64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l16 = lane & 15, G = lane >> 4;
  const int j0 = xcd_logical_block() * 16, M = p.M, N = p.N, K = p.K;
  const int jn = j0 + l16 < N ? j0 + l16 : N - 1;               // rows past the last are read again and not stored
  const char* const w0 = (const char*)p.b[0] + (int64_t)jn * p.ldb[0] * (int64_t)sizeof(E);
  const char* const w1 = GLU ? (const char*)p.b[1] + (int64_t)jn * p.ldb[1] * (int64_t)sizeof(E) : w0;
  const char* const x = (const char*)p.a[0] + (int64_t)(l16 < M ? l16 : 0) * p.lda * (int64_t)sizeof(E);
  const bool xin = l16 < M;
  f4v_t acc[2] = {f4v_t{0.f, 0.f, 0.f, 0.f}, f4v_t{0.f, 0.f, 0.f, 0.f}};
  auto mul = [&](f4v_t c, uint4 w, uint4 xv) __attribute__((always_inline)) {
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float((&w.x)[e]), __uint_as_float((&xv.x)[e]), c, 0, 0, 0);
      return c;
    } else {
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, xv), c, 0, 0, 0);
    }
  };
  // a vector at any element; what follows a row that ends inside one is not the row's
  auto whole = [&](const char* row, int k) __attribute__((always_inline)) {
    const u4v_t t = tk_ld16<E>(reinterpret_cast<const E*>(row) + k);
    return make_uint4(t[0], t[1], t[2], t[3]);
  };
  auto ragged = [&](const char* row, int k) __attribute__((always_inline)) {
    uint32_t t[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (k + e < K) {
        const E* q = reinterpret_cast<const E*>(row) + k + e;
        if constexpr (F32) t[e & 3] = *reinterpret_cast<const uint32_t*>(q);
        else t[(e / 2) & 3] |= (uint32_t)*reinterpret_cast<const uint16_t*>(q) << (16 * (e & 1));
      }
    return make_uint4(t[0], t[1], t[2], t[3]);
  };
  const int turn = 4 * U * V;                                   // reduction elements a wavefront takes per turn
  int k0 = wave * turn;
  for (; k0 + turn <= K; k0 += NW * turn) {
    uint4 a[U], b[U], c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + (u * 4 + G) * V;
      a[u] = whole(w0, k);
      if (GLU) b[u] = whole(w1, k);
      c[u] = make_uint4(0, 0, 0, 0);
      if (xin) c[u] = whole(x, k);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      acc[0] = mul(acc[0], a[u], c[u]);
      if (GLU) acc[1] = mul(acc[1], b[u], c[u]);
    }
  }
  if (k0 < K) {                                                 // the last turn: its whole vectors together, then the one that the row ends in
    uint4 a[U], b[U], c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + (u * 4 + G) * V;
      const bool in = k + V <= K;
      a[u] = b[u] = c[u] = make_uint4(0, 0, 0, 0);
      if (in) a[u] = whole(w0, k);
      if (GLU && in) b[u] = whole(w1, k);
      if (in && xin) c[u] = whole(x, k);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      acc[0] = mul(acc[0], a[u], c[u]);
      if (GLU) acc[1] = mul(acc[1], b[u], c[u]);
    }
    const int k = K / V * V;
    if (k < K && k >= k0) {
      const bool mine = G == 0;
      const uint4 nothing = make_uint4(0, 0, 0, 0), w = mine ? ragged(w0, k) : nothing, t = mine && xin ? ragged(x, k) : nothing;
      acc[0] = mul(acc[0], w, t);
      if (GLU) acc[1] = mul(acc[1], mine ? ragged(w1, k) : nothing, t);
    }
  }
  meet[0][wave][lane] = make_float4(acc[0][0], acc[0][1], acc[0][2], acc[0][3]);
  if (GLU) meet[GLU ? 1 : 0][wave][lane] = make_float4(acc[1][0], acc[1][1], acc[1][2], acc[1][3]);
  __syncthreads();
  if (wave) return;
  float v[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float4 t = meet[0][w][lane];
    v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
    if (GLU) {
      const float4 s = meet[GLU ? 1 : 0][w][lane];
      u[0] += s.x; u[1] += s.y; u[2] += s.z; u[3] += s.w;
    }
  }
  const int n = j0 + 4 * G;
  if (l16 >= M) return;
  if constexpr (GLU) { if (n < p.ldo) tg_glu4<E>(p, l16, n, v, u); }
  else { if (n < N) tg_finish4<E, EPI>(p, l16, n, v); }
}

void tg_skinny(int dt, hipStream_t st, int epi, const TgJob& j) {
  const double es = dt == 1 ? 2 : 4, two = epi == TG_GLU ? 2 : 1;
  KScope ks(st, epi == TG_GLU ? "tok_glu_few" : "tok_linear_few", es * (two * j.N * j.K + (double)j.M * (j.K + j.N)), 2.0 * two * j.M * j.N * j.K,
            j.M, j.K, j.N);
  const int blocks = (j.N + 15) / 16;
  auto go = [&](auto k, int nw) { hipLaunchKernelGGL(k, dim3(blocks), dim3(64 * nw), 0, st, j); };
  if (dt == 1) {
    if (epi == TG_GLU) go(tg_skinny_k<bf16_t, TG_GLU, 4>, 4);
    else go(tg_skinny_k<bf16_t, TG_LINEAR, 8>, 8);
  } else {
    if (epi == TG_GLU) go(tg_skinny_k<float, TG_GLU, 4>, 4);
    else go(tg_skinny_k<float, TG_LINEAR, 8>, 8);
  }
}

}  // namespace ftp
