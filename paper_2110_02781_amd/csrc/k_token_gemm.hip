// Matrix products of the token operators on the matrix cores, their results finished in the tile that made them.
//
// out[m][n] = sum_k A(m,k) B(n,k).  A and B lie in memory with the reduction along their rows (x, the forward's weights) or across
// them (the weights in a data gradient, both operands of a weight gradient); neither is repacked:
//   * a block owns BM x BN of the result and walks the reduction in steps of 128 bytes of a row (64 bfloat16, 32 fp32).  Both
//     operands' parts of a step go from memory straight into one of two LDS buffers (buffer loads that write LDS: no registers,
//     no LDS-write instructions), while the other buffer is multiplied;
//   * such a load puts its 64 lanes' vectors one behind the other, so the order that keeps LDS reads free of bank conflicts is made
//     by which vector each lane asks for: 16-byte vector c of row r lies at place c ^ (r & 7) (reduction along the row), or 32-byte
//     unit p of reduction row r at p ^ g(r) (across), where it is read by the LDS transpose read (fp32: word by word);
//   * loads go through descriptors whose size ends at the operand, or ask for an offset beyond it: what lies outside arrives as
//     zeros, in rows, columns and reduction alike; descriptors are rebuilt per step from a 64-bit base, offsets in them are within a tile;
//   * the operand of the result's columns is the matrix instruction's first: a lane holds four consecutive columns of one row, which the
//     epilogues (bias, activations, residual, gates, 8-bit form with its group maximum over the eight lanes of 32 columns) take together.
// TG_GLU: half of a tile's columns are the gate's, half the up projection's, arranged so that a lane holds both of a column.
// Long reductions with few tiles are split over blocks; partial sums (fp32) are added in a fixed order by tg_join_k, which runs the same epilogues.
#include <algorithm>

#include "mfma_frag.h"
#include "token_dev.h"

namespace ftp {

template <typename E> struct Tg { enum { V = 16 / sizeof(E), KS = 8 * V, F32 = sizeof(E) == 4 }; };
struct TgGroup { TgJob j[3]; int n, blk0[4]; };

typedef __attribute__((address_space(3))) char lds_char;

// one operand's loader: NQ loads of 1024 bytes per wavefront and step fill R * 128 bytes
template <typename E, int ACROSS, int R, int NW>
struct TgLoad {
  static constexpr int NQ = R / (8 * NW);
  static constexpr uint32_t kPast = 0x80000000u;
  uint32_t off[NQ];
  int kc;                                  // along: this lane's first reduction element in a step
  // row0: first row (of the result's side) of the tile, rows: how many the operand has; ld in elements.  half: rows from R / 2 on belong to
  // a second matrix and count from row0 again
  __device__ __forceinline__ void init(int wave, int lane, int row0, int rows, int64_t ld, bool half) {
    kc = 0;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      if (!ACROSS) {
        int r = (q * NW + wave) * 8 + (lane >> 3);
        const int c = (lane & 7) ^ (r & 7);
        kc = c * Tg<E>::V;
        if (half && r >= R / 2) r -= R / 2;
        off[q] = row0 + r < rows ? (uint32_t)(r * (uint32_t)ld * sizeof(E)) + c * 16 : kPast;
      } else {
        constexpr int CPR = R * sizeof(E) / 16;                 // vectors to a reduction row of the tile
        const int i = (q * NW + wave) * 64 + lane, r = i / CPR, c = i % CPR;
        const int sc = Tg<E>::F32 ? ((((c >> 2) ^ ((r >> 2) & 3)) << 2) | (c & 3)) : ((((c >> 1) ^ ((r & 3) | ((r >> 1) & 4))) << 1) | (c & 1));
        off[q] = row0 + sc * Tg<E>::V < rows ? (uint32_t)(r * (uint32_t)ld * sizeof(E)) + sc * 16 : kPast;
      }
    }
  }
};

typedef uint32_t u4s_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u4s_t tg_rsrc(const char* base, uint32_t bytes) {       // raw buffer: base (48 bits), no stride, size in bytes
  const uint64_t b = (uint64_t)base;
  return u4s_t{(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, bytes, 0x00020000u};
}
// 16 bytes per lane from the buffer to LDS, lane after lane from `lds` (an LDS byte address, the same for the wavefront).  In assembly,
// because of the builtin the compiler waits for all of them in front of the next LDS read, whichever buffer that reads: nothing would be in
// flight beside the products.  There is no output register; what orders these loads is tg_wait_loads and the barrier behind it.
__device__ __forceinline__ void tg_load_lds(u4s_t rs, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(rs) : "memory");   // m0: nothing else here uses it
}
// this wavefront's loads are in LDS and its LDS reads done; then everybody's are
__device__ __forceinline__ void tg_meet() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// blocks of one XCD take a patch of GM row tiles by as many column tiles as come: their operands meet in its L2
__device__ __forceinline__ void tg_tile(int t, int tm, int tn, int& it, int& jt) {
  constexpr int GM = 4;
  const int per = GM * tn, g = t / per, r = t - g * per, first = g * GM, h = tm - first < GM ? tm - first : GM;
  it = first + r % h;
  jt = r / h;
}

template <typename E, int LAY, int EPI, int BM, int BN, int WM, int WN, bool PART>
__global__ __launch_bounds__(64 * WM * WN) void tg_gemm_k(const TgGroup grp) {
  constexpr int KS = Tg<E>::KS, NW = WM * WN, S = BM / (16 * WM), T = BN / (16 * WN);
  constexpr bool F32 = Tg<E>::F32, AX = LAY == TG_TN, BX = LAY != TG_NT, GLU = EPI == TG_GLU;
  constexpr int ABYTES = BM * 128, BBYTES = BN * 128, BUF = ABYTES + BBYTES;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const uint32_t smem_at = (uint32_t)(uintptr_t)(lds_char*)smem;

  int gj = 0, lb;
  if (EPI == TG_GRAD) {
    const int b = blockIdx.x;
    gj = (grp.n > 1 && b >= grp.blk0[1]) + (grp.n > 2 && b >= grp.blk0[2]);
    lb = xcd_logical(b - grp.blk0[gj], grp.blk0[gj + 1] - grp.blk0[gj]);
  } else {
    lb = xcd_logical_block();
  }
  const TgJob& p = grp.j[gj];
  const int ntiles = p.tiles_m * p.tiles_n;
  if (lb >= ntiles * p.splits) return;                          // padding of a group's job to a multiple of the XCDs
  const int split = lb / ntiles;
  int it, jt;
  tg_tile(lb - split * ntiles, p.tiles_m, p.tiles_n, it, jt);
  const int m0 = it * BM, j0 = jt * (GLU ? BN / 2 : BN);
  const int M = p.M, N = p.N, K = p.K;

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15, G = lane >> 4;
  const int wm = wave / WN, wn = wave % WN;

  TgLoad<E, AX, BM, NW> la;
  TgLoad<E, BX, BN, NW> lbd;
  la.init(wave, lane, m0, M, p.lda, false);

  // this block's steps of the reduction, counted through both segments
  const int spseg = (K + KS - 1) / KS, total = spseg * p.nseg;
  const int s0 = split * p.steps, s1 = s0 + p.steps < total ? s0 + p.steps : total;

  const char *pa, *pb, *pb2 = nullptr;
  int64_t stepa, stepb, ldb;
  int seg = s0 >= spseg ? 1 : 0, ks = s0 - seg * spseg;          // next step to fetch
  auto aim = [&]() __attribute__((always_inline)) {
    ldb = seg ? p.ldb[1] : p.ldb[0];
    lbd.init(wave, lane, j0, N, ldb, GLU);
    stepa = (AX ? (int64_t)KS * p.lda : KS) * (int64_t)sizeof(E);
    stepb = (BX ? (int64_t)KS * ldb : KS) * (int64_t)sizeof(E);
    pa = (const char*)(seg ? p.a[1] : p.a[0]) + (AX ? (int64_t)m0 : m0 * p.lda) * (int64_t)sizeof(E) + ks * stepa;
    pb = (const char*)(seg ? p.b[1] : p.b[0]) + (BX ? (int64_t)j0 : j0 * ldb) * (int64_t)sizeof(E) + ks * stepb;
    if (GLU) pb2 = (const char*)p.b[1] + j0 * ldb * (int64_t)sizeof(E) + ks * stepb;
  };
  aim();
  auto fetch = [&](int buf) __attribute__((always_inline)) {
    const int left = K - ks * KS;                               // reduction elements from here on
    const uint32_t sa = smem_at + buf * BUF + wave * 1024, sb = sa + ABYTES;
    {
      const int64_t bytes = AX ? (int64_t)left * p.lda * (int64_t)sizeof(E) : 0x7fffffff;
      const u4s_t rs = tg_rsrc(pa, bytes > 0x7fffffff ? 0x7fffffffu : (uint32_t)bytes);
      const bool in = AX || la.kc < left;
#pragma unroll
      for (int q = 0; q < la.NQ; ++q) tg_load_lds(rs, in ? la.off[q] : la.kPast, sa + q * (NW * 1024));
    }
    {
      const int64_t bytes = BX ? (int64_t)left * ldb * (int64_t)sizeof(E) : 0x7fffffff;
      const uint32_t nb = bytes > 0x7fffffff ? 0x7fffffffu : (uint32_t)bytes;
      const u4s_t rs = tg_rsrc(pb, nb), rs2 = tg_rsrc(GLU ? pb2 : pb, nb);
      const bool in = BX || lbd.kc < left;
#pragma unroll
      for (int q = 0; q < lbd.NQ; ++q) tg_load_lds(GLU && q >= lbd.NQ / 2 ? rs2 : rs, in ? lbd.off[q] : lbd.kPast, sb + q * (NW * 1024));
    }
    ++ks;
    pa += stepa; pb += stepb;
    if (GLU) pb2 += stepb;
    if (p.nseg > 1 && ks == spseg && seg == 0) { seg = 1; ks = 0; aim(); }
  };

  f4v_t acc[S][T];
#pragma unroll
  for (int a = 0; a < S; ++a)
#pragma unroll
    for (int b = 0; b < T; ++b) acc[a][b] = f4v_t{0.f, 0.f, 0.f, 0.f};
  // fp32: the sums of a step are a chain of their own, added up outside it (see pw_gemm_deep_k): a reduction of 16384 would otherwise
  // be one chain of as many additions
  f4v_t tot[F32 ? S : 1][F32 ? T : 1];
  if constexpr (F32)
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) tot[a][b] = f4v_t{0.f, 0.f, 0.f, 0.f};

  // where this lane's fragments lie in a buffer
  const int arow = wm * 16 * S, bsub = wn * T;
  auto brow = [&](int b) __attribute__((always_inline)) {        // first column (row of the LDS tile) of fragment b
    return GLU ? (b < T / 2 ? (bsub / 2 + b) * 16 : BN / 2 + (bsub / 2 + b - T / 2) * 16) : (bsub + b) * 16;
  };
  const int gx = F32 ? G : ((l16 >> 2) | ((G & 1) << 2));        // which reduction rows a lane reads: the order's g(r)
  auto frag = [&](const char* tile, int across, int ext, int sub16, int kstep) __attribute__((always_inline)) -> uint4 {
    if (!across) {
      const int r = sub16 + l16;
      return *reinterpret_cast<const uint4*>(tile + r * 128 + (((kstep * 4 + G) ^ (l16 & 7)) << 4));
    }
    if constexpr (F32) {
      const float* t = reinterpret_cast<const float*>(tile + (kstep * 16 + G * 4) * ext * 4 + ((((sub16 >> 4) ^ gx)) << 6) + l16 * 4);
      return make_uint4(__float_as_uint(t[0]), __float_as_uint(t[ext]), __float_as_uint(t[2 * ext]), __float_as_uint(t[3 * ext]));
    } else {
      const char* t = tile + (kstep * 32 + 8 * G + (l16 >> 2)) * ext * 2 + ((((sub16 >> 4) ^ gx)) << 5) + (l16 & 3) * 8;
      const s4v_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s4v_t __attribute__((address_space(3)))*)t);
      const s4v_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s4v_t __attribute__((address_space(3)))*)(t + 8 * ext));
      const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
      return make_uint4(a.x, a.y, b.x, b.y);
    }
  };

  if (s0 < s1) fetch(0);
  tg_meet();
  for (int s = s0; s < s1; ++s) {
    const int buf = (s - s0) & 1;
    if (s + 1 < s1) fetch(buf ^ 1);
    const char* ta = smem + buf * BUF;
    const char* tb = ta + ABYTES;
    if constexpr (F32) {
#pragma unroll
      for (int a = 0; a < S; ++a)
#pragma unroll
        for (int b = 0; b < T; ++b) tot[a][b] += acc[a][b];
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      uint4 af[S], bf[T];
#pragma unroll
      for (int b = 0; b < T; ++b) bf[b] = frag(tb, BX, BN, brow(b), kk);
#pragma unroll
      for (int a = 0; a < S; ++a) af[a] = frag(ta, AX, BM, arow + a * 16, kk);
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int a = 0; a < S; ++a)
#pragma unroll
            for (int b = 0; b < T; ++b)
              acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float((&bf[b].x)[e]), __uint_as_float((&af[a].x)[e]),
                                                               kk + e == 0 ? f4v_t{0.f, 0.f, 0.f, 0.f} : acc[a][b], 0, 0, 0);
      } else {
#pragma unroll
        for (int a = 0; a < S; ++a)
#pragma unroll
          for (int b = 0; b < T; ++b)
            acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, bf[b]), __builtin_bit_cast(bf16x8_t, af[a]), acc[a][b], 0, 0, 0);
      }
    }
    tg_meet();                   // the next step's operands are there, and this buffer is free
  }
  if constexpr (F32) {
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) acc[a][b] += tot[a][b];
  }

  // ---- results: acc[a][b][e] is column brow(b) + 4 G + e of row 16 a + l16 ----
  const int jb = j0 + (GLU ? bsub / 2 : bsub) * 16 + 4 * G;
  if constexpr (PART) {
    const int64_t np = (N + 3) & ~3, plane = (int64_t)M * np;
    float* const part = p.part + (int64_t)split * (GLU ? 2 : 1) * plane;
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) {
        const int m = m0 + arow + a * 16 + l16, n = jb + (GLU ? b % (T / 2) : b) * 16;
        if (m < M && n < np)
          *reinterpret_cast<float4*>(part + (GLU && b >= T / 2 ? plane : 0) + m * np + n) = make_float4(acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]);
      }
  } else if constexpr (GLU) {
    static_assert(T == 4, "a wavefront's 32 gate columns are one group of the 8-bit form");
#pragma unroll
    for (int a = 0; a < S; ++a) {
      const int64_t m = m0 + arow + a * 16 + l16;
      if (p.save == 2) {         // before the rows past M leave: the maximum goes across lanes (of one row)
        float tg = 0.f, tu = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            tg = fmaxf(tg, act8_mag(acc[a][b][e]));
            tu = fmaxf(tu, act8_mag(acc[a][b + 2][e]));
          }
        tg = fmaxf(tg, __shfl_xor(tg, 16)); tu = fmaxf(tu, __shfl_xor(tu, 16));
        tg = fmaxf(tg, __shfl_xor(tg, 32)); tu = fmaxf(tu, __shfl_xor(tu, 32));
        if (m < M) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const float g[4] = {acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]};
            const float u[4] = {acc[a][b + 2][0], acc[a][b + 2][1], acc[a][b + 2][2], acc[a][b + 2][3]};
            const bool vec = p.flags & TG_VEC_Z;
            tg_keep8(p.z, p.ldz, p.zs, p.lds, m, jb + b * 16, N, vec, b == 0 && G == 0, tg, g);
            tg_keep8(p.up, p.ldu, p.us, p.lds, m, jb + b * 16, N, vec, b == 0 && G == 0, tu, u);
          }
        }
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int n = jb + b * 16;
        const float g[4] = {acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]};
        const float u[4] = {acc[a][b + 2][0], acc[a][b + 2][1], acc[a][b + 2][2], acc[a][b + 2][3]};
        if (m < M && n < p.ldo) tg_glu4<E>(p, m, n, g, u);
      }
    }
  } else {
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) {
        const int64_t m = m0 + arow + a * 16 + l16;
        const int n = jb + b * 16;
        float v[4] = {acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]};
        if (m < M && n < (EPI == TG_GLUBWD ? (int)p.ldo : N)) {
          if (EPI == TG_LINEAR) tg_linear4<E>(p, m, n, v);
          if (EPI == TG_GLUBWD) tg_glubwd4<E>(p, m, n, v);
          if (EPI == TG_GRAD) tg_grad4<E>(p, m, n, v);
        }
      }
  }
}

// adds the partial sums of a split reduction, split after split, and finishes the results: a thread has four columns of a row,
// the eight threads of 32 columns lie next to one another
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
#pragma unroll
        for (int x = 1; x < 8; x <<= 1) { tg = fmaxf(tg, __shfl_xor(tg, x)); tu = fmaxf(tu, __shfl_xor(tu, x)); }
        if (in) {
          tg_keep8(p.z, p.ldz, p.zs, p.lds, m, n, p.N, p.flags & TG_VEC_Z, (n & 31) == 0, tg, v);
          tg_keep8(p.up, p.ldu, p.us, p.lds, m, n, p.N, p.flags & TG_VEC_Z, (n & 31) == 0, tu, u);
        }
      }
      if (m < p.M && n < p.ldo) tg_glu4<E>(p, m, n, v, u);
    } else if constexpr (EPI == TG_GLUBWD) {
      if (m < p.M && n < p.ldo) tg_glubwd4<E>(p, m, n, v);
    } else {
      if (in && EPI == TG_LINEAR) tg_linear4<E>(p, m, n, v);
      if (in && EPI == TG_GRAD) tg_grad4<E>(p, m, n, v);
    }
  }
}

// ------------------------------------------------------------------ host
namespace {
struct Tile { int bm, bn; };
Tile tile_of(int dt, int big) { return dt == 1 && big ? Tile{256, 256} : Tile{128, 128}; }
}  // namespace

size_t tg_part_bytes(int epi, int M, int N, int splits) {
  return splits > 1 ? (size_t)splits * (epi == TG_GLU ? 2 : 1) * M * ((N + 3) & ~3) * 4 : 0;
}

TgPlan tg_plan(int dt, int lay, int epi, int M, int N, int K, size_t max_bytes) {
  const int ks = dt == 1 ? 64 : 32, steps = std::max(1, (K + ks - 1) / ks);
  TgPlan best{0, 1};
  double best_t = 1e30;
  for (int big = 0; big <= (dt == 1); ++big) {
    const Tile t = tile_of(dt, big);
    const double tiles = (double)((M + t.bm - 1) / t.bm) * ((N + (epi == TG_GLU ? t.bn / 2 : t.bn) - 1) / (epi == TG_GLU ? t.bn / 2 : t.bn));
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (s > 1 && (steps < 4 * s || tg_part_bytes(epi, M, N, s) > max_bytes)) break;
      const int per = (steps + s - 1) / s;
      const double blocks = tiles * s;
      // microseconds: a big step 1.4 with one block to a CU; a small one 0.45 alone on its CU, 0.6 for two beside each other
      // (fp32 2.6, 4.0)
      double us;
      if (big) us = std::max(1.0, std::ceil(blocks / 256)) * (per * 1.4 + 4.0);
      else {
        const double one = dt == 1 ? 0.45 : 2.6, two = dt == 1 ? 0.6 : 4.6;
        const double full = std::floor(blocks / 512), rest = blocks - full * 512;
        us = full * (per * two + 2.0) + (rest > 256 ? per * two + 2.0 : rest > 0 ? per * one + 2.0 : 0.0);
      }
      if (s > 1) us += 4.0 + 2.0 * (double)tg_part_bytes(epi, M, N, s) / 4e6;
      if (us < best_t) { best_t = us; best = TgPlan{big, s}; }
    }
  }
  return best;
}

template <typename E, int LAY, int EPI, int BM, int BN, int WM, int WN>
static void launch_tile(hipStream_t st, TgGroup& g, bool part) {
  constexpr int KS = Tg<E>::KS, LDS = 2 * (BM + BN) * 128;
  int blocks = 0;
  for (int i = 0; i < g.n; ++i) {
    TgJob& j = g.j[i];
    const int bn = EPI == TG_GLU ? BN / 2 : BN;
    j.tiles_m = (j.M + BM - 1) / BM;
    j.tiles_n = (j.N + bn - 1) / bn;
    const int total = ((j.K + KS - 1) / KS) * j.nseg;
    j.steps = (total + j.splits - 1) / j.splits;
    g.blk0[i] = blocks;
    blocks += g.n > 1 ? (j.tiles_m * j.tiles_n * j.splits + 7) / 8 * 8 : j.tiles_m * j.tiles_n * j.splits;
  }
  g.blk0[g.n] = blocks;
  auto go = [&](auto k) {
    static const hipError_t set = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (set != hipSuccess) { launch_plan_failed("tg_gemm_k: no room for its LDS"); return; }
    hipLaunchKernelGGL(k, dim3(blocks), dim3(64 * WM * WN), LDS, st, g);
  };
  if (part) go(tg_gemm_k<E, LAY, EPI, BM, BN, WM, WN, true>);
  else go(tg_gemm_k<E, LAY, EPI, BM, BN, WM, WN, false>);
}

template <typename E, int LAY, int EPI>
static void launch(hipStream_t st, TgGroup& g, TgPlan plan) {
  const bool part = plan.splits > 1;
  if (sizeof(E) == 2 && plan.big) {
    if constexpr (sizeof(E) == 2) launch_tile<E, LAY, EPI, 256, 256, 2, 4>(st, g, part);
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
// matrices) and its wavefronts share the reduction; a lane reads 64 consecutive bytes of one weight row per turn, four vectors in
// flight, as operands of the matrix instruction (16 weight rows by 16 rows of x), which takes reduction elements in any order as
// long as both operands agree.  The wavefronts' sums meet in LDS in a fixed order.
template <typename E, int EPI, int NW>
__global__ __launch_bounds__(64 * NW) void tg_skinny_k(const TgJob p) {
  constexpr int V = Tg<E>::V, U = 4;                            // vectors a lane reads per turn
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
  const int turn = 4 * U * V;                                   // reduction elements a wavefront takes per turn
  for (int k0 = wave * turn; k0 < K; k0 += NW * turn) {
    uint4 a[U], b[U], c[U];
    const int k = k0 + G * U * V;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = k + u * V < K;                            // K is a multiple of V: a vector is inside or outside
      const int64_t o = (int64_t)(in ? k + u * V : 0) * (int64_t)sizeof(E);
      a[u] = *reinterpret_cast<const uint4*>(w0 + o);
      if (GLU) b[u] = *reinterpret_cast<const uint4*>(w1 + o);
      c[u] = make_uint4(0, 0, 0, 0);
      if (xin && in) c[u] = *reinterpret_cast<const uint4*>(x + o);
      if (!in) { a[u] = make_uint4(0, 0, 0, 0); b[u] = a[u]; }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      acc[0] = mul(acc[0], a[u], c[u]);
      if (GLU) acc[1] = mul(acc[1], b[u], c[u]);
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
  else { if (n < N) tg_linear4<E>(p, l16, n, v); }
}

void tg_skinny(int dt, hipStream_t st, int epi, const TgJob& j) {
  const double es = dt == 1 ? 2 : 4, two = epi == TG_GLU ? 2 : 1;
  KScope ks(st, epi == TG_GLU ? "tok_glu_few" : "tok_linear_few", es * (two * j.N * j.K + (double)j.M * (j.K + j.N)), 2.0 * two * j.M * j.N * j.K,
            j.M, j.K, j.N);
  const int blocks = (j.N + 15) / 16;
  auto go = [&](auto k, int nw) { hipLaunchKernelGGL(k, dim3(blocks), dim3(64 * nw), 0, st, j); };
  if (dt == 1) {
    if (epi == TG_GLU) go(tg_skinny_k<bf16_t, TG_GLU, 8>, 8);
    else go(tg_skinny_k<bf16_t, TG_LINEAR, 16>, 16);
  } else {
    if (epi == TG_GLU) go(tg_skinny_k<float, TG_GLU, 8>, 8);
    else go(tg_skinny_k<float, TG_LINEAR, 16>, 16);
  }
}

}  // namespace ftp
