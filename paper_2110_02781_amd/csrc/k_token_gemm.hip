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
#include <type_traits>

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
  const auto one = [](uint32_t v) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };   // scalar registers
  return u4s_t{one((uint32_t)b), one((uint32_t)(b >> 32) & 0xffffu), one(bytes), 0x00020000u};
}
// 16 bytes per lane from the buffer to LDS, lane after lane from `lds` (an LDS byte address, the same for the wavefront).  In assembly,
// because of the builtin the compiler waits for all of them in front of the next LDS read, whichever buffer that reads: nothing would be in
// flight beside the products.  There is no output register; what orders these loads is tg_wait_loads and the barrier behind it.
__device__ __forceinline__ void tg_load_lds(u4s_t rs, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(rs) : "memory");   // m0: nothing else here uses it
}
// the same in two parts, with one instruction or more between them
template <int ADD> __device__ __forceinline__ void tg_aim_lds(uint32_t lds) { asm volatile("s_add_u32 m0, %0, %1" ::"s"(lds), "n"(ADD) : "memory", "scc"); }
__device__ __forceinline__ void tg_load_aimed(u4s_t rs, uint32_t off) { asm volatile("buffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(rs) : "memory"); }
// this wavefront's loads but the N youngest are in LDS and its LDS reads done; then everybody's are
template <int N = 0>
__device__ __forceinline__ void tg_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
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

// what a block does: its job, tile and steps of the reduction, and the loading of a step
template <typename E, int LAY, int EPI, int BM, int BN, int NW>
struct TgBlock {
  static constexpr int KS = Tg<E>::KS, ABYTES = BM * 128, BUF = (BM + BN) * 128;
  static constexpr bool AX = LAY == TG_TN, BX = LAY != TG_NT, GLU = EPI == TG_GLU;
  int split, m0, j0, s0, s1, wave, lane;
  int K, nseg, spseg, seg, ks;             // seg, ks: the next step to fetch
  uint32_t smem_at;
  const char *pa, *pb, *pb2;
  uint32_t stepa, stepb;                   // bytes
  int64_t lda, ldb;
  TgLoad<E, AX, BM, NW> la;
  TgLoad<E, BX, BN, NW> lb;

  __device__ __forceinline__ static const TgJob& job(const TgGroup& grp, int& lb) {
    if (EPI != TG_GRAD) {
      lb = xcd_logical_block();
      return grp.j[0];
    }
    const int b = blockIdx.x, j = (grp.n > 1 && b >= grp.blk0[1]) + (grp.n > 2 && b >= grp.blk0[2]);
    lb = xcd_logical(b - grp.blk0[j], grp.blk0[j + 1] - grp.blk0[j]);
    return grp.j[j];
  }
  // false: a block of a group's job's padding to a multiple of the XCDs
  __device__ __forceinline__ bool init(const TgJob& p, int b, const char* smem) {
    smem_at = (uint32_t)(uintptr_t)(const lds_char*)smem;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lane = threadIdx.x & 63;
    const int ntiles = p.tiles_m * p.tiles_n;
    if (b >= ntiles * p.splits) return false;
    split = b / ntiles;
    int it, jt;
    tg_tile(b - split * ntiles, p.tiles_m, p.tiles_n, it, jt);
    m0 = it * BM;
    j0 = jt * (GLU ? BN / 2 : BN);
    K = p.K;
    nseg = p.nseg;
    lda = p.lda;
    spseg = (K + KS - 1) / KS;
    const int total = spseg * nseg;
    s0 = split * p.steps;
    s1 = s0 + p.steps < total ? s0 + p.steps : total;
    seg = s0 >= spseg ? 1 : 0;
    ks = s0 - seg * spseg;
    la.init(wave, lane, m0, p.M, lda, false);
    aim(p);
    return true;
  }
  __device__ __forceinline__ void aim(const TgJob& p) {
    ldb = seg ? p.ldb[1] : p.ldb[0];
    lb.init(wave, lane, j0, p.N, ldb, GLU);
    stepa = (uint32_t)((AX ? KS * lda : KS) * (int64_t)sizeof(E));
    stepb = (uint32_t)((BX ? KS * ldb : KS) * (int64_t)sizeof(E));
    pa = (const char*)(seg ? p.a[1] : p.a[0]) + (AX ? (int64_t)m0 : m0 * lda) * (int64_t)sizeof(E) + ks * (int64_t)stepa;
    pb = (const char*)(seg ? p.b[1] : p.b[0]) + (BX ? (int64_t)j0 : j0 * ldb) * (int64_t)sizeof(E) + ks * (int64_t)stepb;
    if (GLU) pb2 = (const char*)p.b[1] + j0 * ldb * (int64_t)sizeof(E) + ks * (int64_t)stepb;
  }
  // the next step's descriptors: a base that moves on by a step, and a size that ends with the reduction where it runs across the rows
  // (past the last step: nothing is inside)
  __device__ __forceinline__ u4s_t source(const char* base, bool across, int64_t ld) const {
    const int left = K - ks * KS, in = left < 0 ? 0 : left < KS ? left : KS;
    return tg_rsrc(base, across ? (uint32_t)in * (uint32_t)ld * (uint32_t)sizeof(E) : 0x7fffffffu);
  }
  __device__ __forceinline__ u4s_t source_a() const { return source(pa, AX, lda); }
  __device__ __forceinline__ u4s_t source_b() const { return source(pb, BX, ldb); }
  __device__ __forceinline__ u4s_t source_b2() const { return source(GLU ? pb2 : pb, BX, ldb); }
  __device__ __forceinline__ bool in_a() const { return AX || la.kc < K - ks * KS; }
  __device__ __forceinline__ bool in_b() const { return BX || lb.kc < K - ks * KS; }
  __device__ __forceinline__ uint32_t place(uint32_t at) const { return smem_at + at + wave * 1024; }
  __device__ __forceinline__ void next(const TgJob& p) {
    ++ks;
    pa += stepa;
    pb += stepb;
    if (GLU) pb2 += stepb;
    if (LAY == TG_NN && nseg > 1 && ks == spseg && seg == 0) { seg = 1; ks = 0; aim(p); }
  }
  // requests the next step's operands into LDS at at_a and at_b
  __device__ __forceinline__ void fetch(const TgJob& p, uint32_t at_a, uint32_t at_b) {
    const u4s_t fa = source_a(), fb = source_b(), fb2 = source_b2();
    const bool ina = in_a(), inb = in_b();
#pragma unroll
    for (int q = 0; q < la.NQ; ++q) tg_load_lds(fa, ina ? la.off[q] : la.kPast, place(at_a) + q * (NW * 1024));
#pragma unroll
    for (int q = 0; q < lb.NQ; ++q) tg_load_lds(GLU && q >= lb.NQ / 2 ? fb2 : fb, inb ? lb.off[q] : lb.kPast, place(at_b) + q * (NW * 1024));
    next(p);
  }
};

// a lane's fragment of 16 rows (of the result's side) from sub16 on, 64 bytes of the reduction: kstep 0 or 1 of a step
template <typename E, bool ACROSS, int EXT>
__device__ __forceinline__ uint4 tg_frag(const char* tile, int sub16, int kstep, int l16, int G) {
  if constexpr (!ACROSS) {
    return *reinterpret_cast<const uint4*>(tile + (sub16 + l16) * 128 + (((kstep * 4 + G) ^ (l16 & 7)) << 4));
  } else if constexpr (Tg<E>::F32) {
    const float* t = reinterpret_cast<const float*>(tile + (kstep * 16 + G * 4) * EXT * 4 + (((sub16 >> 4) ^ G) << 6) + l16 * 4);
    return make_uint4(__float_as_uint(t[0]), __float_as_uint(t[EXT]), __float_as_uint(t[2 * EXT]), __float_as_uint(t[3 * EXT]));
  } else {
    const int g = (l16 >> 2) | ((G & 1) << 2);                   // the order's g(r) of the reduction rows this lane reads
    const char* t = tile + (kstep * 32 + 8 * G + (l16 >> 2)) * EXT * 2 + (((sub16 >> 4) ^ g) << 5) + (l16 & 3) * 8;
    const s4v_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s4v_t __attribute__((address_space(3)))*)t);
    const s4v_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s4v_t __attribute__((address_space(3)))*)(t + 8 * EXT));
    const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
    return make_uint4(a.x, a.y, b.x, b.y);
  }
}

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

template <typename E, int LAY, int EPI, int BM, int BN, int WM, int WN, bool PART>
__global__ __launch_bounds__(64 * WM * WN) void tg_gemm_k(const TgGroup grp) {
  typedef TgBlock<E, LAY, EPI, BM, BN, WM * WN> B;
  constexpr int S = BM / (16 * WM), T = BN / (16 * WN);
  constexpr bool F32 = Tg<E>::F32, GLU = EPI == TG_GLU;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  int lb;
  const TgJob& p = B::job(grp, lb);
  B blk;
  if (!blk.init(p, lb, smem)) return;
  const int l16 = blk.lane & 15, G = blk.lane >> 4, wm = blk.wave / WN, wn = blk.wave % WN;
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
  // fp32: the sums of a step are a chain of their own, added up outside it (see pw_gemm_deep_k): a reduction of 16384 would otherwise
  // be one chain of as many additions
  f4v_t tot[F32 ? S : 1][F32 ? T : 1];
  if constexpr (F32)
#pragma unroll
    for (int a = 0; a < S; ++a)
#pragma unroll
      for (int b = 0; b < T; ++b) tot[a][b] = f4v_t{0.f, 0.f, 0.f, 0.f};

  if (s0 < s1) blk.fetch(p, 0, B::ABYTES);
  tg_meet();
  for (int s = s0; s < s1; ++s) {
    const int buf = (s - s0) & 1;
    if (s + 1 < s1) blk.fetch(p, (buf ^ 1) * B::BUF, (buf ^ 1) * B::BUF + B::ABYTES);
    const char* ta = smem + buf * B::BUF;
    const char* tb = ta + B::ABYTES;
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

  tg_results<E, EPI, S, T, PART>(p, acc, split, m0 + arow + l16, j0 + (GLU ? bsub / 2 : bsub) * 16 + 4 * G, G);
}

// gate and up of four columns of a row; the eight lanes of 32 columns lie next to one another
template <bool PART, bool F>
__device__ __forceinline__ void tg_glu_row(const TgJob& p, int split, int64_t m, int n, const float4 a, const float4 b) {
  if constexpr (PART) {
    const int64_t np = (p.N + 3) & ~3, plane = (int64_t)p.M * np;
    if (m < p.M && n < np) {
      float* const q = p.part + (int64_t)split * 2 * plane + m * np + n;
      *reinterpret_cast<float4*>(q) = a;
      *reinterpret_cast<float4*>(q + plane) = b;
    }
  } else {
    const float g[4] = {a.x, a.y, a.z, a.w}, u[4] = {b.x, b.y, b.z, b.w};
    if (p.save == 2) {
      float tg = 0.f, tu = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) { tg = fmaxf(tg, act8_mag(g[e])); tu = fmaxf(tu, act8_mag(u[e])); }
      tg = tg_max8(tg);
      tu = tg_max8(tu);
      if (m < p.M) {
        const bool vec = p.flags & TG_VEC_Z;
        tg_keep8<F>(p.z, p.ldz, p.zs, p.lds, m, n, p.N, vec, (n & 31) == 0, tg, g);
        tg_keep8<F>(p.up, p.ldu, p.us, p.lds, m, n, p.N, vec, (n & 31) == 0, tu, u);
      }
    }
    if (m < p.M && (F || n < p.ldo)) tg_glu4<bf16_t, F>(p, m, n, g, u);
  }
}

// 64 rows of 128 columns from LDS (rows LD apart), eight rows of a lane at a time.  What the epilogue reads from memory is requested for the next eight
// before these are finished: there is nobody else on the SIMD to fill the wait.  F: all of the tile's columns are inside and go by fours.
template <int EPI, bool PART, bool F, int LD>
__device__ __forceinline__ void tg_rows(const TgJob& p, int split, const float* mine, int row0, int jw, int lane) {
  if constexpr (EPI == TG_GLU) {
    const int c = (lane & 15) * 4;
#pragma unroll 1
    for (int i = 0; i < 64; i += 16) {
      float4 g[4], u[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float* q = mine + (i + 4 * k + (lane >> 4)) * LD + c;
        g[k] = ld4(q);
        u[k] = ld4(q + 64);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) tg_glu_row<PART, F>(p, split, row0 + i + 4 * k + (lane >> 4), jw + c, g[k], u[k]);
    }
  } else {
    const int c = (lane & 31) * 4, n = jw + c, r0 = lane >> 5;
    const int wide = EPI == TG_GLUBWD && !PART ? (int)p.ldo : p.N;
    if (!F && n >= wide) return;
    typedef TgSide<bf16_t, PART ? TG_GRAD : EPI, F> Side;
    Side now[8], next[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) next[k].request(p, row0 + 2 * k + r0, n);
#pragma unroll 1
    for (int i = 0; i < 64; i += 16) {
#pragma unroll
      for (int k = 0; k < 8; ++k) now[k] = next[k];
      if (i < 48) {
#pragma unroll
        for (int k = 0; k < 8; ++k) next[k].request(p, row0 + i + 16 + 2 * k + r0, n);
      }
      float4 t[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) t[k] = ld4(mine + (i + 2 * k + r0) * LD + c);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int64_t m = row0 + i + 2 * k + r0;
        if (m >= p.M) continue;
        if constexpr (PART) {
          const int64_t np = (p.N + 3) & ~3;
          *reinterpret_cast<float4*>(p.part + ((int64_t)split * p.M + m) * np + n) = t[k];
        } else {
          float v[4] = {t[k].x, t[k].y, t[k].z, t[k].w};
          now[k].finish(p, m, n, v);
        }
      }
    }
  }
}

// The large bfloat16 tile: 256 x 256 by four wavefronts of 128 x 128, one to a SIMD.  LDS is read once per 128 columns and rows that way (eight
// wavefronts of 128 x 64 would read half as much again: with the loads' writes all that LDS gives while the matrix cores work), the sums take
// half of a wavefront's 512 registers, and nobody else's instructions fill its gaps: what is read and requested is written between the products here.
// A step's two halves are in registers in turn: while one is multiplied the other is read, and the meeting of the wavefronts lies between the halves,
// behind the last read of the step's operands.
// The instruction is written out because the sums fill all accumulation registers: compiled from the builtin a dozen of them are copied away
// and back in every step.
template <int LAY, int EPI, bool PART>
__global__ __launch_bounds__(256, 1) void tg_big_k(const TgGroup grp) {
  typedef TgBlock<bf16_t, LAY, EPI, 256, 256, 4> B;
  constexpr bool GLU = EPI == TG_GLU;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  int lb;
  const TgJob& p = B::job(grp, lb);
  B blk;
  if (!blk.init(p, lb, smem)) return;
  const int l16 = blk.lane & 15, G = blk.lane >> 4, wm = blk.wave >> 1, wn = blk.wave & 1;
  const int arow = wm * 128, bsub = wn * 8;
  auto brow = [&](int b) __attribute__((always_inline)) { return GLU ? (b < 4 ? (bsub / 2 + b) * 16 : 128 + (bsub / 2 + b - 4) * 16) : (bsub + b) * 16; };
  f4v_t acc[8][8];
#pragma unroll
  for (int a = 0; a < 8; ++a)
#pragma unroll
    for (int b = 0; b < 8; ++b) acc[a][b] = f4v_t{0.f, 0.f, 0.f, 0.f};

  uint4 a0[8], b0[8], a1[8], b1[8];
  // LDS holds five units of 32 KB: both operands of this step and the next, and the rows' operand of the step after that, which is requested during
  // this step's first half; its columns' follows in the second half, where this step's rows lay.  Units are dealt in the order of the requests.
  constexpr uint32_t UNIT = 32768;
  auto mul = [&](const uint4& fa, const uint4 (&fb)[8], int a, int b) __attribute__((always_inline)) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[a][b]) : "v"(__builtin_bit_cast(bf16x8_t, fb[b])), "v"(__builtin_bit_cast(bf16x8_t, fa)));
    __builtin_amdgcn_sched_barrier(0);
  };
  blk.fetch(p, 0, UNIT);
  blk.fetch(p, 2 * UNIT, 3 * UNIT);
  tg_meet<16>();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a0[i] = tg_frag<bf16_t, B::AX, 256>(smem, arow + i * 16, 0, l16, G);
    b0[i] = tg_frag<bf16_t, B::BX, 256>(smem + UNIT, brow(i), 0, l16, G);
  }
  // fragment i of half kk: the columns' eight first, all of which the half's first products need, then the rows', one a turn
  auto read = [&](uint4 (&ra)[8], uint4 (&rb)[8], int i, uint32_t ua, uint32_t ub, int kk) __attribute__((always_inline)) {
    if (i < 8) rb[i] = tg_frag<bf16_t, B::BX, 256>(smem + ub, brow(i), kk, l16, G);
    else if (i < 16) ra[i - 8] = tg_frag<bf16_t, B::AX, 256>(smem + ua, arow + (i - 8) * 16, kk, l16, G);
  };
  // Half a step: its 64 products in eight turns, and between them the eight requests of one operand and the reading of the other half's fragments (Q a
  // turn).  A product keeps the matrix core for as long as four instructions take to issue, so what stands between two products is free as long as it
  // is no more than three; sixteen in front of eight products were 0.66 of the time in products, so 0.75.  Reads that end with the half are waited for
  // at its end: three a turn in the first half leave two turns for the last ones to arrive.
#define TG_TURN(I, fa, fb, ra, rb, ua, ub, kk, Q, at, rs, in, off)                    \
  {                                                                                   \
    tg_aim_lds<I * 4096>(at);                                                         \
    mul(fa[I], fb, I, 0);                                                             \
    tg_load_aimed(rs(I), in ? off[I] : blk.la.kPast);                                 \
    mul(fa[I], fb, I, 1);                                                             \
    read(ra, rb, Q * I, ua, ub, kk);                                                  \
    mul(fa[I], fb, I, 2);                                                             \
    read(ra, rb, Q * I + 1, ua, ub, kk);                                              \
    mul(fa[I], fb, I, 3);                                                             \
    mul(fa[I], fb, I, 4);                                                             \
    mul(fa[I], fb, I, 5);                                                             \
    if (Q == 3) read(ra, rb, Q * I + 2, ua, ub, kk);                                  \
    mul(fa[I], fb, I, 6);                                                             \
  }
  uint32_t u0 = 0, u1 = UNIT, u2 = 2 * UNIT, u3 = 3 * UNIT, u4 = 4 * UNIT;
  u4s_t ra = blk.source_a(), rb = blk.source_b(), rb2 = blk.source_b2();
  bool ina = blk.in_a(), inb = blk.in_b();
  for (int s = blk.s0; s < blk.s1; ++s) {
    const uint32_t at = blk.place(u4), bt = blk.place(u0);
#define TG_A(q) ra
#define TG_B(q) (GLU && q >= 4 ? rb2 : rb)
#define TG_FIRST(I) TG_TURN(I, a0, b0, a1, b1, u0, u1, 1, 3, at, TG_A, ina, blk.la.off) mul(a0[I], b0, I, 7);
#define TG_SECOND(I) TG_TURN(I, a1, b1, a0, b0, u2, u3, 0, 2, bt, TG_B, inb, blk.lb.off)
    TG_FIRST(0) TG_FIRST(1) TG_FIRST(2) TG_FIRST(3) TG_FIRST(4) TG_FIRST(5) TG_FIRST(6) TG_FIRST(7)
    tg_meet<8>();                // all but the requests of this half: the next step is in LDS, and this one's units are free
    TG_SECOND(0) mul(a1[0], b1, 0, 7);
    TG_SECOND(1) mul(a1[1], b1, 1, 7);
    TG_SECOND(2) mul(a1[2], b1, 2, 7);
    TG_SECOND(3) mul(a1[3], b1, 3, 7);
    blk.next(p);                 // the next step's descriptors, between products too (the columns' requests go on until the last turn)
    TG_SECOND(4)
    ra = blk.source_a();
    mul(a1[4], b1, 4, 7);
    TG_SECOND(5)
    const u4s_t nb = blk.source_b();
    mul(a1[5], b1, 5, 7);
    TG_SECOND(6)
    const u4s_t nb2 = blk.source_b2();
    mul(a1[6], b1, 6, 7);
    TG_SECOND(7)
    rb = nb;
    if (GLU) rb2 = nb2;
    ina = blk.in_a(), inb = blk.in_b();
    const uint32_t v0 = u0, v1 = u1;
    u0 = u2; u1 = u3; u2 = u4; u3 = v0; u4 = v1;
    mul(a1[7], b1, 7, 7);
  }
#undef TG_TURN
#undef TG_A
#undef TG_B
#undef TG_FIRST
#undef TG_SECOND
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");           // the last products' results are there (the compiler does not know when)
  // Results: through LDS, half of the wavefront's rows at a time, so that they leave by rows (a lane has four columns, a row is 256 or 512
  // consecutive bytes) in a short loop.  Rows in LDS are 16 bytes more than their 512 apart: the 16 rows of a write are in banks of their own.
  tg_meet();                     // nobody's requests (of steps past the end: zeros) or reads are under way
  constexpr int LD = 132;
  float* const mine = reinterpret_cast<float*>(smem) + blk.wave * (64 * LD);
  const int jw = blk.j0 + (GLU ? bsub / 2 : bsub) * 16;
  const int need = (EPI == TG_GRAD || EPI == TG_LINEAR ? TG_VEC_OUT : 0) | (EPI == TG_LINEAR && p.res ? TG_VEC_RES : 0) |
                   ((EPI == TG_LINEAR && p.z) || EPI == TG_GLUBWD || (GLU && p.save) ? TG_VEC_Z : 0) | (EPI == TG_LINEAR && p.bias ? TG_VEC_BIAS : 0);
  const bool inside = blk.j0 + (GLU ? 128 : 256) <= p.N && (p.flags & need) == need;
  auto write = [&](auto half) __attribute__((always_inline)) {
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int b = 0; b < 8; ++b) *reinterpret_cast<f4v_t*>(mine + (a * 16 + l16) * LD + b * 16 + 4 * G) = acc[half.value * 4 + a][b];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // the other lanes' columns too: a wavefront's LDS accesses are in order
  };
  auto rows = [&](int row0) __attribute__((always_inline)) {
    if (PART || !inside) tg_rows<EPI, PART, false, LD>(p, blk.split, mine, row0, jw, blk.lane);
    else tg_rows<EPI, PART, true, LD>(p, blk.split, mine, row0, jw, blk.lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  const int row0 = blk.m0 + arow;
  write(std::integral_constant<int, 0>());
  rows(row0);
  write(std::integral_constant<int, 1>());
  rows(row0 + 64);
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
      // microseconds.  Large tile: 1.6 a step and 14 around them; small: 0.65 a step and 8 with a CU to itself, 1.12 and 10 for two beside each other
      // (fp32: 2.6, 4.6 a step)
      double us;
      if (big) us = std::ceil(blocks / 256) * (per * 1.6 + 14.0);
      else {
        const double one = dt == 1 ? 0.65 : 2.6, two = dt == 1 ? 1.12 : 4.6;
        const double full = std::floor(blocks / 512), rest = blocks - full * 512;
        us = full * (per * two + 10.0) + (rest > 256 ? per * two + 10.0 : rest > 0 ? per * one + 8.0 : 0.0);
      }
      if (s > 1) us += 4.0 + 2.0 * (double)tg_part_bytes(epi, M, N, s) / 4e6;
      if (us < best_t) { best_t = us; best = TgPlan{big, s}; }
    }
  }
  return best;
}

template <typename E, int LAY, int EPI, int BM, int BN, int WM, int WN>
static void launch_tile(hipStream_t st, TgGroup& g, bool part) {
  constexpr int KS = Tg<E>::KS, LDS = BM == 256 ? 5 * 32768 : 2 * (BM + BN) * 128;
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
  constexpr bool BIG = BM == 256;
  auto go = [&](auto k) {
    static const hipError_t set = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (set != hipSuccess) { launch_plan_failed("tg_gemm_k: no room for its LDS"); return; }
    hipLaunchKernelGGL(k, dim3(blocks), dim3(64 * WM * WN), LDS, st, g);
  };
  if constexpr (BIG) {
    if (part) go(tg_big_k<LAY, EPI, true>);
    else go(tg_big_k<LAY, EPI, false>);
  } else {
    if (part) go(tg_gemm_k<E, LAY, EPI, BM, BN, WM, WN, true>);
    else go(tg_gemm_k<E, LAY, EPI, BM, BN, WM, WN, false>);
  }
}

template <typename E, int LAY, int EPI>
static void launch(hipStream_t st, TgGroup& g, TgPlan plan) {
  const bool part = plan.splits > 1;
  if (sizeof(E) == 2 && plan.big) {
    if constexpr (sizeof(E) == 2) launch_tile<E, LAY, EPI, 256, 256, 2, 2>(st, g, part);
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
  ks.route(dt == 1 && plan.big ? plan.splits > 1 ? "256 split" : "256" : plan.splits > 1 ? "128 split" : "128");
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
  else { if (n < N) tg_finish4<E, EPI>(p, l16, n, v); }
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
