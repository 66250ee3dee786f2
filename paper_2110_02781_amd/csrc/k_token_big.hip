// The large bfloat16 tile of the token operators' products.  A file of its own: its sums fill the accumulation registers, which the other kernels are
// compiled without.
#include <type_traits>

#include "token_tile.h"

namespace ftp {

// gate and up of four columns of a row; the eight lanes of 32 columns lie next to one another
template <bool PART>
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
        tg_keep8(p.z, p.ldz, p.zs, p.lds, m, n, p.N, vec, (n & 31) == 0, tg, g);
        tg_keep8(p.up, p.ldu, p.us, p.lds, m, n, p.N, vec, (n & 31) == 0, tu, u);
      }
    }
    if (m < p.M && n < p.ldo) tg_glu4<bf16_t>(p, m, n, g, u);
  }
}

// `rows` (16, 32, 48 or 64) whole rows of 128 columns from LDS (rows LD apart); a lane's four columns are inside or outside.  Eight rows of a lane at a time,
// and each question (which activation, whether there is a residual) asked once for the eight: nobody else is on the SIMD, so what is not in flight, or
// not next to other rows' instructions, is waited for.  32768 x 512 by 2048 weight rows with bias and GELU: 103 us, 158 asked row by row; without either
// 87 and 108.  What comes from memory is requested eight rows ahead.
template <int EPI, int LD>
__device__ __forceinline__ void tg_rows_inside(const TgJob& p, const float* mine, int row0, int jw, int lane, int rows) {
  if constexpr (EPI == TG_GLU) {
    const int c = (lane & 15) * 4, n = jw + c, first = lane >> 4;
    const bool lead = (n & 31) == 0, in = n < p.N;
    bf16_t* const out = (bf16_t*)p.out + (int64_t)(row0 + first) * p.ldo + n;
#pragma unroll 1
    for (int i = 0; i < rows; i += 16) {
      float g[16], u[16];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float* q = mine + (i + 4 * k + first) * LD + c;
        const float4 a = ld4(q), b = ld4(q + 64);
        g[4 * k] = a.x; g[4 * k + 1] = a.y; g[4 * k + 2] = a.z; g[4 * k + 3] = a.w;
        u[4 * k] = b.x; u[4 * k + 1] = b.y; u[4 * k + 2] = b.z; u[4 * k + 3] = b.w;
      }
      if (p.save == 2) {
        float tg[4], tu[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          tg[k] = tu[k] = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) { tg[k] = fmaxf(tg[k], act8_mag(g[4 * k + e])); tu[k] = fmaxf(tu[k], act8_mag(u[4 * k + e])); }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) { tg[k] = tg_max8(tg[k]); tu[k] = tg_max8(tu[k]); }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (!in) break;                                        // outside only now: the maximum goes across lanes
          const int64_t m = row0 + i + 4 * k + first;
          tg_keep8<true>(p.z, p.ldz, p.zs, p.lds, m, n, p.N, true, lead, tg[k], g + 4 * k);
          tg_keep8<true>(p.up, p.ldu, p.us, p.lds, m, n, p.N, true, lead, tu[k], u + 4 * k);
        }
      }
      if (!in) continue;
      if (p.save == 1) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t m = row0 + i + 4 * k + first;
          put4<bf16_t, true>(p.z, p.ldz, m, n, p.N, true, g + 4 * k);
          put4<bf16_t, true>(p.up, p.ldu, m, n, p.N, true, u + 4 * k);
        }
      }
      tactn<16>(g, p.act);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int e = 0; e < 4; ++e) g[4 * k + e] *= u[4 * k + e];
        put4<bf16_t, true>(out + (i + 4 * k) * p.ldo, 0, 0, 0, 0, true, g + 4 * k);
      }
    }
  } else {
    const int c = (lane & 31) * 4, n = jw + c, r0 = lane >> 5, m0 = row0 + r0;
    if (n >= p.N) return;
    typedef TgSide<bf16_t, EPI, true> Side;
    Side now[8], next[8];
    const bool asks = EPI == TG_GLUBWD || (EPI == TG_LINEAR && p.res);
    auto request = [&](int i) __attribute__((always_inline)) {
      if (asks) {
#pragma unroll
        for (int k = 0; k < 8; ++k) next[k].request(p, m0 + i + 2 * k, n);
      }
    };
    request(0);
    float bias[4] = {0.f, 0.f, 0.f, 0.f};
    if (EPI == TG_LINEAR && p.bias) get4<float, true>(p.bias, 0, 0, n, p.N, true, bias);
#pragma unroll 1
    for (int i = 0; i < rows; i += 16) {
#pragma unroll
      for (int k = 0; k < 8; ++k) now[k] = next[k];
      if (i + 16 < rows) request(i + 16);
      float v[32];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float4 t = ld4(mine + (i + 2 * k + r0) * LD + c);
        v[4 * k] = t.x; v[4 * k + 1] = t.y; v[4 * k + 2] = t.z; v[4 * k + 3] = t.w;
      }
      if constexpr (EPI == TG_LINEAR) {
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] += bias[e & 3];
        if (p.z) {
#pragma unroll
          for (int k = 0; k < 8; ++k) put4<bf16_t, true>(p.z, p.ldz, m0 + i + 2 * k, n, p.N, true, v + 4 * k);
        }
        tactn<32>(v, p.act);
        if (p.res) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            float r[4];
            open4<bf16_t>(now[k].res, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * k + e] += r[e];
          }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) put4<bf16_t, true>(p.out, p.ldo, m0 + i + 2 * k, n, p.N, true, v + 4 * k);
      } else if constexpr (EPI == TG_GLUBWD) {
#pragma unroll
        for (int h = 0; h < 8; h += 4) Side::template finish_rows<4>(now + h, p, m0 + i + 2 * h, n, v + 4 * h);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) now[k].finish(p, m0 + i + 2 * k, n, v + 4 * k);
      }
    }
  }
}

// The same at the matrix's edges and for partial sums: 64 rows of 128 columns from LDS, eight rows of a lane at a time.  What the epilogue reads from memory is
// requested for the next eight before these are finished.
template <int EPI, bool PART, int LD>
__device__ __forceinline__ void tg_rows(const TgJob& p, int split, const float* mine, int row0, int jw, int lane, int from) {
  const int left = p.M - row0, to = left < 64 ? left : 64;
  if constexpr (EPI == TG_GLU) {
    const int c = (lane & 15) * 4;
#pragma unroll 1
    for (int i = from; i < to; i += 16) {
      float4 g[4], u[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float* q = mine + (i + 4 * k + (lane >> 4)) * LD + c;
        g[k] = ld4(q);
        u[k] = ld4(q + 64);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) tg_glu_row<PART>(p, split, row0 + i + 4 * k + (lane >> 4), jw + c, g[k], u[k]);
    }
  } else {
    const int c = (lane & 31) * 4, n = jw + c, r0 = lane >> 5;
    const int wide = EPI == TG_GLUBWD && !PART ? (int)p.ldo : p.N;
    if (n >= wide) return;
    typedef TgSide<bf16_t, PART ? TG_GRAD : EPI> Side;
    Side now[8], next[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) next[k].request(p, row0 + from + 2 * k + r0, n);
#pragma unroll 1
    for (int i = from; i < to; i += 16) {
#pragma unroll
      for (int k = 0; k < 8; ++k) now[k] = next[k];
      if (i + 16 < to) {
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
// Bound by the matrix cores and, with data that is not zeros, by the card's power: a gated block of 8192 rows, 4096 x 14336, runs its products at 1280
// (gate and up with their 8-bit form), 1095 (their gradients), 1500 (down), 1410 (dx) and 1255 TFLOP/s (weight gradients); a library product of the three operand
// orders at 1435 to 1617, 1160 to 1390 and 960 to 1185.  The matrix cores are busy 80, 71 and 68 % of the cycles in the three operand orders, 9, 12 and 15 % of the
// wavefronts' are waits (a library product's: 87, 70, 52 and 4, 9, 11; profiles/token_pmc_matrix.txt).  Requests and reads in front of
// eight products instead of one between two: 4096 x 4096 x 16384 439 us instead of 405; products of 32 x 32 x 16: 441 for 418.
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
  // a product between the setting of m0, to lds + ADD, and the load into LDS that goes by it (tg_load_lds has an idle instruction there): one statement, so that
  // nothing the compiler adds comes between
  auto mul_load = [&](const uint4& fa, const uint4 (&fb)[8], int a, uint32_t lds, auto add, const u4s_t& rs, uint32_t off) __attribute__((always_inline)) {
    asm volatile("s_add_u32 m0, %3, %4\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0\n\tbuffer_load_dwordx4 %5, %6, 0 offen lds"
                 : "+a"(acc[a][0])
                 : "v"(__builtin_bit_cast(bf16x8_t, fb[0])), "v"(__builtin_bit_cast(bf16x8_t, fa)), "s"(lds), "n"(add.value), "v"(off), "s"(rs)
                 : "memory", "scc");
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
    mul_load(fa[I], fb, I, at, std::integral_constant<int, I * 4096>(), rs(I), in ? off[I] : blk.la.kPast); \
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
  u4s_t ra = blk.source_a(), rb = blk.source_b(), rb2 = rb;
  if constexpr (GLU) {
    rb2 = blk.source_b2();
    tg_settle(ra, rb, rb2);
  } else {
    tg_settle(ra, rb);
  }
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
    const bool turned = blk.next_bases(p);   // the next step's descriptors, between products too; the columns' requests go on until the last turn, with the
                                             // descriptor and the offsets of this step
    TG_SECOND(4)
    ra = blk.source_a();         // its first reader is more than five products away, as those of nb and nb2 are
    tg_pin(ra);
    mul(a1[4], b1, 4, 7);
    TG_SECOND(5)
    u4s_t nb = blk.source_b();
    tg_pin(nb);
    mul(a1[5], b1, 5, 7);
    TG_SECOND(6)
    u4s_t nb2 = nb;
    if constexpr (GLU) {
      nb2 = blk.source_b2();
      tg_pin(nb2);
    }
    mul(a1[6], b1, 6, 7);
    TG_SECOND(7)
    if (turned) blk.aim_offsets(p);
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
  // The last products' results are there (the compiler does not know when: tests/test_token_waits.py looks whether it has put a sum's copy in front)
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  // Results: through LDS, half of the wavefront's rows at a time, so that they leave by rows (a lane has four columns, a row is 256 or 512
  // consecutive bytes) in a short loop.  Rows in LDS are 16 bytes more than their 512 apart: the 16 rows of a write are in banks of their own.
  tg_meet();                     // nobody's requests (of steps past the end: zeros) or reads are under way
  constexpr int LD = 132;
  float* const mine = reinterpret_cast<float*>(smem) + blk.wave * (64 * LD);
  const int jw = blk.j0 + (GLU ? bsub / 2 : bsub) * 16;
  const int need = (EPI == TG_GRAD || EPI == TG_LINEAR ? TG_VEC_OUT : 0) | (EPI == TG_LINEAR && p.res ? TG_VEC_RES : 0) |
                   ((EPI == TG_LINEAR && p.z) || EPI == TG_GLUBWD || (GLU && p.save) ? TG_VEC_Z : 0) | (EPI == TG_LINEAR && p.bias ? TG_VEC_BIAS : 0);
  // fours of columns that are accessed as one, and no columns that only pad the rows: whole rows are quick
  const bool quick = (p.flags & need) == need && p.N % 4 == 0 && (EPI == TG_LINEAR || EPI == TG_GRAD || p.ldo == p.N);
  auto write = [&](auto half) __attribute__((always_inline)) {
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int b = 0; b < 8; ++b) *reinterpret_cast<f4v_t*>(mine + (a * 16 + l16) * LD + b * 16 + 4 * G) = acc[half.value * 4 + a][b];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // the other lanes' columns too: a wavefront's LDS accesses are in order
  };
  auto rows = [&](int row0) __attribute__((always_inline)) {
    int done = 0;
    if constexpr (!PART) {
      const int left = p.M - row0;
      done = !quick || left < 0 ? 0 : left < 64 ? left & ~15 : 64;
      if (done) tg_rows_inside<EPI, LD>(p, mine, row0, jw, blk.lane, done);
    }
    if (done < 64) tg_rows<EPI, PART, LD>(p, blk.split, mine, row0, jw, blk.lane, done);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  const int row0 = blk.m0 + arow;
  write(std::integral_constant<int, 0>());
  rows(row0);
  write(std::integral_constant<int, 1>());
  rows(row0 + 64);
}

template <int LAY, int EPI>
static void big_launch(hipStream_t st, const TgGroup& g, int blocks, bool part) {
  constexpr int LDS = 5 * 32768;
  if (part) tg_launch_lds<tg_big_k<LAY, EPI, true>>(st, g, blocks, 256, LDS);
  else tg_launch_lds<tg_big_k<LAY, EPI, false>>(st, g, blocks, 256, LDS);
}
void tg_big_launch(hipStream_t st, int lay, int epi, const TgGroup& g, int blocks, bool part) {
  if (epi == TG_LINEAR && lay == TG_NT) big_launch<TG_NT, TG_LINEAR>(st, g, blocks, part);
  else if (epi == TG_LINEAR) big_launch<TG_NN, TG_LINEAR>(st, g, blocks, part);
  else if (epi == TG_GLU) big_launch<TG_NT, TG_GLU>(st, g, blocks, part);
  else if (epi == TG_GLUBWD) big_launch<TG_NN, TG_GLUBWD>(st, g, blocks, part);
  else big_launch<TG_TN, TG_GRAD>(st, g, blocks, part);
}

}  // namespace ftp
