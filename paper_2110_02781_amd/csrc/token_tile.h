// What the token operators' products share: which tile a block has, how its operands get into LDS and from there into registers.
//
// out[m][n] = sum_k A(m,k) B(n,k).  A and B lie in memory with the reduction along their rows (x, the forward's weights) or across
// them (the weights in a data gradient, both operands of a weight gradient); neither is repacked:
//   * a block owns BM x BN of the result and walks the reduction in steps of 128 bytes of a row (64 bfloat16, 32 fp32).  Both
//     operands' parts of a step go from memory straight into LDS (buffer loads that write it: no registers, no LDS-write
//     instructions), while an earlier step's is multiplied: two buffers, three for tiles of 64, five half ones for the large tile;
//   * such a load puts its 64 lanes' vectors one behind the other, so the order that keeps LDS reads free of bank conflicts is made
//     by which vector each lane asks for: 16-byte vector c of row r lies at place c ^ (r & 7) (reduction along the row), or 32-byte
//     unit p of reduction row r at p ^ g(r) (across; g: the low two bits of r and its bit 3, as many as there are units), where it is read by the LDS transpose read (fp32: word by word);
//   * loads go through descriptors whose size ends at the operand, or ask for an offset beyond it: what lies outside arrives as
//     zeros, in rows, columns and reduction alike; descriptors are rebuilt per step from a 64-bit base, offsets in them are within a tile;
//   * the operand of the result's columns is the matrix instruction's first: a lane holds four consecutive columns of one row, which the
//     epilogues (bias, activations, residual, gates, 8-bit form with its group maximum over the eight lanes of 32 columns) take together.
// TG_GLU: half of a tile's columns are the gate's, half the up projection's, arranged so that a lane holds both of a column.
// Long reductions with few tiles are split over blocks; partial sums (fp32) are added in a fixed order by tg_join_k, which runs the same epilogues.
#pragma once
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
  // a second matrix, whose rows are ld_half apart, and count from row0 again
  __device__ __forceinline__ void init(int wave, int lane, int row0, int rows, int64_t ld, bool half, int64_t ld_half) {
    kc = 0;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      if (!ACROSS) {
        int r = (q * NW + wave) * 8 + (lane >> 3);
        const int c = (lane & 7) ^ (r & 7);
        kc = c * Tg<E>::V;
        uint32_t apart = (uint32_t)ld;
        if (half && r >= R / 2) { r -= R / 2; apart = (uint32_t)ld_half; }
        off[q] = row0 + r < rows ? (uint32_t)(r * apart * sizeof(E)) + c * 16 : kPast;
      } else {
        constexpr int CPR = R * sizeof(E) / 16;                 // vectors to a reduction row of the tile
        const int i = (q * NW + wave) * 64 + lane, r = i / CPR, c = i % CPR;
        const int g = Tg<E>::F32 ? (r >> 2) & 3 : ((r & 3) | ((r >> 1) & 4)) & (R / 16 - 1);
        const int sc = Tg<E>::F32 ? (((c >> 2) ^ g) << 2) | (c & 3) : (((c >> 1) ^ g) << 1) | (c & 1);
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
// A vector instruction that wrote a scalar register (the size's way through tg_rsrc) must be five wait states ahead of the memory instruction that reads it; the
// compiler sees to that only for its own instructions, the loads below are written out.
__device__ __forceinline__ void tg_settle(u4s_t& a, u4s_t& b) { asm volatile("s_nop 4" : "+s"(a), "+s"(b)); }
__device__ __forceinline__ void tg_settle(u4s_t& a, u4s_t& b, u4s_t& c) { asm volatile("s_nop 4" : "+s"(a), "+s"(b), "+s"(c)); }
// the descriptor is complete here, not only where it is used
__device__ __forceinline__ void tg_pin(u4s_t& a) { asm volatile("" : "+s"(a)); }
// 16 bytes per lane from the buffer to LDS, lane after lane from `lds` (an LDS byte address, the same for the wavefront; m0 is set in the statement that goes by it).  In assembly,
// because of the builtin the compiler waits for all of them in front of the next LDS read, whichever buffer that reads: nothing would be in
// flight beside the products.  There is no output register; what orders these loads is tg_meet.
__device__ __forceinline__ void tg_load_lds(u4s_t rs, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(rs) : "memory");
}
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

// LDS buffers of the small tiles: with a CU to itself a block of 64 x 64 multiplies for half the time that its operands take to come
constexpr int tg_buffers(int bm) { return bm == 64 ? 3 : 2; }

// what a block does: its job, tile and steps of the reduction, and the loading of a step
template <typename E, int LAY, int EPI, int BM, int BN, int NW>
struct TgBlock {
  static constexpr int KS = Tg<E>::KS, ABYTES = BM * 128, BUF = (BM + BN) * 128, NL = (BM + BN) / (8 * NW);   // NL: a wavefront's requests a step
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
    seg = nseg > 1 && s0 >= spseg ? 1 : 0;
    ks = s0 - seg * spseg;
    la.init(wave, lane, m0, p.M, lda, false, lda);
    aim(p);
    return true;
  }
  __device__ __forceinline__ void aim(const TgJob& p) {
    aim_bases(p);
    aim_offsets(p);
  }
  __device__ __forceinline__ void aim_offsets(const TgJob& p) {
    lb.init(wave, lane, j0, p.N, ldb, GLU, p.ldb[1]);            // with TG_GLU b[1] is the up projection's weights, in rows of their own distance
  }
  __device__ __forceinline__ void aim_bases(const TgJob& p) {
    ldb = seg ? p.ldb[1] : p.ldb[0];
    stepa = (uint32_t)((AX ? KS * lda : KS) * (int64_t)sizeof(E));
    stepb = (uint32_t)((BX ? KS * ldb : KS) * (int64_t)sizeof(E));
    pa = (const char*)(seg ? p.a[1] : p.a[0]) + (AX ? (int64_t)m0 : m0 * lda) * (int64_t)sizeof(E) + ks * (int64_t)stepa;
    pb = (const char*)(seg ? p.b[1] : p.b[0]) + (BX ? (int64_t)j0 : j0 * ldb) * (int64_t)sizeof(E) + ks * (int64_t)stepb;
    if (GLU) pb2 = (const char*)p.b[1] + j0 * p.ldb[1] * (int64_t)sizeof(E) + ks * (int64_t)stepb;
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
    if (next_bases(p)) aim_offsets(p);
  }
  // true: the second segment begins, whose rows have a distance of their own: aim_offsets() is due, after the last request of this step
  __device__ __forceinline__ bool next_bases(const TgJob& p) {
    ++ks;
    pa += stepa;
    pb += stepb;
    if (GLU) pb2 += stepb;
    if (!(LAY == TG_NN && nseg > 1 && ks == spseg && seg == 0)) return false;
    seg = 1;
    ks = 0;
    aim_bases(p);
    return true;
  }
  // requests the next step's operands into LDS at at_a and at_b
  __device__ __forceinline__ void fetch(const TgJob& p, uint32_t at_a, uint32_t at_b) {
    u4s_t fa = source_a(), fb = source_b(), fb2 = fb;
    if constexpr (GLU) {
      fb2 = source_b2();
      tg_settle(fa, fb, fb2);
    } else {
      tg_settle(fa, fb);
    }
    const bool ina = in_a(), inb = in_b();
#pragma unroll
    for (int q = 0; q < la.NQ; ++q) tg_load_lds(fa, ina ? la.off[q] : la.kPast, place(at_a) + q * (NW * 1024));
#pragma unroll
    for (int q = 0; q < lb.NQ; ++q) {
      const bool up = GLU && (lb.NQ > 1 ? q >= lb.NQ / 2 : wave >= NW / 2);                // rows from BN / 2 on
      tg_load_lds(up ? fb2 : fb, inb ? lb.off[q] : lb.kPast, place(at_b) + q * (NW * 1024));
    }
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
    const int g = ((l16 >> 2) | ((G & 1) << 2)) & (EXT / 16 - 1);   // the order's g(r) of the reduction rows this lane reads
    const char* t = tile + (kstep * 32 + 8 * G + (l16 >> 2)) * EXT * 2 + (((sub16 >> 4) ^ g) << 5) + (l16 & 3) * 8;
    const s4v_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s4v_t __attribute__((address_space(3)))*)t);
    const s4v_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s4v_t __attribute__((address_space(3)))*)(t + 8 * EXT));
    const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
    return make_uint4(a.x, a.y, b.x, b.y);
  }
}

// kernels with more LDS than the runtime gives without being told
template <auto* K>
static void tg_launch_lds(hipStream_t st, const TgGroup& g, int blocks, int threads, int lds) {
  static const hipError_t set = hipFuncSetAttribute((const void*)K, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (set != hipSuccess) { launch_plan_failed("a token product's kernel gets no room for its LDS"); return; }
  hipLaunchKernelGGL(K, dim3(blocks), dim3(threads), lds, st, g);
}
// the large tile's launch (k_token_big.hip)
void tg_big_launch(hipStream_t st, int lay, int epi, const TgGroup& g, int blocks, bool part);

}  // namespace ftp
