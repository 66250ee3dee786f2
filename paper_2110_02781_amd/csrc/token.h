// Launch interface of the token kernels: linear layers, gated feed-forward blocks, 8-bit checkpoints, table lookups.
// Shapes and alignment are the caller's to check (token.cpp); nothing here allocates.
#pragma once
#include <algorithm>

#include "kernels.h"

namespace ftp {

enum { TACT_NONE = 0, TACT_RELU = 1, TACT_RELU6 = 2, TACT_SILU = 3, TACT_GELU = 4 };
enum { kAct8Group = 32 };
static inline int act8_groups(int cols) { return (cols + kAct8Group - 1) / kAct8Group; }

// What becomes of a product's tile.
enum {
  TG_LINEAR = 0,    // (+ bias) [-> z], act, (+ residual) -> out
  TG_GLU = 1,       // act(gate) * up -> out; gate and up kept as they are or in 8 bits
  TG_GLUBWD = 2,    // d hidden -> d gate, d up, hidden, from the gate and up that were kept
  TG_GRAD = 3       // weight gradient: fp32 (may add to what is there) or the call's type
};
// Operands: rows of the reduction ("as" 0: [rows][reduction], 1: [reduction][rows]).  out[m][n] = sum_k A(m,k) B(n,k).
enum { TG_NT = 0, TG_NN = 1, TG_TN = 2 };   // A, B as: (0,0) (0,1) (1,1)

struct TgJob {
  const void* a[2];       // two reduction segments (b[1] of TG_GLU: the up projection's weights instead)
  const void* b[2];
  int64_t lda, ldb[2];    // elements
  int M, N, K, nseg;      // K: one segment's
  // results
  int act, save, flags;   // flags: TG_VEC_*
  const float* bias;
  const void* res; int64_t ldr;
  void* out; int64_t ldo;
  void* z; int64_t ldz;               // TG_LINEAR: z out; TG_GLU, TG_GLUBWD: gate kept
  void* up; int64_t ldu;              // up kept
  uint8_t *zs, *us; int64_t lds;      // their scales (save 2)
  void *dgate, *dup; int64_t ldd;     // TG_GLUBWD
  int out_f32, accumulate;            // TG_GRAD
  float* part;                        // split reductions: [splits][1 or 2][M][Np], Np = N rounded up to 4
  // set by the launcher
  int tiles_m, tiles_n, splits, steps;
};
enum { TG_VEC_OUT = 1, TG_VEC_RES = 2, TG_VEC_Z = 4, TG_VEC_BIAS = 8 };   // four consecutive columns go as one access

struct TgPlan { int tile, splits; };     // tile: 256, 128 or 64 rows and columns
// tile and split of one job's reduction; max_bytes: workspace that its partial sums may take
TgPlan tg_plan(int dt, int epi, int M, int N, int K, size_t max_bytes);
size_t tg_part_bytes(int epi, int M, int N, int splits);
// jobs [0, n): n up to 3, all with the same plan (TG_GRAD), otherwise 1
void tg_launch(int dt, hipStream_t st, int lay, int epi, TgJob* jobs, int n, TgPlan plan);

// few rows against all of the weights: rows <= kSkinnyRows, operands [rows][reduction]; TG_LINEAR and TG_GLU
enum { kSkinnyRows = 16 };
void tg_skinny(int dt, hipStream_t st, int epi, const TgJob& j);

// dz = dy * act'(z) [M][ldd], pad columns zero; partial column sums of it: part[chunks][N]; nothing is written where dz is null
int tk_dz_chunks(int M);
void tk_dz(int dt, hipStream_t st, const void* dy, int64_t lddy, const void* z, int64_t ldz, int act, int M, int N, void* dz,
           int64_t ldd, float* part);
void tk_colsum_join(hipStream_t st, const float* part, int chunks, int N, void* db, int out_dt, int accumulate);
// copies of rows into rows (16-byte aligned) of ldy elements, a multiple of 16 bytes, the rest of a row zero; up to kCopies of them
enum { kCopies = 5 };
struct TkCopy { const void* x; int64_t ldx; void* y; int64_t ldy; int rows, cols; };
void tk_align(int dt, hipStream_t st, const TkCopy* jobs, int n);
void tk_act8_pack(int dt, hipStream_t st, const void* x, int64_t ldx, int64_t M, int N, uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds);
void tk_act8_unpack(int dt, hipStream_t st, const uint8_t* q, int64_t ldq, const uint8_t* s, int64_t lds, int64_t M, int N, int pad_to,
                    void* y, int64_t ldy);

void tk_embed(int dt, hipStream_t st, const void* ids, int ids64, int64_t n, int vocab, int width, float scale, const void* table,
              int64_t ldt, void* out, int64_t ldo);
size_t tk_embed_bwd_bytes(int64_t n, int vocab, int width);
void tk_embed_bwd(int dt, hipStream_t st, const void* ids, int ids64, int64_t n, int vocab, int width, float scale, int64_t pad_id,
                  const void* dy, int64_t lddy, float* dtable, int64_t lddt, int accumulate, void* ws);
void tk_fill(hipStream_t st, void* p, int64_t rows, int64_t row_bytes, int64_t ld_bytes);

// Calls go out in slices of rows whose vectors are numbered below 2^30, so that the division into row and place is a 32-bit one.
template <typename F>
static inline void by_rows(int64_t rows, int64_t per_row, F f) {
  const int64_t step = std::max<int64_t>(1, ((int64_t)1 << 30) / std::max<int64_t>(per_row, 1));
  for (int64_t r = 0; r < rows; r += step) f(r, (int)std::min(step, rows - r));
}
// whether what a call moves is more than the card's last cache (256 MB) holds: then nothing of it is there when it is next asked for
static inline bool past_the_caches(double bytes) { return bytes > 256e6; }
static inline unsigned blocks_of(int64_t n, int most) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((n + 255) / 256, most)); }

}  // namespace ftp
