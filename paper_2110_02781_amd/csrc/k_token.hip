// Memory-bound token kernels: table lookup and its gradient by sorted tokens, the 8-bit form of activations, the gradient behind a
// linear layer's activation, rows copied into the alignment that the matrix products need.
// Rows may start at any element: vectors of 16 bytes are accessed at the element's alignment (global memory takes them unaligned).
#include <algorithm>
#include <type_traits>

#include "token_dev.h"

namespace ftp {

// ---------------------------------------------------------------- table lookup
// out[t] = scale * table[id], 8 columns a thread; a row of NaN where the id is none of the table's.  Memory: 16384 rows of 2048 bfloat16 from 32000
// take 22 us, 6.1 TB/s of rows read (in part from the caches) and written; 8 rows take a launch, 6.5 us with the call.
template <typename E, typename I>
__global__ __launch_bounds__(256) void embed_fwd_k(const I* __restrict__ ids, int64_t t0, int rows, int vocab, int width, float scale,
                                                   const E* __restrict__ table, int64_t ldt, E* __restrict__ out, int64_t ldo) {
  const uint32_t per = (width + 7) / 8, all = (uint32_t)rows * per;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) {
    const uint32_t r = i / per, c = (i - r * per) * 8;
    const int64_t t = t0 + r;
    const int64_t id = (int64_t)ids[t];
    float v[8];
    if (id >= 0 && id < vocab) {
      tk_load8<E>(table + id * ldt + c, width - (int)c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= scale;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(0x7fc00000u);
    }
    tk_store8<E>(out + t * ldo + c, width - (int)c, v);
  }
}

void tk_embed(int dt, hipStream_t st, const void* ids, int ids64, int64_t n, int vocab, int width, float scale, const void* table,
              int64_t ldt, void* out, int64_t ldo) {
  const int es = dt == 1 ? 2 : 4;
  KScope ks(st, "tok_embed", 2.0 * n * width * es + 4.0 * n, (double)n * width, n, vocab, width);
  by_rows(n, (width + 7) / 8, [&](int64_t t0, int rows) {
    const unsigned b = blocks_of((int64_t)rows * ((width + 7) / 8), 1 << 20);
    auto go = [&](auto k, auto* id, auto* tab, auto* o) {
      hipLaunchKernelGGL(k, dim3(b), dim3(256), 0, st, id, t0, rows, vocab, width, scale, tab, ldt, o, ldo);
    };
    if (dt == 1 && ids64) go(embed_fwd_k<bf16_t, int64_t>, (const int64_t*)ids, (const bf16_t*)table, (bf16_t*)out);
    else if (dt == 1) go(embed_fwd_k<bf16_t, int32_t>, (const int32_t*)ids, (const bf16_t*)table, (bf16_t*)out);
    else if (ids64) go(embed_fwd_k<float, int64_t>, (const int64_t*)ids, (const float*)table, (float*)out);
    else go(embed_fwd_k<float, int32_t>, (const int32_t*)ids, (const float*)table, (float*)out);
  });
}

// zeros: block b of nb, blocks of T threads.  Rows start at any element of two bytes or four, and end at one
template <int T>
__device__ __forceinline__ void tk_fill_rows(char* __restrict__ p, uint32_t rows, int64_t row_bytes, int64_t ld_bytes, uint32_t b, uint32_t nb) {
  const uint32_t per = (uint32_t)((row_bytes + 15) / 16), all = rows * per;
  for (uint32_t i = b * T + threadIdx.x; i < all; i += nb * T) {
    const uint32_t r = i / per, c = i - r * per;
    char* const q = p + (int64_t)r * ld_bytes + (int64_t)c * 16;
    const int64_t left = row_bytes - (int64_t)c * 16;
    if (left >= 16) tk_st16<bf16_t>(reinterpret_cast<bf16_t*>(q), u4v_t{0, 0, 0, 0});
    else
      for (int64_t o = 0; o < left; o += 2) *reinterpret_cast<bf16_t*>(q + o) = 0;
  }
}
__global__ __launch_bounds__(256) void tk_fill_k(char* __restrict__ p, uint32_t rows, int64_t row_bytes, int64_t ld_bytes) {
  tk_fill_rows<256>(p, rows, row_bytes, ld_bytes, blockIdx.x, gridDim.x);
}
// rows one behind the other count as longer ones
static void long_rows(int64_t& rows, int64_t& row_bytes, int64_t& ld_bytes) {
  if (ld_bytes != row_bytes || row_bytes >= 65536) return;
  int64_t f = std::min<int64_t>(64, rows);
  while (f > 1 && rows % f) --f;
  rows /= f; row_bytes *= f; ld_bytes *= f;
}

// ---------------------------------------------------------------- its gradient
// Tokens are sorted by id, equal ids in the order of the tokens; then every kRun of them are one block's: it walks them with a running
// sum per column and writes a row of the gradient where the id changes.  What an id has in other runs as well goes to memory as partial
// sums, which embed_join_k adds in the order of the runs.  No atomics: the same tokens give the same bits.
enum { kRun = 16, kChunk = 8192, kChunksMost = 65536, kTile = 4096, kDigit = 8 };
#define FTP_NO_ID 0xffffffffu

// an id as the sort sees it: one that is no row's, or whose gradient is left out, behind all others
__device__ __forceinline__ uint32_t embed_key(int64_t id, int vocab, int64_t pad_id) {
  return id >= 0 && id < vocab && id != pad_id ? (uint32_t)id : FTP_NO_ID;
}
template <typename I>
__global__ __launch_bounds__(256) void embed_keys_k(const I* __restrict__ ids, int n, int vocab, int64_t pad_id, uint32_t* __restrict__ keys,
                                                    uint32_t* __restrict__ pos) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    keys[i] = embed_key((int64_t)ids[i], vocab, pad_id);
    pos[i] = (uint32_t)i;
  }
}
// A token's place among kChunk tokens is how many come before it, counted outright: n^2 comparisons, two instructions for 64 of them, no passes
// that wait for one another.  A block has the chunk's keys in LDS and places 64 tokens, its sixteen wavefronts share the ones compared with, four to a
// read that all lanes make together.  The blocks from `rank` on write the zeros that a gradient written whole starts from, beside the counting,
// which leaves the memory alone.  (Keys by scalar loads, four wavefronts: 16384 tokens at once 85 us; that many beside 262 MB of zeros now 43, the zeros' time.)
template <typename I>
__global__ __launch_bounds__(1024) void embed_rank_k(const I* __restrict__ ids, int n, int vocab, int64_t pad_id, uint32_t* __restrict__ skeys,
                                                     uint32_t* __restrict__ spos, int rank, char* __restrict__ zero, uint32_t rows,
                                                     int64_t row_bytes, int64_t ld_bytes) {
  constexpr int W = 16;
  __shared__ __attribute__((aligned(16))) uint32_t key[kChunk];
  __shared__ uint32_t cnt[W][64];
  if ((int)blockIdx.x >= rank) {
    tk_fill_rows<1024>(zero, rows, row_bytes, ld_bytes, blockIdx.x - rank, gridDim.x - rank);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = blockIdx.x * 64, c0 = first / kChunk * kChunk, m = n - c0 < kChunk ? n - c0 : kChunk, at0 = first - c0;   // first: a multiple of 64
  const int m4 = (m + 3) & ~3;
  for (int j = threadIdx.x; j < m4; j += 1024) key[j] = j < m ? embed_key((int64_t)ids[c0 + j], vocab, pad_id) : 0xffffffffu;
  __syncthreads();
  const int i = at0 + lane;
  const uint32_t k = i < m ? key[i] : 0;
  uint32_t c = 0;
  // tokens in front of this block's count where their id is not larger, those behind it where it is smaller (what pads the last four never is)
  const int per = (((m4 + W - 1) / W) + 3) & ~3, j0 = wave * per, j1 = j0 + per < m4 ? j0 + per : m4;
  const int f1 = j1 < at0 ? j1 : at0, b0 = j0 > at0 + 64 ? j0 : at0 + 64;
#pragma unroll 4
  for (int j = j0; j < f1; j += 4) {
    const uint4 q = *reinterpret_cast<const uint4*>(key + j);
    c += q.x <= k; c += q.y <= k; c += q.z <= k; c += q.w <= k;
  }
  for (int j = j0 > at0 ? j0 : at0; j < j1 && j < at0 + 64; ++j) c += key[j] < k || (key[j] == k && j < i);
#pragma unroll 4
  for (int j = b0; j < j1; j += 4) {
    const uint4 q = *reinterpret_cast<const uint4*>(key + j);
    c += q.x < k; c += q.y < k; c += q.z < k; c += q.w < k;
  }
  cnt[wave][lane] = c;
  __syncthreads();
  if (wave == 0 && i < m) {
    uint32_t at = c0;
#pragma unroll
    for (int w = 0; w < W; ++w) at += cnt[w][lane];
    skeys[at] = k;
    spos[at] = (uint32_t)(first + lane);
  }
}
// From sorted chunks to one order: a token's place is its own in its chunk and, for every other chunk, how many there come before it (ids not larger in
// the chunks in front, smaller ones in those behind), by halving, four chunks at a time.
__global__ __launch_bounds__(256) void embed_merge_k(const uint32_t* __restrict__ keys, const uint32_t* __restrict__ pos, int n,
                                                     uint32_t* __restrict__ okeys, uint32_t* __restrict__ opos) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int own = i / kChunk, chunks = (n + kChunk - 1) / kChunk;
  const uint32_t k = keys[i];
  uint32_t at = (uint32_t)(i - own * kChunk);
  for (int c = 0; c < chunks; c += 4) {
    int lo[4], size[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = (c + u) * kChunk;
      lo[u] = 0;
      size[u] = c + u >= chunks || c + u == own ? 0 : n - s < kChunk ? n - s : kChunk;
    }
    // how many of the chunk's first `size` count: halves of [lo, lo + size]
#pragma unroll 1
    for (int h = kChunk; h > 0; h >>= 1) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int m = lo[u] + h;                                 // do the first m count?  (the m-th decides)
        const bool in = m <= size[u];
        const uint32_t x = in ? keys[(c + u) * kChunk + m - 1] : 0;
        if (in && (c + u < own ? x <= k : x < k)) lo[u] = m;
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) at += lo[u];
  }
  okeys[at] = k;
  opos[at] = pos[i];
}
// Many tokens (more than 65536: 131072 of width 256 took 215 us in chunks, 188 this way; 32768 72 in chunks, more than 110 this way): 8 bits of the
// id at a time, from the lowest.  A block has kTile tokens; counts per block and digit, their running sum over (digit, block), then every token goes to
// its digit's place in its order.
__global__ __launch_bounds__(256) void embed_count_k(const uint32_t* __restrict__ keys, int n, int shift, uint32_t* __restrict__ hist, int blocks) {
  __shared__ uint32_t h[256];
  h[threadIdx.x] = 0;
  __syncthreads();
  for (int u = 0; u < kTile / 256; ++u) {
    const int i = blockIdx.x * kTile + u * 256 + threadIdx.x;
    if (i < n) atomicAdd(&h[(keys[i] >> shift) & 255], 1u);      // counts: their order does not matter
  }
  __syncthreads();
  hist[threadIdx.x * blocks + blockIdx.x] = h[threadIdx.x];
}
__global__ __launch_bounds__(1024) void embed_scan_k(uint32_t* __restrict__ hist, int m) {       // exclusive running sum, one block
  __shared__ uint32_t part[1024];
  const int per = (m + 1023) / 1024, a = threadIdx.x * per, b = a + per < m ? a + per : m;
  uint32_t s = 0;
  for (int i = a; i < b; ++i) s += hist[i];
  part[threadIdx.x] = s;
  __syncthreads();
  for (int d = 1; d < 1024; d <<= 1) {
    const uint32_t t = threadIdx.x >= (unsigned)d ? part[threadIdx.x - d] : 0;
    __syncthreads();
    part[threadIdx.x] += t;
    __syncthreads();
  }
  s = part[threadIdx.x] - s;
  for (int i = a; i < b; ++i) {
    const uint32_t t = hist[i];
    hist[i] = s;
    s += t;
  }
}
__global__ __launch_bounds__(256) void embed_place_k(const uint32_t* __restrict__ keys, const uint32_t* __restrict__ pos, int n, int shift,
                                                     const uint32_t* __restrict__ hist, int blocks, uint32_t* __restrict__ okeys,
                                                     uint32_t* __restrict__ opos) {
  __shared__ uint32_t next[256], have[4][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  next[tid] = hist[tid * blocks + blockIdx.x];
  for (int u = 0; u < kTile / 256; ++u) {
    const int i = blockIdx.x * kTile + u * 256 + tid;
    const bool in = i < n;
    const uint32_t k = in ? keys[i] : 0, p = in ? pos[i] : 0, d = (k >> shift) & 255;
#pragma unroll
    for (int w = 0; w < 4; ++w) have[w][tid] = 0;
    __syncthreads();
    uint64_t same = __ballot(in);                                // lanes of this wavefront with the same digit
#pragma unroll
    for (int b = 0; b < kDigit; ++b) {
      const uint64_t m = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? m : ~m;
    }
    const uint32_t before = __popcll(same & ((1ull << lane) - 1));
    if (in && before == 0) have[wave][d] = (uint32_t)__popcll(same);
    __syncthreads();
    if (in) {
      uint32_t at = next[d] + before;
      for (int w = 0; w < wave; ++w) at += have[w][d];
      okeys[at] = k;
      opos[at] = p;
    }
    __syncthreads();
    next[tid] += have[0][tid] + have[1][tid] + have[2][tid] + have[3][tid];
    __syncthreads();
  }
}

// A block has 256 >> shift runs, of 1 << shift threads with eight columns each (wide rows: blockIdx.y).  16384 tokens of 2048 columns, 32000 rows:
// 36 us for 172 MB, a copy's rate.  Zeros only for the rows that no token has, written beside the sums, move 105 MB less, but counting has nothing
// beside it then: 18 and 65 us instead of 45 (with the zeros) and 36.
template <typename E>
__global__ __launch_bounds__(256) void embed_sum_k(const uint32_t* __restrict__ skeys, const uint32_t* __restrict__ spos, int n, int width, int shift,
                                                   float scale, const E* __restrict__ dy, int64_t lddy, float* __restrict__ dtable,
                                                   int64_t lddt, int accumulate, float* __restrict__ part) {
  constexpr int U = sizeof(E) == 2 ? 16 : 8, K = kRun + 2;
  extern __shared__ uint32_t held[];                             // per run: the id in front of it, its own, the one behind; then its tokens
  const int tid = threadIdx.x, R = 256 >> shift, run0 = blockIdx.x * R;
  uint32_t* const where = held + R * K;
  for (int t = tid; t < R * K; t += 256) {
    const int j = (run0 + t / K) * kRun + t % K - 1;
    held[t] = j >= 0 && j < n ? skeys[j] : FTP_NO_ID;
  }
  for (int t = tid; t < R * kRun; t += 256) {
    const int j = run0 * kRun + t;
    where[t] = j < n ? spos[j] : 0;
  }
  __syncthreads();
  const int sub = tid >> shift, run = run0 + sub, cnt = n - run * kRun < kRun ? n - run * kRun : kRun;
  const uint32_t *key = held + sub * K, *pos = where + sub * kRun;
  const int c = (blockIdx.y * 256 + (tid & ((1 << shift) - 1))) * 8, left = width - c;
  if (left <= 0) return;
  const bool whole = left >= 8;
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = 0.f;
  int start = 0;
  for (int q = 0; q < cnt; q += U) {
    if (key[q + 1] == FTP_NO_ID) return;                         // ids of no row come last
    u4v_t raw[U][sizeof(E) == 2 ? 1 : 2];
    if (whole) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = q + u < cnt && key[q + u + 1] != FTP_NO_ID;
        const E* const p = dy + (int64_t)(in ? pos[q + u] : pos[q]) * lddy + c;
        raw[u][0] = tk_ld16<E>(p);
        if (sizeof(E) == 4) raw[u][sizeof(E) == 4] = tk_ld16<E>(p + 4);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (q + u >= cnt) break;
      const uint32_t k = key[q + u + 1];
      if (k == FTP_NO_ID) break;
      float v[8];
      if (whole) {
        if constexpr (sizeof(E) == 2) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(raw[u][0][i] << 16);
            v[2 * i + 1] = __uint_as_float(raw[u][0][i] & 0xffff0000u);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(raw[u][0][i]); v[i + 4] = __uint_as_float(raw[u][1][i]); }
        }
      } else {
        tk_load8<E>(dy + (int64_t)pos[q + u] * lddy + c, left, v);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += v[e];
      if (q + u + 1 < cnt && key[q + u + 2] == k) continue;
      // the id's last token in this run
      const bool before = start == 0 && key[0] == k, behind = q + u + 1 == cnt && key[q + u + 2] == k;
      if (before || behind) {
        // [run][0]: of an id that began in an earlier run; [run][1]: of one that begins here and goes on
        tk_store8<float>(part + ((int64_t)run * 2 + (before ? 0 : 1)) * width + c, left, s);
      } else {
        float* const d = dtable + (int64_t)k * lddt + c;
        float o[8];
        if (accumulate) tk_load8<float>(d, left, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = accumulate ? fmaf(s[e], scale, o[e]) : s[e] * scale;
        tk_store8<float>(d, left, o);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = 0.f;
      start = q + u + 1;
    }
  }
}
// ids with tokens in several runs: the run in which one begins adds up its parts, sixteen rows in flight (16384 tokens, ids by a power law: 11 us,
// the chain of the most frequent one)
__global__ __launch_bounds__(256) void embed_join_k(const uint32_t* __restrict__ skeys, int n, int width, float scale, float* __restrict__ dtable,
                                                    int64_t lddt, int accumulate, const float* __restrict__ part) {
  const int run = blockIdx.x, last = (run + 1) * kRun - 1;
  if (last + 1 >= n) return;
  const uint32_t k = skeys[last];
  if (k == FTP_NO_ID || skeys[last + 1] != k || (run > 0 && skeys[run * kRun] == k && skeys[run * kRun - 1] == k)) return;
  // the runs that it goes on in: those that begin with it, one behind the other (all lanes are here)
  int cnt = 0;
  for (;;) {
    const int64_t at = (int64_t)(run + 1 + cnt + (int)(threadIdx.x & 63)) * kRun;
    const uint64_t same = __ballot(at < n && skeys[at < n ? at : 0] == k);
    cnt += ~same ? __builtin_ctzll(~same) : 64;
    if (~same) break;
  }
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * 8, left = width - c;
  if (left <= 0) return;
  float s[8], v[8];
  tk_load8<float>(part + ((int64_t)run * 2 + 1) * width + c, left, s);
  const float* q = part + (int64_t)(run + 1) * 2 * width + c;
  int r = 0;
  for (; r + 16 <= cnt; r += 16, q += 32 * (int64_t)width) {
    float t[16][8];
#pragma unroll
    for (int u = 0; u < 16; ++u) tk_load8<float>(q + u * 2 * (int64_t)width, left, t[u]);
#pragma unroll
    for (int u = 0; u < 16; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += t[u][e];
  }
  for (; r < cnt; ++r, q += 2 * (int64_t)width) {
    tk_load8<float>(q, left, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += v[e];
  }
  float* const d = dtable + (int64_t)k * lddt + c;
  if (accumulate) tk_load8<float>(d, left, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = accumulate ? fmaf(s[e], scale, v[e]) : s[e] * scale;
  tk_store8<float>(d, left, v);
}
void tk_fill(hipStream_t st, void* p, int64_t rows, int64_t row_bytes, int64_t ld_bytes) {
  long_rows(rows, row_bytes, ld_bytes);
  by_rows(rows, (row_bytes + 15) / 16, [&](int64_t r, int m) {
    hipLaunchKernelGGL(tk_fill_k, dim3(blocks_of((int64_t)m * ((row_bytes + 15) / 16), 8192)), dim3(256), 0, st, (char*)p + r * ld_bytes,
                       (uint32_t)m, row_bytes, ld_bytes);
  });
}

static inline size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
size_t tk_embed_bwd_bytes(int64_t n, int vocab, int width) {
  const size_t runs = (n + kRun - 1) / kRun, tiles = (n + kTile - 1) / kTile;
  (void)vocab;
  return 4 * up256((size_t)n * 4) + up256(tiles * 256 * 4) + up256(runs * 2 * width * 4);
}
void tk_embed_bwd(int dt, hipStream_t st, const void* ids, int ids64, int64_t n64, int vocab, int width, float scale, int64_t pad_id,
                  const void* dy, int64_t lddy, float* dtable, int64_t lddt, int accumulate, void* ws) {
  const int es = dt == 1 ? 2 : 4, n = (int)n64;
  KScope ks(st, "tok_embed_bwd", (double)n * width * es + (accumulate ? 0.0 : (double)vocab * width * 4) + 4.0 * n, 2.0 * n * width, n, vocab, width);
  // counting among chunks of the tokens, and merging these, or passes over the ids' digits
  const bool rank = n > 0 && n <= kChunksMost;
  int64_t zr = vocab, zb = (int64_t)width * 4, zl = lddt * 4;
  long_rows(zr, zb, zl);
  const bool beside = rank && zr * ((zb + 15) / 16) < ((int64_t)1 << 31);       // the zeros are written beside the counting
  if (!accumulate && !beside) tk_fill(st, dtable, vocab, (int64_t)width * 4, lddt * 4);
  if (n == 0) return;
  char* w = (char*)ws;
  uint32_t* buf[4];
  for (auto& b : buf) { b = (uint32_t*)w; w += up256((size_t)n * 4); }
  const int tiles = (n + kTile - 1) / kTile, runs = (n + kRun - 1) / kRun;
  uint32_t* hist = (uint32_t*)w;
  w += up256((size_t)tiles * 256 * 4);
  float* part = (float*)w;
  uint32_t *k0 = buf[0], *p0 = buf[1], *k1 = buf[2], *p1 = buf[3];
  if (rank) {
    const int blocks = (n + 63) / 64;
    const int64_t vecs = accumulate || !beside ? 0 : zr * ((zb + 15) / 16);
    const int fill = (int)std::min<int64_t>((vecs + 1023) / 1024, 2048);
    auto go = [&](auto k, auto* id) {
      hipLaunchKernelGGL(k, dim3(blocks + fill), dim3(1024), 0, st, id, n, vocab, pad_id, k1, p1, blocks, (char*)dtable, (uint32_t)zr, zb, zl);
    };
    if (ids64) go(embed_rank_k<int64_t>, (const int64_t*)ids);
    else go(embed_rank_k<int32_t>, (const int32_t*)ids);
    if (n > kChunk) {
      hipLaunchKernelGGL(embed_merge_k, dim3((n + 255) / 256), dim3(256), 0, st, k1, p1, n, k0, p0);
      std::swap(k0, k1);
      std::swap(p0, p1);
    }
    k0 = k1; p0 = p1;
  } else {
    if (ids64) hipLaunchKernelGGL(embed_keys_k<int64_t>, dim3(blocks_of(n, 4096)), dim3(256), 0, st, (const int64_t*)ids, n, vocab, pad_id, k0, p0);
    else hipLaunchKernelGGL(embed_keys_k<int32_t>, dim3(blocks_of(n, 4096)), dim3(256), 0, st, (const int32_t*)ids, n, vocab, pad_id, k0, p0);
    // the digits of ids below vocab; no id (all ones) stays behind them because its digits are the largest, where one more bit than the largest id's counts
    int bits = 1;
    while (bits < 32 && ((uint64_t)vocab >> bits)) ++bits;
    for (int shift = 0; shift < bits; shift += kDigit) {
      hipLaunchKernelGGL(embed_count_k, dim3(tiles), dim3(256), 0, st, k0, n, shift, hist, tiles);
      hipLaunchKernelGGL(embed_scan_k, dim3(1), dim3(1024), 0, st, hist, tiles * 256);
      hipLaunchKernelGGL(embed_place_k, dim3(tiles), dim3(256), 0, st, k0, p0, n, shift, hist, tiles, k1, p1);
      std::swap(k0, k1);
      std::swap(p0, p1);
    }
  }
  int shift = 0;
  while (shift < 8 && (8 << shift) < width) ++shift;
  const int per = 256 >> shift, slabs = (width + 2047) / 2048, lds = per * (2 * kRun + 2) * 4;
  const dim3 g((runs + per - 1) / per, slabs);
  if (dt == 1) hipLaunchKernelGGL(embed_sum_k<bf16_t>, g, dim3(256), lds, st, k0, p0, n, width, shift, scale, (const bf16_t*)dy, lddy, dtable, lddt, accumulate, part);
  else hipLaunchKernelGGL(embed_sum_k<float>, g, dim3(256), lds, st, k0, p0, n, width, shift, scale, (const float*)dy, lddy, dtable, lddt, accumulate, part);
  // (the last run has none behind it to add; all 2^26 of 2^30 rows would be more threads than a launch takes)
  if (runs > 1) hipLaunchKernelGGL(embed_join_k, dim3(runs - 1, slabs), dim3(std::max(64, 1 << shift)), 0, st, k0, n, width, scale, dtable, lddt, accumulate, part);
}

// ---------------------------------------------------------------- activations in 8 bits
// Four threads have a group of 32 columns, eight each: the group's largest magnitude goes between them without LDS.  Memory: 16384 x 8192 bfloat16,
// 407 MB either way, packed in 78 us (5.2 TB/s), unpacked in 68 (6.0).
template <typename E>
__global__ __launch_bounds__(256) void act8_pack_k(const E* __restrict__ x, int64_t ldx, int rows, int N, uint8_t* __restrict__ q, int64_t ldq,
                                                   uint8_t* __restrict__ s, int64_t lds) {
  const uint32_t per = (uint32_t)(N + 31) / 32 * 4, all = (uint32_t)rows * per;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) {     // all is a multiple of 4: a group's threads stay together
    const uint32_t r = i / per, c = (i - r * per) * 8;
    const int left = N - (int)c;
    float v[8];
    tk_load8<E>(x + (int64_t)r * ldx + c, left, v);
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, act8_mag(v[e]));
    top = fmaxf(top, dpp_move<0xB1>(top));
    top = fmaxf(top, dpp_move<0x4E>(top));
    const uint32_t b = act8_scale(top);
    const float inv = act8_inv(b);
    const uint32_t lo = act8_pack4(v, inv), hi = act8_pack4(v + 4, inv);
    uint8_t* const p = q + (int64_t)r * ldq + c;
    if (left >= 8) {
      *reinterpret_cast<TkAt<1>::v8*>(p) = u2v_t{lo, hi};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) p[e] = (uint8_t)((e < 4 ? lo : hi) >> (8 * (e & 3)));
    }
    if ((c & 31) == 0) s[(int64_t)r * lds + c / 32] = (uint8_t)b;
  }
}
// pad_to >= N: columns from N to there become zero
template <typename E>
__global__ __launch_bounds__(256) void act8_unpack_k(const uint8_t* __restrict__ q, int64_t ldq, const uint8_t* __restrict__ s, int64_t lds,
                                                     int rows, int N, int pad_to, E* __restrict__ y, int64_t ldy) {
  const uint32_t per = (uint32_t)(pad_to + 7) / 8, all = (uint32_t)rows * per;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) {
    const uint32_t r = i / per, c = (i - r * per) * 8;
    const int left = N - (int)c;
    const uint8_t* const p = q + (int64_t)r * ldq + c;
    uint32_t lo = 0, hi = 0;
    if (left >= 8) {
      const u2v_t t = *reinterpret_cast<const TkAt<1>::v8*>(p);
      lo = t[0]; hi = t[1];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) (e < 4 ? lo : hi) |= (uint32_t)p[e] << (8 * (e & 3));
    }
    const float mul = left > 0 ? act8_mul(s[(int64_t)r * lds + c / 32]) : 0.f;
    float v[8];
    act8_unpack4(lo, mul, v);
    act8_unpack4(hi, mul, v + 4);
    tk_store8<E>(y + (int64_t)r * ldy + c, pad_to - (int)c, v);
  }
}
void tk_act8_pack(int dt, hipStream_t st, const void* x, int64_t ldx, int64_t M, int N, uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds) {
  KScope ks(st, "tok_act8_pack", (double)M * N * ((dt == 1 ? 2 : 4) + 1 + 1.0 / 32), 2.0 * M * N, M, N);
  const int64_t per = (int64_t)act8_groups(N) * 4;
  by_rows(M, per, [&](int64_t r, int m) {
    const unsigned b = blocks_of(m * per, 1 << 20);
    if (dt == 1) hipLaunchKernelGGL(act8_pack_k<bf16_t>, dim3(b), dim3(256), 0, st, (const bf16_t*)x + r * ldx, ldx, m, N, q + r * ldq, ldq, s + r * lds, lds);
    else hipLaunchKernelGGL(act8_pack_k<float>, dim3(b), dim3(256), 0, st, (const float*)x + r * ldx, ldx, m, N, q + r * ldq, ldq, s + r * lds, lds);
  });
}
void tk_act8_unpack(int dt, hipStream_t st, const uint8_t* q, int64_t ldq, const uint8_t* s, int64_t lds, int64_t M, int N, int pad_to,
                    void* y, int64_t ldy) {
  KScope ks(st, "tok_act8_unpack", (double)M * N * ((dt == 1 ? 2 : 4) + 1 + 1.0 / 32), 1.0 * M * N, M, N);
  const int64_t per = (pad_to + 7) / 8;
  by_rows(M, per, [&](int64_t r, int m) {
    const unsigned b = blocks_of(m * per, 1 << 20);
    if (dt == 1) hipLaunchKernelGGL(act8_unpack_k<bf16_t>, dim3(b), dim3(256), 0, st, q + r * ldq, ldq, s + r * lds, lds, m, N, pad_to, (bf16_t*)y + r * ldy, ldy);
    else hipLaunchKernelGGL(act8_unpack_k<float>, dim3(b), dim3(256), 0, st, q + r * ldq, ldq, s + r * lds, lds, m, N, pad_to, (float*)y + r * ldy, ldy);
  });
}

// ---------------------------------------------------------------- linear layers
// All copies of a call go as one launch, blockIdx.y a matrix: 1000 x 1001, fp32, takes 5 us, of which the bytes are 2.
struct AlignGroup { TkCopy j[kCopies]; };
template <typename E>
__global__ __launch_bounds__(256) void tk_align_k(AlignGroup g) {
  constexpr int V = 16 / sizeof(E);
  const TkCopy& j = g.j[blockIdx.y];
  const uint32_t per = (uint32_t)(j.ldy / V), all = (uint32_t)j.rows * per;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) {
    const uint32_t r = i / per, c = (i - r * per) * V;
    const E* const p = (const E*)j.x + (int64_t)r * j.ldx + c;
    const int left = j.cols - (int)c;
    u4v_t t = {0, 0, 0, 0};
    if (left >= V) {
      t = tk_ld16<E>(p);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        uint32_t b = 0;
        if (e < left) b = sizeof(E) == 2 ? (uint32_t)*reinterpret_cast<const uint16_t*>(p + e) : *reinterpret_cast<const uint32_t*>(p + e);
        if (sizeof(E) == 4) t[e & 3] = b;
        else t[e / 2] |= b << (16 * (e & 1));
      }
    }
    *reinterpret_cast<u4v_t*>((E*)j.y + (int64_t)r * j.ldy + c) = t;
  }
}
void tk_align(int dt, hipStream_t st, const TkCopy* jobs, int n) {
  const int es = dt == 1 ? 2 : 4;
  double elements = 0;
  for (int i = 0; i < n; ++i) elements += (double)jobs[i].rows * jobs[i].cols;
  KScope ks(st, "tok_align", 2.0 * elements * es, 0, n, jobs[0].rows, jobs[0].cols);
  auto go = [&](const AlignGroup& g, int m, int64_t most) {
    const dim3 b(blocks_of(most, 1 << 20), m);
    if (dt == 1) hipLaunchKernelGGL(tk_align_k<bf16_t>, b, dim3(256), 0, st, g);
    else hipLaunchKernelGGL(tk_align_k<float>, b, dim3(256), 0, st, g);
  };
  AlignGroup g{};
  int m = 0;
  int64_t most = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t per = jobs[i].ldy * es / 16, all = jobs[i].rows * per;
    if (all <= (int64_t)1 << 30) {
      g.j[m++] = jobs[i];
      most = std::max(most, all);
      continue;
    }
    by_rows(jobs[i].rows, per, [&](int64_t r, int rows) {
      AlignGroup one{};
      one.j[0] = jobs[i];
      one.j[0].x = (const char*)jobs[i].x + r * jobs[i].ldx * es;
      one.j[0].y = (char*)jobs[i].y + r * jobs[i].ldy * es;
      one.j[0].rows = rows;
      go(one, 1, rows * per);
    });
  }
  if (m) go(g, m, most);
}

// dz = dy * act'(z) and its column sums.  A block has 256 columns (64 threads of four) of a chunk of rows, four threads to a column, each with four
// rows in flight; the sums are of dz before it is rounded.  Memory where there are enough rows and columns (8192 x 4096 bfloat16 36 us, 5.6 TB/s), latency
// where not: 22715 x 64 9.3 us (two rows in flight 12.1, one 23), 1000 x 777 fp32 4.2 and its join below 4.6, of which the bytes are 2.  32768 x 2048 84, two rows 80.
static int dz_rows(int M) { return std::max(16, (M + 255) / 256); }
int tk_dz_chunks(int M) { return M > 0 ? (M + dz_rows(M) - 1) / dz_rows(M) : 0; }
// four columns at any alignment, or (not whole) the `left` that there are; as stored, so that a row's wait is not the next one's
template <typename E, bool WHOLE>
__device__ __forceinline__ typename Tg4<E>::raw at4(const E* p, int left) {
  typename Tg4<E>::raw r;
  if constexpr (!WHOLE) return get_raw4<E>(p, 0, 0, 0, left, false);
  else if constexpr (sizeof(E) == 2) { const u2v_t t = *reinterpret_cast<const TkAt<2>::v8*>(p); __builtin_memcpy(&r, &t, 8); }
  else { const u4v_t t = tk_ld16<E>(p); __builtin_memcpy(&r, &t, 16); }
  return r;
}
template <typename E>
__global__ __launch_bounds__(256) void tk_dz_k(const E* __restrict__ dy, int64_t lddy, const E* __restrict__ z, int64_t ldz, int act, int M, int N,
                                               int per, E* __restrict__ dz, int64_t ldd, float* __restrict__ part) {
  constexpr int U = 4;
  __shared__ float4 sum[4][64];
  const int lane = threadIdx.x & 63, ty = threadIdx.x >> 6, n = (blockIdx.x * 64 + lane) * 4;
  const int r0 = blockIdx.y * per, r1 = r0 + per < M ? r0 + per : M;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  const int wide = dz ? (int)ldd : N;
  const auto walk = [&](auto whole) __attribute__((always_inline)) {
    for (int r = r0 + ty; r < r1; r += 4 * U) {
      typename Tg4<E>::raw y[U], x[U];
      float v[4 * U], t[4 * U], a[4 * U], d[4 * U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t m = r + 4 * u < r1 ? r + 4 * u : r;
        y[u] = at4<E, whole.value>(dy + m * lddy + n, N - n);
        if (act != TACT_NONE) x[u] = at4<E, whole.value>(z + m * ldz + n, N - n);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) open4<E>(y[u], v + 4 * u);
      if (act != TACT_NONE) {
#pragma unroll
        for (int u = 0; u < U; ++u) open4<E>(x[u], t + 4 * u);
        tact_gradn<4 * U>(t, a, d, act);
#pragma unroll
        for (int e = 0; e < 4 * U; ++e) v[e] *= d[e];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (r + 4 * u >= r1) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (!whole.value && n + e >= N) v[4 * u + e] = 0.f;    // pad columns
          s[e] += v[4 * u + e];
        }
        if (dz) put4<E>(dz, ldd, r + 4 * u, n, (int)ldd, true, v + 4 * u);
      }
    }
  };
  if (N - n >= 4) walk(std::true_type());
  else if (n < wide) walk(std::false_type());
  if (!part) return;
  sum[ty][lane] = make_float4(s[0], s[1], s[2], s[3]);
  __syncthreads();
  if (ty == 0) {
    const float4 a = sum[0][lane], b = sum[1][lane], c = sum[2][lane], d = sum[3][lane];
    const float t[4] = {(a.x + b.x) + (c.x + d.x), (a.y + b.y) + (c.y + d.y), (a.z + b.z) + (c.z + d.z), (a.w + b.w) + (c.w + d.w)};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < N) part[(int64_t)blockIdx.y * N + n + e] = t[e];
  }
}
void tk_dz(int dt, hipStream_t st, const void* dy, int64_t lddy, const void* z, int64_t ldz, int act, int M, int N, void* dz,
           int64_t ldd, float* part) {
  const int es = dt == 1 ? 2 : 4;
  KScope ks(st, "tok_dz", (double)M * N * es * ((act != TACT_NONE) + 1 + (dz != nullptr)), 4.0 * M * N, M, N);
  const dim3 g((std::max<int64_t>(N, dz ? ldd : 0) + 255) / 256, tk_dz_chunks(M));
  if (dt == 1) hipLaunchKernelGGL(tk_dz_k<bf16_t>, g, dim3(256), 0, st, (const bf16_t*)dy, lddy, (const bf16_t*)z, ldz, act, M, N, dz_rows(M), (bf16_t*)dz, ldd, part);
  else hipLaunchKernelGGL(tk_dz_k<float>, g, dim3(256), 0, st, (const float*)dy, lddy, (const float*)z, ldz, act, M, N, dz_rows(M), (float*)dz, ldd, part);
}
// 64 columns a block, four threads to a column
__global__ __launch_bounds__(256) void tk_colsum_join_k(const float* __restrict__ part, int chunks, int N, void* __restrict__ db, int bf16, int accumulate) {
  __shared__ float sum[4][64];
  const int lane = threadIdx.x & 63, ty = threadIdx.x >> 6, n = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (n < N) {
#pragma unroll 8
    for (int c = ty; c < chunks; c += 4) s += part[(int64_t)c * N + n];
  }
  sum[ty][lane] = s;
  __syncthreads();
  if (ty || n >= N) return;
  s = (sum[0][lane] + sum[1][lane]) + (sum[2][lane] + sum[3][lane]);
  if (bf16) ((bf16_t*)db)[n] = f32_to_bf16(s);
  else ((float*)db)[n] = accumulate ? ((float*)db)[n] + s : s;
}
void tk_colsum_join(hipStream_t st, const float* part, int chunks, int N, void* db, int out_dt, int accumulate) {
  KScope ks(st, "tok_bias_grad", 4.0 * chunks * N, (double)chunks * N, chunks, N);
  hipLaunchKernelGGL(tk_colsum_join_k, dim3((N + 63) / 64), dim3(256), 0, st, part, chunks, N, db, out_dt, accumulate);
}

}  // namespace ftp
