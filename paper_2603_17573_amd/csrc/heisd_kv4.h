// A cache of keys and values held in 4 bits, in blocks of tokens: writing rows into it, reading them back, and attention over
// it.
//
// Format.  A row of head_dim values of one head is cut into groups of 32.  A group is sixteen bytes of 4-bit floats (sign, two
// bits of exponent, one of mantissa: 0 .5 1 1.5 2 3 4 6; in a byte the low half comes first) times 2^(e - 127), one byte e: the
// smallest e >= 1 for which the group's largest magnitude is at most 6 * 2^(e - 127), so nothing saturates.  e = 255 marks a
// group that held a value that is not finite and stands for NaN in all of it.  These are the 4-bit floats and power-of-two
// scales that the conversion instructions of this chip take, so a group becomes bf16 (exactly) with one instruction per two values.
//
// Layout.  One block of one head is a cell of bytes, [n_blocks][kv_heads] of them:
//   key codes        [token][head_dim / 2]
//   value codes      [token / 4][16][token % 4][head_dim / 32]
//   key exponents    [token][head_dim / 32]
//   value exponents  [token / 4][head_dim / 32][token % 4]
// A tile of 16 tokens is what a matrix instruction takes.  Keys are its first operand with tokens as rows: lane l holds token
// l % 16 and a quarter of the head, contiguous.  Values are the first operand with channels as rows and tokens as the summed
// index: lane l holds the four tokens 4 * (l / 16) + 0..3 and head_dim / 16 channels, which this order of bytes makes
// contiguous.  So the part of a tile that a lane uses lies together, a tile's codes are 1 KB (heads of 128) that follow each other, and the attention
// brings them into LDS by direct transfers of 16 bytes a lane, from where every lane reads its part at once.
#pragma once
#include <type_traits>

#include "heisd_common.h"
#include "heisd_paged.h"

namespace heisd {

constexpr int kKv4Tile = 16;
constexpr uint32_t kKv4NotFinite = 253;             // from this exponent on a value may be 2^128 or more, which bf16 does not hold

struct Kv4Cache {
  uint8_t *pool;
  int n_blocks, block_size, block_shift, kv_heads;  // block_size is a power of two, 16 or more
  long long cell;                                   // bytes of one block of one head
  __device__ __forceinline__ uint8_t *at(int id, int head) const { return pool + ((long long)id * kv_heads + head) * cell; }
};
__host__ __device__ constexpr long long kv4_cell_bytes(int block_size, int head_dim) {
  return (long long)block_size * (head_dim + head_dim / 16);
}
template <int HD>
struct Kv4Offsets {                                 // of token t of a cell of bs tokens
  static __device__ __forceinline__ int v_codes(int bs) { return bs * (HD / 2); }
  static __device__ __forceinline__ int k_exp(int bs) { return bs * HD; }
  static __device__ __forceinline__ int v_exp(int bs) { return bs * HD + bs * (HD / 32); }
};

// Requests: which blocks hold the tokens of each, how many tokens there are, which packed rows are theirs.
struct PagedBatch {
  const int32_t *table, *seq_len, *cu_rows;
  int batch, max_blocks, rows;
};

// ---- rows into the cache ------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppXor1, 0xf, 0xf, true));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppXor2, 0xf, 0xf, true));
}

// Four lanes share a group of 32 values, 8 each (16 bytes per access).  gridDim.y: keys and values.  Reads every row once and
// writes 17/64 of the bytes of a bf16 row; bound by memory (20963 rows of 8 heads of 128: 107 MB in 20 us).  VEC: rows are aligned
// for wide loads.
template <typename T, int HD, bool VEC>
__global__ __launch_bounds__(256) void kv4_append(Kv4Cache c, HeadRows<const T> k, HeadRows<const T> v, const int32_t *slot,
                                                  int rows, int per_group, FastDiv by_row) {
  constexpr int LH = HD / 8;                        // lanes per head
  const bool is_v = blockIdx.y;
  const uint32_t per_row = (uint32_t)c.kv_heads * LH;
  const int r0 = blockIdx.x * per_group, nr = min(per_group, rows - r0);
  for (uint32_t u = threadIdx.x; u < nr * per_row; u += 256) {
    const uint32_t r = by_row.of(u), w = u - r * per_row;
    const int h = w / LH, j = w % LH;
    const int s = slot[r0 + r];
    if (s < 0) continue;
    const int id = s >> c.block_shift, t = s & (c.block_size - 1);
    if (id >= c.n_blocks) continue;
    const T *x = (is_v ? v : k).at(r0 + r, h) + j * 8;
    float f[8];
    if constexpr (VEC) {
      if constexpr (sizeof(T) == 2) load_vec<T, 8>(x, f);
      else {
        load_vec<T, 4>(x, f);
        load_vec<T, 4>(x + 4, f + 4);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = (float)x[i];
    }
    uint32_t most = 0;                              // as bits: infinity and NaN are larger than every number
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(f[i]) & 0x7FFFFFFFu);
    most = quad_max(most);
    const bool finite = most < 0x7F800000u;
    const int e = finite ? max((int)(most >> 23) - 2 + ((most & 0x7FFFFFu) > 0x400000u), 1) : 255;
    const float down = __uint_as_float((uint32_t)(254 - min(e, 253)) << 23);        // 2^(127 - e), exact
    uint32_t code = 0;
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[0] * down, f[1] * down, 1.f, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[2] * down, f[3] * down, 1.f, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[4] * down, f[5] * down, 1.f, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[6] * down, f[7] * down, 1.f, 3);
    if (!finite) code = 0;
    uint8_t *cell = c.at(id, h);
    if (!is_v) {
      *reinterpret_cast<uint32_t *>(cell + t * (HD / 2) + j * 4) = code;
      if (j % 4 == 0) cell[Kv4Offsets<HD>::k_exp(c.block_size) + t * (HD / 32) + j / 4] = (uint8_t)e;
    } else {
      uint8_t *to = cell + Kv4Offsets<HD>::v_codes(c.block_size) + (t / 4) * (2 * HD);
      if constexpr (HD == 128) *reinterpret_cast<uint32_t *>(to + j * 16 + (t % 4) * 4) = code;
      else {
        *reinterpret_cast<uint16_t *>(to + 2 * j * 8 + (t % 4) * 2) = (uint16_t)code;
        *reinterpret_cast<uint16_t *>(to + (2 * j + 1) * 8 + (t % 4) * 2) = (uint16_t)(code >> 16);
      }
      if (j % 4 == 0) cell[Kv4Offsets<HD>::v_exp(c.block_size) + ((t / 4) * (HD / 32) + j / 4) * 4 + t % 4] = (uint8_t)e;
    }
  }
}

// ---- cached rows back out -------------------------------------------------------------------------------------------

__device__ __forceinline__ float kv4_scale(uint32_t e) {
  return e == 255 ? __uint_as_float(0x7FC00000u) : e == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(e << 23);
}

// Rows and heads that a workgroup reads back; a lane writes 16 bytes, so that a wave's store is whole lines in either width.
template <typename T>
constexpr int kGatherRows = 32 / sizeof(T);
constexpr int kGatherHeads = 4;

// Some packed rows and heads per workgroup, head by head: the rows of a block that follow each other lie together in the cache.
// A thread requests its values of all heads before it converts the first.  Rows of a block that the pool does not have are
// zero.  Bound by memory, most of it the rows that are written: 4280 rows of 32 heads of 128 into fp32 (159 MB) take 26 us.  One group of all heads
// per sixteen rows, stores of half lines in fp32 and ordinary ones took 55.
template <typename T, int HD, bool VEC>
__global__ __launch_bounds__(256) void kv4_gather(Kv4Cache c, PagedBatch b, const int32_t *cu_seq, int out_rows,
                                                  HeadRows<T> k, HeadRows<T> v) {
  constexpr int E = 16 / sizeof(T), LH = HD / E, ROWS = kGatherRows<T>, PER = 256 / (ROWS * LH);   // values per lane, lanes per row and head, heads at a time
  __shared__ int where[ROWS];                       // slot, -1: no such token (a zero row), -2: nobody's row
  const int r0 = blockIdx.x * ROWS, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const bool is_v = blockIdx.z;
  for (int i = wave; i < ROWS; i += 4) {
    int w = -2;
    if (r0 + i < out_rows) {
      const int q = wave_search(b.batch, r0 + i, [&](int n) { return (long long)cu_seq[n]; });
      const Span s = packed_span(cu_seq, q, out_rows);
      const int t = r0 + i - s.begin;
      if (t >= 0 && t < s.count && t < b.seq_len[q]) {
        const int blk = t >> c.block_shift;
        const int id = blk < b.max_blocks ? b.table[(long long)q * b.max_blocks + blk] : -1;
        w = id >= 0 && id < c.n_blocks ? id * c.block_size + (t & (c.block_size - 1)) : -1;
      }
    }
    if (lane == 0) where[i] = w;
  }
  __syncthreads();
  const int j = threadIdx.x % LH, i = threadIdx.x / LH % ROWS, h0 = blockIdx.y * kGatherHeads + threadIdx.x / (LH * ROWS);
  const int s = where[i];
  if (s == -2) return;
  const int id = max(s, 0) >> c.block_shift, t = s & (c.block_size - 1);
  uint32_t code[kGatherHeads / PER], e[kGatherHeads / PER];
#pragma unroll
  for (int n = 0; n < kGatherHeads / PER; ++n) {
    code[n] = e[n] = 0;
    const int h = h0 + n * PER;
    if (s < 0 || h >= c.kv_heads) continue;
    const uint8_t *cell = c.at(id, h);
    const int d = j * E;                            // the lane's first channel
    if (!is_v) {
      const uint8_t *from = cell + t * (HD / 2) + d / 2;
      code[n] = E == 8 ? *reinterpret_cast<const uint32_t *>(from) : *reinterpret_cast<const uint16_t *>(from);
      e[n] = cell[Kv4Offsets<HD>::k_exp(c.block_size) + t * (HD / 32) + d / 32];
    } else {
      constexpr int PIECE = HD / 16;                // channels that lie together
      const uint8_t *from = cell + Kv4Offsets<HD>::v_codes(c.block_size) + (t / 4) * (2 * HD) + d / PIECE * (2 * PIECE) + (t % 4) * (PIECE / 2) + d % PIECE / 2;
      if constexpr (E <= PIECE) code[n] = E == 8 ? *reinterpret_cast<const uint32_t *>(from) : *reinterpret_cast<const uint16_t *>(from);
      else code[n] = *reinterpret_cast<const uint16_t *>(from) | (uint32_t)*reinterpret_cast<const uint16_t *>(from + 2 * PIECE) << 16;
      e[n] = cell[Kv4Offsets<HD>::v_exp(c.block_size) + ((t / 4) * (HD / 32) + d / 32) * 4 + t % 4];
    }
  }
#pragma unroll
  for (int n = 0; n < kGatherHeads / PER; ++n) {
    const int h = h0 + n * PER;
    if (h >= c.kv_heads) return;
    const float scale = kv4_scale(e[n]);
    float f[8];
    const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[n], 1.f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[n], 1.f, 1);
    f[0] = p0[0] * scale, f[1] = p0[1] * scale, f[2] = p1[0] * scale, f[3] = p1[1] * scale;
    if constexpr (E == 8) {
      const auto p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[n], 1.f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[n], 1.f, 3);
      f[4] = p2[0] * scale, f[5] = p2[1] * scale, f[6] = p3[0] * scale, f[7] = p3[1] * scale;
    }
    T *y = (is_v ? v : k).at(r0 + i, h) + j * E;
    if constexpr (VEC) store_vec_once<T, E>(y, f);
    else {
#pragma unroll
      for (int x = 0; x < E; ++x) y[x] = (T)f[x];
    }
  }
}

// ---- attention ------------------------------------------------------------------------------------------------------

// What a lane holds of two tiles of 16 tokens.
template <int HD>
struct Kv4Pair {
  static constexpr int W = HD / 32;                 // dwords of codes per lane and tile
  uint32_t kc[2][W], vc[2][W];
  uint32_t ke[2], ve[2];                            // the lane's key exponent; the exponents of its four value tokens
};
// Where two tiles lie in LDS: key codes of both, value codes of both, then 64 bytes each of key exponents and of value exponents.  With heads of 128 the
// pieces of a tile's key codes are in the order of the lanes that read them.
// Two pairs are on their way per wave, none of them in registers (a pair held there while the next was fetched: 66 us against 59.5 with 64
// long contexts).  What bounds the kernel then is memory: 246 MB in 50 us when most of them are in the last cache, 57 when none is.
constexpr int kKv4Ring = 2;
template <int HD>
struct Kv4Slot {
  static constexpr int TILE = 16 * HD / 2, V = 2 * TILE, EXP = 4 * TILE, BYTES = EXP + 256;
  static constexpr int TRANSFERS = (HD == 128 ? 4 : 2) + 1;
};

struct Kv4Attend {
  float scale_log2;                                 // magnitude of the softmax scale times log2(e)
  bool flip;                                        // the scale is negative
  int group, q_heads, max_seq, cols;                // cols: columns a workgroup takes (16 or 32)
  float *part, *part_ml;                            // sums of unfinished segments [2 * workgroups][cols][HD], their maxima and sums [..][cols][2]
  float *lse;
};

// Work is counted in units: 128 tokens (a pair of tiles for each wave) of one request, key head and group of columns - a segment is all
// units of such a three.  Every workgroup takes an equal run of the units of the whole call, whatever the requests' lengths are.
// A workgroup per chunk of 1024 tokens instead: 71 us with 64 contexts of 256 to 8191 tokens, where runs took 62 (the last chunks left most of
// the chip idle, and every chunk begins with three round trips to memory).
constexpr int kKv4Unit = 128;

// Workgroups of 256 threads that the registers of a compute unit hold: two column tiles need more of them, heads of 64 fewer.  Queries of two terms
// fit as those of one do.
__host__ __device__ constexpr int kv4_per_unit(int head_dim, int col_tiles) { return col_tiles == 2 ? 2 : head_dim == 64 ? 4 : 3; }

// What a request asks for: its rows, its tokens, units per segment, units in all.
struct Kv4Request {
  Span rows;
  int seq, units;
  long long work;
};
__device__ __forceinline__ Kv4Request kv4_request(const Kv4Cache &c, const PagedBatch &b, const Kv4Attend &a, int i) {
  Kv4Request r;
  r.rows = packed_span(b.cu_rows, i, b.rows);
  r.seq = b.seq_len[i];
  if (r.seq < 0 || r.seq > a.max_seq || (long long)r.seq > (long long)b.max_blocks * c.block_size) r.seq = 0;
  r.units = max((r.seq + kKv4Unit - 1) / kKv4Unit, 1);          // one even without tokens: somebody writes the zeros
  r.work = (long long)r.units * ((r.rows.count * a.group + a.cols - 1) / a.cols * c.kv_heads);
  return r;
}

__device__ __forceinline__ long long wave_sum64(long long v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ long long lane_value64(long long v, int lane) {
  return (long long)((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)v, lane) |
                     (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32);
}
// Quotient of numbers that are not negative; nearly always they fit 32 bits.
__device__ __forceinline__ long long wave_div(long long a, long long b) {
  return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}
// Units per workgroup of a call of `all` units.
__device__ __forceinline__ long long kv4_run(long long all, int groups) { return max(wave_div(all + groups - 1, groups), 1ll); }

// Online softmax state of a column (one query row of one head): maximum and sum in powers of two.
constexpr float kKv4Lazy = 8.f;                     // the maximum is moved only when it grew by more than this (powers of two)

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A part (a wave's or a workgroup's) with maximum m and sum l saw some token.  A maximum of minus infinity alone does not say that it saw none: where all
// scores are NaN nothing moves the maximum, and the sum is NaN.
__device__ __forceinline__ bool kv4_saw(float m, float l) { return m != -INFINITY || l != 0.f; }
// What such a part's sums are multiplied by where the maximum over all parts is `top`.
__device__ __forceinline__ float kv4_weight(float m, float top) { return m == -INFINITY ? 1.f : exp2_fast(m - top); }

// softmax(q K^T) V over the tokens of segments.  The query rows of the heads that share the key head are the columns of the matrix products (CT tiles of
// 16): scores^T = K q^T (tokens are rows), out^T = V^T p^T.  A lane holds the scores of one column and four tokens of each tile, which are
// its summed indices of the second product, so the probabilities never leave their lane.  Four waves take pairs of tiles in turn,
// each with a running maximum and sum of its own, joined through LDS at the end of a segment; what a workgroup has of a segment that it
// shares with others goes to kv4_join.  A probability enters as a bf16 and a bf16 remainder: one bf16 alone (off by up to 2^-8, and with few
// large probabilities nothing averages that out) made the results of single tokens 1.4 times as inexact as their own rounding does, for 3 % of the
// time (59.9 against 62.1 us with 64 contexts of 256 to 8191 tokens).  TERMS 2: so do the queries (fp16 rows, whose 11 bits a bf16 does not hold).
template <typename T, int HD, int CT, int TERMS>
__global__ __launch_bounds__(256, kv4_per_unit(HD, CT)) void kv4_attend(Kv4Cache c, PagedBatch b, HeadRows<const T> q, HeadRows<T> out, Kv4Attend a) {
  constexpr int W = HD / 32, ND = HD / 16, KJ = HD / 32;        // code dwords, tiles of channels, products per score tile
  constexpr int LD = HD + 4;
  typedef Kv4Slot<HD> Slot;
  constexpr int MINE = kKv4Ring * Slot::BYTES;                  // a wave's part of LDS: its ring, at the end of a segment its sums
  static_assert(MINE >= 16 * LD * 4 && MINE % 16 == 0, "the sums take the ring's place");
  __shared__ __attribute__((aligned(16))) unsigned char s_mine[4][MINE];
  __shared__ float s_m[4][16], s_l[4][16];
  __shared__ long long s_start[4][64];                          // a wave's own: on its way to a later request another may be behind
  __shared__ int4 s_req[4][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int bs = c.block_size;

  // This workgroup's run of units.  Every wave finds it for itself: 64 requests are at hand (in LDS, a request per lane), 64 more while the
  // run lies behind them.
  int first = 0;
  long long end;                                                // units before the end of these 64
  auto requests = [&](long long before) {
    Kv4Request r = kv4_request(c, b, a, min(first + lane, b.batch - 1));
    if (first + lane >= b.batch) r.work = 0;
    long long start = r.work;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const long long t = __shfl_up(start, o);
      if (lane >= o) start += t;
    }
    end = before + lane_value64(start, 63);
    s_start[wave][lane] = start + before - r.work;
    s_req[wave][lane] = make_int4(r.rows.begin, r.rows.count, r.seq, r.units);
  };
  requests(0);
  long long all = end;
  for (int i = 64; i < b.batch; i += 64) all += wave_sum64(i + lane < b.batch ? kv4_request(c, b, a, i + lane).work : 0);
  const long long per = kv4_run(all, gridDim.x), run0 = blockIdx.x * per, run1 = min(run0 + per, all);

  for (long long at = run0; at < run1;) {
    while (at >= end && first + 64 < b.batch) {
      first += 64;
      requests(end);
    }
    if (at >= end) break;                                       // not reached while the lengths stay as they are
    const int local = 63 - __clzll(__ballot(s_start[wave][lane] <= at));      // the last of those that begin here has the work
    const int req = first + local;
    const int4 rq = s_req[wave][local];
    const Span rows{__builtin_amdgcn_readfirstlane(rq.x), __builtin_amdgcn_readfirstlane(rq.y)};
    const int seq = __builtin_amdgcn_readfirstlane(rq.z), units = __builtin_amdgcn_readfirstlane(rq.w);
    const long long in_req = at - lane_value64(s_start[wave][lane], local);
    const int segment = __builtin_amdgcn_readfirstlane((int)wave_div(in_req, units));
    const int u0 = __builtin_amdgcn_readfirstlane((int)(in_req - (long long)segment * units));
    const int u1 = __builtin_amdgcn_readfirstlane((int)min((long long)units, u0 + (run1 - at)));
    const int head = segment % c.kv_heads, col0 = segment / c.kv_heads * (16 * CT);
    const bool whole = u0 == 0 && u1 == units;
    const long long slot = 2 * (long long)blockIdx.x + (at != run0);
    const int n_cols = rows.count * a.group;
    const int t1 = min(seq, u1 * kKv4Unit);

    // the columns' queries and how many tokens each may see
    typename VecOf<T, 8>::type qr[CT][KJ];
    int seen[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const int n = min(col0 + ct * 16 + col, n_cols - 1), i = n / a.group;       // columns past the end: the last again, not stored
      seen[ct] = seq - rows.count + i + 1;
      const T *p = q.at(rows.begin + i, head * a.group + (n - i * a.group)) + quad * (HD / 4);
#pragma unroll
      for (int j = 0; j < KJ; ++j) qr[ct][j] = *reinterpret_cast<const typename VecOf<T, 8>::type *>(p + j * 8);
    }
    f32x4 acc[CT][ND];
    float m[CT], l[CT];
    uint32_t odd = 0;                                           // met a value that is not finite among tokens that not everybody may see
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      m[ct] = -INFINITY;
      l[ct] = 0.f;
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[ct][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    int t0 = 0, my_id = -1;                                     // tokens t0 .. t0 + 4095 are at hand
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)s_mine[wave];
    // Requests pair i: codes 16 bytes a lane, all exponents in one transfer of 4 bytes a lane.
    auto fetch = [&](int i) {
      const uint32_t to = __builtin_amdgcn_readfirstlane(ring + i % kKv4Ring * Slot::BYTES);
      const uint8_t *cell[2];
      int t[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        cell[n] = c.at(max(__builtin_amdgcn_readlane(my_id, 2 * i + n), 0), head);   // a missing block: any block, masked below
        t[n] = (t0 + 32 * (wave + 4 * i) + 16 * n) & (bs - 1);
        if constexpr (HD == 128) {
          lds_dma16_s(cell[n] + t[n] * (HD / 2), col * (HD / 2) + quad * (HD / 8), to + n * Slot::TILE);
          lds_dma16_s(cell[n] + Kv4Offsets<HD>::v_codes(bs) + t[n] * (HD / 2), lane * 16, to + Slot::V + n * Slot::TILE);
        }
      }
      const int n = lane >> 4 & 1;                              // the exponents: both tiles' keys, then both tiles' values
      const uint8_t *e = (n ? cell[1] : cell[0]) + (n ? t[1] : t[0]) * (HD / 32) + lane % (HD / 8) * 4;
      if constexpr (HD == 64) {                                 // a transfer brings both tiles
        const uint8_t *x = (lane >> 5 ? cell[1] : cell[0]) + (lane >> 5 ? t[1] : t[0]) * (HD / 2) + lane % 32 * 16;
        lds_dma16(x, to);
        lds_dma16(x + Kv4Offsets<HD>::v_codes(bs), to + Slot::V);
      }
      lds_dma4(e + (lane >> 5 ? Kv4Offsets<HD>::v_exp(bs) : Kv4Offsets<HD>::k_exp(bs)), to + Slot::EXP);
    };
    auto take = [&](Kv4Pair<HD> &p, int i) {
      const unsigned char *from = s_mine[wave] + i % kKv4Ring * Slot::BYTES;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        if constexpr (W == 4) {
          const u32x4 x = *reinterpret_cast<const u32x4 *>(from + n * Slot::TILE + lane * 16);
          const u32x4 y = *reinterpret_cast<const u32x4 *>(from + Slot::V + n * Slot::TILE + lane * 16);
#pragma unroll
          for (int w = 0; w < W; ++w) p.kc[n][w] = x[w], p.vc[n][w] = y[w];
        } else {
          const u32x2 x = *reinterpret_cast<const u32x2 *>(from + n * Slot::TILE + col * (HD / 2) + quad * (HD / 8));
          const u32x2 y = *reinterpret_cast<const u32x2 *>(from + Slot::V + n * Slot::TILE + lane * 8);
#pragma unroll
          for (int w = 0; w < W; ++w) p.kc[n][w] = x[w], p.vc[n][w] = y[w];
        }
        p.ke[n] = from[Slot::EXP + n * 64 + col * (HD / 32) + quad * (HD / 4) / 32];
        p.ve[n] = *reinterpret_cast<const uint32_t *>(from + Slot::EXP + 128 + n * 64 + (quad * (HD / 32) + col * (HD / 16) / 32) * 4);
      }
    };
    bf16x8 qf[CT][KJ][TERMS];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int j = 0; j < KJ; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float f = a.flip ? -(float)qr[ct][j][e] : (float)qr[ct][j][e];   // a negative scale: larger products are larger scores
          qf[ct][j][0][e] = (__bf16)f;
          if constexpr (TERMS == 2) qf[ct][j][1][e] = (__bf16)(f - (float)qf[ct][j][0][e]);
        }
    auto use_pair = [&](const Kv4Pair<HD> &p, int i) {
      const int base = t0 + 32 * (wave + 4 * i);
      f32x4 s[CT][2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float ks = __uint_as_float(p.ke[n] << 23);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) s[ct][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < KJ; ++j) {
          bf16x8 kf;
          const uint32_t w = p.kc[n][j];
          const auto x0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 1),
                     x2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 3);
          kf[0] = x0[0], kf[1] = x0[1], kf[2] = x1[0], kf[3] = x1[1], kf[4] = x2[0], kf[5] = x2[1], kf[6] = x3[0], kf[7] = x3[1];
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int e = 0; e < TERMS; ++e)
              s[ct][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[ct][j][e], s[ct][n], 0, 0, 0);
        }
      }
      // tokens that some column must not see: the last ones, and those of missing blocks
      const bool gone0 = __builtin_amdgcn_readlane(my_id, 2 * i) < 0, gone1 = __builtin_amdgcn_readlane(my_id, 2 * i + 1) < 0;
      uint32_t ve[2] = {p.ve[0], p.ve[1]};
      float x[CT][8];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[ct][e] = s[ct][e >> 2][e & 3];
      if (gone0 || gone1 || base + 32 > seq - rows.count + 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int t = base + 16 * (e >> 2) + 4 * quad + (e & 3);
          const bool gone = (e < 4 ? gone0 : gone1) || t >= seq;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
            if (gone || t >= seen[ct]) x[ct][e] = -INFINITY;
          // a probability of zero times a value that is not finite would be NaN: such values leave the product
          const uint32_t mask = 0xFFu << (8 * (e & 3));
          const bool large = ((ve[e >> 2] >> (8 * (e & 3))) & 0xFFu) >= kKv4NotFinite;
          odd |= (uint32_t)(large && !gone);
          if (large || gone) ve[e >> 2] &= ~mask;
        }
      }
      bf16x8 pf[CT][2];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float top = x[ct][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, x[ct][e]);
        top = max_xor32(max_xor16(top)) * a.scale_log2;
        if (__ballot(top > m[ct] + kKv4Lazy)) {
          const float next = fmaxf(m[ct], top);
          const float by = next == -INFINITY ? 1.f : exp2_fast(m[ct] - next);
          m[ct] = next;
          l[ct] *= by;
#pragma unroll
          for (int d = 0; d < ND; ++d) acc[ct][d] *= by;
        }
        const float use = m[ct] == -INFINITY ? 0.f : m[ct];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float pr = exp2_fast(__builtin_fmaf(x[ct][e], a.scale_log2, -use));
          l[ct] += pr;
          pf[ct][0][e] = (__bf16)pr;
          pf[ct][1][e] = (__bf16)(pr - (float)pf[ct][0][e]);
        }
      }
      float vs[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        vs[n][0] = __uint_as_float(ve[n] << 23);    // of a scale the conversion reads the exponent only: the bits beside it may stay
        vs[n][1] = __uint_as_float(ve[n] << 15);
        vs[n][2] = __uint_as_float(ve[n] << 7);
        vs[n][3] = __uint_as_float(ve[n] >> 1);
      }
      // two channels at a time: a conversion gives channels 2 d, 2 d + 1 of one token, a product takes one channel of eight tokens
      auto channels = [&](auto which) {
        constexpr int dd = decltype(which)::value;
        uint32_t r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int n = e >> 2;
          if constexpr (HD == 128)
            r[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(p.vc[n][e & 3], vs[n][e & 3], dd));
          else if (e & 1)
            r[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(p.vc[n][(e & 3) >> 1], vs[n][e & 3], 2 + (dd & 1)));
          else
            r[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(p.vc[n][(e & 3) >> 1], vs[n][e & 3], dd & 1));
        }
        u32x4 lo, hi;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          lo[w] = __builtin_amdgcn_perm(r[2 * w + 1], r[2 * w], 0x05040100u);
          hi[w] = __builtin_amdgcn_perm(r[2 * w + 1], r[2 * w], 0x07060302u);
        }
        const bf16x8 v0 = __builtin_bit_cast(bf16x8, lo), v1 = __builtin_bit_cast(bf16x8, hi);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            acc[ct][2 * dd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pf[ct][e], acc[ct][2 * dd], 0, 0, 0);
            acc[ct][2 * dd + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pf[ct][e], acc[ct][2 * dd + 1], 0, 0, 0);
          }
      };
      // one after the other: the compiler would convert them all first and run out of registers
      channels(std::integral_constant<int, 0>{});
      __builtin_amdgcn_sched_barrier(0);
      channels(std::integral_constant<int, 1>{});
      if constexpr (HD == 128) {
        __builtin_amdgcn_sched_barrier(0);
        channels(std::integral_constant<int, 2>{});
        __builtin_amdgcn_sched_barrier(0);
        channels(std::integral_constant<int, 3>{});
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    for (t0 = u0 * kKv4Unit; t0 < t1; t0 += 32 * kKv4Unit) {
      // the blocks of the wave's tiles: lane 2 i + n holds that of tile n of its i-th pair of these 32
      const int t = t0 + 32 * (wave + 4 * (lane >> 1)) + 16 * (lane & 1);
      my_id = t < t1 ? b.table[(long long)req * b.max_blocks + (t >> c.block_shift)] : -1;
      if (my_id >= c.n_blocks) my_id = -1;
      const int n_pairs = max((min(t1 - t0, 32 * kKv4Unit) + 127 - 32 * wave) >> 7, 0);
      wait_vmcnt_all();                                         // the compiler's own loads: none may be waited for among the transfers
      for (int i = 0; i < min(n_pairs, kKv4Ring); ++i) fetch(i);
      for (int i = 0; i < n_pairs; ++i) {
        if (i + kKv4Ring - 1 < n_pairs) wait_vmcnt<(kKv4Ring - 1) * Slot::TRANSFERS>();
        else wait_vmcnt<0>();
        Kv4Pair<HD> p;
        take(p, i);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the pair is in registers: its place may be written again
        if (i + kKv4Ring < n_pairs) fetch(i + kKv4Ring);
        use_pair(p, i);
      }
    }
    // what is not finite makes NaN of the columns that do see it (rare: the exponents of all of the wave's tokens are read again)
    uint32_t nan_out = 0;                                       // bit ct: the lane's column of tile ct, in the lane's channels
    if (__ballot(odd)) {
      for (int t = u0 * kKv4Unit; t < t1; ++t) {
        if ((t / 32 - wave) % 4) continue;
        const int id = b.table[(long long)req * b.max_blocks + (t >> c.block_shift)], o = t & (bs - 1);
        if (id < 0 || id >= c.n_blocks) continue;
        const uint8_t e = c.at(id, head)[Kv4Offsets<HD>::v_exp(bs) + ((o / 4) * (HD / 32) + quad * (HD / 4) / 32) * 4 + o % 4];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) nan_out |= (uint32_t)(e >= kKv4NotFinite && t < seen[ct]) << ct;
      }
    }
    // join the waves, a tile of columns at a time
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      l[ct] = sum_xor32(sum_xor16(l[ct]));
      if (quad == 0) {
        s_m[wave][col] = m[ct];
        s_l[wave][col] = l[ct];
      }
      float *to = reinterpret_cast<float *>(s_mine[wave]) + col * LD;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int d = 0; d < ND; ++d) to[(4 * quad + e) * ND + d] = nan_out >> ct & 1 ? __uint_as_float(0x7FC00000u) : acc[ct][d][e];
      __syncthreads();
      for (int u = threadIdx.x; u < 16 * (HD / 4); u += 256) {
        const int n = u / (HD / 4), d = u % (HD / 4) * 4, cn = col0 + ct * 16 + n;
        if (cn >= n_cols) continue;
        const float top = fmaxf(fmaxf(s_m[0][n], s_m[1][n]), fmaxf(s_m[2][n], s_m[3][n]));
        float sum = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w)
          if (kv4_saw(s_m[w][n], s_l[w][n])) {
            const float by = kv4_weight(s_m[w][n], top);
            sum += s_l[w][n] * by;
            o += *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(s_mine[w]) + n * LD + d) * by;
          }
        const int i = cn / a.group, h = head * a.group + (cn - i * a.group);
        const long long r = rows.begin + i;
        if (whole) {
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          float f[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
          store_vec<T, 4>(out.at(r, h) + d, f);
          if (a.lse && d == 0) a.lse[r * a.q_heads + h] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
        } else {
          const long long at_col = slot * a.cols + ct * 16 + n;
          *reinterpret_cast<f32x4 *>(a.part + at_col * HD + d) = o;
          if (d == 0) *reinterpret_cast<float2 *>(a.part_ml + at_col * 2) = make_float2(top, sum);
        }
      }
      __syncthreads();
    }
    at += u1 - u0;
  }
}

// Joins the parts of segments that several workgroups worked on, in the order of their tokens.  A workgroup per segment; 16 bytes of
// a column per thread.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_join(Kv4Cache c, PagedBatch b, HeadRows<T> out, Kv4Attend a, int grid) {
  const int req = blockIdx.y, lane = threadIdx.x & 63;
  long long before = 0, all = 0;
  for (int i = lane; i < b.batch; i += 64) {
    const long long work = kv4_request(c, b, a, i).work;
    all += work;
    if (i < req) before += work;
  }
  const Kv4Request r = kv4_request(c, b, a, req);
  before = wave_sum64(before);
  const long long per = kv4_run(wave_sum64(all), grid);
  const int segments = (int)wave_div(r.work, r.units);
  for (int seg = blockIdx.x; seg < segments; seg += gridDim.x) {
    const long long s0 = before + (long long)seg * r.units;
    const int w0 = (int)wave_div(s0, per), w1 = (int)wave_div(s0 + r.units - 1, per);   // who has the first, the last unit
    if (w0 == w1) continue;
    const int first_slot = 2 * w0 + (w0 * per != s0);                              // the others begin their runs inside the segment
    const int head = seg % c.kv_heads, col0 = seg / c.kv_heads * a.cols, n_cols = min(r.rows.count * a.group - col0, a.cols);
    for (int u = threadIdx.x; u < n_cols * (HD / 4); u += 256) {
      const int n = u / (HD / 4), d = u % (HD / 4) * 4;
      float top = -INFINITY, sum = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      constexpr int K = 8;                                                         // parts requested at once
      for (int w = w0; w <= w1; w += K) {
        float2 ml[K];
        f32x4 x[K];
#pragma unroll
        for (int i = 0; i < K; ++i) {
          const int wi = min(w + i, w1);
          const long long at = (long long)(wi == w0 ? first_slot : 2 * wi) * a.cols + n;
          ml[i] = *reinterpret_cast<const float2 *>(a.part_ml + at * 2);
          x[i] = *reinterpret_cast<const f32x4 *>(a.part + at * HD + d);
          if (w + i > w1) ml[i] = make_float2(-INFINITY, 0.f);
        }
        float next = top;
#pragma unroll
        for (int i = 0; i < K; ++i) next = fmaxf(next, ml[i].x);
        const float keep = kv4_weight(top, next);
        sum *= keep;
        o *= keep;
        top = next;
#pragma unroll
        for (int i = 0; i < K; ++i)
          if (kv4_saw(ml[i].x, ml[i].y)) {
            const float by = kv4_weight(ml[i].x, top);
            sum += ml[i].y * by;
            o += x[i] * by;
          }
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const int i = (col0 + n) / a.group, h = head * a.group + (col0 + n - i * a.group);
      float f[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
      store_vec<T, 4>(out.at(r.rows.begin + i, h) + d, f);
      if (a.lse && d == 0) a.lse[(long long)(r.rows.begin + i) * a.q_heads + h] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    }
  }
}

}  // namespace heisd
