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
// contiguous.  So every lane fetches its part of a tile in one load, a wave's loads are consecutive, and nothing passes through LDS.
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
// writes 17/64 of the bytes of a bf16 row; bound by memory.  VEC: rows are aligned for wide loads.
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

constexpr int kGatherRows = 16;

// Sixteen packed rows per workgroup, head by head: the rows of a block that follow each other lie together in the cache.  Rows
// of a block that the pool does not have are zero.  Bound by memory.
template <typename T, int HD, bool VEC>
__global__ __launch_bounds__(256) void kv4_gather(Kv4Cache c, PagedBatch b, const int32_t *cu_seq, int out_rows,
                                                  HeadRows<T> k, HeadRows<T> v) {
  constexpr int LH = HD / 8;
  __shared__ int where[kGatherRows];                // slot, -1: no such token (a zero row), -2: nobody's row
  const int r0 = blockIdx.x * kGatherRows, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const bool is_v = blockIdx.y;
  for (int i = wave; i < kGatherRows; i += 4) {
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
  for (int u = threadIdx.x; u < c.kv_heads * kGatherRows * LH; u += 256) {
    const int j = u % LH, i = u / LH % kGatherRows, h = u / (LH * kGatherRows);
    const int s = where[i];
    if (s == -2) continue;
    float f[8];
    if (s < 0) {
#pragma unroll
      for (int n = 0; n < 8; ++n) f[n] = 0.f;
    } else {
      const int id = s >> c.block_shift, t = s & (c.block_size - 1);
      const uint8_t *cell = c.at(id, h);
      uint32_t code, e;
      if (!is_v) {
        code = *reinterpret_cast<const uint32_t *>(cell + t * (HD / 2) + j * 4);
        e = cell[Kv4Offsets<HD>::k_exp(c.block_size) + t * (HD / 32) + j / 4];
      } else {
        const uint8_t *from = cell + Kv4Offsets<HD>::v_codes(c.block_size) + (t / 4) * (2 * HD);
        if constexpr (HD == 128) code = *reinterpret_cast<const uint32_t *>(from + j * 16 + (t % 4) * 4);
        else
          code = *reinterpret_cast<const uint16_t *>(from + 2 * j * 8 + (t % 4) * 2) |
                 (uint32_t)*reinterpret_cast<const uint16_t *>(from + (2 * j + 1) * 8 + (t % 4) * 2) << 16;
        e = cell[Kv4Offsets<HD>::v_exp(c.block_size) + ((t / 4) * (HD / 32) + j / 4) * 4 + t % 4];
      }
      const float scale = kv4_scale(e);
      const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.f, 1),
                 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.f, 3);
      f[0] = p0[0] * scale, f[1] = p0[1] * scale, f[2] = p1[0] * scale, f[3] = p1[1] * scale;
      f[4] = p2[0] * scale, f[5] = p2[1] * scale, f[6] = p3[0] * scale, f[7] = p3[1] * scale;
    }
    T *y = (is_v ? v : k).at(r0 + i, h) + j * 8;
    if constexpr (VEC) {
      if constexpr (sizeof(T) == 2) store_vec<T, 8>(y, f);
      else {
        store_vec<T, 4>(y, f);
        store_vec<T, 4>(y + 4, f + 4);
      }
    } else {
#pragma unroll
      for (int n = 0; n < 8; ++n) y[n] = (T)f[n];
    }
  }
}

// ---- attention ------------------------------------------------------------------------------------------------------

// What a wave holds of two tiles of 16 tokens.
template <int HD>
struct Kv4Pair {
  static constexpr int W = HD / 32;                 // dwords of codes per lane and tile
  uint32_t kc[2][W], vc[2][W];
  uint32_t ke[2], ve[2];                            // the lane's key exponent; the exponents of its four value tokens
};

struct Kv4Attend {
  float scale_log2;                                 // softmax scale times log2(e)
  int group, q_heads, chunk, n_chunks, max_seq;
  float *part, *lse;                                // part: [row][query head][chunk][HD + 2] sums of chunks
};

// Online softmax state of a column (one query row of one head): maximum and sum in powers of two.
constexpr float kKv4Lazy = 8.f;                     // the maximum is moved only when it grew by more than this (powers of two)

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// softmax(q K^T) V over the tokens of one chunk of one request and one key head.  The query rows of the heads that share the key head
// are the columns of the matrix products (CT tiles of 16): scores^T = K q^T (tokens are rows), out^T = V^T p^T.  A lane holds the
// scores of one column and four tokens of each tile, which are its summed indices of the second product, so the probabilities
// never leave their lane.  Four waves take pairs of tiles in turn, each with a running maximum and sum of its own, joined
// through LDS at the end; chunks are joined by kv4_join.  TERMS 2: queries and probabilities enter as a bf16 and a bf16
// remainder (fp16 rows, whose 11 bits a bf16 does not hold); 1: as one bf16, rounding the probabilities by 2^-9.
template <typename T, int HD, int CT, int TERMS>
__global__ __launch_bounds__(256) void kv4_attend(Kv4Cache c, PagedBatch b, HeadRows<const T> q, HeadRows<T> out, Kv4Attend a) {
  constexpr int W = HD / 32, ND = HD / 16, KJ = HD / 32;        // code dwords, tiles of channels, products per score tile
  constexpr int LD = HD + 4;
  __shared__ __attribute__((aligned(16))) float s_out[4][16 * LD];
  __shared__ float s_m[4][16], s_l[4][16];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int head = blockIdx.x % c.kv_heads, req = blockIdx.z, chunk = blockIdx.y;
  const Span rows = packed_span(b.cu_rows, req, b.rows);
  int seq = b.seq_len[req];
  if (seq > a.max_seq || (long long)seq > (long long)b.max_blocks * c.block_size) seq = 0;
  seq = max(seq, 0);
  const int t0 = chunk * a.chunk, t1 = min(seq, t0 + a.chunk);
  if (rows.count == 0 || (chunk > 0 && t0 >= seq)) return;
  const int n_cols = rows.count * a.group;
  const int bs = c.block_size;
  const bool whole = seq <= a.chunk;

  for (int col0 = blockIdx.x / c.kv_heads * (16 * CT); col0 < n_cols; col0 += gridDim.x / c.kv_heads * (16 * CT)) {
    // the columns' queries and how many tokens each may see
    bf16x8 qf[CT][KJ][TERMS];
    int seen[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const int n = col0 + ct * 16 + col, i = n / a.group;
      const bool there = n < n_cols;
      seen[ct] = there ? seq - rows.count + i + 1 : 0;
      const T *p = there ? q.at(rows.begin + i, head * a.group + (n - i * a.group)) + quad * (HD / 4) : nullptr;
#pragma unroll
      for (int j = 0; j < KJ; ++j) {
        float f[8];
        if (there) load_vec<T, 8>(p + j * 8, f);
        else
          for (int e = 0; e < 8; ++e) f[e] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          qf[ct][j][0][e] = (__bf16)f[e];
          if constexpr (TERMS == 2) qf[ct][j][1][e] = (__bf16)(f[e] - (float)qf[ct][j][0][e]);
        }
      }
    }
    f32x4 acc[CT][ND];
    float m[CT], l[CT];
    bool nan_out[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      m[ct] = -INFINITY;
      l[ct] = 0.f;
      nan_out[ct] = false;
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[ct][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // the blocks of the wave's tiles: lane 2 i + n holds that of tile n of its i-th pair (32 pairs: a chunk has at most 4096 tokens)
    const int n_pairs = max((t1 - t0 + 127 - 32 * wave) >> 7, 0);
    int my_id = -1;
    {
      const int t = t0 + 32 * (wave + 4 * (lane >> 1)) + 16 * (lane & 1);
      if (t < t1) my_id = b.table[(long long)req * b.max_blocks + (t >> c.block_shift)];
      if (my_id >= c.n_blocks) my_id = -1;
    }
    auto load_pair = [&](Kv4Pair<HD> &p, int i) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int id = max(__builtin_amdgcn_readlane(my_id, 2 * i + n), 0);          // a missing block: any block, masked below
        const int t = (t0 + 32 * (wave + 4 * i) + 16 * n) & (bs - 1);
        const uint8_t *cell = c.at(id, head);
        const uint8_t *kp = cell + t * (HD / 2) + col * (HD / 2) + quad * (HD / 8);
        const uint8_t *vp = cell + Kv4Offsets<HD>::v_codes(bs) + t * (HD / 2) + quad * (2 * HD) + col * (HD / 8);
        if constexpr (W == 4) {
          const u32x4 x = *reinterpret_cast<const u32x4 *>(kp), y = *reinterpret_cast<const u32x4 *>(vp);
#pragma unroll
          for (int w = 0; w < W; ++w) p.kc[n][w] = x[w], p.vc[n][w] = y[w];
        } else {
          const u32x2 x = *reinterpret_cast<const u32x2 *>(kp), y = *reinterpret_cast<const u32x2 *>(vp);
#pragma unroll
          for (int w = 0; w < W; ++w) p.kc[n][w] = x[w], p.vc[n][w] = y[w];
        }
        p.ke[n] = cell[Kv4Offsets<HD>::k_exp(bs) + (t + col) * (HD / 32) + quad * (HD / 4) / 32];
        p.ve[n] = *reinterpret_cast<const uint32_t *>(cell + Kv4Offsets<HD>::v_exp(bs) + t * (HD / 32) +
                                                      (quad * (HD / 32) + col * (HD / 16) / 32) * 4);
      }
    };
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
        for (int e = 0; e < 8; ++e) x[ct][e] = s[ct][e >> 2][e & 3] * a.scale_log2;
      if (gone0 || gone1 || base + 32 > seq - rows.count + 1) {
        bool odd = false;
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
          odd = odd || (large && !gone);
          if (large || gone) ve[e >> 2] &= ~mask;
        }
        if (__ballot(odd)) {                        // and what is NaN makes NaN of the columns that do see it
          for (int t = base; t < min(base + 32, seq); ++t) {
            const int id = __builtin_amdgcn_readlane(my_id, 2 * i + ((t - base) >> 4));
            if (id < 0) continue;
            const int o = t & (bs - 1);
            const uint8_t e = c.at(id, head)[Kv4Offsets<HD>::v_exp(bs) + ((o / 4) * (HD / 32) + quad * (HD / 4) / 32) * 4 + o % 4];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) nan_out[ct] = nan_out[ct] || (e >= kKv4NotFinite && t < seen[ct]);
          }
        }
      }
      bf16x8 pf[CT][TERMS];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float top = x[ct][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, x[ct][e]);
        top = max_xor32(max_xor16(top));
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
          const float pr = exp2_fast(x[ct][e] - use);
          l[ct] += pr;
          pf[ct][0][e] = (__bf16)pr;
          if constexpr (TERMS == 2) pf[ct][1][e] = (__bf16)(pr - (float)pf[ct][0][e]);
        }
      }
      float vs[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        vs[n][0] = __uint_as_float((ve[n] << 23) & 0x7F800000u);
        vs[n][1] = __uint_as_float((ve[n] << 15) & 0x7F800000u);
        vs[n][2] = __uint_as_float((ve[n] << 7) & 0x7F800000u);
        vs[n][3] = __uint_as_float((ve[n] >> 1) & 0x7F800000u);
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
          for (int e = 0; e < TERMS; ++e) {
            acc[ct][2 * dd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pf[ct][e], acc[ct][2 * dd], 0, 0, 0);
            acc[ct][2 * dd + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pf[ct][e], acc[ct][2 * dd + 1], 0, 0, 0);
          }
      };
      channels(std::integral_constant<int, 0>{});
      channels(std::integral_constant<int, 1>{});
      if constexpr (HD == 128) {
        channels(std::integral_constant<int, 2>{});
        channels(std::integral_constant<int, 3>{});
      }
    };
    Kv4Pair<HD> now, next;
    if (n_pairs > 0) load_pair(now, 0);
    for (int i = 0; i < n_pairs; i += 2) {
      if (i + 1 < n_pairs) load_pair(next, i + 1);
      use_pair(now, i);
      if (i + 1 >= n_pairs) break;
      if (i + 2 < n_pairs) load_pair(now, i + 2);
      use_pair(next, i + 1);
    }
    // join the waves, a tile of columns at a time
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      l[ct] = sum_xor32(sum_xor16(l[ct]));
      if (quad == 0) {
        s_m[wave][col] = m[ct];
        s_l[wave][col] = l[ct];
      }
      float *to = s_out[wave] + col * LD;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int d = 0; d < ND; ++d) to[(4 * quad + e) * ND + d] = nan_out[ct] ? __uint_as_float(0x7FC00000u) : acc[ct][d][e];
      __syncthreads();
      for (int u = threadIdx.x; u < 16 * (HD / 4); u += 256) {
        const int n = u / (HD / 4), d = u % (HD / 4) * 4, cn = col0 + ct * 16 + n;
        if (cn >= n_cols) continue;
        const float top = fmaxf(fmaxf(s_m[0][n], s_m[1][n]), fmaxf(s_m[2][n], s_m[3][n]));
        float sum = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w)
          if (s_m[w][n] != -INFINITY) {             // a wave that saw nothing holds nothing
            const float by = exp2_fast(s_m[w][n] - top);
            sum += s_l[w][n] * by;
            o += *reinterpret_cast<const f32x4 *>(s_out[w] + n * LD + d) * by;
          }
        const int i = cn / a.group, h = head * a.group + (cn - i * a.group);
        const long long r = rows.begin + i;
        if (whole) {
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          float f[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
          store_vec<T, 4>(out.at(r, h) + d, f);
          if (a.lse && d == 0) a.lse[r * a.q_heads + h] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
        } else {
          float *p = a.part + ((r * a.q_heads + h) * a.n_chunks + chunk) * (HD + 2);
          *reinterpret_cast<float2 *>(p + d) = make_float2(o[0], o[1]);
          *reinterpret_cast<float2 *>(p + d + 2) = make_float2(o[2], o[3]);
          if (d == 0) {
            p[HD] = top;
            p[HD + 1] = sum;
          }
        }
      }
      __syncthreads();
    }
  }
}

// Joins the chunks of rows that have more than one: a wave per row and head.  Chunks are added in their order.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_join(Kv4Cache c, PagedBatch b, HeadRows<T> out, Kv4Attend a) {
  constexpr int V = HD / 64;
  const int lane = threadIdx.x & 63;
  const long long at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long long r = at / a.q_heads;
  const int h = (int)(at - r * a.q_heads);
  if (r >= b.rows) return;
  const int req = wave_search(b.batch, r, [&](int n) { return (long long)b.cu_rows[n]; });
  const Span rows = packed_span(b.cu_rows, req, b.rows);
  if (r < rows.begin || r >= rows.begin + rows.count) return;
  const int seq = b.seq_len[req];
  if (seq > a.max_seq || (long long)seq > (long long)b.max_blocks * c.block_size || seq <= a.chunk) return;
  const int n = (seq + a.chunk - 1) / a.chunk;
  const float *p = a.part + at * a.n_chunks * (HD + 2);
  float top = -INFINITY;
  for (int i = lane; i < n; i += 64) top = fmaxf(top, p[(long long)i * (HD + 2) + HD]);
  top = wave_max(top);
  float sum = 0.f, o[V] = {};
  for (int i = 0; i < n; ++i) {
    const float *x = p + (long long)i * (HD + 2);
    const float m = x[HD];
    if (m == -INFINITY) continue;
    const float by = exp2_fast(m - top);
    sum += x[HD + 1] * by;
#pragma unroll
    for (int v = 0; v < V; ++v) o[v] += x[lane * V + v] * by;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int v = 0; v < V; ++v) o[v] *= inv;
  store_vec<T, V>(out.at(r, h) + lane * V, o);
  if (a.lse && lane == 0) a.lse[r * a.q_heads + h] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace heisd
