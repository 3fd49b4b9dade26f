// What stays in the 4-bit cache: tokens copied from one request to another, the attention weight that every cached token has received, and
// eviction of the tokens that received least.  Weights are fp32, [n_blocks][kv_heads][block_size]: a token's lies where its cell does.
#pragma once
#include "heisd_common.h"
#include "heisd_kv4.h"
#include "heisd_paged.h"

namespace heisd {

// ---- tokens copied from one request to another --------------------------------------------------------------------------

struct CopyArgs {
  const int32_t *from;
  float *weight;                                    // or null
  long long layer_bytes, layer_weights;
  int max_seq, head_dim;
};

// One workgroup per block of 16-byte pieces of a request, block and layer.  A block's cells of all heads lie together in the source and in the
// destination; of a block that is not full, only the tiles of 16 tokens that hold tokens are copied.  Sources and destinations are different
// blocks.  Reads and writes (head_dim + head_dim / 16) bytes per token and head: a third of 128 requests of up to 500 tokens, 8 heads of 128, two layers in 10 us, with
// two thirds of the workgroups finding nothing to copy.
constexpr int kCopyPieces = 4;
__global__ __launch_bounds__(256) void kv4_copy_blocks(Kv4Cache c, PagedBatch b, CopyArgs a, int per_block) {
  const int req = blockIdx.y, from = a.from[req];
  if (from < 0 || from >= b.batch || from == req) return;
  const int all = b.seq_len[req], n = min(all, a.max_seq), j = blockIdx.x / per_block, bs = c.block_size;
  if (n <= 0 || (long long)all > (long long)b.max_blocks * bs || (long long)j * bs >= n) return;
  const int to_id = b.table[(long long)req * b.max_blocks + j], from_id = b.table[(long long)from * b.max_blocks + j];
  if (to_id < 0 || to_id >= c.n_blocks || from_id < 0 || from_id >= c.n_blocks || to_id == from_id) return;
  const int used = min((n - j * bs + 15) & ~15, bs);
  c.pool += blockIdx.z * a.layer_bytes;
  const int piece0 = (blockIdx.x % per_block) * (256 * kCopyPieces) + threadIdx.x;
  const uint8_t *src = c.at(from_id, 0);
  uint8_t *dst = c.at(to_id, 0);
  const int codes = bs * (a.head_dim / 2), pieces = c.kv_heads * (int)(c.cell / 16);
  u32x4 x[kCopyPieces];
  bool ok[kCopyPieces];
#pragma unroll
  for (int i = 0; i < kCopyPieces; ++i) {
    const int p = piece0 + 256 * i;
    int o = p * 16 % (int)c.cell;                   // the place in the cell, then in its part
    const int per_token = o < 2 * codes ? a.head_dim / 2 : a.head_dim / 32;
    if (o < 2 * codes) o = o < codes ? o : o - codes;
    else {
      o -= 2 * codes;
      if (o >= bs * per_token) o -= bs * per_token;
    }
    ok[i] = p < pieces && o < used * per_token;
    if (ok[i]) x[i] = *reinterpret_cast<const u32x4 *>(src + (long long)p * 16);
  }
#pragma unroll
  for (int i = 0; i < kCopyPieces; ++i)
    if (ok[i]) *reinterpret_cast<u32x4 *>(dst + (long long)(piece0 + 256 * i) * 16) = x[i];
  if (a.weight && blockIdx.x % per_block == 0) {
    float *w = a.weight + blockIdx.z * a.layer_weights;
    for (int u = threadIdx.x; u < c.kv_heads * bs; u += 256)
      if ((u & (bs - 1)) < n - j * bs) w[(long long)to_id * c.kv_heads * bs + u] = w[(long long)from_id * c.kv_heads * bs + u];
  }
}

// ---- attention weights of cached tokens ---------------------------------------------------------------------------------

struct WeighArgs {
  float scale_log2, decay;                          // softmax scale times log2(e)
  int group, q_heads, max_seq;
  const float *lse, *weight_in;
  float *weight_out;
};
constexpr int kWeighPairs = 8;                      // pairs of tiles that a wave takes at most
constexpr int kWeighUnit = 128;                     // tokens of a pair for each of the four waves

// The same for four tiles: a quarter of a token's head in each of them, and the weight that the lane's token of the 64 had.
template <int HD>
struct WeighFour {
  uint32_t kc[4][HD / 32], ke[4];
  float old;
};
// What a lane holds of the keys of two tiles of 16 tokens: a quarter of one token's head in each, and the weight that one of the tokens had.
template <int HD>
struct WeighPair {
  uint32_t kc[2][HD / 32], ke[2];
  float old;
};
__device__ __forceinline__ bf16x8 weigh_keys(uint32_t w, uint32_t e) {
  const float ks = __uint_as_float(e << 23);
  const auto x0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 1),
             x2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 3);
  bf16x8 k;
  k[0] = x0[0], k[1] = x0[1], k[2] = x1[0], k[3] = x1[1], k[4] = x2[0], k[5] = x2[1], k[6] = x3[0], k[7] = x3[1];
  return k;
}

// The weights of tokens [t0, t1) of a request with at most four columns (a single token and up to four query heads per key head, four single heads' tokens).  Of a product
// for sixteen columns these would be a quarter, so tokens are its columns here and the queries its rows, four times over: of tile k's scores the lanes 16 k on keep
// theirs, and four tiles give every lane one token with all of its scores.  Nothing is exchanged between lanes, and there are a quarter of the exponents
// (64 contexts of up to 7847 tokens: 35.8 us, 44 with rows as columns).
template <typename T, int HD, int TERMS>
__device__ __forceinline__ void weigh_four(const Kv4Cache &c, const PagedBatch &b, const HeadRows<const T> &q, const WeighArgs &a, int req, int head, Span own, int had,
                                           int t0, int t1) {
  constexpr int KJ = HD / 32;
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4, bs = c.block_size;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = t0 + wave * 64;
  const int units = max((t1 - first + 255) / 256, 0);
  if (!units) return;
  int my_id = -1;                                   // lane 4 i + k: the block of tile k of the i-th 64 tokens
  {
    const int t = first + 256 * (lane >> 2) + 16 * (lane & 3);
    if (lane < 4 * units && t < t1) my_id = b.table[(long long)req * b.max_blocks + (t >> c.block_shift)];
    if (my_id >= c.n_blocks) my_id = -1;
  }
  const int n_cols = own.count * a.group;
  bf16x8 qf[KJ][TERMS];
  float lse[4];
  int seen[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int n = min(e, n_cols - 1), i = n / a.group;
    const float x = n_cols ? a.lse[(long long)(own.begin + i) * a.q_heads + head * a.group + (n - i * a.group)] : 0.f;
    lse[e] = x * 1.4426950408889634f;
    seen[e] = e >= n_cols || x == -INFINITY ? 0 : had + 1 + i;
  }
  {
    const int n = min(col & 3, n_cols - 1), i = n_cols ? n / a.group : 0;
    const T *from = n_cols ? q.at(own.begin + i, head * a.group + (n - i * a.group)) + quad * (HD / 4) : nullptr;
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      typename VecOf<T, 8>::type v{};
      if (n_cols) v = *reinterpret_cast<const typename VecOf<T, 8>::type *>(from + j * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = (float)v[e];
        qf[j][0][e] = (__bf16)f;
        if constexpr (TERMS == 2) qf[j][1][e] = (__bf16)(f - (float)qf[j][0][e]);
      }
    }
  }
  auto weight_at = [&](int u) {
    const int id = __builtin_amdgcn_ds_bpermute((4 * u + quad) * 4, my_id), t = first + 256 * u + lane;
    return id < 0 || t >= t1 ? -1ll : ((long long)id * c.kv_heads + head) * bs + (t & (bs - 1));
  };
  auto fetch = [&](int u) {
    WeighFour<HD> r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint8_t *cell = c.at(max(__builtin_amdgcn_readlane(my_id, 4 * u + k), 0), head);      // a missing block: any block, not written
      const int o = ((first + 256 * u + 16 * k) & (bs - 1)) + col;
      const uint32_t *codes = reinterpret_cast<const uint32_t *>(cell + o * (HD / 2) + quad * (HD / 8));
#pragma unroll
      for (int j = 0; j < KJ; ++j) r.kc[k][j] = codes[j];
      r.ke[k] = cell[Kv4Offsets<HD>::k_exp(bs) + o * (HD / 32) + quad * (HD / 4) / 32];
    }
    const long long at = weight_at(u);
    r.old = at >= 0 && first + 256 * u + lane < had ? a.weight_in[at] : 0.f;
    return r;
  };
  WeighFour<HD> next = fetch(0);
  for (int u = 0; u < units; ++u) {
    const WeighFour<HD> now = next;
    if (u + 1 < units) next = fetch(u + 1);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KJ; ++j) {
        const bf16x8 kf = weigh_keys(now.kc[k][j], now.ke[k]);
#pragma unroll
        for (int e = 0; e < TERMS; ++e) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[j][e], kf, x, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = quad == k ? x[e] : s[e];
    }
    const int t = first + 256 * u + lane;
    float fresh = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float pr = exp2_fast(__builtin_fmaf(s[e], a.scale_log2, -lse[e]));
      fresh += t < seen[e] ? pr : 0.f;
    }
    const long long at = weight_at(u);
    if (at >= 0) a.weight_out[at] = __builtin_fmaf(a.decay, now.old, fresh);
  }
}

// weight[t] = decay * weight[t] + sum over the rows that see token t and the query heads of its key head of exp(scale q . k - lse).  Scores are one
// matrix product of keys (tokens are rows) and the rows' queries (columns, 16 at a time); lane l has column l % 16 and four
// tokens of a tile, adds up its columns' probabilities, and the 16 lanes of a token are added at the end.  Every token's weight is written by one wave, whose order of
// additions is fixed.  A token that one of its request's rows brought (the last n) had no weight before.  Queries enter as in the attention.
// A wave takes `pairs` pairs of tiles, the next one on its way while it works.  Where 16 columns hold all rows (single tokens and few), their queries
// stay in registers; up to four columns are weigh_four's.  64 contexts of up to 7847 tokens, 8 key heads of 128 (137 MB): 35.8 us, 3.8 TB/s, by latency and vector work about
// equally; without queries in registers and the next pair on its way 77.  Four prefixes of up to 3475 tokens and 64 columns each: 10 us.
template <typename T, int HD, int TERMS>
__global__ __launch_bounds__(256, 4) void kv4_weigh(Kv4Cache c, PagedBatch b, PrefixGroups p, HeadRows<const T> q, WeighArgs a, int pairs) {
  constexpr int KJ = HD / 32;
  const int req = blockIdx.z, head = blockIdx.y, lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), bs = c.block_size;
  const int seq = b.seq_len[req], t0 = blockIdx.x * (kWeighUnit * pairs) + wave * 32;
  if (seq <= (int)blockIdx.x * (kWeighUnit * pairs) || seq > max(a.max_seq, p.groups ? p.max_prefix : 0) || (long long)seq > (long long)b.max_blocks * bs) return;
  Span own = wave_span(b.cu_rows, req, b.rows);
  const int had = seq - own.count;                  // tokens that had a weight before
  if (seq > a.max_seq) own.count = 0;
  unsigned long long any = 0;                       // is it anybody's prefix?
  for (int g0 = 0; g0 < p.groups && !any; g0 += 64) any = __ballot(g0 + lane < p.groups && p.prefix[min(g0 + lane, p.groups - 1)] == req);
  if (!any && own.count * a.group <= 4) {
    weigh_four<T, HD, TERMS>(c, b, q, a, req, head, own, had, blockIdx.x * (kWeighUnit * pairs), min(seq, (int)(blockIdx.x + 1) * (kWeighUnit * pairs)));
    return;
  }
  if (seq <= t0) return;
  const int n_pairs = min((seq - t0 + kWeighUnit - 1) / kWeighUnit, pairs);
  int my_id = -1;                                   // lane 2 i + n: the block of tile n of the i-th pair
  {
    const int t = t0 + kWeighUnit * (lane >> 1) + 16 * (lane & 1);
    if (lane < 2 * n_pairs && t < seq) my_id = b.table[(long long)req * b.max_blocks + (t >> c.block_shift)];
    if (my_id >= c.n_blocks) my_id = -1;
  }
  // tokens this lane writes: 4 quad + e of tile n, with col = 4 n + e below 8
  auto my_token = [&](int i) { return t0 + kWeighUnit * i + 16 * (col >> 2) + 4 * quad + (col & 3); };
  auto weight_at = [&](int i) {
    const int id0 = __builtin_amdgcn_readlane(my_id, 2 * i), id1 = __builtin_amdgcn_readlane(my_id, 2 * i + 1), id = col >> 2 ? id1 : id0;
    return col >= 8 || id < 0 || my_token(i) >= seq ? -1ll : ((long long)id * c.kv_heads + head) * bs + (my_token(i) & (bs - 1));
  };
  auto fetch = [&](int i) {
    WeighPair<HD> r;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const uint8_t *cell = c.at(max(__builtin_amdgcn_readlane(my_id, 2 * i + n), 0), head);      // a missing block: any block, not written
      const int o = ((t0 + kWeighUnit * i + 16 * n) & (bs - 1)) + col;
      const uint32_t *codes = reinterpret_cast<const uint32_t *>(cell + o * (HD / 2) + quad * (HD / 8));
#pragma unroll
      for (int j = 0; j < KJ; ++j) r.kc[n][j] = codes[j];
      r.ke[n] = cell[Kv4Offsets<HD>::k_exp(bs) + o * (HD / 32) + quad * (HD / 4) / 32];
    }
    const long long at = weight_at(i);
    r.old = at >= 0 && my_token(i) < had ? a.weight_in[at] : 0.f;
    return r;
  };
  // a column's query: column c0 + col of rows [begin, begin + count)
  struct Column {
    bf16x8 q[KJ][TERMS];
    float lse;                                      // in powers of two
    int seen;
  };
  auto column = [&](Column &x, Span rows, int c0, int seen0, bool causal) {
    const int n_cols = rows.count * a.group, n = min(c0 + col, n_cols - 1), i = n / a.group, h = head * a.group + (n - i * a.group);
    const T *from = q.at(rows.begin + i, h) + quad * (HD / 4);
    const float lse = a.lse[(long long)(rows.begin + i) * a.q_heads + h];
    x.lse = lse * 1.4426950408889634f;
    x.seen = c0 + col >= n_cols || lse == -INFINITY ? 0 : causal ? seen0 + i : seq;
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      const auto v = *reinterpret_cast<const typename VecOf<T, 8>::type *>(from + j * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = (float)v[e];
        x.q[j][0][e] = (__bf16)f;
        if constexpr (TERMS == 2) x.q[j][1][e] = (__bf16)(f - (float)x.q[j][0][e]);
      }
    }
  };
  auto collect = [&](float (&sum)[2][4], const f32x4 (&s)[2], const Column &x, int base) {
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float pr = exp2_fast(__builtin_fmaf(s[n][e], a.scale_log2, -x.lse));
        sum[n][e] += base + 16 * n + 4 * quad + e < x.seen ? pr : 0.f;
      }
  };
  auto add = [&](float (&sum)[2][4], const bf16x8 (&kf)[2][KJ], const Column &x, int base) {
    f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int j = 0; j < KJ; ++j)
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < TERMS; ++e) s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[n][j], x.q[j][e], s[n], 0, 0, 0);
    collect(sum, s, x, base);
  };
  const int own_cols = own.count * a.group, seen0 = had + 1;
  const bool few = !any && own_cols <= 16;
  Column only;
  if (few && own_cols) column(only, own, 0, seen0, true);
  // the weights of pair i: the columns' sums, added up by the 16 lanes of a token
  auto finish = [&](int i, const float (&sum)[2][4], float old) {
    const long long at = weight_at(i);
    float fresh = 0.f;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float all = sum16(sum[n][e]);
        fresh = col == 4 * n + e ? all : fresh;
      }
    if (at >= 0) a.weight_out[at] = __builtin_fmaf(a.decay, old, fresh);
  };
  if (few) {
    WeighPair<HD> next = fetch(0);
    for (int i = 0; i < n_pairs; ++i) {
      const WeighPair<HD> now = next;
      if (i + 1 < n_pairs) next = fetch(i + 1);
      f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
      float sum[2][4] = {};
      if (own_cols) {
#pragma unroll
        for (int j = 0; j < KJ; ++j)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const bf16x8 kf = weigh_keys(now.kc[n][j], now.ke[n]);
#pragma unroll
            for (int e = 0; e < TERMS; ++e) s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, only.q[j][e], s[n], 0, 0, 0);
          }
        collect(sum, s, only, t0 + kWeighUnit * i);
      }
      finish(i, sum, now.old);
    }
    return;
  }
  WeighPair<HD> next = fetch(0);
  for (int i = 0; i < n_pairs; ++i) {
    const WeighPair<HD> now = next;
    if (i + 1 < n_pairs) next = fetch(i + 1);
    const int base = t0 + kWeighUnit * i;
    bf16x8 kf[2][KJ];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int j = 0; j < KJ; ++j) kf[n][j] = weigh_keys(now.kc[n][j], now.ke[n]);
    float sum[2][4] = {};
    Column x;
    for (int c0 = max(base - seen0 + 1, 0) * a.group & ~15; c0 < own_cols; c0 += 16) {        // rows before see none of these tokens
      column(x, own, c0, seen0, true);
      add(sum, kf, x, base);
    }
    for (int g0 = 0; g0 < p.groups; g0 += 64) {     // the groups that this request is the prefix of
      unsigned long long mine = __ballot(g0 + lane < p.groups && p.prefix[min(g0 + lane, p.groups - 1)] == req);
      for (; mine; mine &= mine - 1) {
        const PrefixSpan s = prefix_span(c, b, p, g0 + __builtin_ctzll(mine));
        if (s.request != req) continue;
        const Span rows{__builtin_amdgcn_readfirstlane(s.rows.begin), __builtin_amdgcn_readfirstlane(s.rows.count)};
        for (int c0 = 0; c0 < rows.count * a.group; c0 += 16) {
          column(x, rows, c0, 0, false);
          add(sum, kf, x, base);
        }
      }
    }
    finish(i, sum, now.old);
  }
}

// ---- eviction -----------------------------------------------------------------------------------------------------------

struct EvictArgs {
  const int32_t *keep;
  int recent, max_seq;
  long long layer_bytes, layer_weights;
  const float *weight_in;
  float *weight_out;
  int32_t *seq_out;
};

// Weights as whole numbers in the same order; what is not a number is the lightest.
__device__ __forceinline__ uint32_t evict_key(float w) {
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w + 0.f);      // no negative zero
  return u >> 31 ? ~u : u | 0x80000000u;
}

constexpr int kEvictThreads = 1024;
constexpr int kEvictQueue = 4 * kEvictThreads;

// A sixteenth of a token's bytes on their way from one place to another, in one lane of 16: 4 (2) bytes of key codes and of value codes each, an
// exponent of a key (value) group in one of the first lanes, the weight in the first.
template <int HD>
struct EvictPiece {
  typedef std::conditional_t<HD == 128, uint32_t, uint16_t> Codes;
  Codes k, v;
  float w;
  uint8_t e;
  static constexpr int G = HD / 32;
  __device__ __forceinline__ static int value_at(int t, int bs, int lane16) {
    return Kv4Offsets<HD>::v_codes(bs) + (t / 4) * (2 * HD) + lane16 * (HD / 8) + (t % 4) * G;
  }
  __device__ __forceinline__ static int exp_at(int t, int bs, int lane16) {
    const int g = lane16 % G;
    return lane16 < G ? Kv4Offsets<HD>::k_exp(bs) + t * G + g : Kv4Offsets<HD>::v_exp(bs) + ((t / 4) * G + g) * 4 + t % 4;
  }
  __device__ __forceinline__ void load(const uint8_t *cell, const float *weight, int t, int bs, int lane16) {
    k = reinterpret_cast<const Codes *>(cell + t * (HD / 2))[lane16];
    v = *reinterpret_cast<const Codes *>(cell + value_at(t, bs, lane16));
    if (lane16 < 2 * G) e = cell[exp_at(t, bs, lane16)];
    if (lane16 == 0) w = *weight;
  }
  __device__ __forceinline__ void store(uint8_t *cell, float *weight, int t, int bs, int lane16) const {
    reinterpret_cast<Codes *>(cell + t * (HD / 2))[lane16] = k;
    *reinterpret_cast<Codes *>(cell + value_at(t, bs, lane16)) = v;
    if (lane16 < 2 * G) cell[exp_at(t, bs, lane16)] = e;
    if (lane16 == 0) *weight = w;
  }
};

// What a workgroup of an eviction has to do: one request, head and layer.  Every thread of the workgroup makes it (a barrier is in it).
struct EvictTask {
  Kv4Cache c;
  const int32_t *table;
  const float *w_in;
  float *w_out;
  int head, n, keep, recent, cand, first;           // cand: tokens that may go, of which `first` stay
  bool whole, cut;
  __device__ __forceinline__ EvictTask(const Kv4Cache &cache, const PagedBatch &b, const EvictArgs &a) : c(cache) {
    const int req = blockIdx.y, bs = c.block_size;
    head = blockIdx.x;
    table = b.table + (long long)req * b.max_blocks;
    n = b.seq_len[req];
    keep = a.keep[req];
    c.pool += blockIdx.z * a.layer_bytes;
    w_in = a.weight_in + blockIdx.z * a.layer_weights;
    w_out = a.weight_out + blockIdx.z * a.layer_weights;
    whole = n >= 0 && n <= a.max_seq && (long long)n <= (long long)b.max_blocks * bs;
    bool missing = false;
    if (whole)
      for (int j = threadIdx.x; (long long)j * bs < n; j += blockDim.x) missing |= table[j] < 0 || table[j] >= c.n_blocks;
    whole = !__syncthreads_or(missing) && whole;
    cut = whole && keep >= 0 && keep < n;
    recent = min(a.recent, cut ? keep : 0);
    cand = n - recent;
    first = keep - recent;
    if (head == 0 && blockIdx.z == 0 && threadIdx.x == 0) a.seq_out[req] = cut ? keep : n;
  }
  __device__ __forceinline__ long long weight_at(int t) const {
    return ((long long)table[t >> c.block_shift] * c.kv_heads + head) * c.block_size + (t & (c.block_size - 1));
  }
  __device__ __forceinline__ uint8_t *cell(int t) const { return c.at(table[t >> c.block_shift], head); }
  template <int HD>
  __device__ __forceinline__ void load(EvictPiece<HD> &p, int t, int lane16) const {
    p.load(cell(t), w_in + weight_at(t), t & (c.block_size - 1), c.block_size, lane16);
  }
  template <int HD>
  __device__ __forceinline__ void store(const EvictPiece<HD> &p, int t, int lane16) const {
    p.store(cell(t), w_out + weight_at(t), t & (c.block_size - 1), c.block_size, lane16);
  }
  // A request that loses nothing: its weights go where they are wanted.
  __device__ __forceinline__ void pass_weights() const {
    if (whole && w_in != w_out)
      for (int t = threadIdx.x; t < n; t += blockDim.x) w_out[weight_at(t)] = w_in[weight_at(t)];
  }
};

// Inclusive sum over the lanes of a wave, in the vector ALU: within rows of 16, then from row to row.
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true);      // row_shr 1, 2, 4, 8
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true);
  const uint32_t r0 = __builtin_amdgcn_readlane((int)v, 15), r1 = __builtin_amdgcn_readlane((int)v, 31), r2 = __builtin_amdgcn_readlane((int)v, 47);
  const int row = (threadIdx.x & 63) >> 4;
  return v + (row > 0 ? r0 : 0) + (row > 1 ? r1 : 0) + (row > 2 ? r2 : 0);
}
// Sum over the workgroup's threads before this one; total: over all.  part: W values of LDS that nothing else uses before the next barrier but one.
template <int W>
__device__ __forceinline__ uint32_t evict_scan(uint32_t v, uint32_t &total, uint32_t *part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t upto = wave_scan(v);
  if (lane == 63) part[wave] = upto;
  __syncthreads();
  const uint32_t parts = wave_scan(lane < W ? part[lane] : 0);
  total = __builtin_amdgcn_readlane((int)parts, W - 1);
  const uint32_t before = __builtin_amdgcn_ds_bpermute(max(wave - 1, 0) * 4, (int)parts);
  return upto - v + (wave ? before : 0);
}

// The bin, counted from the last, in which the `left`-th lies: {bin, how many of it are wanted}.  Clears the bins.  All of the workgroup's threads.
template <int W, int BINS>
__device__ __forceinline__ uint2 evict_bin(uint32_t *hist, uint32_t left, uint32_t *part, uint2 *pick) {
  constexpr int PER = BINS / (W * 64);
  static_assert(PER >= 1 && BINS % (W * 64) == 0, "bins per thread");
  uint32_t h[PER], sum = 0, all;
  const int top = BINS - 1 - threadIdx.x * PER;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    h[i] = hist[top - i];
    hist[top - i] = 0;
    sum += h[i];
  }
  uint32_t before = evict_scan<W>(sum, all, part);
  if (before < left && left <= before + sum) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (before < left && left <= before + h[i]) *pick = make_uint2(top - i, left - before);
      before += h[i];
    }
  }
  __syncthreads();
  return *pick;
}

// Of the first n - recent tokens of a request the heaviest stay (in each layer and head for itself), and all of the last `recent`.  Tokens that
// stay and lie behind the first keep - recent places fill the places of those that go, in order; then the last ones move up.  So
// only what has to move is moved: a context at its budget that loses 64 of 2112 tokens moves 64 + the last ones, not 2048.
// One workgroup per request, head and layer.  A thread holds the keys of E tokens that follow each other; the threshold is found 11 bits at a time (a
// histogram in LDS; counts do not depend on the order of the atomics), then two sums over the workgroup say which of the tokens at the threshold stay (the
// lowest) and where every hole and every filler stands in its list.  The moves are read in lots, all of a lot before any of it is written: places lie
// before the tokens of later lots, so what is read is never new.  One context of 2112 tokens to 2048, two layers of 8 heads: 13.5 us, latency; sixteen of
// 1137 to 8192 tokens to 1024: 30, by the moves: a token's values lie in four lines, of which a quarter each is its own.  Weights read again for every eight bits, and sums
// through LDS: 44.5 and 89.
constexpr int kEvictLot = 4;                        // moves that a sixteenth of a wave's lanes reads at once
template <int HD, int E>
__global__ __launch_bounds__(kEvictThreads) void kv4_evict_held(Kv4Cache cache, PagedBatch b, EvictArgs a) {
  constexpr int N = kEvictThreads, W = N / 64, BINS = 2048;
  __shared__ uint32_t hist[BINS], part[5][W];
  __shared__ uint2 pick[3];
  __shared__ uint16_t holes[N * E / 2], fillers[N * E / 2];
  const int tid = threadIdx.x;
  for (int i = tid; i < BINS; i += N) hist[i] = 0;
  const EvictTask k(cache, b, a);
  if (!k.cut) {
    k.pass_weights();
    return;
  }
  const int t0 = tid * E;
  uint32_t key[E];
  float w[E];
  if (t0 < k.n) {                                   // E is a part of 16, so these are in one block
    const float *from = k.w_in + k.weight_at(t0);
    typedef f32x4 __attribute__((aligned(4))) four;              // weights may begin at any float
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const four x = *reinterpret_cast<const four *>(from + i);
      w[i] = x[0], w[i + 1] = x[1], w[i + 2] = x[2], w[i + 3] = x[3];
    }
  }
#pragma unroll
  for (int i = 0; i < E; ++i) key[i] = t0 + i < k.cand ? evict_key(w[i]) : 0;
  uint32_t prefix = 0, left = (uint32_t)k.first;
  if (k.first) {
    auto digit = [&](int n, int shift, int above, uint32_t mask) {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (t0 + i < k.cand && (above > 31 || key[i] >> above == prefix >> above)) atomicAdd(&hist[key[i] >> shift & mask], 1u);
      __syncthreads();
      const uint2 d = evict_bin<W, BINS>(hist, left, part[n], &pick[n]);
      prefix |= d.x << shift;
      left = d.y;
    };
    digit(0, 21, 32, 2047);
    digit(1, 10, 21, 2047);
    digit(2, 0, 10, 1023);
  }
  // tokens at the threshold: the first `left` stay
  uint32_t equal = 0, none;
#pragma unroll
  for (int i = 0; i < E; ++i) equal += t0 + i < k.cand && key[i] == prefix;
  uint32_t before = evict_scan<W>(equal, none, part[3]);
  uint32_t stays = 0, counts = 0;                   // holes in the low half, fillers in the high
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const bool in = t0 + i < k.cand && k.first, eq = in && key[i] == prefix;
    const bool yes = in && (key[i] > prefix || (eq && before < left));
    before += eq;
    stays |= (uint32_t)yes << i;
    counts += t0 + i < k.first ? !yes : yes ? 0x10000u : 0u;
  }
  uint32_t at = evict_scan<W>(counts, none, part[4]);
  const int fills = (int)(none & 0xFFFFu);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const bool yes = stays >> i & 1;
    if (t0 + i < k.first) {
      if (!yes) holes[at & 0xFFFFu] = (uint16_t)(t0 + i), ++at;
      else if (k.w_in != k.w_out) k.w_out[k.weight_at(t0 + i)] = w[i];
    } else if (yes) fillers[at >> 16] = (uint16_t)(t0 + i), at += 0x10000u;
  }
  __syncthreads();
  const int moves = fills + k.recent, lane16 = tid & 15;
  for (int m0 = 0; m0 < moves; m0 += N / 16 * kEvictLot) {
    EvictPiece<HD> p[kEvictLot];
    int to[kEvictLot];
#pragma unroll
    for (int i = 0; i < kEvictLot; ++i) {
      const int m = m0 + i * (N / 16) + tid / 16;
      to[i] = m >= moves ? -1 : m < fills ? (int)holes[m] : k.first + m - fills;
      if (to[i] >= 0) k.load(p[i], m < fills ? (int)fillers[m] : k.cand + m - fills, lane16);
    }
    wait_vmcnt_all();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEvictLot; ++i)
      if (to[i] >= 0) k.store(p[i], to[i], lane16);
  }
}

// The same for any length: the weights are read again where they are needed, eight bits of the threshold at a time, and holes and fillers are listed chunk by
// chunk, both in order; as many pairs as both lists hold are moved.
template <int HD>
__global__ __launch_bounds__(kEvictThreads) void kv4_evict(Kv4Cache cache, PagedBatch b, EvictArgs a) {
  constexpr int N = kEvictThreads, W = N / 64, BINS = 1024;
  __shared__ uint32_t hist[BINS], part[W];
  __shared__ uint2 pick;
  __shared__ int holes[kEvictQueue + N], fillers[kEvictQueue + N];
  const int tid = threadIdx.x;
  hist[tid] = 0;
  const EvictTask k(cache, b, a);
  if (!k.cut) {
    k.pass_weights();
    return;
  }
  const int cand = k.cand, first = k.first;
  auto key_of = [&](int t) { return evict_key(k.w_in[k.weight_at(t)]); };
  // the key of the lightest that stays, and how many with that key stay
  uint32_t prefix = 0, left = (uint32_t)first;
  for (int shift = 24; shift >= 0 && first; shift -= 8) {
    for (int t = tid; t < cand; t += N) {
      const uint32_t key = key_of(t);
      if (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[key >> shift & 255], 1u);
    }
    __syncthreads();
    const uint2 d = evict_bin<W, BINS>(hist, left, part, &pick);
    prefix |= d.x << shift;
    left = d.y;
    __syncthreads();
  }
  // which tokens stay, chunk by chunk and in order: equal ones from the lowest on
  uint32_t equal_holes = 0, equal_behind = 0;       // tokens with the threshold's key before the chunk, in either region
  for (int t0 = 0; t0 < first; t0 += N) plan_scan<W>((uint32_t)(t0 + tid < first && key_of(t0 + tid) == prefix), equal_behind, part);
  auto stays = [&](int t, int end, uint32_t &equal_before) {
    const uint32_t key = t < end ? key_of(t) : 0;
    const bool eq = t < end && key == prefix;
    const uint32_t rank = plan_scan<W>((uint32_t)eq, equal_before, part);
    return t < end && first && (key > prefix || (eq && rank <= left));
  };
  int at_hole = 0, at_filler = first, n_holes = 0, n_fillers = 0;
  while (true) {
    while (n_holes < kEvictQueue && at_hole < first) {
      const int t = at_hole + tid;
      const bool yes = stays(t, first, equal_holes), hole = t < first && !yes;
      uint32_t count = (uint32_t)n_holes;
      const uint32_t rank = plan_scan<W>((uint32_t)hole, count, part);
      if (hole) holes[rank - 1] = t;
      if (yes && k.w_in != k.w_out) k.w_out[k.weight_at(t)] = k.w_in[k.weight_at(t)];
      n_holes = (int)count;
      at_hole += N;
    }
    while (n_fillers < kEvictQueue && at_filler < cand) {
      const int t = at_filler + tid;
      const bool yes = stays(t, cand, equal_behind);
      uint32_t count = (uint32_t)n_fillers;
      const uint32_t rank = plan_scan<W>((uint32_t)yes, count, part);
      if (yes) fillers[rank - 1] = t;
      n_fillers = (int)count;
      at_filler += N;
    }
    __syncthreads();
    const int moves = min(n_holes, n_fillers);
    if (!moves) break;
    for (int i = tid / 16; i < moves; i += N / 16) {
      EvictPiece<HD> p;
      k.load(p, fillers[i], tid & 15);
      k.store(p, holes[i], tid & 15);
    }
    __syncthreads();
    // what is left of either list moves to its front
    const int left_holes = n_holes - moves, left_fillers = n_fillers - moves;
    for (int i = 0; i < max(left_holes, left_fillers); i += N) {
      const int h = i + tid < left_holes ? holes[moves + i + tid] : 0, f = i + tid < left_fillers ? fillers[moves + i + tid] : 0;
      __syncthreads();
      if (i + tid < left_holes) holes[i + tid] = h;
      if (i + tid < left_fillers) fillers[i + tid] = f;
      __syncthreads();
    }
    n_holes = left_holes, n_fillers = left_fillers;
  }
  // the last ones move up; a chunk is read before it is written, and its places lie before the tokens of later chunks
  wait_vmcnt_all();
  __syncthreads();
  for (int i0 = 0; i0 < k.recent; i0 += N / 16) {
    const int i = i0 + tid / 16;
    EvictPiece<HD> p;
    if (i < k.recent) k.load(p, cand + i, tid & 15);
    wait_vmcnt_all();
    __syncthreads();
    if (i < k.recent) k.store(p, first + i, tid & 15);
  }
}

}  // namespace heisd
