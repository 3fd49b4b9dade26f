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
  int blocks, head_dim;                             // blocks: of the longest request
};

// One workgroup per block of 16-byte pieces of a request, block and layer.  A block's cells of all heads lie together in the source and in the
// destination; of a block that is not full, only the tiles of 16 tokens that hold tokens are copied.  Sources and destinations are different
// blocks.  Reads and writes (head_dim + head_dim / 16) bytes per token and head.
constexpr int kCopyPieces = 4;
__global__ __launch_bounds__(256) void kv4_copy_blocks(Kv4Cache c, PagedBatch b, CopyArgs a, int per_block) {
  const int req = blockIdx.y, from = a.from[req];
  if (from < 0 || from >= b.batch || from == req) return;
  const int n = b.seq_len[req], j = blockIdx.x / per_block, bs = c.block_size;
  if (n <= 0 || (long long)n > (long long)b.max_blocks * bs || (long long)j * bs >= n) return;
  const int to_id = b.table[(long long)req * b.max_blocks + j], from_id = b.table[(long long)from * b.max_blocks + j];
  if (to_id < 0 || to_id >= c.n_blocks || from_id < 0 || from_id >= c.n_blocks || to_id == from_id) return;
  const int used = min((n - j * bs + 15) & ~15, bs);
  c.pool += blockIdx.z * a.layer_bytes;
  const int piece0 = (blockIdx.x % per_block) * (256 * kCopyPieces) + threadIdx.x;
  const uint8_t *src = c.at(from_id, 0);
  uint8_t *dst = c.at(to_id, 0);
  const int codes = bs * (a.head_dim / 2), all = c.kv_heads * (int)(c.cell / 16);
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
    ok[i] = p < all && o < used * per_token;
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
constexpr int kWeighTokens = 128;                   // per workgroup: 32 per wave

// weight[t] = decay * weight[t] + sum over the rows that see token t and the query heads of its key head of exp(scale q . k - lse).  Scores are one
// matrix product of keys (tokens are rows, held in registers) and the rows' queries (columns, 16 at a time); lane l has column l % 16 and four
// tokens of a tile, adds up its columns' probabilities and the 16 lanes of a token are added at the end.  Every token's weight is written by one wave, whose order of
// additions is fixed.  A token that one of its request's rows brought (the last n) had no weight before.  Queries enter as in the attention.
template <typename T, int HD, int TERMS>
__global__ __launch_bounds__(256) void kv4_weigh(Kv4Cache c, PagedBatch b, PrefixGroups p, HeadRows<const T> q, WeighArgs a) {
  constexpr int KJ = HD / 32;
  const int req = blockIdx.z, head = blockIdx.y, lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), bs = c.block_size;
  const int seq = b.seq_len[req], base = blockIdx.x * kWeighTokens + wave * 32;
  if (seq <= base || seq > max(a.max_seq, p.groups ? p.max_prefix : 0) || (long long)seq > (long long)b.max_blocks * bs) return;
  const Span own = wave_span(b.cu_rows, req, b.rows);
  // keys of 32 tokens
  bf16x8 kf[2][KJ];
  int id[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int t = base + 16 * n;
    id[n] = t < seq ? b.table[(long long)req * b.max_blocks + (t >> c.block_shift)] : -1;
    if (id[n] >= c.n_blocks) id[n] = -1;
    id[n] = __builtin_amdgcn_readfirstlane(id[n]);
    if (id[n] < 0) continue;
    const uint8_t *cell = c.at(id[n], head);
    const int o = (t & (bs - 1)) + col;
    const uint8_t *codes = cell + o * (HD / 2) + quad * (HD / 8);
    const float ks = __uint_as_float((uint32_t)cell[Kv4Offsets<HD>::k_exp(bs) + o * (HD / 32) + quad * (HD / 4) / 32] << 23);
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      const uint32_t w = reinterpret_cast<const uint32_t *>(codes)[j];
      const auto x0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 1),
                 x2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ks, 3);
      kf[n][j][0] = x0[0], kf[n][j][1] = x0[1], kf[n][j][2] = x1[0], kf[n][j][3] = x1[1];
      kf[n][j][4] = x2[0], kf[n][j][5] = x2[1], kf[n][j][6] = x3[0], kf[n][j][7] = x3[1];
    }
  }
  float sum[2][4] = {};
  // all columns of rows [r0, r0 + count), of which row i sees tokens below seen0 + i (causal) or all
  auto add_rows = [&](Span rows, int seen0, bool causal) {
    const int n_cols = rows.count * a.group;
    const int i0 = causal ? max(base - seen0 + 1, 0) : 0;         // rows before see none of these tokens
    for (int c0 = i0 * a.group & ~15; c0 < n_cols; c0 += 16) {
      const int n = min(c0 + col, n_cols - 1), i = n / a.group, h = head * a.group + (n - i * a.group);
      const T *x = q.at(rows.begin + i, h) + quad * (HD / 4);
      const float lse = a.lse[(long long)(rows.begin + i) * a.q_heads + h] * 1.4426950408889634f;
      const int seen = c0 + col >= n_cols || lse == -INFINITY ? 0 : causal ? seen0 + i : seq;
      f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int j = 0; j < KJ; ++j) {
        const auto v = *reinterpret_cast<const typename VecOf<T, 8>::type *>(x + j * 8);
        bf16x8 qf[TERMS];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float f = (float)v[e];
          qf[0][e] = (__bf16)f;
          if constexpr (TERMS == 2) qf[1][e] = (__bf16)(f - (float)qf[0][e]);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < TERMS; ++e) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][j], qf[e], s[t], 0, 0, 0);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float pr = exp2f(__builtin_fmaf(s[t][e], a.scale_log2, -lse));
          sum[t][e] += base + 16 * t + 4 * quad + e < seen ? pr : 0.f;
        }
    }
  };
  if (own.count && seq <= a.max_seq) add_rows(own, seq - own.count + 1, true);
  for (int g0 = 0; g0 < p.groups; g0 += 64) {       // the groups that this request is the prefix of
    unsigned long long mine = __ballot(g0 + lane < p.groups && p.prefix[min(g0 + lane, p.groups - 1)] == req);
    for (; mine; mine &= mine - 1) {
      const PrefixSpan s = prefix_span(c, b, p, g0 + __builtin_ctzll(mine));
      if (s.request == req) add_rows(Span{__builtin_amdgcn_readfirstlane(s.rows.begin), __builtin_amdgcn_readfirstlane(s.rows.count)}, 0, false);
    }
  }
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float fresh = sum16(sum[n][e]);
      const int t = base + 16 * n + 4 * quad + e;
      if (col != 4 * n + e || t >= seq || id[n] < 0) continue;
      const long long at = ((long long)id[n] * c.kv_heads + head) * bs + (t & (bs - 1));
      const float old = t < seq - own.count ? a.weight_in[at] : 0.f;
      a.weight_out[at] = __builtin_fmaf(a.decay, old, fresh);
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

// Of the first n - recent tokens of a request the heaviest stay (in each layer and head for itself), and all of the last `recent`.  Tokens that
// stay and lie behind the first keep - recent places fill the places of those that go, in order; then the last ones move up.  So
// only what has to move is moved: a context at its budget that loses 64 of 2112 tokens moves 64 + the last ones, not 2048.
// One workgroup per request, head and layer.  The threshold is found eight bits at a time (a histogram in LDS; counts do not depend on the order
// of the atomics); holes and fillers are then listed chunk by chunk, both in order, and as many pairs as both lists hold are moved.
template <int HD>
__global__ __launch_bounds__(kEvictThreads) void kv4_evict(Kv4Cache c, PagedBatch b, EvictArgs a) {
  constexpr int N = kEvictThreads, W = N / 64;
  __shared__ uint32_t hist[256], part[W];
  __shared__ uint32_t s_pick[3];
  __shared__ int holes[kEvictQueue + N], fillers[kEvictQueue + N];
  const int head = blockIdx.x, req = blockIdx.y, tid = threadIdx.x, bs = c.block_size;
  const int32_t *table = b.table + (long long)req * b.max_blocks;
  const int n = b.seq_len[req], keep = a.keep[req];
  c.pool += blockIdx.z * a.layer_bytes;
  const float *w_in = a.weight_in + blockIdx.z * a.layer_weights;
  float *w_out = a.weight_out + blockIdx.z * a.layer_weights;
  bool whole = n >= 0 && n <= a.max_seq && (long long)n <= (long long)b.max_blocks * bs;
  bool missing = false;
  if (whole)
    for (int j = tid; (long long)j * bs < n; j += N) missing |= table[j] < 0 || table[j] >= c.n_blocks;
  whole = !__syncthreads_or(missing) && whole;
  const bool cut = whole && keep >= 0 && keep < n;
  if (head == 0 && blockIdx.z == 0 && tid == 0) a.seq_out[req] = cut ? keep : n;
  if (!whole) return;
  auto place = [&](int t) { return ((long long)table[t >> c.block_shift] * c.kv_heads + head) * bs + (t & (bs - 1)); };
  const int recent = min(a.recent, cut ? keep : 0), cand = n - recent, first = keep - recent;   // candidates, and how many of them stay
  if (!cut) {
    if (w_in != w_out)
      for (int t = tid; t < n; t += N) w_out[place(t)] = w_in[place(t)];
    return;
  }
  // the key of the lightest that stays, and how many with that key stay
  uint32_t prefix = 0, left = (uint32_t)first;
  for (int shift = 24; shift >= 0 && first; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int t = tid; t < cand; t += N) {
      const uint32_t key = evict_key(w_in[place(t)]);
      if (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[key >> shift & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      uint32_t sum = 0;
      int d = 255;
      for (; d > 0 && sum + hist[d] < left; --d) sum += hist[d];
      s_pick[0] = prefix | (uint32_t)d << shift;
      s_pick[1] = left - sum;
    }
    __syncthreads();
    prefix = s_pick[0], left = s_pick[1];
    __syncthreads();
  }
  // which tokens stay, chunk by chunk and in order: equal ones from the lowest on
  uint32_t equal_holes = 0, equal_behind = 0;       // tokens with the threshold's key before the chunk, in either region
  for (int t0 = 0; t0 < first; t0 += N) {
    const bool eq = t0 + tid < first && evict_key(w_in[place(t0 + tid)]) == prefix;
    plan_scan<W>((uint32_t)eq, equal_behind, part);
  }
  auto stays = [&](int t, int end, uint32_t &equal_before) {
    const uint32_t key = t < end ? evict_key(w_in[place(t)]) : 0;
    const bool eq = t < end && key == prefix;
    const uint32_t rank = plan_scan<W>((uint32_t)eq, equal_before, part);
    return t < end && first && (key > prefix || (eq && rank <= left));
  };
  const uint32_t behind0 = equal_behind;
  (void)behind0;
  int at_hole = 0, at_filler = first, n_holes = 0, n_fillers = 0;
  auto move_token = [&](int to, int from, int lane16) {
    // 16 lanes move a token: 4 (2) bytes of key codes and of value codes each, exponents by the first
    const int ti = to & (bs - 1), fi = from & (bs - 1);
    uint8_t *d = c.at(table[to >> c.block_shift], head);
    const uint8_t *s = c.at(table[from >> c.block_shift], head);
    const int vd = Kv4Offsets<HD>::v_codes(bs) + (ti / 4) * (2 * HD) + lane16 * (HD / 8) + (ti % 4) * (HD / 32);
    const int vs = Kv4Offsets<HD>::v_codes(bs) + (fi / 4) * (2 * HD) + lane16 * (HD / 8) + (fi % 4) * (HD / 32);
    typedef std::conditional_t<HD == 128, uint32_t, uint16_t> Piece;
    const Piece k = reinterpret_cast<const Piece *>(s + fi * (HD / 2))[lane16], v = *reinterpret_cast<const Piece *>(s + vs);
    uint8_t e = 0;
    const bool is_k = lane16 < HD / 32, is_v = lane16 >= HD / 32 && lane16 < HD / 16;
    const int g = lane16 % (HD / 32);
    const int ed = is_k ? Kv4Offsets<HD>::k_exp(bs) + ti * (HD / 32) + g : Kv4Offsets<HD>::v_exp(bs) + ((ti / 4) * (HD / 32) + g) * 4 + ti % 4;
    const int es = is_k ? Kv4Offsets<HD>::k_exp(bs) + fi * (HD / 32) + g : Kv4Offsets<HD>::v_exp(bs) + ((fi / 4) * (HD / 32) + g) * 4 + fi % 4;
    if (is_k || is_v) e = s[es];
    const float w = w_in[place(from)];
    return [=]() {
      reinterpret_cast<Piece *>(d + ti * (HD / 2))[lane16] = k;
      *reinterpret_cast<Piece *>(d + vd) = v;
      if (is_k || is_v) d[ed] = e;
      if (lane16 == 0) w_out[place(to)] = w;
    };
  };
  while (true) {
    while (n_holes < kEvictQueue && at_hole < first) {
      const int t = at_hole + tid;
      const bool yes = stays(t, first, equal_holes), hole = t < first && !yes;
      uint32_t count = (uint32_t)n_holes;
      const uint32_t rank = plan_scan<W>((uint32_t)hole, count, part);
      if (hole) holes[rank - 1] = t;
      if (yes && w_in != w_out) w_out[place(t)] = w_in[place(t)];
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
    for (int i = tid / 16; i < moves; i += N / 16) move_token(holes[i], fillers[i], tid & 15)();
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
  // the last ones move up; a chunk is read before it is written, and its places lie before those of later chunks
  __syncthreads();
  for (int i0 = 0; i0 < recent; i0 += N / 16) {
    const int i = i0 + tid / 16;
    const bool in = i < recent;
    const auto write = move_token(first + (in ? i : recent - 1), cand + (in ? i : recent - 1), tid & 15);
    __syncthreads();
    if (in) write();
    __syncthreads();
  }
}

}  // namespace heisd
