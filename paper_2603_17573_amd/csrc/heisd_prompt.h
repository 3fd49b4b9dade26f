// Attention of packed prompts: whole sequences or chunks of them behind earlier rows, grouped heads, causal or not.
#pragma once
#include "heisd_common.h"
#include "heisd_paged.h"

namespace heisd {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;

// kLazy: the running maximum is moved only when it grew by more than this (powers of two).  kLift: a probability is held as 2^kLift times its
// ratio to that maximum, at most 2^(kLazy + kLift).  fp16 is normal from 2^-14 on and ends at 2^16: with 4 and 11 a probability keeps its 11
// bits down to 2^-25 of the largest and is off by at most 2^-36 of it below, which 2^24 of them turn into 2^-12.  With 8 and 0, as bf16 has it,
// 65536 keys of 2^-24.5 of the largest weight got 1.4 times their share beside it, and smaller ones nothing.  Five chunks of up to 276 rows, fp16, heads of
// 64: 15.9 us with 8 and 0, 16.0 with 8 and 7, 16.3 with 4 and 11, 16.7 with 2 and 13 (the maximum moves more often).
template <typename T>
struct MatrixOf;
template <>
struct MatrixOf<__bf16> {
  typedef bf16x8 x8;
  static __device__ __forceinline__ f32x16 mul(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static constexpr uint32_t kExp = 0x7F807F80u, kOne = 0x00800080u;
  static constexpr float kLazy = 8.f, kLift = 0.f;
};
template <>
struct MatrixOf<_Float16> {
  typedef f16x8 x8;
  static __device__ __forceinline__ f32x16 mul(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static constexpr uint32_t kExp = 0x7C007C00u, kOne = 0x04000400u;
  static constexpr float kLazy = 4.f, kLift = 11.f;
};
// Nonzero if one of two 16-bit floats has an exponent of ones (infinite or NaN).
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t two) {
  return ((two & MatrixOf<T>::kExp) + MatrixOf<T>::kOne) & 0x80008000u;
}

constexpr int kPromptRows = 128, kPromptKeys = 64, kPromptWaves = 4;

// The join of two sets takes less than their buffers.
template <int HD>
constexpr int prompt_lds_bytes(int split) { return split * 2 * 2 * kPromptKeys * HD * 2; }

// Where the 16-byte pieces of an LDS row go: piece c of row r lies at c ^ prompt_swizzle(r).  A read of K takes the same piece of 16
// rows at a time, a transposed read of V 64 bytes of four rows: both must meet all 64 banks once.  A row of 256 bytes is all banks, of
// 128 bytes half of them; the two lowest bits of r that leave the banks as they are move the 64-byte piece.
template <int CH>
__device__ __forceinline__ int prompt_swizzle(int r) {
  return CH == 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 2) & 3);
}

struct PromptArgs {
  const int32_t *cu_q, *cu_k;
  const int32_t *seq_len;                           // NULL, or negative for sequences that are to see nothing
  int batch, rows, k_rows, q_heads, kv_heads, group;
  int tiles;                                        // row tiles in the grid
  float scale_log2;                                 // magnitude of the softmax scale times log2(e)
  uint32_t flip;                                    // 0x80008000 where the scale is negative
  float *lse;
};

// The plain loop, for the rows of a wave that met a value that is not finite among masked ones: a matrix product would multiply it
// by a probability of zero, which is NaN.  One token after the other, 64 lanes over the channels.
template <typename T, int HD, bool CAUSAL>
__device__ __forceinline__ void prompt_rows_plain(HeadRows<const T> q, HeadRows<const T> k, HeadRows<const T> v, HeadRows<T> out, PromptArgs a,
                                               int row0, int n_rows, int head, int k_row0, int n_keys, int shift) {
  constexpr int V = HD / 64;
  const int lane = threadIdx.x & 63, kvh = head / a.group;
  for (int i = 0; i < n_rows; ++i) {
    float x[V], y[V], o[V] = {}, m = -INFINITY, l = 0.f;
    load_vec<T, V>(q.at(row0 + i, head) + lane * V, x);
    const int seen = CAUSAL ? min(n_keys, shift + i + 1) : n_keys;
    for (int t = 0; t < seen; ++t) {
      load_vec<T, V>(k.at(k_row0 + t, kvh) + lane * V, y);
      float s = 0.f;
      for (int n = 0; n < V; ++n) s += x[n] * y[n];
      s = wave_sum(s) * (a.flip ? -a.scale_log2 : a.scale_log2);
      load_vec<T, V>(v.at(k_row0 + t, kvh) + lane * V, y);
      const float next = fmaxf(m, s), use = next == -INFINITY ? 0.f : next;
      const float by = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - use), p = __builtin_amdgcn_exp2f(s - use);
      m = next;
      l = l * by + p;
      for (int n = 0; n < V; ++n) o[n] = o[n] * by + p * y[n];
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    for (int n = 0; n < V; ++n) o[n] *= inv;
    store_vec<T, V>(out.at(row0 + i, head) + lane * V, o);
    if (a.lse && lane == 0) a.lse[(long long)(row0 + i) * a.q_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
  }
}

// softmax(q K^T) V.  A workgroup has 128 rows of one sequence and head, a wave 32 of them as the columns of its products:
// scores^T = K q^T (64 keys at a time), out^T = V^T p^T.  A lane then holds 32 scores of one row, so maximum and sum need one exchange
// (with lane + 32), rescaling is a multiplication by the lane's own factor, and the probabilities are the second product's
// operand as they stand: its eight summed indices per lane are two runs of four keys, and the transposed LDS read delivers V in just that
// order.  K and V go to LDS by direct transfers, two buffers, one barrier per 64 keys; 16-byte pieces are permuted within a row by
// the row's number so that neither read meets bank conflicts.  SPLIT 2: two such sets of four waves, each with buffers of its own, take every
// other block of keys and are joined through LDS: half as many steps one after the other, for calls too small to fill the chip.
// A probability enters the second product as one number of the rows' type.  That rounding is as large as the result's own and makes the error against
// 64 bits up to 1.3 times what a single rounding leaves (bf16 prompts 0.0021 for 0.0016, fp16 chunks 0.00026 for 0.00021); a remainder as a second product, as the
// attention over the cache has it, would take 477 us for 363 with packed prompts and 22.4 for 16.7 with chunks, for it is bound by these products.
// Packed causal prompts of 15805 rows, 32 heads of 128 over 8, bf16: 362 to 370 us (866 to 885 TFLOP/s at 1.95 to 2.1 GHz, which is what the chip
// clocks meanwhile).  The matrix cores are busy 44 % of that, the vector units (exponents, sums, maxima) about as much, LDS 23 % without
// conflicts: a wave does one after the other, the two waves of a SIMD fall into step, and a quarter of the wave cycles is waiting for data or a barrier.
template <typename T, int HD, bool CAUSAL, int SPLIT>
__global__ __launch_bounds__(256 * SPLIT, HD == 64 && SPLIT == 1 ? 3 : 2) void prompt_attend(HeadRows<const T> q, HeadRows<const T> k, HeadRows<const T> v,
                                                                                             HeadRows<T> out, PromptArgs a) {
  typedef typename MatrixOf<T>::x8 x8;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int RB = HD * 2, CH = RB / 16, TILE = kPromptKeys * RB;                // bytes of a row, 16-byte pieces of it, a tile
  constexpr int NS = HD / 16, ND = HD / 32, NT = kPromptKeys / 32, NK = kPromptKeys / 16;
  const int wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), set = wave8 / kPromptWaves, wave = wave8 % kPromptWaves;
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int kvh = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads;
  const int head = kvh * a.group + rest % a.group, tile = a.tiles - 1 - rest / a.group;
  // which sequence: sequence i is given tiles floor(cu[i] / 128) + i and on, enough for any length
  const int seq = wave_search(a.batch, tile, [&](int i) { return (long long)max(a.cu_q[i], 0) / kPromptRows + i; });
  const Span rows = wave_span(a.cu_q, seq, a.rows);
  Span keys = wave_span(a.cu_k, seq, a.k_rows);
  if (a.seq_len && __builtin_amdgcn_readfirstlane(a.seq_len[seq]) < 0) keys.count = 0;
  const int first = (tile - (rows.begin / kPromptRows + seq)) * kPromptRows;
  if (first < 0 || first >= rows.count) return;
  const int shift = CAUSAL ? keys.count - rows.count : 0;                          // row i sees keys 0 .. shift + i
  const int n_keys = CAUSAL ? max(min(keys.count, shift + min(first + kPromptRows, rows.count)), 0) : keys.count;
  const int mine = first + wave * 32, my_rows = min(max(rows.count - mine, 0), 32);   // the wave's rows
  const int my_row = min(mine + col, rows.count - 1);
  const int seen = CAUSAL ? min(keys.count, shift + my_row + 1) : keys.count;
  const int all_see = CAUSAL ? min(keys.count, shift + mine + 1) : keys.count;        // keys that every row of the wave sees
  const int some_see = CAUSAL ? min(n_keys, shift + min(mine + 32, rows.count)) : keys.count;   // ... that some row sees

  x8 qf[NS];
  {
    const T *p = q.at(rows.begin + my_row, head) + half * 8;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      u32x4 w = *reinterpret_cast<const u32x4 *>(p + s * 16);
      w ^= a.flip;                                  // a negative scale: the queries' signs, so that larger products are larger scores
      qf[s] = __builtin_bit_cast(x8, w);
    }
  }
  f32x16 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;
  float m = -INFINITY, l[4] = {};                   // the row's maximum so far (powers of two), parts of its sum
  uint32_t odd = 0;

  const unsigned char *mine_lds = smem + set * 4 * TILE;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem + set * 4 * TILE;
  constexpr int RP = 1024 / RB, NP = kPromptKeys / RP / kPromptWaves;              // rows per transfer, transfers per wave and matrix
  constexpr int STEP = RP * kPromptWaves;                                          // rows from one transfer of a wave to its next
  const int lane_row = wave * RP + lane / CH, lane_chunk = (lane % CH) ^ prompt_swizzle<CH>(lane_row);   // STEP is a multiple of 16
  const uint32_t k_off = (uint32_t)(lane_row * k.rs + lane_chunk * 8) * sizeof(T), v_off = (uint32_t)(lane_row * v.rs + lane_chunk * 8) * sizeof(T);
  const T *k_next = k.at(keys.begin + set * kPromptKeys, kvh), *v_next = v.at(keys.begin + set * kPromptKeys, kvh);   // the next transfer's first row
  auto stage = [&](int block, int buf) __attribute__((always_inline)) {
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + buf * 2 * TILE + wave * 1024);
    if ((block + 1) * kPromptKeys <= n_keys) {
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        lds_dma16_s(k_next, k_off, to + n * kPromptWaves * 1024);
        lds_dma16_s(v_next, v_off, to + TILE + n * kPromptWaves * 1024);
        k_next += STEP * k.rs;
        v_next += STEP * v.rs;
      }
      k_next += (SPLIT - 1) * kPromptKeys * k.rs;
      v_next += (SPLIT - 1) * kPromptKeys * v.rs;
    } else {                                        // past the end: the last row again, masked
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        const long long row = keys.begin + min(block * kPromptKeys + n * STEP + lane_row, n_keys - 1);
        lds_dma16(k.at(row, kvh) + lane_chunk * 8, to + n * kPromptWaves * 1024);
        lds_dma16(v.at(row, kvh) + lane_chunk * 8, to + TILE + n * kPromptWaves * 1024);
      }
    }
  };
  // byte offsets of the lane's reads; rows further on are constants away
  uint32_t k_at[NS], v_at[ND][2];
#pragma unroll
  for (int s = 0; s < NS; ++s) k_at[s] = col * RB + (((2 * s + half) ^ prompt_swizzle<CH>(col)) << 4);
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = 8 * e + 4 * half + ((lane & 15) >> 2), chunk = d * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
      v_at[d][e] = row * RB + ((chunk ^ prompt_swizzle<CH>(row)) << 4) + (lane & 1) * 8;
    }

  const int n_blocks = (n_keys + kPromptKeys - 1) / kPromptKeys;
  wait_vmcnt_all();
  if (set < n_blocks) stage(set, 0);
  for (int step = 0; step * SPLIT < n_blocks; ++step) {
    const int blk = step * SPLIT + set, buf = step & 1, base = blk * kPromptKeys;
    wait_vmcnt<0>();
    __syncthreads();
    if (blk + SPLIT < n_blocks) stage(blk + SPLIT, buf ^ 1);
    if (base >= some_see) continue;                 // some_see is at most n_keys: a set's last block may not be there
    const unsigned char *kt = mine_lds + buf * 2 * TILE, *vt = kt + TILE;
    f32x16 s[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        s[t] = MatrixOf<T>::mul(*reinterpret_cast<const x8 *>(kt + k_at[n] + t * 32 * RB), qf[n], s[t]);
    if (base + kPromptKeys > all_see) {             // some row must not see some of these keys
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (base + 32 * t + 8 * (e >> 2) + 4 * half + (e & 3) >= seen) s[t][e] = -INFINITY;
#pragma unroll 4
      for (int i = 0; i < TILE / 1024; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4 *>(vt + i * 1024 + lane * 16);
        odd |= not_finite<T>(w[0]) | not_finite<T>(w[1]) | not_finite<T>(w[2]) | not_finite<T>(w[3]);
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[t][e]);
    top = max_xor32(top) * a.scale_log2;
    if (__ballot(top > m + MatrixOf<T>::kLazy)) {
      const float next = fmaxf(m, top);
      const float by = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - next);
      m = next;
#pragma unroll
      for (int i = 0; i < 4; ++i) l[i] *= by;
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[d] *= by;
    }
    const float use = m == -INFINITY ? 0.f : m - MatrixOf<T>::kLift;
    x8 pf[NK];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], a.scale_log2, -use));
        l[e & 3] += p;
        pf[2 * t + (e >> 3)][e & 7] = (T)p;
      }
#pragma unroll
    for (int n = 0; n < NK; ++n)
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + v_at[d][0] + n * 16 * RB));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + v_at[d][1] + n * 16 * RB));
        struct Both { s16x4 a, b; } both = {lo, hi};
        const x8 vf = __builtin_bit_cast(x8, both);
        acc[d] = MatrixOf<T>::mul(vf, pf[n], acc[d]);
      }
  }
  if constexpr (SPLIT == 2) {                       // the second set's sums through LDS, a register after the other
    __syncthreads();
    float *to = reinterpret_cast<float *>(smem) + wave * 64 + lane;
    if (set) {
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) to[(d * 16 + e) * 256] = acc[d][e];
      to[ND * 16 * 256] = m;
      to[(ND * 16 + 1) * 256] = (l[0] + l[1]) + (l[2] + l[3]);
      to[(ND * 16 + 2) * 256] = __uint_as_float(odd);
    }
    __syncthreads();
    if (set) return;
    const float m2 = to[ND * 16 * 256], next = fmaxf(m, m2);
    const float by = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - next), by2 = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m2 - next);
    m = next;
    l[0] = ((l[0] + l[1]) + (l[2] + l[3])) * by + to[(ND * 16 + 1) * 256] * by2;
    l[1] = l[2] = l[3] = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[d][e] = acc[d][e] * by + to[(d * 16 + e) * 256] * by2;
    odd |= __float_as_uint(to[(ND * 16 + 2) * 256]);
  }
  if (my_rows == 0) return;
  if (__ballot(odd != 0)) {
    prompt_rows_plain<T, HD, CAUSAL>(q, k, v, out, a, rows.begin + mine, my_rows, head, keys.begin, keys.count, shift + mine);
    return;
  }
  const float sum = sum_xor32((l[0] + l[1]) + (l[2] + l[3]));
  if (col >= my_rows) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const long long r = rows.begin + mine + col;
  T *o = out.at(r, head);
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = acc[d][4 * e + i] * inv;
      store_vec<T, 4>(o + d * 32 + e * 8 + half * 4, f);
    }
  if (a.lse && half == 0) a.lse[r * a.q_heads + head] = sum == 0.f ? -INFINITY : (m - MatrixOf<T>::kLift + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace heisd
