// Attention over a prefix that a group of requests shares and over the requests' own tokens, both in the 4-bit cache: the parts of a row, joined.
#pragma once
#include "heisd_common.h"
#include "heisd_kv4.h"
#include "heisd_paged.h"
#include "heisd_prompt.h"

namespace heisd {

// ---- a prefix, for many rows ----------------------------------------------------------------------------------------------

// Values enter the second product as fp16 (and keys the first, where the queries are fp16) where those of a run allow it: times 2^13 over the largest exponent of their
// group of 32 channels (of all keys).  The sixteen codes times 2^-36 of that are still fp16 numbers, so nothing is rounded.  Where exponents lie further apart, or something
// is not finite, all of it is bf16, with probabilities (and fp16 queries) as a bf16 and a remainder.  (Groups of e = 1, 6 2^-126 at most, may become zero beside others.)
constexpr int kWideShift = 13, kWideSpread = 36, kWideTop = 127 + 64;      // (sums of 2^15 times larger values might pass fp32)
template <int HD>
constexpr int wide_lds_bytes = 2 * 2 * kWideTokens * HD * 2 + 2 * kWideTokens;

// softmax(q K^T) V over a run of a prefix's tokens.  A workgroup has 32 * W columns (rows of the group times the query heads of one key head), a wave
// 32 of them; the products are those of prompt_attend.  64 tokens at a time become bf16 once for all columns, on their way into LDS: a lane brings 32
// keys' values of a token, or four tokens' values of eight channels, 16 bytes of codes either way, requested a step ahead and its block's number two.  Which
// bytes of LDS a row's pieces take is as in prompt_attend; K goes by tokens across the lanes and V by channels, so that no two lanes of a write
// meet in a bank.  All columns see the same tokens: what nobody sees (behind the end, in missing blocks) has scores of minus infinity and values of zero.
// Every workgroup takes an equal run of the work of all groups, as in kv4_attend; a unit is a step for 32 * W columns of a key head.
// A probability enters the second product as two 16-bit numbers, itself and what its rounding left: bf16s (off by 2^-16 of it together) or fp16s (2^-21, or 2^-36 of the
// largest), so that a prefix is as exact for many columns as for few.  One fp16 alone takes 87 us for 108, but it is off by up to 2^-11, which nothing averages out: fp16 rows
// are then off by 0.00027 to 0.00029 where their own rounding gives 0.00021, and more bf16 rows get another last bit.
// W 8 where there are as many columns: the tokens become bf16 half as often (two prefixes of 3029 and 3855 tokens, 1792 columns, 8 key heads of 128, bf16: 108 us; with the own
// tokens a call takes 118 to 122, with W 4 137).  51 GFLOP (77 with the second terms) at 470 TFLOP/s: matrix cores busy 31 %, vector units 35 %, the rest waiting, mostly for the
// step's barrier (two waves per SIMD are all that the registers allow).  Tried, with one term: one set of waves bringing tokens before and one after its products (90 for 87), equal
// runs given up for a fixed number of cuts (134 for 120 then).  The scaled products, which take the 4-bit keys as they are, hold their sums to 2^-14 only.
template <typename T, int HD, int W>
__global__ __launch_bounds__(64 * W, 2) void kv4_prefix(Kv4Cache c, PagedBatch b, HeadRows<const T> q, Kv4SharedAttend a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int RB = HD * 2, CH = RB / 16, TILE = kWideTokens * RB, G = HD / 32;
  constexpr int NS = HD / 16, ND = HD / 32, NT = kWideTokens / 32, NK = kWideTokens / 16;
  constexpr int NU = (2 * G + W - 1) / W;           // of a wave's 2 * G lots of 64 lanes' loads
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  __shared__ int2 s_e[W][G + 1];
  const int bs = c.block_size;
  int first = 0;                                    // 64 groups are at hand, a lane each
  Kv4Request mine;
  long long start, end;
  auto groups = [&](long long before) {
    mine = wide_request(c, b, a, min(first + lane, a.prefix.groups - 1));
    if (first + lane >= a.prefix.groups) mine.work = 0, mine.units = 0;
    start = mine.work;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const long long t = __shfl_up(start, o);
      if (lane >= o) start += t;
    }
    end = before + lane_value64(start, 63);
    start += before - mine.work;
  };
  groups(0);
  long long all = end;
  for (int i = 64; i < a.prefix.groups; i += 64) all += wave_sum64(i + lane < a.prefix.groups ? wide_request(c, b, a, i + lane).work : 0);
  const long long per = kv4_run(all, gridDim.x), run0 = blockIdx.x * per, run1 = min(run0 + per, all);
  if (blockIdx.x == gridDim.x - 1) {                // the books for whoever joins the parts
    for (int i = threadIdx.x; i < b.batch; i += 64 * W) a.group_at[i] = -1;
    __syncthreads();
    long long before = 0;
    for (int g0 = 0; g0 < a.prefix.groups; g0 += 64) {
      if (g0) groups(before);
      before = end;
      const int n = min(64, a.prefix.groups - g0);
      if (wave == 0 && lane < n) a.book[g0 + lane] = WideBook{mine.rows.begin, mine.rows.count, mine.units, 0, start, per};
      for (int i = wave; i < n; i += W) {
        if (__builtin_amdgcn_readlane(mine.units, i) == 0) continue;
        const int r0 = a.prefix.first[g0 + i], r1 = a.prefix.first[g0 + i + 1];
        for (int r = r0 + lane; r < r1; r += 64) a.group_at[r] = g0 + i;
      }
      first = g0 + 64;
    }
    if (a.prefix.groups > 64) first = 0, groups(0);
    else first = 0;
  }
  int head = 0, t_begin = 0, t_end = 0;
  const int32_t *table = b.table;

  // what this lane brings of a step: lots 0 .. G - 1 are keys' groups, the others a G-th of the values each
  struct Lot {
    u32x4 code;
    uint32_t e;
    int id;
  };
  Lot lot[NU];
  auto lot_of = [&](int n) { return wave + n * W; };
  auto token_of = [&](int n) {                      // within a step
    if (lot_of(n) < G) return lane;
    const int v = (lot_of(n) - G) * 64 + lane;
    return v / (HD / 8) * 4;
  };
  auto ask_block = [&](int step, int n) {
    const int t = t_begin + step * kWideTokens + token_of(n);
    int id = t < t_end ? table[t >> c.block_shift] : -1;
    return id >= c.n_blocks ? -1 : id;
  };
  auto ask_codes = [&](int step, int n) {
    if (lot_of(n) >= 2 * G) return;
    const int o = (t_begin + step * kWideTokens + token_of(n)) & (bs - 1);
    const uint8_t *cell = c.at(max(lot[n].id, 0), head);
    if (lot_of(n) < G) {
      lot[n].code = *reinterpret_cast<const u32x4 *>(cell + o * (HD / 2) + lot_of(n) * 16);
      lot[n].e = cell[Kv4Offsets<HD>::k_exp(bs) + o * G + lot_of(n)];
    } else {
      const int piece = lane % (HD / 8);
      lot[n].code = *reinterpret_cast<const u32x4 *>(cell + Kv4Offsets<HD>::v_codes(bs) + o / 4 * (2 * HD) + piece * 16);
      lot[n].e = *reinterpret_cast<const uint32_t *>(cell + Kv4Offsets<HD>::v_exp(bs) + (o / 4 * G + piece / 4) * 4);
    }
  };
  auto widen = [&](uint32_t w, uint32_t e) {
    const float s = __uint_as_float(e << 23);
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
    return r;
  };
  int top_e[G], top_k = 0;                          // largest exponent of each group of channels in the run, and of the keys
  auto widen_half = [&](uint32_t w, int e, int top) {
    const float s = __uint_as_float((uint32_t)max(e - top + (127 + kWideShift), 0) << 23);
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3));
    return r;
  };
  auto put = [&](int step, int n, int buf, auto fast) {
    unsigned char *kt = smem + buf * 2 * TILE, *vt = kt + TILE, *seen = smem + 4 * TILE + buf * kWideTokens;
    if (lot_of(n) >= 2 * G) return;
    if (lot_of(n) < G) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        u32x4 x;
        if constexpr (decltype(fast)::value && std::is_same_v<T, _Float16>) x = widen_half(lot[n].code[d], (int)lot[n].e, top_k);
        else x = widen(lot[n].code[d], lot[n].e);
        *reinterpret_cast<u32x4 *>(kt + lane * RB + (((lot_of(n) * 4 + d) ^ prompt_swizzle<CH>(lane)) << 4)) = x;
      }
      if (lot_of(n) == 0) seen[lane] = lot[n].id >= 0;
    } else {
      const int t4 = token_of(n), piece = lane % (HD / 8), left = t_end - (t_begin + step * kWideTokens + t4);
      const bool cut = __ballot(lot[n].id < 0 || left < 4) != 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t w;
        if constexpr (HD == 128) w = lot[n].code[j];
        else w = __builtin_amdgcn_perm(lot[n].code[2 + j / 2], lot[n].code[j / 2], j & 1 ? 0x07060302u : 0x05040100u);
        u32x4 x;
        if constexpr (decltype(fast)::value) {
          int of = top_e[0];
#pragma unroll
          for (int k = 1; k < G; ++k) of = piece / 4 == k ? top_e[k] : of;
          x = widen_half(w, (int)(lot[n].e >> (8 * j) & 255), of);
        } else x = widen(w, lot[n].e >> (8 * j));   // of a scale the conversion reads the exponent only
        if (cut) {
          asm volatile("" ::: "memory");            // a branch
          if (lot[n].id < 0 || j >= left) x = u32x4{0, 0, 0, 0};
        }
        *reinterpret_cast<u32x4 *>(vt + (t4 + j) * RB + ((piece ^ prompt_swizzle<CH>(t4 + j)) << 4)) = x;
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

  for (long long at = run0; at < run1;) {
    while (at >= end && first + 64 < a.prefix.groups) {
      first += 64;
      groups(end);
    }
    if (at >= end) break;                           // not reached while the lengths stay as they are
    const int local = 63 - __clzll(__ballot(start <= at)), g = first + local;      // the last of those that begin here has the work
    const int row0 = __builtin_amdgcn_readlane(mine.rows.begin, local), n_cols = __builtin_amdgcn_readlane(mine.rows.count, local) * a.group;
    const int tokens = __builtin_amdgcn_readlane(mine.seq, local), units = __builtin_amdgcn_readlane(mine.units, local);
    const long long in_group = at - lane_value64(start, local);
    const int segment = __builtin_amdgcn_readfirstlane((int)wave_div(in_group, units));
    const int u0 = __builtin_amdgcn_readfirstlane((int)(in_group - (long long)segment * units));
    const int u1 = __builtin_amdgcn_readfirstlane((int)min((long long)units, u0 + (run1 - at))), steps = u1 - u0;
    const bool whole = steps == units;
    const long long slot = 2 * (long long)blockIdx.x + (at != run0);
    at += steps;
    head = segment % c.kv_heads;
    t_begin = u0 * kWideTokens;
    t_end = min(tokens, u1 * kWideTokens);
    table = b.table + (long long)__builtin_amdgcn_readfirstlane(a.prefix.prefix[g]) * b.max_blocks;
    const int col0 = (segment / c.kv_heads * W + wave) * 32;
    const int my_col = min(col0 + col, n_cols - 1), my_row = row0 + my_col / a.group, my_head = head * a.group + my_col % a.group;

    typename MatrixOf<T>::x8 qf[NS];
    {
      const T *p = q.at(my_row, my_head) + half * 8;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        u32x4 w = *reinterpret_cast<const u32x4 *>(p + s * 16);
        w ^= a.flip ? 0x80008000u : 0u;             // a negative scale: the queries' signs, so that larger products are larger scores
        qf[s] = __builtin_bit_cast(typename MatrixOf<T>::x8, w);
      }
    }
    f32x16 acc[ND];
  #pragma unroll
    for (int d = 0; d < ND; ++d)
  #pragma unroll
      for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;
    float m = -INFINITY, l[4] = {};

    // the run's exponents
    int e_max = 0, e_min = 255;
    for (int i = threadIdx.x; i < (t_end - t_begin + 3) / 4 * G; i += 64 * W) {         // of channels 32 (lane % G) on
      const int t = t_begin + i / G * 4, id = table[t >> c.block_shift];
      if (id < 0 || id >= c.n_blocks) continue;
      const uint32_t e = *reinterpret_cast<const uint32_t *>(c.at(id, head) + Kv4Offsets<HD>::v_exp(bs) + ((t & (bs - 1)) / 4 * G + i % G) * 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int x = t + j < t_end ? (int)(e >> (8 * j) & 255) : 0;
        e_max = max(e_max, x);
        if (x > 1) e_min = min(e_min, x);
      }
    }
#pragma unroll
    for (int o = G; o < 64; o <<= 1) {
      e_max = max(e_max, __shfl_xor(e_max, o));
      e_min = min(e_min, __shfl_xor(e_min, o));
    }
    if (lane < G) s_e[wave][lane] = make_int2(e_max, e_min);
    if constexpr (std::is_same_v<T, _Float16>) {
      e_max = 0, e_min = 255;
      for (int t = t_begin + threadIdx.x; t < t_end; t += 64 * W) {
        const int id = table[t >> c.block_shift];
        if (id < 0 || id >= c.n_blocks) continue;
        const uint8_t *from = c.at(id, head) + Kv4Offsets<HD>::k_exp(bs) + (t & (bs - 1)) * G;
        const uint32_t e = G == 4 ? *reinterpret_cast<const uint32_t *>(from) : *reinterpret_cast<const uint16_t *>(from);
#pragma unroll
        for (int j = 0; j < G; ++j) {
          const int x = (int)(e >> (8 * j) & 255);
          e_max = max(e_max, x);
          if (x > 1) e_min = min(e_min, x);
        }
      }
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        e_max = max(e_max, __shfl_xor(e_max, o));
        e_min = min(e_min, __shfl_xor(e_min, o));
      }
      if (lane == 0) s_e[wave][G] = make_int2(e_max, e_min);
    }
    __syncthreads();                                // LDS is free, too
    bool narrow = true;
#pragma unroll
    for (int k = 0; k < G; ++k) {
      int2 e = s_e[0][k];
#pragma unroll
      for (int w = 1; w < W; ++w) e.x = max(e.x, s_e[w][k].x), e.y = min(e.y, s_e[w][k].y);
      top_e[k] = __builtin_amdgcn_readfirstlane(e.x);
      narrow = narrow && e.x <= kWideTop && e.x - e.y <= kWideSpread;
    }
    if constexpr (std::is_same_v<T, _Float16>) {
      int2 e = s_e[0][G];
#pragma unroll
      for (int w = 1; w < W; ++w) e.x = max(e.x, s_e[w][G].x), e.y = min(e.y, s_e[w][G].y);
      top_k = __builtin_amdgcn_readfirstlane(e.x);
      narrow = narrow && e.x <= kWideTop && e.x - e.y <= kWideSpread;
    }
    narrow = __builtin_amdgcn_readfirstlane(narrow);
    auto walk = [&](auto fast) {
      constexpr bool FAST = decltype(fast)::value;
      constexpr float kLazy = FAST ? MatrixOf<_Float16>::kLazy : kKv4Lazy, kLift = FAST ? MatrixOf<_Float16>::kLift : 0.f;
      const float scale_log2 = FAST && std::is_same_v<T, _Float16> ? fmaxf(ldexpf(a.scale_log2, top_k - (127 + kWideShift)), 1e-37f) : a.scale_log2;      // not 0: minus infinity stands for masked scores
      typedef std::conditional_t<FAST, _Float16, __bf16> PE;
      typedef typename MatrixOf<PE>::x8 P8;
      int next_id[NU];
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        lot[n].id = ask_block(0, n);
        next_id[n] = ask_block(1, n);
        ask_codes(0, n);
      }
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        put(0, n, 0, fast);
        lot[n].id = next_id[n];
        next_id[n] = ask_block(2, n);
        ask_codes(1, n);
      }
      for (int step = 0; step < steps; ++step) {
        const int buf = step & 1;
        __syncthreads();                                // this step's tokens are in LDS, the step's before have been used
        if (step + 1 < steps) {
#pragma unroll
          for (int n = 0; n < NU; ++n) {
            put(step + 1, n, buf ^ 1, fast);
            lot[n].id = next_id[n];
            next_id[n] = ask_block(step + 3, n);
            ask_codes(step + 2, n);
          }
        }
        if (col0 >= n_cols) continue;                   // a wave without columns only brings tokens
        const unsigned char *kt = smem + buf * 2 * TILE, *vt = kt + TILE, *seen = smem + 4 * TILE + buf * kWideTokens;
        const unsigned long long live = __ballot(seen[lane] != 0);
        f32x16 s[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            if constexpr (FAST || std::is_same_v<T, __bf16>)
              s[t] = MatrixOf<T>::mul(*reinterpret_cast<const typename MatrixOf<T>::x8 *>(kt + k_at[n] + t * 32 * RB), qf[n], s[t]);
            else {                                  // fp16 queries as a bf16 and a remainder
              const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(kt + k_at[n] + t * 32 * RB);
              u32x4 held = __builtin_bit_cast(u32x4, qf[n]);
              asm volatile("" : "+v"(held));        // converted in every step: kept, they are 64 registers that have to be spilled
              const typename MatrixOf<T>::x8 qh = __builtin_bit_cast(typename MatrixOf<T>::x8, held);
              bf16x8 hi, lo;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                hi[e] = (__bf16)(float)qh[e];
                lo[e] = (__bf16)((float)qh[e] - (float)hi[e]);
              }
              s[t] = MatrixOf<__bf16>::mul(kf, hi, s[t]);
              s[t] = MatrixOf<__bf16>::mul(kf, lo, s[t]);
            }
          }
        if (live != ~0ull) {
        asm volatile("" ::: "memory");              // a branch: selects would cost every step a hundred instructions
          const unsigned long long my = live >> (4 * half);
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (!(my >> (32 * t + 8 * (e >> 2) + (e & 3)) & 1)) s[t][e] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) top = fmaxf(top, s[t][e]);
        top = max_xor32(top) * scale_log2;
        if (__ballot(top > m + kLazy)) {
          const float next = fmaxf(m, top);
          const float by = next == -INFINITY ? 1.f : exp2_fast(m - next);
          m = next;
#pragma unroll
          for (int i = 0; i < 4; ++i) l[i] *= by;
#pragma unroll
          for (int d = 0; d < ND; ++d) acc[d] *= by;
        }
        const float use = m == -INFINITY ? 0.f : m - kLift;
        P8 pf[NK][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float p0 = exp2_fast(__builtin_fmaf(s[t][e], scale_log2, -use)), p1 = exp2_fast(__builtin_fmaf(s[t][e + 1], scale_log2, -use));
            l[e & 3] += p0;
            l[(e & 3) + 1] += p1;
            typedef __attribute__((ext_vector_type(2))) float f32x2;
            typedef __attribute__((ext_vector_type(2))) PE two;
            uint32_t held = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{p0, p1}, two));
            asm("" : "+v"(held));                   // converted once, and two at a time
            const two hi = __builtin_bit_cast(two, held), lo = __builtin_convertvector(f32x2{p0 - (float)hi[0], p1 - (float)hi[1]}, two);
            P8 *const to = pf[2 * t + (e >> 3)];
            to[0][e & 7] = hi[0], to[0][(e & 7) + 1] = hi[1];
            to[1][e & 7] = lo[0], to[1][(e & 7) + 1] = lo[1];
          }
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + v_at[d][0] + n * 16 * RB));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + v_at[d][1] + n * 16 * RB));
            struct Both { s16x4 a, b; } both = {lo, hi};
            const P8 vf = __builtin_bit_cast(P8, both);
#pragma unroll
            for (int e = 0; e < 2; ++e) acc[d] = MatrixOf<PE>::mul(vf, pf[n][e], acc[d]);
          }
      }
      m -= kLift;
      if constexpr (FAST) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[d][e] = ldexpf(acc[d][e], top_e[d] - (127 + kWideShift));
      }
    };
    if (narrow) walk(std::true_type{});
    else walk(std::false_type{});
    const float sum = sum_xor32((l[0] + l[1]) + (l[2] + l[3]));
    if (col0 + col >= n_cols) continue;
    const long long to = whole ? ((long long)b.rows + my_row) * a.q_heads + my_head : slot * (32 * W) + wave * 32 + col;
    float *o = (whole ? a.whole : a.wide_part) + to * HD;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4 *>(o + d * 32 + e * 8 + half * 4) = f32x4{acc[d][4 * e], acc[d][4 * e + 1], acc[d][4 * e + 2], acc[d][4 * e + 3]};
    if (half == 0) *reinterpret_cast<float2 *>((whole ? a.whole_ml : a.wide_ml) + to * 2) = make_float2(m, sum);
  }
}

// ---- joining ---------------------------------------------------------------------------------------------------------------

// Joins what kv4_attend left of a row: its own tokens' part and its group's prefix', each whole or in parts of several workgroups (wide: only rows whose own
// tokens are in parts).  A workgroup takes some columns (rows times query heads) of a request, 16 bytes of a column per thread.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_shared_join(Kv4Cache c, PagedBatch b, HeadRows<T> out, Kv4SharedAttend a, int grid) {
  const int req = blockIdx.y, lane = threadIdx.x & 63;
  Kv4Parts own{kv4_request(c, b, a, req), 0, 0, a.cols_shift, a.part, a.part_ml}, shared = own;
  const int n_cols = own.r.rows.count * a.q_heads;
  constexpr int PER = 256 / (HD / 4);
  if ((long long)blockIdx.x * PER >= n_cols) return;
  PrefixSpan span;
  const int g = a.wide ? -1 : group_of(c, b, a.prefix, req, &span);
  long long all = 0;
  shared.r.work = 0;
  for (int i = lane; i < kv4_requests(b, a); i += 64) {
    const long long work = kv4_request(c, b, a, i).work;
    all += work;
    if (i < req) own.before += work;
    if (i < b.batch + g) shared.before += work;
  }
  own.before = wave_sum64(own.before);
  own.per = shared.per = kv4_run(wave_sum64(all), grid);
  if (kv4_live(c, b, a, req)) {
    if (a.wide) shared = wide_parts(a, req);
    else if (g >= 0) {
      shared.r = kv4_request(c, b, a, b.batch + g);
      shared.before = wave_sum64(shared.before);
    }
  }
  for (int u = blockIdx.x * PER + threadIdx.x / (HD / 4); u < n_cols; u += gridDim.x * PER) {
    const int d = threadIdx.x % (HD / 4) * 4, i = u / a.q_heads, h = u - i * a.q_heads, head = h / a.group, in_head = h - head * a.group;
    const long long r = own.r.rows.begin + i, at = r * a.q_heads + h, at_prefix = ((long long)b.rows + r) * a.q_heads + h;
    const Kv4Parts::Place mine = own.place(c.kv_heads, head, i * a.group + in_head);
    if (a.wide && mine.w0 == mine.w1) continue;     // done
    Kv4Sums<1> s;
    own.add<HD, 1>(s, mine, d, a.whole + at * HD, a.whole_ml + at * 2);
    const long long in_group = r - shared.r.rows.begin;
    if (shared.r.work && in_group >= 0 && in_group < shared.r.rows.count)
      shared.add<HD, 1>(s, shared.place(c.kv_heads, head, (int)in_group * a.group + in_head), d, a.whole + at_prefix * HD, a.whole_ml + at_prefix * 2);
    s.store(out.at(r, h) + d, a.lse && d == 0 ? a.lse + at : nullptr);
  }
}

// The same where every segment is whole: own tokens, and the runs of the prefix, all kept by row.  Four requests of 32 heads behind 95 tokens 4.1 us (kv4_shared
// 8.7, latency), 64 behind eight prefixes of up to 3158 5.5 (23.6: half of it vector work, mostly widening the prefix for 32 columns).
constexpr int kSplitsMost = 32;
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_direct_join(Kv4Cache c, PagedBatch b, HeadRows<T> out, Kv4SharedAttend a) {
  constexpr int PER = 256 / (HD / 4), K = 8;
  const int req = blockIdx.y;
  const Span rows = wave_span(b.cu_rows, req, b.rows);
  const int n_cols = rows.count * a.q_heads;
  if ((long long)blockIdx.x * PER >= n_cols) return;
  PrefixSpan span{{0, 0}, -1, 0};
  group_of(c, b, a.prefix, req, &span);
  if (!kv4_live(c, b, a, req)) span = PrefixSpan{{0, 0}, -1, 0};
  const int run = span.tokens ? kv4_split(span.tokens, a.split_shift) : 1, runs = (span.tokens + run - 1) / run;
  for (int u = blockIdx.x * PER + threadIdx.x / (HD / 4); u < n_cols; u += gridDim.x * PER) {
    const int d = threadIdx.x % (HD / 4) * 4;
    const long long first = (long long)rows.begin * a.q_heads, at = first + u, apart = (long long)b.rows * a.q_heads;
    const int i = u / a.q_heads, h = u - i * a.q_heads, in_group = rows.begin + i - span.rows.begin;
    const int parts = 1 + (in_group >= 0 && in_group < span.rows.count ? runs : 0);      // own tokens first
    Kv4Sums<1> s;
    for (int p = 0; p < parts; p += K) {
      float2 ml[K];
      f32x4 x[K][1];
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const long long from = at + min(p + k, parts - 1) * apart;
        ml[k] = *reinterpret_cast<const float2 *>(a.whole_ml + from * 2);
        x[k][0] = *reinterpret_cast<const f32x4 *>(a.whole + from * HD + d);
        if (p + k >= parts) ml[k] = make_float2(-INFINITY, 0.f);
      }
      s.add(ml, x);
    }
    s.store(out.at(rows.begin + i, h) + d, a.lse && d == 0 ? a.lse + at : nullptr);
  }
}

// ---- positions -----------------------------------------------------------------------------------------------------------

// Rows of a request whose cached tokens begin later than at 0 (behind a shared prefix, after an eviction): a wave finds the requests of its first row, a
// lane goes on from there.
__global__ __launch_bounds__(256) void offset_positions(PagedBatch b, const int32_t *offset, int32_t *position) {
  const int r0 = blockIdx.x * 256 + (threadIdx.x & ~63), r = r0 + (threadIdx.x & 63);
  if (r0 >= b.rows) return;
  int lo = wave_search(b.batch, r0, [&](int i) { return (long long)b.cu_rows[i]; });
  if (r >= b.rows) return;
  int hi = b.batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (b.cu_rows[mid] <= r) lo = mid;
    else hi = mid - 1;
  }
  const Span s = packed_span(b.cu_rows, lo, b.rows);
  const int p = position[r];
  if (r < s.begin || r >= s.begin + s.count || p < 0) return;
  const long long moved = (long long)p + offset[lo];
  position[r] = moved < 0 || moved > 0x7FFFFFFF ? -1 : (int)moved;
}

}  // namespace heisd
