// Continuations of requests: beam search's choice over beams and vocabulary, and block tables when requests go on as continuations of others.
#pragma once
#include <float.h>
#include "heisd_common.h"
#include "heisd_paged.h"

namespace heisd {

// ---- the next beams ---------------------------------------------------------------------------------------------------

constexpr int kBeamMost = 64;                       // beams and width at most: a lane each
constexpr int kBeamWave = 2048;                     // logits that a wave of beam_scan reads
constexpr int kBeamWaves = 8;                       // waves of a workgroup of beam_pick
constexpr int kBeamList = 448;                      // candidates that a wave ranks at once: up to 256 come at a time
template <typename T>
constexpr int kBeamSegment = 64 * 16 / sizeof(T);   // logits of one load of a wave

struct BeamArgs {
  const void *logits;
  long long row_stride;
  int groups, beams, width, vocab, segments, end_token;   // segments: of a row, a multiple of those that a wave reads
  double power;
  const float *score_in;
  const int32_t *length_in, *done_in;
  float *score_out;
  int32_t *beam, *token, *length_out, *done_out, *parent;
  int first, stride;
  float2 *ms;                                       // [rows][segments / segments of a wave]: maximum and sum of exponentials
  float *top;                                       // [rows][segments] maxima
};

// Is (v, i) in front of (w, j)?  Larger values first, lower tokens among equals.
__device__ __forceinline__ bool beam_before(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// The best (value, index) of the wave, in every lane.
__device__ __forceinline__ void beam_wave_best(float &v, int &i) {
  const float top = wave_max(v);
  i = (int)wave_min_u(v == top ? (uint32_t)i : 0x7FFFFFFFu);
  v = top;
}

// The lane's part of segment s of a row: logits V * lane on of kBeamSegment.  Returns the token of f[0].  What is not there is minus infinity.  Which tokens a lane has does
// not depend on the row's address, so that beams with the same logits have the same sums, bit for bit, and are equal; loads of 16 bytes begin at any element.
template <typename T>
__device__ __forceinline__ int beam_load(const T *x, int vocab, int s, float *f) {
  constexpr int V = 16 / sizeof(T);
  typedef typename VecOf<T, V>::type __attribute__((aligned(sizeof(T)))) vec;
  const int t0 = s * kBeamSegment<T> + (threadIdx.x & 63) * V;
  if (t0 + V <= vocab) {
    const vec v = *reinterpret_cast<const vec *>(x + t0);
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = (float)v[e];
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = t0 + e < vocab ? (float)x[t0 + e] : -INFINITY;
  }
  return t0;
}

// Maxima of N segments of a row from s on, and (maximum, sum of exponentials) of all of them, in every lane.
template <typename T, int N, typename Top>
__device__ __forceinline__ float2 beam_segments(const T *x, int vocab, int s, Top top) {
  constexpr int V = 16 / sizeof(T);
  float f[N * V], m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) beam_load(x, vocab, s + k, f + k * V);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    float mine = -INFINITY;
#pragma unroll
    for (int e = 0; e < V; ++e) mine = fmaxf(mine, f[k * V + e]);       // fmaxf drops NaN
    mine = wave_max(mine);
    top(s + k, mine);
    m = fmaxf(m, mine);
  }
  if (m > -INFINITY) {
#pragma unroll
    for (int e = 0; e < N * V; ++e) {
      const float p = __builtin_amdgcn_exp2f((f[e] - m) * 1.4426950408889634f);
      sum += f[e] == f[e] ? p : 0.f;
    }
  }
  return make_float2(m, wave_sum(sum));
}

// One read of the logits: the sum of exponentials, a wave's part at a time, and the maximum of every segment.  The `width` largest logits of a row lie
// in the `width` segments with the largest maxima (the lower ones among equals: each of them holds a logit that comes before whatever lies outside), so
// nothing else has to be kept.  Bound by memory: 512 rows of 131071 fp16 logits (134 MB) in 30.9 us, 4.3 TB/s (28 with loads at multiples of 16 bytes, whose sums went by the row's
// address: copies of a beam then had other last bits and another order); ranking candidates here, chunk by chunk with a maximum over the workgroup for each, took 181.
template <typename T>
__global__ __launch_bounds__(256) void beam_scan(BeamArgs a) {
  constexpr int N = kBeamWave / kBeamSegment<T>;
  const int row = blockIdx.y, part = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (part * N >= a.segments) return;
  if ((a.done_in && a.done_in[row]) || !(a.score_in[row] > -INFINITY)) return;      // beam_pick does not look here
  const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
  float mine = 0.f;
  const float2 ms = beam_segments<T, N>(x, a.vocab, part * N, [&](int s, float v) { mine = s - part * N == lane ? v : mine; });
  if (lane < N) a.top[(long long)row * a.segments + part * N + lane] = mine;
  if (lane == 0) a.ms[(long long)row * (a.segments / N) + part] = ms;
}

template <int CTRL>
__device__ __forceinline__ double dpp_move64(double v) {
  const unsigned long long u = __double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)u, CTRL, 0xf, 0xf, true), hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xf, 0xf, true);
  return __longlong_as_double((unsigned long long)hi << 32 | lo);
}
// Maximum over the lanes of a row of 16 (rows != 0: over the wave), in every lane.
__device__ __forceinline__ double wave_max64(double v, int rows) {
  v = fmax(v, dpp_move64<kDppXor1>(v));
  v = fmax(v, dpp_move64<kDppXor2>(v));
  v = fmax(v, dpp_move64<kDppHalfMirror>(v));
  v = fmax(v, dpp_move64<kDppMirror>(v));
  if (rows) {
    unsigned long long u = __double_as_longlong(v);
    auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false), hi = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    v = fmax(__longlong_as_double((unsigned long long)hi[0] << 32 | lo[0]), __longlong_as_double((unsigned long long)hi[1] << 32 | lo[1]));
    u = __double_as_longlong(v);
    lo = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false), hi = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    v = fmax(__longlong_as_double((unsigned long long)hi[0] << 32 | lo[0]), __longlong_as_double((unsigned long long)hi[1] << 32 | lo[1]));
  }
  return v;
}
__device__ __forceinline__ double wave_sum64d(double v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// The best `most` of `count` candidates of the wave in LDS, in order, to the front of the list; the new count.
__device__ __forceinline__ int beam_rank(float2 *list, int count, int most) {
  constexpr int K = kBeamList / 64;
  const int lane = threadIdx.x & 63;
  float v[K], last = INFINITY, keep = 0.f;
  int i[K], last_i = -1, keep_i = 0, n = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const float2 c = lane + 64 * k < count ? list[lane + 64 * k] : make_float2(-INFINITY, 0.f);
    v[k] = c.x, i[k] = __float_as_int(c.y);
  }
  for (; n < min(count, most); ++n) {
    float best = -INFINITY;
    int at = 0x7FFFFFFF;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (64 * k >= count) break;
      if (beam_before(last, last_i, v[k], i[k]) && beam_before(v[k], i[k], best, at)) best = v[k], at = i[k];
    }
    beam_wave_best(best, at);
    last = best, last_i = at;
    if (lane == n) keep = best, keep_i = at;
  }
  if (lane < n) list[lane] = make_float2(keep, __int_as_float(keep_i));
  return n;
}

// A group's next beams.  A wave takes a beam: its segments with the largest maxima are read again (eight requested at once), and what is not below the last of
// those maxima is ranked (a list that gets full is cut to the best `width`).  Then the beams' candidates, which are in order, are merged by one wave (a lane a
// beam).  Scores are held in 64 bits: what decides between two beams' candidates are differences of sums.  DIRECT: rows of few segments, which the wave
// reads here for the first time, so that one launch does.  Bound by latency, a chain of loads and maxima over a wave: four beams over 256 bins 8.5 us, of four over
// 32000 11, of eight over 131071 21 to 23 (segments one after the other and 64-bit maxima through LDS: 9.3, 17.5, 30).
template <typename T, bool DIRECT>
__global__ __launch_bounds__(kBeamWaves * 64) void beam_pick(BeamArgs a) {
  constexpr int V = 16 / sizeof(T), N = kBeamWave / kBeamSegment<T>, W = kBeamWaves;
  constexpr int K = DIRECT ? 1 : (1 << 19) / kBeamSegment<T> / 64;      // maxima per lane
  __shared__ float2 s_list[W][kBeamList];
  __shared__ float2 s_best[kBeamMost * kBeamMost];  // a beam's best logits in order, and their tokens
  __shared__ double s_add[kBeamMost], s_norm[kBeamMost];    // what a beam's logits are added to; its length's power
  __shared__ int s_len[kBeamMost], s_done[kBeamMost], s_count[kBeamMost];
  const int g = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int b = wave; b < a.beams; b += W) {
    const int row = g * a.beams + b;
    const float before = a.score_in[row];
    const int ended = a.done_in ? a.done_in[row] : 0, had = a.length_in ? a.length_in[row] : 0;
    float tops[K], m = -INFINITY;
    constexpr int P = DIRECT ? 1 : (1 << 19) / kBeamWave / 64;          // parts per lane
    float2 ms[P];
    if constexpr (!DIRECT) {                        // requested before it is known whether they are wanted
#pragma unroll
      for (int k = 0; k < P; ++k) ms[k] = lane + 64 * k < a.segments / N ? a.ms[(long long)row * (a.segments / N) + lane + 64 * k] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int k = 0; k < K; ++k) tops[k] = lane + 64 * k < a.segments ? a.top[(long long)row * a.segments + lane + 64 * k] : -INFINITY;
    }
    const bool done = ended != 0, alive = before > -INFINITY;
    const int length = had + !done;
    int count = 0;
    double add = before;
    if (alive && done) {
      if (lane == 0) s_best[b * a.width] = make_float2(0.f, __int_as_float(a.end_token));
      count = 1;
    } else if (alive) {
      const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
      double sum = 0;
      if constexpr (DIRECT) {
        tops[0] = -INFINITY;
        for (int s = 0; s < a.segments; s += N) {
          const float2 ms = beam_segments<T, N>(x, a.vocab, s, [&](int at, float v) { tops[0] = at == lane ? v : tops[0]; });
          const float next = fmaxf(m, ms.x);
          if (ms.x > -INFINITY) sum = sum * exp((double)m - (double)next) + (double)ms.y * exp((double)ms.x - (double)next);
          m = next;
        }
      } else {
#pragma unroll
        for (int k = 0; k < P; ++k) m = fmaxf(m, ms[k].x);
        m = wave_max(m);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          if (64 * k >= a.segments / N) break;
          sum += ms[k].x > -INFINITY ? (double)ms[k].y * exp((double)ms[k].x - (double)m) : 0.0;
        }
        sum = wave_sum64d(sum);
      }
      if (m > -INFINITY && m < INFINITY) {
        add -= (double)m + log(sum);
        // the segments, and what a candidate has to reach
        int mine = 0, chosen = 0, last_i = -1;
        float last = INFINITY;
        for (; chosen < a.width; ++chosen) {
          float best = -INFINITY;
          int at = 0x7FFFFFFF;
#pragma unroll
          for (int k = 0; k < K; ++k) {
            if (64 * k >= a.segments) break;
            if (beam_before(last, last_i, tops[k], lane + 64 * k) && beam_before(tops[k], lane + 64 * k, best, at)) best = tops[k], at = lane + 64 * k;
          }
          beam_wave_best(best, at);
          if (!(best > -INFINITY)) break;
          last = best, last_i = at;
          if (lane == chosen) mine = at;
        }
        float floor = chosen == a.width ? last : -INFINITY;
        int floor_i = 0x7FFFFFFF;
        constexpr int B = 8;                        // segments requested at once
        for (int n0 = 0; n0 < chosen; n0 += B) {
          float f[B][V];
          int t0[B];
#pragma unroll
          for (int n = 0; n < B; ++n)
            if (n0 + n < chosen) t0[n] = beam_load(x, a.vocab, __builtin_amdgcn_readlane(mine, n0 + n), f[n]);
#pragma unroll
          for (int n = 0; n < B; ++n) {
            if (n0 + n >= chosen) break;
#pragma unroll
            for (int e0 = 0; e0 < V; e0 += 4) {
              if (count > kBeamList - 256) {
                count = beam_rank(s_list[wave], count, a.width);
                if (count == a.width) floor = s_list[wave][count - 1].x, floor_i = __float_as_int(s_list[wave][count - 1].y);
              }
#pragma unroll
              for (int e = e0; e < e0 + 4; ++e) {
                const bool yes = f[n][e] > -INFINITY && !beam_before(floor, floor_i, f[n][e], t0[n] + e);
                const unsigned long long all = __ballot(yes);
                if (!all) continue;
                if (yes) s_list[wave][count + __popcll(all & ((1ull << lane) - 1))] = make_float2(f[n][e], __int_as_float(t0[n] + e));
                count += __popcll(all);
              }
            }
          }
        }
        count = beam_rank(s_list[wave], count, a.width);
        if (lane < count) s_best[b * a.width + lane] = s_list[wave][lane];
      }
    }
    if (lane == 0) {
      s_add[b] = add;
      s_norm[b] = a.power == 0 ? 1.0 : fmin(fmax(exp(-a.power * log((double)max(length, 1))), DBL_MIN), DBL_MAX);      // not 0 or infinite: a score of 0 would rank as NaN
      s_len[b] = length;
      s_done[b] = done;
      s_count[b] = count;
    }
  }
  __syncthreads();
  if (wave) return;
  int at = 0;
  const bool in = lane < a.beams;
  const double add = in ? s_add[lane] : 0, norm = in ? s_norm[lane] : 0;
  const int count = in ? s_count[lane] : 0;
  for (int n = 0; n < a.width; ++n) {
    const float2 next = at < count ? s_best[lane * a.width + at] : make_float2(0.f, 0.f);
    const double score = at < count ? add + (double)next.x : -INFINITY;
    const double rank = at < count ? score * norm : -INFINITY;
    const double best = wave_max64(rank, a.beams > 16);
    const unsigned long long who = __ballot(at < count && rank == best) & (a.beams > 16 ? ~0ull : 0xFFFFull);      // (of one row: the others hold their own maxima)
    const long long to = (long long)g * a.width + n;
    if (!who) {                                     // no more candidates
      if (lane == 0) {
        a.score_out[to] = -INFINITY;
        a.beam[to] = a.token[to] = -1;
        if (a.length_out) a.length_out[to] = 0;
        if (a.done_out) a.done_out[to] = 1;
        if (a.parent) a.parent[a.first + (long long)g * a.stride + n] = -1;
      }
      continue;
    }
    const int b = __builtin_ctzll(who);
    if (lane == b) {
      const int token = __float_as_int(next.y);
      a.score_out[to] = (float)score;
      a.beam[to] = b;
      a.token[to] = token;
      if (a.length_out) a.length_out[to] = s_len[b];
      if (a.done_out) a.done_out[to] = s_done[b] || (a.end_token >= 0 && token == a.end_token);
      if (a.parent) a.parent[a.first + (long long)g * a.stride + n] = a.first + g * a.stride + b;
      ++at;
    }
  }
}

// ---- requests that continue others ------------------------------------------------------------------------------------

struct ReorderArgs {
  int batch, block_size, max_blocks, n_blocks, trim;
  const int32_t *parent, *len_in, *owned_in, *table_in;
  int32_t *len_out, *owned_out, *table_out, *copy_from, *free_ids;
  const int32_t *free_in;
  int32_t *free_out;
};

__device__ __forceinline__ int reorder_blocks(const ReorderArgs &a, int length) {
  return length <= 0 ? 0 : (int)(((long long)length + a.block_size - 1) / a.block_size);
}
// What is left of a request's blocks when `length` tokens go on in them.
__device__ __forceinline__ int reorder_kept(const ReorderArgs &a, int owned, int length) {
  return a.trim ? min(owned, reorder_blocks(a, length)) : owned;
}

// A wave writes row b of the table: its parent's blocks, or those from the free ones; -1 behind them.
__device__ __forceinline__ void reorder_row(const ReorderArgs &a, int b, int lane) {
  int32_t *row = a.table_out + (long long)b * a.max_blocks;
  const int at = __builtin_amdgcn_readfirstlane(row[0]), owned = __builtin_amdgcn_readfirstlane(a.owned_out[b]);
  const int32_t *from = at < 0 ? a.table_in + (long long)(-1 - at) * a.max_blocks : nullptr;
  for (int j = lane; j < a.max_blocks; j += 64) row[j] = j >= owned ? -1 : from ? from[j] : a.free_ids[at - j];
}

// The books, on one workgroup: who takes its parent's blocks over, what goes back to the free ones, who takes how many of them.  Between the
// passes owned_out holds who goes on in a request's blocks (-1: itself, else the lowest), and the first entry of a row of table_out where its blocks
// are: -1 - parent for those that take them over, else the place of its first one among the free ones.  Everything is a function of the inputs (the
// minimum does not depend on the order of the atomics).  TABLES: the rows of the table too, of no more requests than threads; otherwise reorder_tables
// writes them.  Bound by latency (two sums, six round trips to memory): 6.1 us for four requests on one wave, 11.4 for 128 on four with their tables (8.9 and 4.9 in
// two launches).
template <int W, bool TABLES>
__global__ __launch_bounds__(W * 64) void reorder_books(ReorderArgs a) {
  constexpr int N = W * 64, kNobody = 0x7FFFFFFF;
  __shared__ uint32_t part[W], ends[N];
  __shared__ int lengths[N], skip[N];
  const int tid = threadIdx.x;
  const uint32_t free0 = (uint32_t)min(max(a.free_in[0], 0), a.n_blocks);
  auto heir_of = [&](int p) { return __hip_atomic_load(&a.owned_out[p], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };   // past the cache that the atomics pass
  auto parent_of = [&](int b) {
    const int p = b < a.batch ? a.parent[b] : -1;
    return p < a.batch ? p : -1;
  };
  for (int b = tid; b < a.batch; b += N) __hip_atomic_store(&a.owned_out[b], kNobody, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __threadfence();
  __syncthreads();
  for (int b = tid; b < a.batch; b += N) {
    const int p = parent_of(b);
    if (p >= 0) atomicMin(&a.owned_out[p], p == b ? -1 : b);
  }
  __threadfence();
  __syncthreads();
  // blocks that nobody goes on with, in the order of the requests that had them
  uint32_t back_sum = 0;
  for (int b0 = 0; b0 < a.batch; b0 += N) {
    const int b = b0 + tid;
    int owned = 0, kept = 0;
    if (b < a.batch) {
      owned = min(max(a.owned_in[b], 0), a.max_blocks);
      kept = heir_of(b) == kNobody ? 0 : reorder_kept(a, owned, a.len_in[b]);
    }
    if (!__syncthreads_or(owned - kept)) continue;
    const uint32_t before = back_sum;
    ends[tid] = plan_scan<W>((uint32_t)(owned - kept), back_sum, part);
    lengths[tid] = owned - kept;
    skip[tid] = kept;
    __syncthreads();
    for (uint32_t j = before + tid; j < back_sum && free0 + j < (uint32_t)a.n_blocks; j += N) {
      const int i = plan_owner(ends, N, j);
      a.free_ids[free0 + j] = a.table_in[(long long)(b0 + i) * a.max_blocks + skip[i] + (j - (ends[i] - lengths[i]))];
    }
    back_sum = min(back_sum, (uint32_t)a.n_blocks);
    __syncthreads();
  }
  const int n_free = (int)min(free0 + back_sum, (uint32_t)a.n_blocks);
  // the other continuations take blocks, first come, first served
  uint32_t need_sum = 0, granted = 0;               // blocks asked for, blocks given
  for (int b0 = 0; b0 < a.batch; b0 += N) {
    const int b = b0 + tid, p = parent_of(b);
    const int key = p >= 0 ? heir_of(p) : kNobody;
    const bool heir = p >= 0 && key == (p == b ? -1 : b);
    const int length = p >= 0 ? a.len_in[p] : -1;
    const bool fits = (long long)length <= (long long)a.max_blocks * a.block_size;
    const int need = p >= 0 && !heir && fits ? reorder_blocks(a, length) : 0;
    const uint32_t end = plan_scan<W>((uint32_t)need, need_sum, part);
    need_sum = min(need_sum, (uint32_t)a.n_blocks + 1);
    const bool live = heir || (p >= 0 && fits && (need == 0 || end <= (uint32_t)n_free));
    if (b < a.batch) {
      a.len_out[b] = live ? length : -1;
      a.copy_from[b] = live && need ? (key < 0 ? p : key) : -1;
      a.table_out[(long long)b * a.max_blocks] = heir ? -1 - p : max(n_free - 1 - (int)(end - need), 0);
    }
    ends[tid] = end;
    __syncthreads();
    const int last = plan_owner(ends, N, (uint32_t)n_free);       // the first that gets nothing more
    granted = max(granted, last > 0 ? ends[last - 1] : 0u);
    __syncthreads();
  }
  if (tid == 0) a.free_out[0] = n_free - (int)granted;
  __threadfence();
  __syncthreads();
  for (int b = tid; b < a.batch; b += N) {
    const int at = a.table_out[(long long)b * a.max_blocks];
    const int owned = at < 0 ? reorder_kept(a, min(max(a.owned_in[-1 - at], 0), a.max_blocks), a.len_in[-1 - at])
                             : a.copy_from[b] < 0 ? 0 : reorder_blocks(a, a.len_out[b]);
    a.owned_out[b] = owned;
    if (TABLES) lengths[b] = at, skip[b] = owned;
  }
  if (!TABLES) return;
  __threadfence();
  __syncthreads();
  for (int n = tid; n < a.batch * a.max_blocks; n += N) {
    const int b = n / a.max_blocks, j = n - b * a.max_blocks, at = lengths[b];
    a.table_out[n] = j >= skip[b] ? -1 : at < 0 ? a.table_in[(long long)(-1 - at) * a.max_blocks + j] : a.free_ids[at - j];
  }
}

__global__ __launch_bounds__(256) void reorder_tables(ReorderArgs a) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (b < a.batch) reorder_row(a, b, threadIdx.x & 63);
}

}  // namespace heisd
