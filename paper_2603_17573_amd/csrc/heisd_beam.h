// Continuations of requests: beam search's choice over beams and vocabulary, and block tables when requests go on as continuations of others.
#pragma once
#include "heisd_common.h"
#include "heisd_paged.h"

namespace heisd {

// ---- the next beams ---------------------------------------------------------------------------------------------------

constexpr int kBeamMost = 64;                       // beams and width at most: a lane each
constexpr int kBeamValues = 32;                     // logits that a thread holds
constexpr int kBeamChunk = 256 * kBeamValues;       // logits that a workgroup takes
constexpr int kBeamKeep = 512;                      // candidates of a workgroup that are ranked among each other

struct BeamArgs {
  const void *logits;
  long long row_stride;
  int groups, beams, width, vocab, chunks, end_token;
  double power;
  const float *score_in;
  const int32_t *length_in, *done_in;
  float *score_out;
  int32_t *beam, *token, *length_out, *done_out, *parent;
  int first, stride;
  float *ms;                                        // [rows][chunks][2]: maximum and sum of a chunk
  float *value;                                     // [rows][chunks][width] the largest logits of a chunk, in order
  int32_t *index;                                   // and their tokens (-1: no more)
};

// Is (v, i) in front of (w, j)?  Larger values first, lower tokens among equals.
__device__ __forceinline__ bool beam_before(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// The best (value, index) of the wave, in every lane.
__device__ __forceinline__ void beam_wave_best(float &v, int &i) {
  const float top = wave_max(v);
  i = (int)wave_min_u(v == top ? (uint32_t)i : 0x7FFFFFFFu);
  v = top;
}

// A chunk of one row: its maximum, its sum of exponentials and its `width` largest logits, with one read of it.  Within a beam scores are logits and
// one constant, so the order of the logits is that of the scores.
template <typename T>
__global__ __launch_bounds__(256) void beam_rows(BeamArgs a) {
  constexpr int V = 16 / sizeof(T), NV = kBeamValues / V;
  __shared__ float s_v[4], s_s[4];
  __shared__ int s_i[4];
  const int row = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x, wave = tid >> 6;
  const long long part = (long long)row * a.chunks + chunk;
  const float before = a.score_in[row];
  if ((a.done_in && a.done_in[row]) || !(before > -INFINITY)) return;       // beam_join does not look here
  const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
  // vectors are aligned whatever the row's address is: the first and the last of a row may be cut
  const int shift = (int)(((uintptr_t)x & 15) / sizeof(T));
  float f[kBeamValues];
  auto token_of = [&](int n) { return chunk * kBeamChunk + ((n / V) * 256 + tid) * V + n % V - shift; };
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int t0 = token_of(k * V);
    if (t0 >= 0 && t0 + V <= a.vocab) load_vec<T, V>(x + t0, f + k * V);
    else {
#pragma unroll
      for (int e = 0; e < V; ++e) f[k * V + e] = t0 + e >= 0 && t0 + e < a.vocab ? (float)x[t0 + e] : -INFINITY;
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int n = 0; n < kBeamValues; ++n) {
    if (!(f[n] > -INFINITY)) f[n] = -INFINITY;      // NaN
    top = fmaxf(top, f[n]);
  }
  top = wave_max(top);
  if ((tid & 63) == 0) s_v[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(s_v[0], s_v[1]), fmaxf(s_v[2], s_v[3]));
  float sum = 0.f;
  if (top > -INFINITY) {
#pragma unroll
    for (int n = 0; n < kBeamValues; ++n) sum += expf(f[n] - top);
  }
  sum = wave_sum(sum);
  if ((tid & 63) == 0) s_s[wave] = sum;
  __syncthreads();
  if (tid == 0) *reinterpret_cast<float2 *>(a.ms + part * 2) = make_float2(top, (s_s[0] + s_s[1]) + (s_s[2] + s_s[3]));
  float last = INFINITY;                            // the one that was taken last
  int last_i = -1;
  for (int n = 0; n < a.width; ++n) {
    float best = -INFINITY;
    int at = 0x7FFFFFFF;
#pragma unroll
    for (int k = 0; k < kBeamValues; ++k) {
      const int i = token_of(k);
      if (f[k] > -INFINITY && beam_before(last, last_i, f[k], i) && beam_before(f[k], i, best, at)) best = f[k], at = i;
    }
    beam_wave_best(best, at);
    __syncthreads();
    if ((tid & 63) == 0) s_v[wave] = best, s_i[wave] = at;
    __syncthreads();
    last = -INFINITY, last_i = 0x7FFFFFFF;
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (beam_before(s_v[w], s_i[w], last, last_i)) last = s_v[w], last_i = s_i[w];
    if (tid == 0) a.value[part * a.width + n] = last, a.index[part * a.width + n] = last > -INFINITY ? last_i : -1;
  }
}

__device__ __forceinline__ double wave_max64(double v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmax(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ double wave_sum64d(double v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// A group's next beams.  A wave joins the chunks of one beam (a lane each); then the beams' candidates, which are in order, are merged by one wave
// (a lane a beam).  Scores are held in 64 bits: what decides between two beams' candidates are differences of sums.
template <int W>
__global__ __launch_bounds__(W * 64) void beam_join(BeamArgs a) {
  __shared__ double s_add[kBeamMost];               // what a beam's logits are added to; its length's power
  __shared__ double s_norm[kBeamMost];
  __shared__ float s_value[kBeamMost * kBeamMost];  // a beam's best logits in order
  __shared__ int s_token[kBeamMost * kBeamMost];
  __shared__ int s_len[kBeamMost], s_done[kBeamMost], s_count[kBeamMost];
  const int g = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int b = wave; b < a.beams; b += W) {
    const int row = g * a.beams + b;
    const float before = a.score_in[row];
    const bool done = a.done_in && a.done_in[row] != 0, alive = before > -INFINITY;
    const int length = (a.length_in ? a.length_in[row] : 0) + !done;
    int count = 0;
    double add = before;
    if (alive && done) {
      if (lane == 0) s_value[b * a.width] = 0.f, s_token[b * a.width] = a.end_token;
      count = 1;
    } else if (alive) {
      const long long part = (long long)row * a.chunks + lane;
      const float2 ms = lane < a.chunks ? *reinterpret_cast<const float2 *>(a.ms + part * 2) : make_float2(-INFINITY, 0.f);
      const float top = wave_max(ms.x);
      const double sum = wave_sum64d(ms.x > -INFINITY && top < INFINITY ? (double)ms.y * exp((double)ms.x - (double)top) : 0.0);
      if (sum > 0) {
        add -= (double)top + log(sum);
        int at = 0;                                 // this lane's chunk has given so many
        for (; count < a.width; ++count) {
          float v = -INFINITY;
          int i = 0x7FFFFFFF;
          if (lane < a.chunks && at < a.width) {
            i = a.index[part * a.width + at];
            v = i < 0 ? -INFINITY : a.value[part * a.width + at];
            if (i < 0) i = 0x7FFFFFFF;
          }
          const int mine = i;
          beam_wave_best(v, i);
          if (!(v > -INFINITY)) break;
          at += mine == i;
          if (lane == 0) s_value[b * a.width + count] = v, s_token[b * a.width + count] = i;
        }
      }
    }
    if (lane == 0) {
      s_add[b] = add;
      s_norm[b] = a.power == 0 ? 1.0 : pow((double)max(length, 1), -a.power);
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
    const double score = at < count ? add + (double)s_value[lane * a.width + at] : -INFINITY;
    const double rank = at < count ? score * norm : -INFINITY;
    const double best = wave_max64(rank);
    const unsigned long long who = __ballot(at < count && rank == best);
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
      const int token = s_token[lane * a.width + at];
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
// minimum does not depend on the order of the atomics).  TABLES: the rows of the table too; otherwise reorder_tables writes them.
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
  }
  if (!TABLES) return;
  __threadfence();
  __syncthreads();
  for (int b = tid >> 6; b < a.batch; b += W) reorder_row(a, b, tid & 63);
}

__global__ __launch_bounds__(256) void reorder_tables(ReorderArgs a) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (b < a.batch) reorder_row(a, b, threadIdx.x & 63);
}

}  // namespace heisd
