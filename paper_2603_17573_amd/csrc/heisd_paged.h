// Requests that share one pool of cache blocks: block tables, slots and positions from their lengths, and rotary positions
// of packed rows.
#pragma once
#include "heisd_common.h"

namespace heisd {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// Rows of heads as a caller lays them out: element (r, h, i) at p[r * rs + h * hs + i].
template <typename T>
struct HeadRows {
  T *p;
  long long rs, hs;
  __device__ __forceinline__ T *at(long long r, int h) const { return p + r * rs + h * hs; }
};

// n / d for n < 2^32 / d by one multiplication (mul = 0 stands for d = 1).
struct FastDiv {
  uint32_t mul;
  explicit FastDiv(uint32_t d) : mul(d <= 1 ? 0 : (uint32_t)(0x100000000ull / d) + 1) {}
  __device__ __forceinline__ uint32_t of(uint32_t n) const { return mul ? __umulhi(n, mul) : n; }
};

// The last i in [0, n) with key(i) <= want, for keys that do not decrease; 0 if there is none.  A whole wave searches: a round
// of 64 pivots divides what is left by 64.
template <typename Key>
__device__ __forceinline__ int wave_search(int n, long long want, Key key) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;
  while (len > 1) {
    const int step = (len + 63) >> 6;
    const int at = lo + lane * step;
    const bool le = lane * step < len && key(at) <= want;
    const unsigned long long m = __ballot(le);
    const int last = m ? 63 - __clzll(m) : 0;
    lo += last * step;
    len = min(step, len - last * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Rows [begin, begin + count) of sequence i of n packed in `rows` rows, as cu says; count 0 where cu makes no sense.
struct Span {
  int begin, count;
};
__device__ __forceinline__ Span packed_span(const int32_t *cu, int i, int rows) {
  const int a = cu[i], b = cu[i + 1];
  return (a < 0 || b < a || b > rows) ? Span{0, 0} : Span{a, b - a};
}

// The same for a sequence that is the whole wave's, in scalar registers.
__device__ __forceinline__ Span wave_span(const int32_t *cu, int i, int rows) {
  const Span s = packed_span(cu, i, rows);
  return Span{__builtin_amdgcn_readfirstlane(s.begin), __builtin_amdgcn_readfirstlane(s.count)};
}

// ---- block tables, slots and positions ---------------------------------------------------------------------------

struct PlanArgs {
  int batch, block_size, max_blocks, n_blocks, rows;
  const int32_t *cached, *fresh, *owned_in;
  int32_t *owned_out, *table, *free_ids;
  const int32_t *free_in;
  int32_t *free_out, *cu_rows, *seq_len, *slot, *position, *cu_seq;
};

// Inclusive sum over a workgroup of W waves, plus `carry`; carry becomes the total.  part: W values of LDS.
template <int W, typename N>
__device__ __forceinline__ N plan_scan(N v, N &carry, N *part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const N t = __shfl_up(v, o);
    if (lane >= o) v += t;
  }
  if (W == 1) {
    v += carry;
    carry = __shfl(v, 63);
    return v;
  }
  if (lane == 63) part[wave] = v;
  __syncthreads();
  N before = carry, total = carry;
#pragma unroll 4
  for (int w = 0; w < W; ++w) {
    const N x = part[w];
    if (w < wave) before += x;
    total += x;
  }
  __syncthreads();
  carry = total;
  return v + before;
}

// The first i of n values in LDS that do not decrease with end[i] > want (n: none).
template <typename N>
__device__ __forceinline__ int plan_owner(const N *end, int n, N want) {
  int lo = 0;
  while (lo < n) {
    const int mid = (lo + n) >> 1;
    if (end[mid] > want) n = mid;
    else lo = mid + 1;
  }
  return lo;
}

// The slot and the position of row r, which is row `i` of request b's new rows.
__device__ __forceinline__ void plan_row(const PlanArgs &a, int r, int cached, int i, int b, bool live) {
  int slot = -1, pos = -1;
  if (live) {
    pos = cached + i;
    const int blk = pos / a.block_size;
    const int id = a.table[(long long)b * a.max_blocks + blk];
    if (id >= 0 && id < a.n_blocks) slot = id * a.block_size + (pos - blk * a.block_size);
  }
  a.slot[r] = slot;
  a.position[r] = pos;
}

// One workgroup keeps the books: prefix sums over the requests decide who gets which free block.  Blocks that finished requests
// give back go on top of the free ones first; a request that needs blocks then takes them from the top, first come, first
// served.  Everything is a function of the inputs alone, so the outputs may be the inputs' own buffers.  A request per thread for the
// sums; then a block (or a row) per thread, which finds its request by bisection in LDS: with a wave per request, each waited for its own
// few blocks (512 requests: 17.7 us).  SLOTS: the rows' slots too; otherwise plan_slots fills them.  Sums of rows are held in 64 bits; those
// of blocks stay below 2^32 because a request has at most 2^20 and the carries are clamped.  Bound by latency: three sums and four
// round trips to memory, 3.9 us for one request on one wave (10.7 on sixteen), 10.2 for 512 requests of which a quarter are prompts; plan_slots
// takes 4.0 more for their 56260 rows.
template <int W, bool SLOTS>
__global__ __launch_bounds__(W * 64) void plan_books(PlanArgs a) {
  constexpr int N = W * 64;
  __shared__ uint32_t part[W], ends[N];
  __shared__ unsigned long long wide[W], row_ends[N];
  __shared__ int firsts[N], lengths[N];
  const int tid = threadIdx.x;
  const uint32_t free0 = (uint32_t)min(max(a.free_in[0], 0), a.n_blocks);
  // finished requests' blocks
  uint32_t back_sum = 0;
  for (int b0 = 0; b0 < a.batch; b0 += N) {
    const int b = b0 + tid;
    const int back = b < a.batch && a.cached[b] < 0 ? min(max(a.owned_in[b], 0), a.max_blocks) : 0;
    if (!__syncthreads_or(back)) continue;
    const uint32_t before = back_sum;
    ends[tid] = plan_scan<W>((uint32_t)back, back_sum, part);
    lengths[tid] = back;
    __syncthreads();
    for (uint32_t j = before + tid; j < back_sum && free0 + j < (uint32_t)a.n_blocks; j += N) {
      const int i = plan_owner(ends, N, j);
      a.free_ids[free0 + j] = a.table[(long long)(b0 + i) * a.max_blocks + (j - (ends[i] - lengths[i]))];
    }
    back_sum = min(back_sum, (uint32_t)a.n_blocks);
    __syncthreads();
  }
  const uint32_t n_free = min(free0 + back_sum, (uint32_t)a.n_blocks);
  unsigned long long row_sum = 0, seq_sum = 0;
  uint32_t need_sum = 0, granted = 0;               // blocks asked for, blocks given
  const unsigned long long rows = (unsigned long long)a.rows;
  for (int b0 = 0; b0 < a.batch; b0 += N) {
    const int b = b0 + tid;
    const bool in = b < a.batch;
    const int cached = in ? a.cached[b] : -1, fresh = in ? a.fresh[b] : 0;
    const int owned = in ? min(max(a.owned_in[b], 0), a.max_blocks) : 0;
    const unsigned long long n = (unsigned long long)max(fresh, 0);
    const unsigned long long rows_before = row_sum, row_end = plan_scan<W>(n, row_sum, wide);
    const long long total = (long long)cached + fresh;
    bool live = in && cached >= 0 && fresh >= 0 && total <= (long long)a.max_blocks * a.block_size && row_end <= rows;
    int need = live ? max((int)((total + a.block_size - 1) / a.block_size) - owned, 0) : 0;
    const uint32_t need_end = plan_scan<W>((uint32_t)need, need_sum, part);
    need_sum = min(need_sum, (uint32_t)a.n_blocks + 1);
    live = live && (need == 0 || need_end <= n_free);
    const unsigned long long seq_end = plan_scan<W>(live ? (unsigned long long)total : 0ull, seq_sum, wide);
    if (in) {
      if (b == 0) {
        a.cu_rows[0] = 0;
        if (a.cu_seq) a.cu_seq[0] = 0;
      }
      a.cu_rows[b + 1] = (int)min(row_end, rows);
      a.seq_len[b] = live ? (int)total : -1;
      if (a.cu_seq) a.cu_seq[b + 1] = (int)min(seq_end, 0x7FFFFFFFull);
      a.owned_out[b] = cached < 0 ? 0 : owned + (live ? need : 0);
    }
    // requests are granted in order until one is refused: what they get is a run of the free blocks
    ends[tid] = need_end;
    firsts[tid] = need;
    lengths[tid] = owned;
    __syncthreads();
    const int last = plan_owner(ends, N, n_free);     // the first that gets nothing more
    const uint32_t upto = last > 0 ? ends[last - 1] : granted;
    for (uint32_t j = granted + tid; j < upto; j += N) {
      const int i = plan_owner(ends, N, j);
      a.table[(long long)(b0 + i) * a.max_blocks + lengths[i] + (j - (ends[i] - firsts[i]))] = a.free_ids[n_free - 1 - j];
    }
    granted = max(granted, upto);
    __syncthreads();
    if (SLOTS) {
      row_ends[tid] = row_end;
      firsts[tid] = live ? cached : -1;
      ends[tid] = (uint32_t)min(n, rows);
      __syncthreads();
      for (unsigned long long r = rows_before + tid; r < min(row_sum, rows); r += N) {
        const int i = plan_owner(row_ends, N, r);
        plan_row(a, (int)r, firsts[i], (int)(r - (row_ends[i] - ends[i])), b0 + i, firsts[i] >= 0);
      }
      __syncthreads();
    }
  }
  if (SLOTS)
    for (int r = (int)min(row_sum, rows) + tid; r < a.rows; r += N) {
      a.slot[r] = -1;
      a.position[r] = -1;
    }
  if (tid == 0) a.free_out[0] = (int)(n_free - granted);
}

// Slots and positions of many rows: a wave finds the requests of its first and its last row, a lane those between.
__global__ __launch_bounds__(256) void plan_slots(PlanArgs a) {
  const int r0 = (blockIdx.x * 256 + (threadIdx.x & ~63));
  if (r0 >= a.rows) return;
  auto begin = [&](int i) { return (long long)a.cu_rows[i]; };
  int lo = wave_search(a.batch, r0, begin);
  const int r = r0 + (threadIdx.x & 63);
  int hi = lo;
  if (a.cu_rows[lo + 1] < r0 + 64) hi = wave_search(a.batch, r0 + 63, begin);
  if (r >= a.rows) return;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.cu_rows[mid] <= r) lo = mid;
    else hi = mid - 1;
  }
  const int at = a.cu_rows[lo];
  plan_row(a, r, a.cached[lo], r - at, lo, r < a.cu_rows[lo + 1] && a.seq_len[lo] >= 0);
}

// ---- rotary positions -----------------------------------------------------------------------------------------------

struct RopeArgs {
  const double *turns;            // turns per position of every pair
  float magnitude;                // what cos and sin are multiplied by; its sine is negated for the transposed rotation
  float sine;
  const int32_t *position;
  int rows, pairs, rest, q_heads, heads, per_group;   // rest: elements of a head behind the rotated ones (0: nothing to copy)
  FastDiv by_units;               // units of work per head
  int units;
  FastDiv by_row;                 // units of work per row
};

constexpr int kRopeThreads = 256, kRopePairs = 256;

template <typename T, int V>
struct VecOf {
  typedef __attribute__((ext_vector_type(V))) T type;
};
template <typename T>
struct VecOf<T, 1> {
  typedef T type;
};
template <typename T, int V>
__device__ __forceinline__ void load_vec(const T *p, float *x) {
  if constexpr (V == 1) x[0] = (float)p[0];
  else {
    const typename VecOf<T, V>::type v = *reinterpret_cast<const typename VecOf<T, V>::type *>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (float)v[i];
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T *p, const float *x) {
  if constexpr (V == 1) p[0] = (T)x[0];
  else {
    typename VecOf<T, V>::type v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (T)x[i];
    *reinterpret_cast<typename VecOf<T, V>::type *>(p) = v;
  }
}

// The same past the caches' keeping: rows that are written once and are too many to stay.
template <typename T, int V>
__device__ __forceinline__ void store_vec_once(T *p, const float *x) {
  typename VecOf<T, V>::type v;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = (T)x[i];
  __builtin_nontemporal_store(v, reinterpret_cast<typename VecOf<T, V>::type *>(p));
}

// (a, b) -> (a cos - b sin, b cos + a sin) for every pair of a row's heads.  The angle is position * frequency, reduced in 64
// bits to a fraction of a turn (at position 100000 a 32-bit product is off by 1e-3 of a radian), then sine and cosine in 32 (off by 2^-22
// at most: fp32 rows come out 3.7e-8 off, with sines of 64 bits 3.0e-8).
// They are the same for all heads of a row: a workgroup computes them once into LDS, then every thread turns V pairs at a
// time, 16 bytes per access.  Bound by memory: 2 * heads * head_dim values per row; 16384 rows of 40 heads of 128 in bf16 (336 MB) take
// 64 us, 5.3 TB/s, the rate of a large copy.
template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kRopeThreads) void rope_rows(RopeArgs a, HeadRows<const T> q, HeadRows<T> q_out, HeadRows<const T> k,
                                                         HeadRows<T> k_out) {
  __shared__ __attribute__((aligned(16))) float cs[kRopePairs], sn[kRopePairs];
  __shared__ int live[kRopePairs];
  const int r0 = blockIdx.x * a.per_group, nr = min(a.per_group, a.rows - r0);
  for (int i = threadIdx.x; i < nr * a.pairs; i += kRopeThreads) {
    const int r = i / a.pairs, j = i - r * a.pairs;
    const int pos = a.position[r0 + r];
    double t = (double)pos * a.turns[j];
    t -= rint(t);
    float s, c;
    sincospif(2.f * (float)t, &s, &c);
    cs[i] = c * a.magnitude;
    sn[i] = s * a.sine;
    if (j == 0) live[r] = pos >= 0;
  }
  __syncthreads();
  const uint32_t per_row = (uint32_t)(a.heads * a.units);
  for (uint32_t u = threadIdx.x; u < nr * per_row; u += kRopeThreads) {
    const uint32_t r = V == 1 ? u / per_row : a.by_row.of(u), w = u - r * per_row;
    if (!live[r]) continue;
    uint32_t h = a.by_units.of(w);
    const int j = (int)(w - h * a.units) * V;
    const bool is_q = h < (uint32_t)a.q_heads;
    if (!is_q) h -= a.q_heads;
    const T *x = is_q ? q.at(r0 + r, h) : k.at(r0 + r, h);
    T *y = is_q ? q_out.at(r0 + r, h) : k_out.at(r0 + r, h);
    if (j >= a.pairs) {                                      // behind the rotated part
      const int e = 2 * a.pairs + (j - a.pairs);
      float v[V];
      load_vec<T, V>(x + e, v);
      store_vec<T, V>(y + e, v);
      continue;
    }
    float v[2 * V], o[2 * V];
    float c[V], s[V];
    load_vec<float, V % 4 ? V : 4>(cs + r * a.pairs + j, c);
    load_vec<float, V % 4 ? V : 4>(sn + r * a.pairs + j, s);
    if constexpr (V == 8) {
      load_vec<float, 4>(cs + r * a.pairs + j + 4, c + 4);
      load_vec<float, 4>(sn + r * a.pairs + j + 4, s + 4);
    }
    if (HALF) {
      load_vec<T, V>(x + j, v);
      load_vec<T, V>(x + a.pairs + j, v + V);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        o[i] = v[i] * c[i] - v[V + i] * s[i];
        o[V + i] = v[V + i] * c[i] + v[i] * s[i];
      }
      store_vec<T, V>(y + j, o);
      store_vec<T, V>(y + a.pairs + j, o + V);
    } else {
      load_vec<T, V>(x + 2 * j, v);
      load_vec<T, V>(x + 2 * j + V, v + V);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        o[2 * i] = v[2 * i] * c[i] - v[2 * i + 1] * s[i];
        o[2 * i + 1] = v[2 * i + 1] * c[i] + v[2 * i] * s[i];
      }
      store_vec<T, V>(y + 2 * j, o);
      store_vec<T, V>(y + 2 * j + V, o + V);
    }
  }
}

}  // namespace heisd
