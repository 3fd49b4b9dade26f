// Attention over a prefix that a group of requests shares and over the requests' own tokens, both in the 4-bit cache: the parts of a row, joined.
#pragma once
#include "heisd_common.h"
#include "heisd_kv4.h"
#include "heisd_paged.h"

namespace heisd {

// Which group request i belongs to (-1: none).  Groups that are described follow each other, so at most one does.
__device__ __forceinline__ int group_of(const PrefixGroups &p, int i) {
  const int lane = threadIdx.x & 63;
  for (int g0 = 0; g0 < p.groups; g0 += 64) {
    const int g = min(g0 + lane, p.groups - 1);
    const unsigned long long m = __ballot(p.first[g] <= i && i < p.first[g + 1]);
    if (m) return g0 + __builtin_ctzll(m);
  }
  return -1;
}

// Joins what kv4_attend left of a row: its own tokens' part and its group's prefix', each whole or in parts of several workgroups.  A workgroup takes some
// columns (rows times query heads) of a request, 16 bytes of a column per thread.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_shared_join(Kv4Cache c, PagedBatch b, HeadRows<T> out, Kv4SharedAttend a, int grid) {
  const int req = blockIdx.y, lane = threadIdx.x & 63;
  const Kv4Request own = kv4_request(c, b, a, req);
  const int n_cols = own.rows.count * a.q_heads;
  constexpr int PER = 256 / (HD / 4);
  if ((long long)blockIdx.x * PER >= n_cols) return;
  const int g = group_of(a.prefix, req), seq = b.seq_len[req];
  const bool live = seq >= 0 && seq <= a.max_seq && (long long)seq <= (long long)b.max_blocks * c.block_size;
  long long before[2] = {0, 0}, all = 0;
  for (int i = lane; i < b.batch + a.prefix.groups; i += 64) {
    const long long work = kv4_request(c, b, a, i).work;
    all += work;
    if (i < req) before[0] += work;
    if (i < b.batch + g) before[1] += work;
  }
  before[0] = wave_sum64(before[0]);
  before[1] = wave_sum64(before[1]);
  const long long per = kv4_run(wave_sum64(all), grid);
  Kv4Request shared{};
  if (g >= 0) shared = kv4_request(c, b, a, b.batch + g);
  for (int u = blockIdx.x * PER + threadIdx.x / (HD / 4); u < n_cols; u += gridDim.x * PER) {
    const int d = threadIdx.x % (HD / 4) * 4, i = u / a.q_heads, h = u - i * a.q_heads, head = h / a.group;
    const long long r = own.rows.begin + i;
    Kv4Sums s;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const Kv4Request &q = part ? shared : own;
      if (!live || !q.work || r < q.rows.begin || r >= q.rows.begin + q.rows.count) continue;
      const int col = (int)(r - q.rows.begin) * a.group + h - head * a.group, tile = col / a.cols, n = col - tile * a.cols;
      const long long s0 = before[part] + ((long long)tile * c.kv_heads + head) * q.units;
      const int w0 = (int)wave_div(s0, per), w1 = (int)wave_div(s0 + q.units - 1, per);
      if (w0 == w1) {
        const long long at = ((long long)part * b.rows + r) * a.q_heads + h;
        const float2 ml[1] = {*reinterpret_cast<const float2 *>(a.whole_ml + at * 2)};
        const f32x4 x[1] = {*reinterpret_cast<const f32x4 *>(a.whole + at * HD + d)};
        s.add(ml, x);
        continue;
      }
      const int first_slot = 2 * w0 + (w0 * per != s0);
      constexpr int K = 8;
      for (int w = w0; w <= w1; w += K) {
        float2 ml[K];
        f32x4 x[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int wi = min(w + k, w1);
          const long long at = (long long)(wi == w0 ? first_slot : 2 * wi) * a.cols + n;
          ml[k] = *reinterpret_cast<const float2 *>(a.part_ml + at * 2);
          x[k] = *reinterpret_cast<const f32x4 *>(a.part + at * HD + d);
          if (w + k > w1) ml[k] = make_float2(-INFINITY, 0.f);
        }
        s.add(ml, x);
      }
    }
    const float inv = s.sum == 0.f ? 0.f : 1.f / s.sum;
    float f[4] = {s.o[0] * inv, s.o[1] * inv, s.o[2] * inv, s.o[3] * inv};
    store_vec<T, 4>(out.at(r, h) + d, f);
    if (a.lse && d == 0) a.lse[r * a.q_heads + h] = s.sum == 0.f ? -INFINITY : (s.top + log2f(s.sum)) * 0.6931471805599453f;
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
