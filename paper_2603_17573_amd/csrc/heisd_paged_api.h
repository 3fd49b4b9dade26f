// C ABI of the operators on paged requests: argument checks and launches (part of heisd_api.hip).
#pragma once

static size_t dtype_bytes(int32_t t) { return t == HEISD_DTYPE_F32 ? 4 : t == HEISD_DTYPE_BF16 || t == HEISD_DTYPE_F16 ? 2 : 0; }

template <typename T>
static HeadRows<T> head_rows(const heisd_head_rows &r) {
  return HeadRows<T>{static_cast<T *>(r.data), r.row_stride, r.head_stride};
}

// Are all rows of these heads reachable by accesses of `bytes` bytes (a power of two)?
static bool rows_aligned(const heisd_head_rows &r, size_t bytes) {
  const int64_t n = (int64_t)(bytes / dtype_bytes(r.dtype));
  return ((uintptr_t)r.data & (bytes - 1)) == 0 && r.row_stride % n == 0 && r.head_stride % n == 0;
}

// rows: how many there are (without any, there need not be memory for them).
static int rows_ok(const char *who, const char *name, const heisd_head_rows *r, int64_t rows) {
  if (!r || (!r->data && rows > 0)) return fail(nullptr, HEISD_EINVAL, "%s: NULL %s", who, name);
  if (!dtype_bytes(r->dtype)) return fail(nullptr, HEISD_EINVAL, "%s: %s has unknown dtype %d", who, name, r->dtype);
  if (r->heads < 1 || r->heads > 512) return fail(nullptr, HEISD_EINVAL, "%s: %s has %d heads (1..512)", who, name, r->heads);
  if (r->row_stride < 0 || r->head_stride < 0) return fail(nullptr, HEISD_EINVAL, "%s: %s has a negative stride", who, name);
  if ((uintptr_t)r->data % dtype_bytes(r->dtype)) return fail(nullptr, HEISD_EINVAL, "%s: %s is misaligned", who, name);
  return HEISD_OK;
}

// Rows that are written must not lie on each other (a broadcast tensor's do): workgroups would write, or read and write, the same bytes at
// once.
static int apart_ok(const char *who, const char *name, const heisd_head_rows &r, int64_t rows, int head_dim) {
  if ((rows > 1 && r.row_stride < head_dim) || (r.heads > 1 && r.head_stride < head_dim))
    return fail(nullptr, HEISD_EINVAL, "%s: rows or heads of %s lie on each other (strides %lld and %lld, head_dim %d)", who, name,
                (long long)r.row_stride, (long long)r.head_stride, head_dim);
  return HEISD_OK;
}

static int launched(const char *who) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(nullptr, HEISD_EHIP, "%s: %s", who, hipGetErrorString(e));
  g_init_err[0] = 0;
  return HEISD_OK;
}

// A launch has fewer than 2^32 threads in each direction: this many workgroups of 256.
constexpr int64_t kMostGroups = 0xFFFFFFFFll / 256;
static int groups_ok(const char *who, int64_t groups) {
  if (groups <= kMostGroups) return HEISD_OK;
  return fail(nullptr, HEISD_EINVAL, "%s: too many rows for one call (%lld workgroups, at most %lld)", who, (long long)groups, (long long)kMostGroups);
}

// ---- block tables, slots and positions ---------------------------------------------------------------------------

// Up to this many packed rows the one workgroup that keeps the books writes the slots as well.  us, one launch / two: 8 requests, 1024 rows
// 8.1 / 9.4, 4096 12.2 / 9.9, 8192 16.4 / 9.7; 64 requests, 1024 8.2 / 9.6, 4096 12.1 / 9.7; 512 requests, 4096 12.5 / 13.1, 8192 16.7 / 13.0.
constexpr int kPlanOneGroupRows = 2048;

extern "C" int heisd_paged_plan(const heisd_plan_desc *p, void *stream) {
  const char *who = "paged_plan";
  if (!p) return fail(nullptr, HEISD_EINVAL, "%s: NULL description", who);
  if (p->batch < 1 || p->batch > 65535 || p->rows < 0 || p->rows > (1 << 30))
    return fail(nullptr, HEISD_EINVAL, "%s: batch=%d (1..65535) rows=%d (0..2^30)", who, p->batch, p->rows);
  if (p->block_size < 1 || p->n_blocks < 1 || p->max_blocks < 1 || p->max_blocks > (1 << 20) ||
      (int64_t)p->n_blocks * p->block_size > 0x7FFFFFFF || (int64_t)p->max_blocks * p->block_size > 0x7FFFFFFF)
    return fail(nullptr, HEISD_EINVAL, "%s: block_size=%d n_blocks=%d max_blocks=%d (at most 2^31 - 1 slots, 2^20 blocks per request)", who,
                p->block_size, p->n_blocks, p->max_blocks);
  if (!p->cached_len || !p->new_len || !p->owned_in || !p->owned_out || !p->block_table || !p->free_ids || !p->free_count_in ||
      !p->free_count_out || !p->cu_rows || !p->seq_len || (p->rows > 0 && (!p->slot || !p->position)))
    return fail(nullptr, HEISD_EINVAL, "%s: NULL pointer", who);
  const PlanArgs a{p->batch, p->block_size, p->max_blocks, p->n_blocks, p->rows, p->cached_len, p->new_len, p->owned_in, p->owned_out,
                   p->block_table, p->free_ids, p->free_count_in, p->free_count_out, p->cu_rows, p->seq_len, p->slot, p->position, p->cu_seq};
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const int most = std::max(p->batch, p->rows / 4);            // threads that have something to do
  if (p->rows > kPlanOneGroupRows) {
    if (p->batch <= 256) plan_books<4, false><<<dim3(1), dim3(256), 0, st>>>(a);
    else plan_books<16, false><<<dim3(1), dim3(1024), 0, st>>>(a);
    plan_slots<<<dim3((p->rows + 255) / 256), dim3(256), 0, st>>>(a);
  } else if (most <= 64) plan_books<1, true><<<dim3(1), dim3(64), 0, st>>>(a);
  else if (most <= 256) plan_books<4, true><<<dim3(1), dim3(256), 0, st>>>(a);
  else plan_books<16, true><<<dim3(1), dim3(1024), 0, st>>>(a);
  return launched(who);
}

// ---- rotary positions ---------------------------------------------------------------------------------------------

extern "C" int heisd_rope_table(const heisd_rope_desc *d, double *turns, float *magnitude) {
  const char *who = "rope_table";
  if (!d || !turns || !magnitude) return fail(nullptr, HEISD_EINVAL, "%s: NULL pointer", who);
  const int n = d->rotary_dim;
  if (n < 2 || n > 256 || n % 2) return fail(nullptr, HEISD_EINVAL, "%s: rotary_dim=%d (even, 2..256)", who, n);
  if (!(d->base > 1) || !std::isfinite(d->base)) return fail(nullptr, HEISD_EINVAL, "%s: base %g", who, d->base);
  if (d->scaling < HEISD_ROPE_NONE || d->scaling > HEISD_ROPE_BANDS) return fail(nullptr, HEISD_EINVAL, "%s: scaling %d", who, d->scaling);
  const bool by_length = d->scaling == HEISD_ROPE_PARTS || d->scaling == HEISD_ROPE_BANDS;
  if (d->scaling != HEISD_ROPE_NONE && (!(d->factor >= 1) || !std::isfinite(d->factor)))
    return fail(nullptr, HEISD_EINVAL, "%s: factor %g (1 or more)", who, d->factor);
  if (by_length && d->original_len < 1) return fail(nullptr, HEISD_EINVAL, "%s: original_len %d", who, d->original_len);
  if (d->scaling == HEISD_ROPE_PARTS && !(d->beta_slow > 0 && d->beta_fast > d->beta_slow && std::isfinite(d->beta_fast)))
    return fail(nullptr, HEISD_EINVAL, "%s: beta_fast %g, beta_slow %g", who, d->beta_fast, d->beta_slow);
  if (d->scaling == HEISD_ROPE_BANDS && !(d->low_freq > 0 && d->high_freq > d->low_freq && std::isfinite(d->high_freq)))
    return fail(nullptr, HEISD_EINVAL, "%s: low_freq %g, high_freq %g", who, d->low_freq, d->high_freq);
  const double two_pi = 6.283185307179586476925286766559;
  double base = d->base, lo = 0, hi = 0;
  if (d->scaling == HEISD_ROPE_BASE && n > 2) base *= std::pow(d->factor, (double)n / (n - 2));
  if (d->scaling == HEISD_ROPE_PARTS) {
    auto pair = [&](double rotations) { return n * std::log(d->original_len / (rotations * two_pi)) / (2 * std::log(base)); };
    lo = std::max(0.0, std::floor(pair(d->beta_fast)));
    hi = std::min((double)(n - 1), std::ceil(pair(d->beta_slow)));
  }
  for (int i = 0; i < n / 2; ++i) {
    double f = std::pow(base, -2.0 * i / n), keep = 1;
    if (d->scaling == HEISD_ROPE_LINEAR) keep = 0;
    if (d->scaling == HEISD_ROPE_PARTS) keep = 1 - std::min(1.0, std::max(0.0, (i - lo) / std::max(hi - lo, 0.001)));
    if (d->scaling == HEISD_ROPE_BANDS)
      keep = std::min(1.0, std::max(0.0, (d->original_len * f / two_pi - d->low_freq) / (d->high_freq - d->low_freq)));
    if (keep != 1) f = f * keep + f / d->factor * (1 - keep);
    turns[i] = f / two_pi;
  }
  *magnitude = d->scaling == HEISD_ROPE_PARTS ? (float)(0.1 * std::log(d->factor) + 1) : 1.f;
  g_init_err[0] = 0;
  return HEISD_OK;
}

template <typename T, int V>
static void rope_launch(const RopeArgs &a, const heisd_head_rows *q, const heisd_head_rows *q_out, const heisd_head_rows *k,
                        const heisd_head_rows *k_out, bool half, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)a.rows + a.per_group - 1) / a.per_group)), block(kRopeThreads);
  const HeadRows<T> ki = k ? head_rows<T>(*k) : HeadRows<T>{}, ko = k ? head_rows<T>(*k_out) : HeadRows<T>{};
  const HeadRows<T> qi = head_rows<T>(*q), qo = head_rows<T>(*q_out);
  const HeadRows<const T> qc{qi.p, qi.rs, qi.hs}, kc{ki.p, ki.rs, ki.hs};
  if (half) rope_rows<T, V, true><<<grid, block, 0, st>>>(a, qc, qo, kc, ko);
  else rope_rows<T, V, false><<<grid, block, 0, st>>>(a, qc, qo, kc, ko);
}

extern "C" int heisd_rope(const double *turns, float magnitude, int32_t rotary_dim, int32_t layout, int32_t inverse, const int32_t *position,
                          int32_t rows, int32_t head_dim, const heisd_head_rows *q, const heisd_head_rows *q_out,
                          const heisd_head_rows *k, const heisd_head_rows *k_out, void *stream) {
  const char *who = "rope";
  if (rows < 0 || head_dim < 2 || head_dim > 256 || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > head_dim)
    return fail(nullptr, HEISD_EINVAL, "%s: rows=%d head_dim=%d (2..256) rotary_dim=%d (even, at most head_dim)", who, rows, head_dim, rotary_dim);
  if (layout != HEISD_ROPE_HALF && layout != HEISD_ROPE_INTERLEAVED) return fail(nullptr, HEISD_EINVAL, "%s: layout %d", who, layout);
  if (!turns || ((uintptr_t)turns & 7) || !std::isfinite(magnitude)) return fail(nullptr, HEISD_EINVAL, "%s: bad table", who);
  if ((k == nullptr) != (k_out == nullptr)) return fail(nullptr, HEISD_EINVAL, "%s: k without k_out, or k_out without k", who);
  const heisd_head_rows *all[4] = {q, q_out, k, k_out};
  const char *names[4] = {"q", "q_out", "k", "k_out"};
  bool wide = true, copies = false;
  const int per = 16 / (q && dtype_bytes(q->dtype) ? (int)dtype_bytes(q->dtype) : 2);
  for (int i = 0; i < (k ? 4 : 2); ++i) {
    const int rc = rows_ok(who, names[i], all[i], rows);
    if (rc != HEISD_OK) return rc;
    if (all[i]->dtype != q->dtype) return fail(nullptr, HEISD_EINVAL, "%s: dtypes differ", who);
    wide = wide && rows_aligned(*all[i], 16);
  }
  for (int i = 0; i < (k ? 4 : 2); i += 2) {
    if (all[i]->heads != all[i + 1]->heads) return fail(nullptr, HEISD_EINVAL, "%s: %s and its output differ in heads", who, names[i]);
    const bool same = all[i]->data == all[i + 1]->data;
    if (same && (all[i]->row_stride != all[i + 1]->row_stride || all[i]->head_stride != all[i + 1]->head_stride))
      return fail(nullptr, HEISD_EINVAL, "%s: %s is rotated in place with other strides", who, names[i]);
    copies = copies || !same;
    if (const int rc = apart_ok(who, names[i + 1], *all[i + 1], rows, head_dim)) return rc;
  }
  if (rows == 0) return HEISD_OK;
  if (!position) return fail(nullptr, HEISD_EINVAL, "%s: NULL positions", who);
  const int pairs = rotary_dim / 2, rest = copies ? head_dim - rotary_dim : 0;
  wide = wide && pairs % per == 0 && rest % per == 0;
  const int units = (pairs + rest) / (wide ? per : 1), heads = q->heads + (k ? k->heads : 0);
  // Rows per workgroup: as many as there are sines for its threads, but no fewer than eight workgroups per compute unit, and few
  // enough for the division by multiplication (see FastDiv).
  const int64_t per_row = (int64_t)heads * units;
  int64_t group = std::min<int64_t>(kRopePairs / pairs, (rows + 2047) / 2048);
  group = std::max<int64_t>(1, std::min<int64_t>(group, wide ? (int64_t)0xFFFFFFFF / (per_row * per_row) : group));
  if (const int rc = groups_ok(who, (rows + group - 1) / group)) return rc;
  const RopeArgs a{turns, magnitude, inverse ? -magnitude : magnitude, position, rows, pairs, rest, q->heads, heads, (int)group,
                   FastDiv((uint32_t)units), units, FastDiv((uint32_t)per_row)};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool half = layout == HEISD_ROPE_HALF;
  (void)hipGetLastError();
  if (q->dtype == HEISD_DTYPE_F32) {
    if (wide) rope_launch<float, 4>(a, q, q_out, k, k_out, half, st);
    else rope_launch<float, 1>(a, q, q_out, k, k_out, half, st);
  } else if (q->dtype == HEISD_DTYPE_BF16) {
    if (wide) rope_launch<__bf16, 8>(a, q, q_out, k, k_out, half, st);
    else rope_launch<__bf16, 1>(a, q, q_out, k, k_out, half, st);
  } else {
    if (wide) rope_launch<_Float16, 8>(a, q, q_out, k, k_out, half, st);
    else rope_launch<_Float16, 1>(a, q, q_out, k, k_out, half, st);
  }
  return launched(who);
}

// ---- the cache in 4 bits -------------------------------------------------------------------------------------------

static bool kv4_shape_ok(int32_t n_blocks, int32_t block_size, int32_t kv_heads, int32_t head_dim) {
  return n_blocks >= 1 && block_size >= kKv4Tile && block_size <= 4096 && (block_size & (block_size - 1)) == 0 && kv_heads >= 1 &&
         kv_heads <= 512 && (head_dim == 64 || head_dim == 128) && (int64_t)n_blocks * block_size <= 0x7FFFFFFF;
}

extern "C" size_t heisd_kv4_pool_bytes(int32_t n_blocks, int32_t block_size, int32_t kv_heads, int32_t head_dim) {
  if (!kv4_shape_ok(n_blocks, block_size, kv_heads, head_dim)) return 0;
  return (size_t)n_blocks * kv_heads * (size_t)kv4_cell_bytes(block_size, head_dim);
}

static int kv4_ok(const char *who, const heisd_kv4_desc *c, Kv4Cache *out) {
  if (!c || !c->pool || ((uintptr_t)c->pool & 15)) return fail(nullptr, HEISD_EINVAL, "%s: NULL or misaligned pool", who);
  if (c->head_dim != 64 && c->head_dim != 128) return fail(nullptr, HEISD_EUNSUPPORTED, "%s: head_dim %d (64 or 128)", who, c->head_dim);
  if (!kv4_shape_ok(c->n_blocks, c->block_size, c->kv_heads, c->head_dim))
    return fail(nullptr, HEISD_EINVAL, "%s: n_blocks=%d block_size=%d (a power of two, 16..4096) kv_heads=%d (1..512)", who, c->n_blocks,
                c->block_size, c->kv_heads);
  *out = Kv4Cache{static_cast<uint8_t *>(c->pool), c->n_blocks, c->block_size, __builtin_ctz(c->block_size), c->kv_heads,
                  kv4_cell_bytes(c->block_size, c->head_dim)};
  return HEISD_OK;
}

static int batch_ok(const char *who, const heisd_paged_batch *b, bool rows, PagedBatch *out) {
  if (!b || !b->block_table || !b->seq_len || (rows && !b->cu_rows)) return fail(nullptr, HEISD_EINVAL, "%s: NULL batch or pointer of it", who);
  if (b->batch < 1 || b->batch > 65535 || b->max_blocks < 1 || b->rows < 0)
    return fail(nullptr, HEISD_EINVAL, "%s: batch=%d (1..65535) max_blocks=%d rows=%d", who, b->batch, b->max_blocks, b->rows);
  *out = PagedBatch{b->block_table, b->seq_len, b->cu_rows, b->batch, b->max_blocks, b->rows};
  return HEISD_OK;
}

// Rows a workgroup takes: about `units` 256-thread rounds' worth, at most what the division by multiplication allows.
static int rows_per_group(int64_t per_row, int rounds) {
  return (int)std::max<int64_t>(1, std::min<int64_t>((int64_t)rounds * 256 / per_row, (int64_t)0xFFFFFFFF / (per_row * per_row)));
}

template <typename T, int HD>
static void kv4_append_launch(const Kv4Cache &c, const heisd_head_rows *k, const heisd_head_rows *v, const int32_t *slot, int rows, int per,
                              int64_t per_row, bool wide, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)rows + per - 1) / per), 2), block(256);
  const HeadRows<T> ki = head_rows<T>(*k), vi = head_rows<T>(*v);
  const HeadRows<const T> kc{ki.p, ki.rs, ki.hs}, vc{vi.p, vi.rs, vi.hs};
  if (wide) kv4_append<T, HD, true><<<grid, block, 0, st>>>(c, kc, vc, slot, rows, per, FastDiv((uint32_t)per_row));
  else kv4_append<T, HD, false><<<grid, block, 0, st>>>(c, kc, vc, slot, rows, per, FastDiv((uint32_t)per_row));
}

extern "C" int heisd_kv4_append(const heisd_kv4_desc *cache, const heisd_head_rows *k, const heisd_head_rows *v, const int32_t *slot,
                                int32_t rows, void *stream) {
  const char *who = "kv4_append";
  Kv4Cache c;
  int rc = kv4_ok(who, cache, &c);
  if (rc == HEISD_OK) rc = rows_ok(who, "k", k, rows);
  if (rc == HEISD_OK) rc = rows_ok(who, "v", v, rows);
  if (rc != HEISD_OK) return rc;
  if (k->dtype != v->dtype || k->heads != c.kv_heads || v->heads != c.kv_heads)
    return fail(nullptr, HEISD_EINVAL, "%s: k and v differ in dtype, or in heads from the cache", who);
  if (rows < 0 || (rows > 0 && !slot)) return fail(nullptr, HEISD_EINVAL, "%s: rows=%d or NULL slots", who, rows);
  if (rows == 0) return HEISD_OK;
  const int64_t per_row = (int64_t)c.kv_heads * (cache->head_dim / 8);
  const int per = rows_per_group(per_row, rows * per_row > (1 << 20) ? 4 : 1);
  if ((rc = groups_ok(who, ((int64_t)rows + per - 1) / per)) != HEISD_OK) return rc;
  const bool wide = rows_aligned(*k, 16) && rows_aligned(*v, 16), big = cache->head_dim == 128;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (k->dtype == HEISD_DTYPE_F32) {
    if (big) kv4_append_launch<float, 128>(c, k, v, slot, rows, per, per_row, wide, st);
    else kv4_append_launch<float, 64>(c, k, v, slot, rows, per, per_row, wide, st);
  } else if (k->dtype == HEISD_DTYPE_BF16) {
    if (big) kv4_append_launch<__bf16, 128>(c, k, v, slot, rows, per, per_row, wide, st);
    else kv4_append_launch<__bf16, 64>(c, k, v, slot, rows, per, per_row, wide, st);
  } else {
    if (big) kv4_append_launch<_Float16, 128>(c, k, v, slot, rows, per, per_row, wide, st);
    else kv4_append_launch<_Float16, 64>(c, k, v, slot, rows, per, per_row, wide, st);
  }
  return launched(who);
}

template <typename T, int HD>
static void kv4_gather_launch(const Kv4Cache &c, const PagedBatch &b, const int32_t *cu_seq, int out_rows, const heisd_head_rows *k,
                              const heisd_head_rows *v, bool wide, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)out_rows + kGatherRows<T> - 1) / kGatherRows<T>), (c.kv_heads + kGatherHeads - 1) / kGatherHeads, 2), block(256);
  if (wide) kv4_gather<T, HD, true><<<grid, block, 0, st>>>(c, b, cu_seq, out_rows, head_rows<T>(*k), head_rows<T>(*v));
  else kv4_gather<T, HD, false><<<grid, block, 0, st>>>(c, b, cu_seq, out_rows, head_rows<T>(*k), head_rows<T>(*v));
}

extern "C" int heisd_kv4_gather(const heisd_kv4_desc *cache, const heisd_paged_batch *batch, const int32_t *cu_seq, int32_t out_rows,
                                const heisd_head_rows *k_out, const heisd_head_rows *v_out, void *stream) {
  const char *who = "kv4_gather";
  Kv4Cache c;
  PagedBatch b;
  int rc = kv4_ok(who, cache, &c);
  if (rc == HEISD_OK) rc = batch_ok(who, batch, false, &b);
  if (rc == HEISD_OK) rc = rows_ok(who, "k_out", k_out, out_rows);
  if (rc == HEISD_OK) rc = rows_ok(who, "v_out", v_out, out_rows);
  if (rc != HEISD_OK) return rc;
  if (k_out->dtype != v_out->dtype || k_out->heads != c.kv_heads || v_out->heads != c.kv_heads)
    return fail(nullptr, HEISD_EINVAL, "%s: k_out and v_out differ in dtype, or in heads from the cache", who);
  if (out_rows < 0 || !cu_seq) return fail(nullptr, HEISD_EINVAL, "%s: out_rows=%d or NULL cu_seq", who, out_rows);
  if (out_rows == 0) return HEISD_OK;
  if ((rc = apart_ok(who, "k_out", *k_out, out_rows, cache->head_dim)) != HEISD_OK) return rc;
  if ((rc = apart_ok(who, "v_out", *v_out, out_rows, cache->head_dim)) != HEISD_OK) return rc;
  const int per = k_out->dtype == HEISD_DTYPE_F32 ? kGatherRows<float> : kGatherRows<__bf16>;
  if ((rc = groups_ok(who, ((int64_t)out_rows + per - 1) / per)) != HEISD_OK) return rc;
  const bool wide = rows_aligned(*k_out, 16) && rows_aligned(*v_out, 16), big = cache->head_dim == 128;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (k_out->dtype == HEISD_DTYPE_F32) {
    if (big) kv4_gather_launch<float, 128>(c, b, cu_seq, out_rows, k_out, v_out, wide, st);
    else kv4_gather_launch<float, 64>(c, b, cu_seq, out_rows, k_out, v_out, wide, st);
  } else if (k_out->dtype == HEISD_DTYPE_BF16) {
    if (big) kv4_gather_launch<__bf16, 128>(c, b, cu_seq, out_rows, k_out, v_out, wide, st);
    else kv4_gather_launch<__bf16, 64>(c, b, cu_seq, out_rows, k_out, v_out, wide, st);
  } else {
    if (big) kv4_gather_launch<_Float16, 128>(c, b, cu_seq, out_rows, k_out, v_out, wide, st);
    else kv4_gather_launch<_Float16, 64>(c, b, cu_seq, out_rows, k_out, v_out, wide, st);
  }
  return launched(who);
}

// How a call is cut: column tiles per workgroup, and workgroups: as many as are resident at once (kv4_per_unit), fewer where there is
// little to do - four units of 128 tokens for each, counted with the largest lengths (one context of 4000 tokens, 8 key heads, 1 / 2 / 4 / 8 / 16
// units each: 13.4 / 11.9 / 12.4 / 15.6 / 22.1 us; eight of them: 20.2 / 20.0 / 16.5 / 17.4 / 22.9).  More than 16 columns are two tiles, for which the
// cache is read once, where the work fills the grid even so: drafts of seven, 4 query heads per key head, one tile / two: 64 contexts of 256 to 4000
// tokens 64.3 / 62.4 us, 16 of up to 2000 30.4 / 26.8, one of 4000 15.5 / 21.0.
constexpr int kKv4Units = 256;                       // compute units that the grid is made for (a fixed number: results do not depend on the device)
struct Kv4Plan {
  int col_tiles, segments;
  int64_t units;
  size_t part_ml, total;
  int groups(int head_dim) const {
    return (int)std::max<int64_t>(1, std::min<int64_t>((units + 3) / 4, kv4_per_unit(head_dim, col_tiles) * kKv4Units));
  }
  // (With 2^22 columns the products stay below 2^59, and more change nothing: there are 65535 segments already.)
  Kv4Plan(int64_t batch, int64_t kv_heads, int64_t group, int64_t max_q, int64_t max_seq, int64_t head_dim) {
    const int64_t cols = std::min<int64_t>(max_q * group, 1 << 22), lengths = (max_seq + 4 * kKv4Unit - 1) / (4 * kKv4Unit);
    col_tiles = cols > 16 && batch * kv_heads * ((cols + 15) / 16) * lengths >= kv4_per_unit((int)head_dim, 1) * kKv4Units ? 2 : 1;
    segments = (int)std::min<int64_t>(kv_heads * ((cols + 16 * col_tiles - 1) / (16 * col_tiles)), 65535);
    units = batch * segments * ((max_seq + kKv4Unit - 1) / kKv4Unit);
    const size_t rows = (size_t)2 * groups((int)head_dim) * 16 * col_tiles;
    part_ml = align256(rows * (size_t)head_dim * sizeof(float));
    total = part_ml + align256(rows * 2 * sizeof(float));
  }
};

static int kv4_attention_sizes_ok(const char *who, int32_t kv_heads, int32_t q_heads, int32_t rows, int32_t max_q, int32_t max_seq) {
  if (q_heads < 1 || q_heads > 512 || q_heads % kv_heads)
    return fail(nullptr, HEISD_EINVAL, "%s: %d query heads over %d key heads", who, q_heads, kv_heads);
  if (rows < 0 || max_q < 1 || max_seq < 1 || max_seq > (1 << 24) || (int64_t)rows * q_heads > 0x7FFFFF00)
    return fail(nullptr, HEISD_EINVAL, "%s: rows=%d max_q=%d max_seq=%d (1..2^24)", who, rows, max_q, max_seq);
  return HEISD_OK;
}

extern "C" size_t heisd_kv4_attention_workspace_bytes(const heisd_kv4_desc *cache, int32_t batch, int32_t rows, int32_t q_heads, int32_t max_q,
                                                      int32_t max_seq) {
  if (!cache || !kv4_shape_ok(cache->n_blocks, cache->block_size, cache->kv_heads, cache->head_dim) || batch < 1 || batch > 65535 ||
      kv4_attention_sizes_ok("kv4_attention_workspace_bytes", cache->kv_heads, q_heads, rows, max_q, max_seq) != HEISD_OK)
    return 0;
  return Kv4Plan(batch, cache->kv_heads, q_heads / cache->kv_heads, max_q, max_seq, cache->head_dim).total;
}

template <typename T, int HD, int TERMS>
static void kv4_attention_launch(const Kv4Cache &c, const PagedBatch &b, const heisd_head_rows *q, const heisd_head_rows *out,
                                 const Kv4Attend &a, const Kv4Plan &plan, hipStream_t st) {
  const HeadRows<T> qi = head_rows<T>(*q), o = head_rows<T>(*out);
  const HeadRows<const T> qc{qi.p, qi.rs, qi.hs};
  const dim3 block(256);
  const int groups = plan.groups(HD);
  if (plan.col_tiles == 2) kv4_attend<T, HD, 2, TERMS><<<dim3(groups), block, 0, st>>>(c, b, qc, o, a);
  else kv4_attend<T, HD, 1, TERMS><<<dim3(groups), block, 0, st>>>(c, b, qc, o, a);
  if (groups > 1) kv4_join<T, HD><<<dim3(plan.segments, b.batch), block, 0, st>>>(c, b, o, a, groups);
}

extern "C" int heisd_kv4_attention(const heisd_kv4_desc *cache, const heisd_paged_batch *batch, const heisd_head_rows *q,
                                   const heisd_head_rows *out, float *lse, float scale, int32_t max_q, int32_t max_seq, void *workspace,
                                   size_t workspace_bytes, void *stream) {
  const char *who = "kv4_attention";
  Kv4Cache c;
  PagedBatch b;
  int rc = kv4_ok(who, cache, &c);
  if (rc == HEISD_OK) rc = batch_ok(who, batch, true, &b);
  if (rc == HEISD_OK) rc = rows_ok(who, "q", q, b.rows);
  if (rc == HEISD_OK) rc = rows_ok(who, "out", out, b.rows);
  if (rc == HEISD_OK) rc = kv4_attention_sizes_ok(who, c.kv_heads, q->heads, b.rows, max_q, max_seq);
  if (rc != HEISD_OK) return rc;
  if (q->dtype != out->dtype || q->heads != out->heads) return fail(nullptr, HEISD_EINVAL, "%s: q and out differ in dtype or heads", who);
  if (q->dtype == HEISD_DTYPE_F32) return fail(nullptr, HEISD_EUNSUPPORTED, "%s: q in fp32 (bf16 or fp16)", who);
  if (!rows_aligned(*q, 16) || !rows_aligned(*out, 8)) return fail(nullptr, HEISD_EINVAL, "%s: q (16 bytes) or out (8 bytes) misaligned", who);
  if (!std::isfinite(scale)) return fail(nullptr, HEISD_EINVAL, "%s: scale %g", who, scale);
  if (b.rows == 0) return HEISD_OK;
  if ((rc = apart_ok(who, "out", *out, b.rows, cache->head_dim)) != HEISD_OK) return rc;
  const Kv4Plan plan(b.batch, c.kv_heads, q->heads / c.kv_heads, max_q, max_seq, cache->head_dim);
  const size_t need = plan.total;
  if (!workspace || ((uintptr_t)workspace & 255)) return fail(nullptr, HEISD_EINVAL, "%s: NULL or misaligned workspace", who);
  if (workspace_bytes < need) return fail(nullptr, HEISD_ENOMEM, "%s: workspace %zu bytes < %zu needed", who, workspace_bytes, need);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  const Kv4Attend a{std::max(std::fabs(scale) * 1.4426950408889634f, 1e-30f),      // not 0: minus infinity stands for masked scores
                    scale < 0, q->heads / c.kv_heads, q->heads, max_seq, 16 * plan.col_tiles,
                    reinterpret_cast<float *>(ws), reinterpret_cast<float *>(ws + plan.part_ml), lse};
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (q->dtype == HEISD_DTYPE_BF16) {
    if (cache->head_dim == 128) kv4_attention_launch<__bf16, 128, 1>(c, b, q, out, a, plan, st);
    else kv4_attention_launch<__bf16, 64, 1>(c, b, q, out, a, plan, st);
  } else {
    if (cache->head_dim == 128) kv4_attention_launch<_Float16, 128, 2>(c, b, q, out, a, plan, st);
    else kv4_attention_launch<_Float16, 64, 2>(c, b, q, out, a, plan, st);
  }
  return launched(who);
}

// ---- attention of packed prompts -------------------------------------------------------------------------------------

// Two sets of waves share a workgroup's keys where the workgroups are few and the keys of a sequence (on average) many.  us, one set / two, one
// causal sequence: 1024 keys, heads of 128, 36 workgroups 22.8 / 20.6, 288 25.2 / 23.3, 576 29.9 / 34.6, 1152 50.7 / 66.9; heads of 64, 288
// 17.7 / 14.9, 576 19.0 / 20.5; 4096 keys, 264 77.6 / 63.0, 528 90.3 / 79.5; 276 keys, heads of 128, 12 9.9 / 10.8, 192 11.2 / 12.0.
constexpr int64_t kPromptSplitGroups = 320, kPromptSplitKeys = 512;

template <typename T, int HD, bool CAUSAL, int SPLIT>
static hipError_t prompt_launch_one(const PromptArgs &a, const heisd_head_rows *q, const heisd_head_rows *k, const heisd_head_rows *v,
                                    const heisd_head_rows *out, hipStream_t st) {
  const HeadRows<T> qi = head_rows<T>(*q), ki = head_rows<T>(*k), vi = head_rows<T>(*v);
  const HeadRows<const T> qc{qi.p, qi.rs, qi.hs}, kc{ki.p, ki.rs, ki.hs}, vc{vi.p, vi.rs, vi.hs};
  constexpr int lds = prompt_lds_bytes<HD>(SPLIT);
  if constexpr (lds > 65536) {                       // above the usual limit of a workgroup, which is raised once per device
    static std::atomic<bool> raised[kRetrieveMaxDevices];
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess && (dev < 0 || dev >= kRetrieveMaxDevices)) e = hipErrorInvalidDevice;
    if (e == hipSuccess && !raised[dev].load()) {
      e = hipFuncSetAttribute(reinterpret_cast<const void *>(&prompt_attend<T, HD, CAUSAL, SPLIT>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (e == hipSuccess) raised[dev].store(true);
    }
    if (e != hipSuccess) return e;
  }
  prompt_attend<T, HD, CAUSAL, SPLIT><<<dim3((unsigned)((int64_t)a.tiles * a.q_heads)), dim3(256 * SPLIT), lds, st>>>(qc, kc, vc, head_rows<T>(*out), a);
  return hipSuccess;
}

template <typename T, int HD, bool CAUSAL>
static hipError_t prompt_launch(const PromptArgs &a, const heisd_head_rows *q, const heisd_head_rows *k, const heisd_head_rows *v,
                                const heisd_head_rows *out, hipStream_t st) {
  const bool split = (int64_t)a.tiles * a.q_heads <= kPromptSplitGroups && a.k_rows >= kPromptSplitKeys * a.batch;
  return split ? prompt_launch_one<T, HD, CAUSAL, 2>(a, q, k, v, out, st) : prompt_launch_one<T, HD, CAUSAL, 1>(a, q, k, v, out, st);
}

static int prompt_attention(const char *who, const heisd_head_rows *q, const heisd_head_rows *k, const heisd_head_rows *v, const heisd_head_rows *out,
                            float *lse, const int32_t *cu_q, const int32_t *cu_k, const int32_t *seq_len, int32_t batch, int32_t rows, int32_t k_rows,
                            int32_t head_dim, float scale, int32_t causal, void *stream) {
  int rc = rows_ok(who, "q", q, rows);
  if (rc == HEISD_OK) rc = rows_ok(who, "k", k, k_rows);
  if (rc == HEISD_OK) rc = rows_ok(who, "v", v, k_rows);
  if (rc == HEISD_OK) rc = rows_ok(who, "out", out, rows);
  if (rc != HEISD_OK) return rc;
  if (head_dim != 64 && head_dim != 128) return fail(nullptr, HEISD_EUNSUPPORTED, "%s: head_dim %d (64 or 128)", who, head_dim);
  if (q->dtype == HEISD_DTYPE_F32) return fail(nullptr, HEISD_EUNSUPPORTED, "%s: fp32 rows (bf16 or fp16)", who);
  if (k->dtype != q->dtype || v->dtype != q->dtype || out->dtype != q->dtype) return fail(nullptr, HEISD_EINVAL, "%s: dtypes differ", who);
  if (k->heads != v->heads || q->heads != out->heads || q->heads % k->heads)
    return fail(nullptr, HEISD_EINVAL, "%s: %d query heads, %d key heads, %d value heads, %d output heads", who, q->heads, k->heads, v->heads, out->heads);
  if (!rows_aligned(*q, 16) || !rows_aligned(*k, 16) || !rows_aligned(*v, 16) || !rows_aligned(*out, 8))
    return fail(nullptr, HEISD_EINVAL, "%s: q, k, v (16 bytes) or out (8 bytes) misaligned", who);
  if (!cu_q || !cu_k || batch < 1 || batch > 65535 || rows < 0 || k_rows < 0 || !std::isfinite(scale))
    return fail(nullptr, HEISD_EINVAL, "%s: NULL lengths, batch=%d (1..65535) rows=%d k_rows=%d scale=%g", who, batch, rows, k_rows, scale);
  if (k->row_stride > (1 << 25) || v->row_stride > (1 << 25))                       // 16 rows apart stays below 2^32 bytes
    return fail(nullptr, HEISD_EUNSUPPORTED, "%s: rows of k or v more than 2^25 elements apart", who);
  const int64_t tiles = (int64_t)rows / kPromptRows + batch;
  if (rows == 0) return HEISD_OK;
  if ((rc = groups_ok(who, tiles * q->heads)) != HEISD_OK) return rc;
  if ((rc = apart_ok(who, "out", *out, rows, head_dim)) != HEISD_OK) return rc;
  const PromptArgs a{cu_q, cu_k, seq_len, batch, rows, k_rows, q->heads, k->heads, q->heads / k->heads, (int)tiles,
                     std::max(std::fabs(scale) * 1.4426950408889634f, 1e-30f),   // not 0: minus infinity stands for masked scores
                     scale < 0 ? 0x80008000u : 0u, lse};
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  hipError_t e;
  if (q->dtype == HEISD_DTYPE_BF16) {
    if (head_dim == 128) e = causal ? prompt_launch<__bf16, 128, true>(a, q, k, v, out, st) : prompt_launch<__bf16, 128, false>(a, q, k, v, out, st);
    else e = causal ? prompt_launch<__bf16, 64, true>(a, q, k, v, out, st) : prompt_launch<__bf16, 64, false>(a, q, k, v, out, st);
  } else {
    if (head_dim == 128) e = causal ? prompt_launch<_Float16, 128, true>(a, q, k, v, out, st) : prompt_launch<_Float16, 128, false>(a, q, k, v, out, st);
    else e = causal ? prompt_launch<_Float16, 64, true>(a, q, k, v, out, st) : prompt_launch<_Float16, 64, false>(a, q, k, v, out, st);
  }
  if (e != hipSuccess) return fail(nullptr, HEISD_EHIP, "%s: %s", who, hipGetErrorString(e));
  return launched(who);
}

extern "C" int heisd_prompt_attention(const heisd_head_rows *q, const heisd_head_rows *k, const heisd_head_rows *v, const heisd_head_rows *out,
                                      float *lse, const int32_t *cu_q, const int32_t *cu_k, int32_t batch, int32_t rows, int32_t k_rows,
                                      int32_t head_dim, float scale, int32_t causal, void *stream) {
  return prompt_attention("prompt_attention", q, k, v, out, lse, cu_q, cu_k, nullptr, batch, rows, k_rows, head_dim, scale, causal, stream);
}

extern "C" int heisd_paged_prompt_attention(const heisd_paged_batch *batch, const heisd_head_rows *q, const heisd_head_rows *k,
                                            const heisd_head_rows *v, const heisd_head_rows *out, float *lse, int32_t head_dim, float scale,
                                            void *stream) {
  const char *who = "paged_prompt_attention";
  PagedBatch b;
  const int rc = batch_ok(who, batch, true, &b);
  if (rc != HEISD_OK) return rc;
  return prompt_attention(who, q, k, v, out, lse, b.cu_rows, b.cu_rows, b.seq_len, b.batch, b.rows, b.rows, head_dim, scale, 1, stream);
}
