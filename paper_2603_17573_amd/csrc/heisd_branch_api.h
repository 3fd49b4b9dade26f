// C ABI of the operators on requests that continue others: argument checks and launches (part of heisd_api.hip).
#pragma once

// ---- the next beams --------------------------------------------------------------------------------------------------

constexpr int kBeamMostVocab = (1 << 19) - 8;       // not more segments than beam_pick's lanes hold
constexpr int kBeamDirectVocab = 4096;              // up to here one launch does.  us, one / two: four beams over 256 logits 8.8 / 12.7, 4000 10.4 / 12.6,
                                                    // 8000 15.0 / 13.3; 64 beams over 1000 11.2 / 14.6, 4000 12.3 / 13.9, 8000 15.6 / 13.8

static int beam_sizes_ok(const char *who, int32_t groups, int32_t beams, int32_t width, int32_t vocab) {
  if (groups < 1 || groups > 65535 || beams < 1 || beams > kBeamMost || width < 1 || width > kBeamMost || vocab < 1 || vocab > kBeamMostVocab)
    return fail(nullptr, HEISD_EINVAL, "%s: groups=%d (1..65535) beams=%d width=%d (1..%d) vocab=%d (1..%d)", who, groups, beams, width, kBeamMost,
                vocab, kBeamMostVocab);
  if ((int64_t)groups * beams > 65535) return fail(nullptr, HEISD_EINVAL, "%s: %lld beams in all (at most 65535)", who, (long long)groups * beams);
  return HEISD_OK;
}
struct BeamLayout {
  int segments;
  size_t top, total;
  BeamLayout(int64_t rows, int64_t vocab, size_t size) {
    const int64_t waves = (vocab + kBeamWave - 1) / kBeamWave;
    segments = (int)(waves * (kBeamWave * size / 1024));
    top = align256((size_t)(rows * waves) * sizeof(float2));
    total = top + align256((size_t)rows * segments * sizeof(float));
  }
};

extern "C" size_t heisd_beam_select_workspace_bytes(int32_t groups, int32_t beams, int32_t width, int32_t vocab) {
  if (beam_sizes_ok("beam_select_workspace_bytes", groups, beams, width, vocab) != HEISD_OK) return 0;
  return BeamLayout((int64_t)groups * beams, vocab, 4).total;        // fp32 has most segments, and every dtype as many parts
}

template <typename T>
static void beam_launch(const BeamArgs &a, hipStream_t st) {
  const dim3 groups(a.groups), block(kBeamWaves * 64);
  if (a.vocab <= kBeamDirectVocab) {
    beam_pick<T, true><<<groups, block, 0, st>>>(a);
    return;
  }
  const int per = 4 * kBeamWave / kBeamSegment<T>;
  beam_scan<T><<<dim3((a.segments + per - 1) / per, a.groups * a.beams), dim3(256), 0, st>>>(a);
  beam_pick<T, false><<<groups, block, 0, st>>>(a);
}

extern "C" int heisd_beam_select(const heisd_beam_desc *d, void *workspace, size_t workspace_bytes, void *stream) {
  const char *who = "beam_select";
  if (!d) return fail(nullptr, HEISD_EINVAL, "%s: NULL description", who);
  if (const int rc = beam_sizes_ok(who, d->groups, d->beams, d->width, d->vocab)) return rc;
  const size_t size = dtype_bytes(d->dtype);
  if (!size) return fail(nullptr, HEISD_EINVAL, "%s: logits have unknown dtype %d", who, d->dtype);
  if (!d->logits || (uintptr_t)d->logits % size || d->row_stride < 0)
    return fail(nullptr, HEISD_EINVAL, "%s: NULL or misaligned logits, or a negative stride", who);
  if (!d->score_in || !d->score_out || !d->beam || !d->token) return fail(nullptr, HEISD_EINVAL, "%s: NULL pointer", who);
  if (!d->length_in != !d->length_out || !d->done_in != !d->done_out)
    return fail(nullptr, HEISD_EINVAL, "%s: length_in without length_out, done_in without done_out, or the other way round", who);
  if (d->end_token < -1 || d->end_token >= d->vocab || (d->end_token >= 0 && !d->done_in))
    return fail(nullptr, HEISD_EINVAL, "%s: end_token %d (-1..vocab - 1; with done_in)", who, d->end_token);
  if (!std::isfinite(d->length_power) || (d->length_power != 0 && !d->length_in))
    return fail(nullptr, HEISD_EINVAL, "%s: length_power %g (with length_in)", who, d->length_power);
  if (d->parent && (d->first < 0 || d->stride < d->width || d->first + (int64_t)d->groups * d->stride > 0x7FFFFFFF))
    return fail(nullptr, HEISD_EINVAL, "%s: parents from %d on, %d apart", who, d->first, d->stride);
  const void *in[3] = {d->score_in, d->length_in, d->done_in}, *out[3] = {d->score_out, d->length_out, d->done_out};
  for (int i = 0; i < 3; ++i)
    if (in[i] && in[i] == out[i] && d->width != d->beams) return fail(nullptr, HEISD_EINVAL, "%s: in place with another number of beams", who);
  const BeamLayout lay((int64_t)d->groups * d->beams, d->vocab, size);
  if (!workspace || ((uintptr_t)workspace & 255)) return fail(nullptr, HEISD_EINVAL, "%s: NULL or misaligned workspace", who);
  if (workspace_bytes < lay.total) return fail(nullptr, HEISD_ENOMEM, "%s: workspace %zu bytes < %zu needed", who, workspace_bytes, lay.total);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  const BeamArgs a{d->logits, d->row_stride, d->groups, d->beams, d->width, d->vocab, lay.segments, d->end_token, d->length_power, d->score_in, d->length_in,
                   d->done_in, d->score_out, d->beam, d->token, d->length_out, d->done_out, d->parent, d->first, d->stride,
                   reinterpret_cast<float2 *>(ws), reinterpret_cast<float *>(ws + lay.top)};
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (d->dtype == HEISD_DTYPE_F32) beam_launch<float>(a, st);
  else if (d->dtype == HEISD_DTYPE_BF16) beam_launch<__bf16>(a, st);
  else beam_launch<_Float16>(a, st);
  return launched(who);
}

// ---- requests that continue others --------------------------------------------------------------------------------------

extern "C" int heisd_paged_reorder(const heisd_reorder_desc *d, void *stream) {
  const char *who = "paged_reorder";
  if (!d) return fail(nullptr, HEISD_EINVAL, "%s: NULL description", who);
  if (d->batch < 1 || d->batch > 65535) return fail(nullptr, HEISD_EINVAL, "%s: batch=%d (1..65535)", who, d->batch);
  if (d->block_size < 1 || d->n_blocks < 1 || d->max_blocks < 1 || d->max_blocks > (1 << 20) ||
      (int64_t)d->n_blocks * d->block_size > 0x7FFFFFFF || (int64_t)d->max_blocks * d->block_size > 0x7FFFFFFF)
    return fail(nullptr, HEISD_EINVAL, "%s: block_size=%d n_blocks=%d max_blocks=%d (at most 2^31 - 1 slots, 2^20 blocks per request)", who,
                d->block_size, d->n_blocks, d->max_blocks);
  if (!d->parent || !d->len_in || !d->owned_in || !d->table_in || !d->len_out || !d->owned_out || !d->table_out || !d->copy_from || !d->free_ids ||
      !d->free_count_in || !d->free_count_out)
    return fail(nullptr, HEISD_EINVAL, "%s: NULL pointer", who);
  if (d->len_out == d->len_in || d->owned_out == d->owned_in || d->table_out == d->table_in || d->len_out == d->parent || d->copy_from == d->parent ||
      d->copy_from == d->len_in)
    return fail(nullptr, HEISD_EINVAL, "%s: lengths, owned blocks, tables or parents in place", who);
  const ReorderArgs a{d->batch, d->block_size, d->max_blocks, d->n_blocks, d->trim != 0, d->parent, d->len_in, d->owned_in, d->table_in, d->len_out,
                      d->owned_out, d->table_out, d->copy_from, d->free_ids, d->free_count_in, d->free_count_out};
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const int64_t entries = (int64_t)d->batch * d->max_blocks;
  if (d->batch <= 64 && entries <= 1024) reorder_books<1, true><<<dim3(1), dim3(64), 0, st>>>(a);
  else if (d->batch <= 256 && entries <= 8192) reorder_books<4, true><<<dim3(1), dim3(256), 0, st>>>(a);
  else {
    if (d->batch <= 256) reorder_books<4, false><<<dim3(1), dim3(256), 0, st>>>(a);
    else reorder_books<16, false><<<dim3(1), dim3(1024), 0, st>>>(a);
    reorder_tables<<<dim3((d->batch + 3) / 4), dim3(256), 0, st>>>(a);
  }
  return launched(who);
}

// Layers of a cache: `layer_bytes` from one pool to the next.
static int layers_ok(const char *who, const heisd_kv4_desc *cache, int32_t layers, int64_t layer_bytes) {
  if (layers < 1 || layers > 65535) return fail(nullptr, HEISD_EINVAL, "%s: %d layers (1..65535)", who, layers);
  const size_t pool = heisd_kv4_pool_bytes(cache->n_blocks, cache->block_size, cache->kv_heads, cache->head_dim);
  if (layers > 1 && (layer_bytes < (int64_t)pool || (layer_bytes & 15) || layer_bytes > (int64_t)1 << 42))
    return fail(nullptr, HEISD_EINVAL, "%s: layers %lld bytes apart (at least %zu, a multiple of 16)", who, (long long)layer_bytes, pool);
  return HEISD_OK;
}
static int64_t kv4_weights(const Kv4Cache &c) { return (int64_t)c.n_blocks * c.kv_heads * c.block_size; }

extern "C" int heisd_kv4_copy(const heisd_kv4_desc *cache, int32_t layers, int64_t layer_bytes, const heisd_paged_batch *batch, const int32_t *copy_from,
                              float *weight, int32_t max_seq, void *stream) {
  const char *who = "kv4_copy";
  Kv4Cache c;
  PagedBatch b;
  int rc = kv4_ok(who, cache, &c);
  if (rc == HEISD_OK) rc = batch_ok(who, batch, false, &b);
  if (rc == HEISD_OK) rc = layers_ok(who, cache, layers, layer_bytes);
  if (rc != HEISD_OK) return rc;
  if (!copy_from || max_seq < 1) return fail(nullptr, HEISD_EINVAL, "%s: NULL copy_from or max_seq=%d", who, max_seq);
  const int64_t blocks = std::min<int64_t>(((int64_t)max_seq + c.block_size - 1) / c.block_size, b.max_blocks);
  const int64_t pieces = c.kv_heads * (c.cell / 16), per_block = (pieces + 256 * kCopyPieces - 1) / (256 * kCopyPieces);
  if ((rc = groups_ok(who, blocks * per_block)) != HEISD_OK) return rc;
  const CopyArgs a{copy_from, weight, layer_bytes, kv4_weights(c), max_seq, cache->head_dim};
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  kv4_copy_blocks<<<dim3((unsigned)(blocks * per_block), b.batch, layers), dim3(256), 0, st>>>(c, b, a, (int)per_block);
  return launched(who);
}

// ---- attention over a shared prefix ---------------------------------------------------------------------------------------

static int groups_desc_ok(const char *who, const heisd_prefix_groups *g, PrefixGroups *out) {
  if (!g || !g->groups) {                            // nobody shares anything
    *out = PrefixGroups{nullptr, nullptr, 0, 0, 0};
    return HEISD_OK;
  }
  if (!g->first || !g->prefix) return fail(nullptr, HEISD_EINVAL, "%s: NULL pointer of the groups", who);
  if (g->groups < 0 || g->groups > 65535 || g->max_rows < 1 || g->max_prefix < 1 || g->max_prefix > (1 << 24))
    return fail(nullptr, HEISD_EINVAL, "%s: groups=%d (0..65535) max_rows=%d max_prefix=%d (1..2^24)", who, g->groups, g->max_rows, g->max_prefix);
  *out = PrefixGroups{g->first, g->prefix, g->groups, g->max_rows, g->max_prefix};
  return HEISD_OK;
}

// As Kv4Plan, with the groups' work beside the requests'.  Groups of many columns are kv4_prefix's.  Where the requests' own tokens are few, nothing of them is cut, and a
// workgroup knows by its number what it has to do (`direct`): prefixes are cut into a power of two of runs then, so that there are kSplitGroups workgroups for them
// (four requests behind 95 tokens: 12.8 us in two kernels, 18.8 as runs).
// us a call, narrow / wide on four waves / on eight, 4 query heads per key head, 8 key heads of 128, bf16, prefixes of up to 8191 tokens: eight groups of 64 columns 71.0 / 64.3 /
// 63.8, of 96 90.8 / 68.4 / 67.0, of 128 166 / 77.7 / 74.1, of 192 200 / 101 / 90.1; two of 64 31.3 / 40.9 / 31.1, of 1792 394 / 137 / 122; one of 128 40.4 / 36.2 / 33.5, of 256 59.8 /
// 39.6 / 42.2.  fp16: eight of 64 76.1 / 71.4 / 68.2, of 128 178 / 86.1 / 78.5; two of 64 32.9 / 44.6 / 32.8.  Heads of 64: eight of 64 59.7 / 45.7 / 50.1, of 128 144 / 57.8 / 60.1.  So the
// two numbers below fit heads of 64; heads of 128 would nearly always have eight waves.
// Own tokens whole (up to kWholeTokens) / cut, two groups of four requests of up to 250, 500 and 1000 own tokens 20.8 / 21.6, 17.4 / 20.1 and 21.6 / 23.6, eight of eight of up to 1000
// 42.7 / 46.3, two of 64 of up to 900 with seven rows each 148 / 199; of up to 2000, for which the limit would have to be 4096, 23.8 / 26.7 and 50.6 / 56.9.
constexpr int64_t kWideLeast = 64, kWideMany = 192, kWholeTokens = 1024, kSplitGroups = 512, kSplitTokens = 4096;
struct SharedPlan {
  int col_tiles, unit, wide_waves, direct, split_shift;
  int64_t groups, wide, tiles, depth;
  size_t part_ml, whole, whole_ml, wide_part, wide_ml, book, group_of, total;
  SharedPlan(int64_t batch, int64_t rows, int64_t kv_heads, int64_t group, int64_t max_q, int64_t max_seq, const PrefixGroups &p, int64_t head_dim) {
    const int64_t own_cols = std::min<int64_t>(max_q * group, 1 << 22), cols = std::min<int64_t>(p.max_rows * group, 1 << 22);
    wide_waves = cols >= kWideMany ? 8 : 4;
    const int64_t wide_cols = 32 * wide_waves;
    wide = p.groups && cols >= kWideLeast
               ? std::min<int64_t>(p.groups * kv_heads * ((cols + wide_cols - 1) / wide_cols) * ((p.max_prefix + 255) / 256), 8 / wide_waves * kKv4Units) : 0;
    col_tiles = (wide ? own_cols : std::max(own_cols, cols)) > 16 ? 2 : 1;
    const int64_t tile = 16 * col_tiles, most = kv4_shared_per_unit(col_tiles) * kKv4Units;
    const int64_t own_tiles = (own_cols + tile - 1) / tile, group_tiles = wide ? 0 : (cols + tile - 1) / tile;
    tiles = std::max<int64_t>(own_tiles, group_tiles);
    for (split_shift = 0; !wide && p.groups && (1 << split_shift) < kSplitsMost && ((int64_t)p.groups * kv_heads * group_tiles << split_shift) < kSplitGroups &&
                          (kKv4Unit << split_shift) < p.max_prefix;) ++split_shift;
    depth = batch + (wide ? 0 : (int64_t)p.groups << split_shift);
    direct = max_seq <= kWholeTokens && (wide || p.max_prefix <= kSplitTokens << split_shift) && tiles <= 65535 && depth <= 65535;
    unit = direct ? kWholeTokens : kKv4Unit;
    const int64_t own = batch * std::min<int64_t>(kv_heads * own_tiles, 65535) * ((max_seq + unit - 1) / unit);
    const int64_t shared = wide ? 0 : (int64_t)p.groups * std::min<int64_t>(kv_heads * group_tiles, 65535) * ((p.max_prefix + kKv4Unit - 1) / kKv4Unit);
    groups = direct ? 0 : std::max<int64_t>(1, std::min<int64_t>((own + shared + 1) / 2, most));
    part_ml = align256((size_t)2 * groups * tile * head_dim * sizeof(float));
    whole = part_ml + align256((size_t)2 * groups * tile * 2 * sizeof(float));
    const size_t parts = 1 + (direct && !wide ? (size_t)1 << split_shift : 1);      // by row: own tokens, the prefix or its runs
    whole_ml = whole + align256(parts * rows * group * kv_heads * head_dim * sizeof(float));
    wide_part = whole_ml + align256(parts * rows * group * kv_heads * 2 * sizeof(float));
    wide_ml = wide_part + align256((size_t)2 * wide * wide_cols * head_dim * sizeof(float));
    book = wide_ml + align256((size_t)2 * wide * wide_cols * 2 * sizeof(float));
    group_of = book + align256(wide ? p.groups * sizeof(WideBook) : 0);
    total = group_of + align256(wide ? batch * sizeof(int32_t) : 0);
  }
};

extern "C" size_t heisd_kv4_shared_attention_workspace_bytes(const heisd_kv4_desc *cache, int32_t batch, int32_t rows, int32_t q_heads, int32_t max_q,
                                                             int32_t max_seq, const heisd_prefix_groups *groups) {
  const char *who = "kv4_shared_attention_workspace_bytes";
  PrefixGroups p;
  if (!cache || !kv4_shape_ok(cache->n_blocks, cache->block_size, cache->kv_heads, cache->head_dim) || batch < 1 || batch > 65535 ||
      kv4_attention_sizes_ok(who, cache->kv_heads, q_heads, rows, max_q, max_seq) != HEISD_OK || groups_desc_ok(who, groups, &p) != HEISD_OK)
    return 0;
  return SharedPlan(batch, rows, cache->kv_heads, q_heads / cache->kv_heads, max_q, max_seq, p, cache->head_dim).total;
}

template <typename T, int HD, int W>
static hipError_t kv4_prefix_launch(const Kv4Cache &c, const PagedBatch &b, const HeadRows<const T> &q, const Kv4SharedAttend &a, hipStream_t st) {
  constexpr int lds = wide_lds_bytes<HD>;
  if constexpr (lds > 65536 - 1024) {                // above the usual limit of a workgroup (which has 1 KB beside it), which is raised once per device
    static std::atomic<bool> raised[kRetrieveMaxDevices];
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess && (dev < 0 || dev >= kRetrieveMaxDevices)) e = hipErrorInvalidDevice;
    if (e == hipSuccess && !raised[dev].load()) {
      e = hipFuncSetAttribute(reinterpret_cast<const void *>(&kv4_prefix<T, HD, W>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (e == hipSuccess) raised[dev].store(true);
    }
    if (e != hipSuccess) return e;
  }
  kv4_prefix<T, HD, W><<<dim3((unsigned)a.wide), dim3(64 * W), lds, st>>>(c, b, q, a);
  return hipSuccess;
}

template <typename T, int HD, int TERMS>
static hipError_t kv4_shared_launch(const Kv4Cache &c, const PagedBatch &b, const heisd_head_rows *q, const heisd_head_rows *out, const Kv4SharedAttend &a,
                              const SharedPlan &plan, int max_q, hipStream_t st) {
  const HeadRows<T> qi = head_rows<T>(*q), o = head_rows<T>(*out);
  const HeadRows<const T> qc{qi.p, qi.rs, qi.hs};
  const dim3 block(256), grid = plan.direct ? dim3(c.kv_heads, (unsigned)plan.tiles, (unsigned)plan.depth) : dim3((unsigned)plan.groups);
  if (plan.wide) {
    const hipError_t e = plan.wide_waves == 8 ? kv4_prefix_launch<T, HD, 8>(c, b, qc, a, st) : kv4_prefix_launch<T, HD, 4>(c, b, qc, a, st);
    if (e != hipSuccess) return e;
  }
  if (plan.col_tiles == 2) kv4_shared<T, HD, 2, TERMS><<<grid, block, 0, st>>>(c, b, qc, o, a);
  else kv4_shared<T, HD, 1, TERMS><<<grid, block, 0, st>>>(c, b, qc, o, a);
  if (plan.direct && plan.wide) return hipSuccess;
  const int64_t per = 256 / (HD / 4), cols = std::min<int64_t>((int64_t)max_q * a.q_heads, (int64_t)b.rows * a.q_heads);
  const dim3 joins((unsigned)std::min<int64_t>((cols + per - 1) / per, 65535), b.batch);
  if (plan.direct) kv4_direct_join<T, HD><<<joins, block, 0, st>>>(c, b, o, a);
  else kv4_shared_join<T, HD><<<joins, block, 0, st>>>(c, b, o, a, (int)plan.groups);
  return hipSuccess;
}

extern "C" int heisd_kv4_shared_attention(const heisd_kv4_desc *cache, const heisd_paged_batch *batch, const heisd_prefix_groups *groups,
                                          const heisd_head_rows *q, const heisd_head_rows *out, float *lse, float scale, int32_t max_q,
                                          int32_t max_seq, void *workspace, size_t workspace_bytes, void *stream) {
  const char *who = "kv4_shared_attention";
  Kv4Cache c;
  PagedBatch b;
  PrefixGroups p;
  int rc = kv4_ok(who, cache, &c);
  if (rc == HEISD_OK) rc = batch_ok(who, batch, true, &b);
  if (rc == HEISD_OK) rc = groups_desc_ok(who, groups, &p);
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
  const SharedPlan plan(b.batch, b.rows, c.kv_heads, q->heads / c.kv_heads, max_q, max_seq, p, cache->head_dim);
  if (!workspace || ((uintptr_t)workspace & 255)) return fail(nullptr, HEISD_EINVAL, "%s: NULL or misaligned workspace", who);
  if (workspace_bytes < plan.total) return fail(nullptr, HEISD_ENOMEM, "%s: workspace %zu bytes < %zu needed", who, workspace_bytes, plan.total);
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  Kv4SharedAttend a;
  static_cast<Kv4Attend &>(a) = Kv4Attend{std::max(std::fabs(scale) * 1.4426950408889634f, 1e-30f),      // not 0: minus infinity stands for masked scores
                                          scale < 0, q->heads / c.kv_heads, q->heads, max_seq, 16 * plan.col_tiles,
                                          reinterpret_cast<float *>(ws), reinterpret_cast<float *>(ws + plan.part_ml), lse};
  a.prefix = p;
  a.unit_shift = __builtin_ctz(plan.unit);
  a.cols_shift = __builtin_ctz(a.cols);
  a.group_shift = (a.group & (a.group - 1)) ? -1 : __builtin_ctz(a.group);
  a.wide = (int)plan.wide;
  a.wide_shift = __builtin_ctz(32 * plan.wide_waves);
  a.direct = plan.direct;
  a.split_shift = plan.split_shift;
  a.wide_part = reinterpret_cast<float *>(ws + plan.wide_part);
  a.wide_ml = reinterpret_cast<float *>(ws + plan.wide_ml);
  a.book = reinterpret_cast<WideBook *>(ws + plan.book);
  a.group_at = reinterpret_cast<int32_t *>(ws + plan.group_of);
  a.whole = reinterpret_cast<float *>(ws + plan.whole);
  a.whole_ml = reinterpret_cast<float *>(ws + plan.whole_ml);
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  hipError_t e;
  if (q->dtype == HEISD_DTYPE_BF16) {
    if (cache->head_dim == 128) e = kv4_shared_launch<__bf16, 128, 1>(c, b, q, out, a, plan, max_q, st);
    else e = kv4_shared_launch<__bf16, 64, 1>(c, b, q, out, a, plan, max_q, st);
  } else {
    if (cache->head_dim == 128) e = kv4_shared_launch<_Float16, 128, 2>(c, b, q, out, a, plan, max_q, st);
    else e = kv4_shared_launch<_Float16, 64, 2>(c, b, q, out, a, plan, max_q, st);
  }
  if (e != hipSuccess) return fail(nullptr, HEISD_EHIP, "%s: %s", who, hipGetErrorString(e));
  return launched(who);
}

extern "C" int heisd_paged_offset(const heisd_paged_batch *batch, const int32_t *offset, int32_t *position, void *stream) {
  const char *who = "paged_offset";
  PagedBatch b;
  if (const int rc = batch_ok(who, batch, true, &b)) return rc;
  if (!offset || (!position && b.rows > 0)) return fail(nullptr, HEISD_EINVAL, "%s: NULL pointer", who);
  if (b.rows == 0) return HEISD_OK;
  (void)hipGetLastError();
  offset_positions<<<dim3((b.rows + 255) / 256), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(b, offset, position);
  return launched(who);
}

// ---- attention weights and eviction ----------------------------------------------------------------------------------------

constexpr int64_t kWeighFill = 4096;

extern "C" int heisd_kv4_weigh(const heisd_kv4_desc *cache, const heisd_paged_batch *batch, const heisd_prefix_groups *groups, const heisd_head_rows *q,
                               const float *lse, float scale, float decay, const float *weight_in, float *weight_out, int32_t max_seq, void *stream) {
  const char *who = "kv4_weigh";
  Kv4Cache c;
  PagedBatch b;
  PrefixGroups p;
  int rc = kv4_ok(who, cache, &c);
  if (rc == HEISD_OK) rc = batch_ok(who, batch, true, &b);
  if (rc == HEISD_OK) rc = groups_desc_ok(who, groups, &p);
  if (rc == HEISD_OK) rc = rows_ok(who, "q", q, b.rows);
  if (rc == HEISD_OK) rc = kv4_attention_sizes_ok(who, c.kv_heads, q->heads, b.rows, 1, max_seq);
  if (rc != HEISD_OK) return rc;
  if (q->dtype == HEISD_DTYPE_F32) return fail(nullptr, HEISD_EUNSUPPORTED, "%s: q in fp32 (bf16 or fp16)", who);
  if (!rows_aligned(*q, 16)) return fail(nullptr, HEISD_EINVAL, "%s: q (16 bytes) misaligned", who);
  if ((!lse && b.rows > 0) || !weight_in || !weight_out || !std::isfinite(scale) || !std::isfinite(decay))
    return fail(nullptr, HEISD_EINVAL, "%s: NULL pointer, scale %g or decay %g", who, scale, decay);
  const WeighArgs a{scale * 1.4426950408889634f, decay, q->heads / c.kv_heads, q->heads, max_seq, lse, weight_in, weight_out};
  // As many pairs per wave as leave some workgroups per compute unit, counted with the largest lengths (kWeighFill 8192 / 4096 / 2048 / 1024: 38.9 / 35.8 / 53.6 / 74.1 us
  // with 64 contexts of up to 7847 tokens).
  const int64_t units = ((int64_t)std::max(max_seq, p.max_prefix) + kWeighUnit - 1) / kWeighUnit;
  const int pairs = (int)std::max<int64_t>(1, std::min<int64_t>(kWeighPairs, units * c.kv_heads * b.batch / kWeighFill));
  const dim3 grid((unsigned)((units + pairs - 1) / pairs), c.kv_heads, b.batch), block(256);
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const HeadRows<__bf16> qb = head_rows<__bf16>(*q);
  const HeadRows<const __bf16> qc{qb.p, qb.rs, qb.hs};
  const HeadRows<const _Float16> qh{reinterpret_cast<const _Float16 *>(qb.p), qb.rs, qb.hs};
  if (q->dtype == HEISD_DTYPE_BF16) {
    if (cache->head_dim == 128) kv4_weigh<__bf16, 128, 1><<<grid, block, 0, st>>>(c, b, p, qc, a, pairs);
    else kv4_weigh<__bf16, 64, 1><<<grid, block, 0, st>>>(c, b, p, qc, a, pairs);
  } else {
    if (cache->head_dim == 128) kv4_weigh<_Float16, 128, 2><<<grid, block, 0, st>>>(c, b, p, qh, a, pairs);
    else kv4_weigh<_Float16, 64, 2><<<grid, block, 0, st>>>(c, b, p, qh, a, pairs);
  }
  return launched(who);
}

// Keys are held in registers up to 16384 tokens.  us, eight keys per thread / sixteen / read again: 16 contexts of 2000 tokens to 1024 21.8 / 25.0 / 25.7, of 8192 to 1024
// 30.3 / 33.4 / 54.7, to 8000 19.5 / 24.6 / 51.4; of 16384 to 16000 - / 35.7 / 96.7.  (256 threads for up to 2048 tokens: 31.7, the moves take them all.)
template <int HD>
static void kv4_evict_launch(const Kv4Cache &c, const PagedBatch &b, const EvictArgs &a, dim3 grid, hipStream_t st) {
  const dim3 block(kEvictThreads);
  if (a.max_seq <= 8 * kEvictThreads) kv4_evict_held<HD, 8><<<grid, block, 0, st>>>(c, b, a);
  else if (a.max_seq <= 16 * kEvictThreads) kv4_evict_held<HD, 16><<<grid, block, 0, st>>>(c, b, a);
  else kv4_evict<HD><<<grid, block, 0, st>>>(c, b, a);
}

extern "C" int heisd_kv4_evict(const heisd_kv4_desc *cache, int32_t layers, int64_t layer_bytes, const heisd_paged_batch *batch, const int32_t *keep,
                               int32_t recent, const float *weight_in, float *weight_out, int32_t *seq_out, int32_t max_seq, void *stream) {
  const char *who = "kv4_evict";
  Kv4Cache c;
  PagedBatch b;
  int rc = kv4_ok(who, cache, &c);
  if (rc == HEISD_OK) rc = batch_ok(who, batch, false, &b);
  if (rc == HEISD_OK) rc = layers_ok(who, cache, layers, layer_bytes);
  if (rc != HEISD_OK) return rc;
  if (!keep || !weight_in || !weight_out || !seq_out || recent < 0 || max_seq < 1 || max_seq > (1 << 24))
    return fail(nullptr, HEISD_EINVAL, "%s: NULL pointer, recent=%d or max_seq=%d (1..2^24)", who, recent, max_seq);
  if (seq_out == b.seq_len || seq_out == keep) return fail(nullptr, HEISD_EINVAL, "%s: lengths in place", who);
  const EvictArgs a{keep, recent, max_seq, layer_bytes, kv4_weights(c), weight_in, weight_out, seq_out};
  const dim3 grid(c.kv_heads, b.batch, layers);
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (cache->head_dim == 128) kv4_evict_launch<128>(c, b, a, grid, st);
  else kv4_evict_launch<64>(c, b, a, grid, st);
  return launched(who);
}
