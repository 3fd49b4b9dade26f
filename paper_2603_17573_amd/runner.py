"""Torch-facing plumbing around the C ABI: device buffers, pointers, streams.  No arithmetic."""
import numpy as np
import torch

from . import binding as B

_SHAPE_KEYS = ("n_layers", "d_model", "n_heads", "head_dim", "d_ffn", "vocab", "n_bins", "rms_eps",
               "rope_base")
_LAYER_MATS = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down")


def _to_dev(a, device):
    """numpy uint16 (bf16 bits) -> bf16 tensor; float -> fp32 tensor; tensors pass through."""
    if isinstance(a, torch.Tensor):
        return a.to(device)
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(a.astype(np.float32)).to(device)


class DeviceModel:
    """The target model's weights resident in HBM (caller-owned from the library's point of view)."""

    def __init__(self, shape, weights, device="cuda:0"):
        self.shape = {k: getattr(shape, k) for k in _SHAPE_KEYS}
        self.shape["bin_token_base"] = shape.vocab - shape.n_bins
        self.device = torch.device(device)
        self.t = {}
        for k in ("tok_emb", "lm_head", "final_norm"):
            self.t[k] = _to_dev(weights[k], self.device)
        for k in _LAYER_MATS + ("attn_norm", "ffn_norm"):
            self.t[k] = [_to_dev(w, self.device) for w in weights[k]]

    def pointers(self):
        p = {k: self.t[k].data_ptr() for k in ("tok_emb", "lm_head", "final_norm")}
        for k in _LAYER_MATS + ("attn_norm", "ffn_norm"):
            p[k] = [w.data_ptr() for w in self.t[k]]
        return p


class Verifier:
    """Owns a heisd_verify_ctx and its workspace; step() marshals tensors into one C call."""

    def __init__(self, model: DeviceModel, max_batch: int, max_k: int, kv_capacity: int):
        self.model = model
        self.max_batch, self.max_k, self.kv_capacity = max_batch, max_k, kv_capacity
        desc, self._keep = B.make_model_desc(model.shape, model.pointers(), max_batch, max_k, kv_capacity)
        nbytes = B.heisd_verify_workspace_bytes(desc)
        if nbytes == 0:
            raise ValueError("invalid model description")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=model.device)
        desc.workspace, desc.workspace_bytes = self.workspace.data_ptr(), nbytes
        self.desc = desc
        rc, ctx = B.heisd_verify_init(desc)
        if rc != 0:
            raise RuntimeError("heisd_verify_init failed (%d): %s" % (rc, B.heisd_last_error(None)))
        self.ctx = ctx

    def new_cache(self, batch: int):
        s = self.model.shape
        shp = (s["n_layers"], batch, s["n_heads"], self.kv_capacity, s["head_dim"])
        return (torch.zeros(shp, dtype=torch.bfloat16, device=self.model.device),
                torch.zeros(shp, dtype=torch.bfloat16, device=self.model.device))

    def step(self, k_cache, v_cache, prefix_len, first_pred, draft_tokens, accept, skip_mask=None,
             want_aux=True, out=None, stream=None):
        """draft_tokens i32[batch,K] on the device.  Returns dict of device tensors (enqueued on the
        stream, not synchronised).  `out` lets a timing loop reuse the output tensors."""
        batch, K = draft_tokens.shape
        dev = self.model.device
        if out is None:
            out = {"accepted_len": torch.empty(batch, dtype=torch.int32, device=dev),
                   "next_token": torch.empty(batch, dtype=torch.int32, device=dev)}
            if want_aux:
                out["target_bins"] = torch.empty(batch, K + 1, dtype=torch.int32, device=dev)
                out["bin_logits"] = torch.empty(batch, K, self.model.shape["n_bins"], dtype=torch.float32,
                                                device=dev)
        kv = B.heisd_kv_desc(k_cache.data_ptr(), v_cache.data_ptr(), prefix_len.data_ptr(),
                             first_pred.data_ptr())
        st = (stream or torch.cuda.current_stream(dev)).cuda_stream
        rc = B.heisd_verify_step(self.ctx, kv, draft_tokens.data_ptr(), K, batch, accept,
                                 skip_mask.data_ptr() if skip_mask is not None else None,
                                 out["accepted_len"].data_ptr(), out["next_token"].data_ptr(),
                                 out["target_bins"].data_ptr() if "target_bins" in out else None,
                                 out["bin_logits"].data_ptr() if "bin_logits" in out else None, st)
        if rc != 0:
            raise RuntimeError("heisd_verify_step failed (%d): %s" % (rc, B.heisd_last_error(self.ctx)))
        return out

    def tree_step(self, k_cache, v_cache, prefix_len, first_pred, tree_tokens, parent, accept, skip_mask=None,
                  want_aux=True, out=None, stream=None):
        """tree_tokens, parent: i32[batch,T] on the device.  Returns dict of device tensors."""
        batch, T = tree_tokens.shape
        dev = self.model.device
        if out is None:
            out = {"accepted_len": torch.empty(batch, dtype=torch.int32, device=dev),
                   "next_token": torch.empty(batch, dtype=torch.int32, device=dev),
                   "accepted_path": torch.empty(batch, T, dtype=torch.int32, device=dev)}
            if want_aux:
                out["target_bins"] = torch.empty(batch, T + 1, dtype=torch.int32, device=dev)
                out["bin_logits"] = torch.empty(batch, T, self.model.shape["n_bins"], dtype=torch.float32,
                                                device=dev)
        kv = B.heisd_kv_desc(k_cache.data_ptr(), v_cache.data_ptr(), prefix_len.data_ptr(),
                             first_pred.data_ptr())
        st = (stream or torch.cuda.current_stream(dev)).cuda_stream
        rc = B.heisd_verify_tree_step(self.ctx, kv, tree_tokens.data_ptr(), parent.data_ptr(), T, batch, accept,
                                      skip_mask.data_ptr() if skip_mask is not None else None,
                                      out["accepted_len"].data_ptr(), out["next_token"].data_ptr(),
                                      out["accepted_path"].data_ptr(),
                                      out["target_bins"].data_ptr() if "target_bins" in out else None,
                                      out["bin_logits"].data_ptr() if "bin_logits" in out else None, st)
        if rc != 0:
            raise RuntimeError("heisd_verify_tree_step failed (%d): %s" % (rc, B.heisd_last_error(self.ctx)))
        return out

    def prefill_chunk(self, k_cache, v_cache, prefix_len, token_ids=None, x_rows=None, want_logits=False,
                      out=None, stream=None):
        """token_ids i32[batch,n], x_rows f32[batch,n,d] on the device, or both (then a row whose id is
        negative takes its embedding from x_rows).  Returns dict of device tensors: next_bin i32[batch]
        (and last_logits f32[batch,n_bins])."""
        src = token_ids if token_ids is not None else x_rows
        batch, n = src.shape[0], src.shape[1]
        dev = self.model.device
        if out is None:
            out = {"next_bin": torch.empty(batch, dtype=torch.int32, device=dev)}
            if want_logits:
                out["last_logits"] = torch.empty(batch, self.model.shape["n_bins"], dtype=torch.float32, device=dev)
        kv = B.heisd_kv_desc(k_cache.data_ptr(), v_cache.data_ptr(), prefix_len.data_ptr(), None)
        st = (stream or torch.cuda.current_stream(dev)).cuda_stream
        rc = B.heisd_prefill_chunk(self.ctx, kv, token_ids.data_ptr() if token_ids is not None else None,
                                   x_rows.data_ptr() if x_rows is not None else None, n, batch,
                                   out["next_bin"].data_ptr(),
                                   out["last_logits"].data_ptr() if "last_logits" in out else None, st)
        if rc != 0:
            raise RuntimeError("heisd_prefill_chunk failed (%d): %s" % (rc, B.heisd_last_error(self.ctx)))
        return out

    def close(self):
        if self.ctx is not None:
            B.heisd_free(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def build_sequence_tree(candidates, accept, max_tokens):
    """Host call: candidates i32[R,K] (numpy) -> (tokens[T], parent[T]) numpy arrays."""
    cand = np.ascontiguousarray(candidates, dtype=np.int32)
    R, K = cand.shape
    tokens = np.zeros(max_tokens, np.int32)
    parent = np.zeros(max_tokens, np.int32)
    rc, n = B.heisd_build_sequence_tree(cand.ctypes.data, R, K, accept, max_tokens, tokens.ctypes.data,
                                        parent.ctypes.data)
    if rc != 0:
        raise RuntimeError("heisd_build_sequence_tree failed (%d): %s" % (rc, B.heisd_last_error(None)))
    return tokens[:n].copy(), parent[:n].copy()


# ---- requests that share one pool ---------------------------------------------------------------------------------

_DTYPE = {torch.bfloat16: B.HEISD_DTYPE_BF16, torch.float16: B.HEISD_DTYPE_F16, torch.float32: B.HEISD_DTYPE_F32}


def head_rows(t: torch.Tensor) -> B.heisd_head_rows:
    """[rows, heads, head_dim] in any order of rows and heads; the values of a head must be adjacent."""
    if t.dim() != 3 or t.dtype not in _DTYPE or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError("expected [rows, heads, head_dim] of bf16, fp16 or fp32 with adjacent values, got %s %s strides %s"
                         % (tuple(t.shape), t.dtype, t.stride()))
    return B.heisd_head_rows(t.data_ptr(), t.stride(0), t.stride(1), t.shape[1], _DTYPE[t.dtype])


def _ints(t, shape, what, device):
    if t.dtype != torch.int32 or not t.is_contiguous() or tuple(t.shape) != tuple(shape) or t.device != device or not t.is_cuda:
        raise ValueError("%s: expected contiguous int32 %s on %s, got %s %s on %s"
                         % (what, tuple(shape), device if device.type == "cuda" else "a GPU", t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _floats(t, n, what, device):
    if t.dtype != torch.float32 or not t.is_contiguous() or t.numel() != n or t.device != device or not t.is_cuda:
        raise ValueError("%s: expected %d contiguous float32 on %s, got %s %s on %s"
                         % (what, n, device if device.type == "cuda" else "a GPU", t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def make_plan_desc(block_size, n_blocks, cached_len, new_len, owned_in, owned_out, block_table, free_ids, free_count_in, free_count_out,
                   seq_len, cu_rows, slot, position, cu_seq=None) -> B.heisd_plan_desc:
    """The tensors of one heisd_paged_plan call, which must stay alive as long as the descriptor is used."""
    b, rows = cached_len.shape[0], slot.shape[0]
    d = B.heisd_plan_desc(b, block_size, block_table.shape[1], n_blocks, rows)
    for name, t, shape in (("cached_len", cached_len, (b,)), ("new_len", new_len, (b,)), ("owned_in", owned_in, (b,)),
                           ("owned_out", owned_out, (b,)), ("block_table", block_table, (b, block_table.shape[1])),
                           ("free_ids", free_ids, (n_blocks,)), ("free_count_in", free_count_in, (1,)),
                           ("free_count_out", free_count_out, (1,)), ("cu_rows", cu_rows, (b + 1,)), ("seq_len", seq_len, (b,)),
                           ("slot", slot, (rows,)), ("position", position, (rows,))):
        setattr(d, name, _ints(t, shape, name, cached_len.device))
    if cu_seq is not None:
        d.cu_seq = _ints(cu_seq, (b + 1,), "cu_seq", cached_len.device)
    return d


def make_rope_desc(rotary_dim, base=10000.0, scaling="none", factor=1.0, original_len=0, beta_fast=32.0, beta_slow=1.0, low_freq=1.0,
                   high_freq=4.0) -> B.heisd_rope_desc:
    return B.heisd_rope_desc(rotary_dim, B.ROPE_SCALING[scaling], original_len, base, factor, beta_fast, beta_slow, low_freq, high_freq)


def rope_table(desc: B.heisd_rope_desc, device):
    """(turns per position of every pair, fp64 on the device, and the magnitude): once per model."""
    rc, turns, magnitude = B.heisd_rope_table(desc)
    if rc != 0:
        raise ValueError("heisd_rope_table failed (%d): %s" % (rc, B.heisd_last_error(None)))
    return torch.tensor(turns, dtype=torch.float64, device=device), magnitude


def make_kv4_desc(pool: torch.Tensor, block_size, kv_heads, head_dim) -> B.heisd_kv4_desc:
    """pool: contiguous uint8 whose size is that of a whole number of blocks; it must stay alive as long as the descriptor is used."""
    cell = block_size * (head_dim + head_dim // 16) * kv_heads
    if pool.dtype != torch.uint8 or not pool.is_contiguous() or cell <= 0 or pool.numel() % cell or not pool.is_cuda:
        raise ValueError("pool: expected contiguous uint8 of a multiple of %d bytes on a GPU" % cell)
    return B.heisd_kv4_desc(pool.data_ptr(), pool.numel() // cell, block_size, kv_heads, head_dim)


def make_paged_batch(block_table, seq_len, cu_rows, rows) -> B.heisd_paged_batch:
    (b, most), dev = block_table.shape, block_table.device
    return B.heisd_paged_batch(_ints(block_table, (b, most), "block_table", dev), _ints(seq_len, (b,), "seq_len", dev),
                               _ints(cu_rows, (b + 1,), "cu_rows", dev) if cu_rows is not None else None, b, most, rows)


def make_beam_desc(logits, beams, width, score_in, score_out, beam, token, length_in=None, length_out=None, done_in=None, done_out=None,
                   end_token=-1, length_power=0.0, parent=None, first=0, stride=0) -> B.heisd_beam_desc:
    """The tensors of heisd_beam_select calls, which must stay alive as long as the descriptor is used.  logits: [groups * beams, vocab] with
    adjacent tokens; score_out, beam, token, length_out, done_out: [groups, width]; parent: i32, entries first + group * stride + n are written."""
    if logits.dim() != 2 or logits.dtype not in _DTYPE or not logits.is_cuda or (logits.shape[1] > 1 and logits.stride(1) != 1) or \
            beams < 1 or logits.shape[0] % beams:
        raise ValueError("logits: expected [groups * %d, vocab] of bf16, fp16 or fp32 with adjacent tokens on a GPU, got %s %s strides %s on %s"
                         % (beams, tuple(logits.shape), logits.dtype, logits.stride(), logits.device))
    rows, dev = logits.shape[0], logits.device
    groups = rows // beams
    d = B.heisd_beam_desc(logits.data_ptr(), logits.stride(0), _DTYPE[logits.dtype], groups, beams, width, logits.shape[1], end_token, length_power)
    d.score_in, d.score_out = _floats(score_in, rows, "score_in", dev), _floats(score_out, groups * width, "score_out", dev)
    for name, t, n in (("beam", beam, groups * width), ("token", token, groups * width), ("length_in", length_in, rows),
                       ("length_out", length_out, groups * width), ("done_in", done_in, rows), ("done_out", done_out, groups * width)):
        if t is not None:
            if t.numel() != n:
                raise ValueError("%s: expected %d values, got %s" % (name, n, tuple(t.shape)))
            setattr(d, name, _ints(t, t.shape, name, dev))
    if parent is not None:
        if parent.numel() < first + (groups - 1) * stride + width:
            raise ValueError("parent: %d entries, groups of %d from %d on, %d apart" % (parent.numel(), width, first, stride))
        d.parent, d.first, d.stride = _ints(parent, parent.shape, "parent", dev), first, stride
    return d


def make_reorder_desc(block_size, n_blocks, parent, len_in, owned_in, table_in, len_out, owned_out, table_out, copy_from, free_ids, free_count_in,
                      free_count_out, trim=False) -> B.heisd_reorder_desc:
    """The tensors of one heisd_paged_reorder call, which must stay alive as long as the descriptor is used."""
    b, most = table_in.shape
    d = B.heisd_reorder_desc(b, block_size, most, n_blocks, int(trim))
    for name, t, shape in (("parent", parent, (b,)), ("len_in", len_in, (b,)), ("owned_in", owned_in, (b,)), ("table_in", table_in, (b, most)),
                           ("len_out", len_out, (b,)), ("owned_out", owned_out, (b,)), ("table_out", table_out, (b, most)),
                           ("copy_from", copy_from, (b,)), ("free_ids", free_ids, (n_blocks,)), ("free_count_in", free_count_in, (1,)),
                           ("free_count_out", free_count_out, (1,))):
        setattr(d, name, _ints(t, shape, name, parent.device))
    return d


def make_prefix_groups(first, prefix, max_rows, max_prefix) -> B.heisd_prefix_groups:
    """first i32 [groups + 1], prefix i32 [groups]: group g is requests first[g] .. first[g + 1] - 1, which all see request prefix[g]'s tokens."""
    n = prefix.shape[0]
    return B.heisd_prefix_groups(_ints(first, (n + 1,), "first", prefix.device), _ints(prefix, (n,), "prefix", prefix.device), n, max_rows, max_prefix)


class PagedCache:
    """The caches of every layer of a batch of requests, held in 4 bits in one pool of blocks per layer, and the calls of a step in
    the order a decoder makes them: begin() once, then for every layer rotate(), append() and one of attend() (single
    tokens and drafts), prompt() (whole prompts into empty caches) or chunk() (chunks behind cached rows).

    Requests that continue others: share() says which ones see another request's tokens in front of their own, attend_shared() then takes the place of attend();
    fork() lets requests go on as continuations of others; weigh() adds up what attention the tokens receive (weights=True), evict() keeps those that received
    most.  offset() gives rows the positions that they have behind a prefix or after an eviction.

    max_batch requests of at most max_len tokens (rounded up to whole blocks); a step has at most max_rows packed rows.  Everything the calls need is allocated
    here (and by share()), so a step can be captured into a HIP graph (chunk() too, once its buffers have been made by a first call)."""

    def __init__(self, n_layers, q_heads, kv_heads, head_dim, max_batch, max_len, max_rows, n_blocks, block_size=64, rope=None,
                 layout="half", max_new=1, device="cuda:0", weights=False):
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.q_heads, self.kv_heads, self.head_dim, self.max_new = q_heads, kv_heads, head_dim, max_new
        self.block_size, self.n_blocks = block_size, n_blocks
        nbytes = B.heisd_kv4_pool_bytes(n_blocks, block_size, kv_heads, head_dim)
        if nbytes == 0:
            raise ValueError("invalid cache: %d blocks of %d tokens, %d heads of %d" % (n_blocks, block_size, kv_heads, head_dim))
        self.max_len = -(-max_len // block_size) * block_size      # what begin() takes: the plan knows blocks only
        i32 = dict(dtype=torch.int32, device=self.device)
        with torch.cuda.device(self.device):
            self.pools = torch.empty((n_layers, nbytes), dtype=torch.uint8, device=self.device)
            self.table = torch.full((max_batch, self.max_len // block_size), -1, **i32)
            self.owned = torch.zeros(max_batch, **i32)
            self.free_ids = torch.arange(n_blocks, **i32)
            self.free_count = torch.full((1,), n_blocks, **i32)
            self.seq_len = torch.full((max_batch,), -1, **i32)
            self.cu_rows, self.cu_seq = torch.zeros(max_batch + 1, **i32), torch.zeros(max_batch + 1, **i32)
            self.slot, self.position = torch.full((max_rows,), -1, **i32), torch.full((max_rows,), -1, **i32)
            self.descs = [make_kv4_desc(p, block_size, kv_heads, head_dim) for p in self.pools]
            n = B.heisd_kv4_attention_workspace_bytes(self.descs[0], max_batch, max_rows, q_heads, max_new, self.max_len)
            if n == 0:
                raise ValueError("invalid attention: %d query heads, %d rows, max_new %d, max_len %d" % (q_heads, max_rows, max_new, self.max_len))
            self.workspace = torch.empty(n, dtype=torch.uint8, device=self.device)
            self.weights = torch.empty((n_layers, n_blocks, kv_heads, block_size), device=self.device) if weights else None
            self.lengths, self.copy_from = torch.empty(max_batch, **i32), torch.empty(max_batch, **i32)
            self._cached = torch.full((max_batch,), -1, **i32) if weights else None      # tokens of requests that seq_len has none of, for evict()
            self._table, self._owned = torch.empty_like(self.table), torch.empty_like(self.owned)
            desc = rope if rope is not None else make_rope_desc(head_dim)
            self.rotary_dim, self.layout = desc.rotary_dim, B.ROPE_LAYOUT[layout]
            self.turns, self.magnitude = rope_table(desc, self.device)
        self.rows, self._kv, self._captured, self._shared = 0, {}, [], None
        self.batch = make_paged_batch(self.table, self.seq_len, self.cu_rows, 0)

    def _call(self, fn, *args):
        with torch.cuda.device(self.device):
            rc = fn(*args, torch.cuda.current_stream(self.device).cuda_stream)
        if rc != 0:
            raise RuntimeError("%s failed (%d): %s" % (fn.__name__, rc, B.heisd_last_error(None)))

    def _of_step(self, t, heads, what):
        if tuple(t.shape) != (self.rows, heads, self.head_dim) or t.device != self.device:
            raise ValueError("%s: expected [%d, %d, %d] on %s, got %s on %s" % (what, self.rows, heads, self.head_dim, self.device,
                                                                              tuple(t.shape), t.device))
        return head_rows(t)

    def _lse(self, t):
        if t is None:
            return None
        if t.dtype != torch.float32 or t.dim() != 2 or t.shape[0] < self.rows or t.shape[1] != self.q_heads or not t.is_contiguous() or t.device != self.device:
            raise ValueError("lse: expected contiguous float32 [%d or more, %d] on %s, got %s %s strides %s on %s"
                             % (self.rows, self.q_heads, self.device, t.dtype, tuple(t.shape), t.stride(), t.device))
        return t.data_ptr()

    def begin(self, cached_len, new_len, rows):
        """cached_len, new_len i32[max_batch] on the device (a negative cached_len: the request is finished and gives its blocks back);
        rows: packed rows of this step, at least the sum of new_len.  A request that does not fit has seq_len -1 afterwards."""
        if not 0 <= rows <= self.slot.shape[0]:
            raise ValueError("rows=%d, made for at most %d" % (rows, self.slot.shape[0]))
        if cached_len.data_ptr() == self.seq_len.data_ptr():
            cached_len = cached_len.clone()
        self._call(B.heisd_paged_plan, make_plan_desc(self.block_size, self.n_blocks, cached_len, new_len, self.owned, self.owned, self.table,
                                                      self.free_ids, self.free_count, self.free_count, self.seq_len, self.cu_rows,
                                                      self.slot[:rows], self.position[:rows], self.cu_seq))
        if self._cached is not None:
            self._cached.copy_(cached_len)
        self.rows, self.batch = rows, make_paged_batch(self.table, self.seq_len, self.cu_rows, rows)

    def rotate(self, q, k):
        """q and k of this step's rows, in place."""
        hq, hk = self._of_step(q, self.q_heads, "q"), self._of_step(k, self.kv_heads, "k")
        self._call(B.heisd_rope, self.turns.data_ptr(), self.magnitude, self.rotary_dim, self.layout, 0, self.position.data_ptr(), self.rows,
                   self.head_dim, hq, hq, hk, hk)

    def append(self, layer, k, v):
        self._call(B.heisd_kv4_append, self.descs[layer], self._of_step(k, self.kv_heads, "k"), self._of_step(v, self.kv_heads, "v"),
                   self.slot.data_ptr(), self.rows)

    def attend(self, layer, q, scale=None, out=None, lse=None):
        """Attention of this step's rows over everything their requests have cached, the rows themselves included."""
        out = torch.empty_like(q) if out is None else out
        hq, ho = self._of_step(q, self.q_heads, "q"), self._of_step(out, self.q_heads, "out")
        self._call(B.heisd_kv4_attention, self.descs[layer], self.batch, hq, ho, self._lse(lse),
                   self.head_dim ** -0.5 if scale is None else scale, self.max_new, self.max_len, self.workspace.data_ptr(),
                   self.workspace.numel())
        return out

    def offset(self, offset):
        """Adds offset i32[max_batch] to the positions of this step's rows, request by request: the length of the prefix that a request's tokens lie behind, the
        number of its tokens that were evicted.  Once per step, before rotate().  They are the caller's: after fork() a request has those of its parent (offset[parent])."""
        self._call(B.heisd_paged_offset, self.batch, _ints(offset, self.seq_len.shape, "offset", self.device), self.position.data_ptr())

    def share(self, first, prefix, max_rows, max_prefix=None, max_own=None):
        """first i32[groups + 1], prefix i32[groups]: the requests first[g] .. first[g + 1] - 1 see the tokens of request prefix[g] in front of their own, from
        now on (both may change between steps).  max_rows: at least the rows of a group in a step; max_prefix, max_own (max_len if not given): at least the longest prefix, and the
        longest request that has rows."""
        groups = make_prefix_groups(first, prefix, max_rows, self.max_len if max_prefix is None else max_prefix)
        if first.device != self.device:
            raise ValueError("first, prefix: expected on %s, got on %s" % (self.device, first.device))
        own = self.max_len if max_own is None else max_own
        n = B.heisd_kv4_shared_attention_workspace_bytes(self.descs[0], self.table.shape[0], self.slot.shape[0], self.q_heads, self.max_new, own, groups)
        if n == 0:
            raise ValueError("invalid groups: max_rows %d, max_prefix %d, max_own %d" % (max_rows, groups.max_prefix, own))
        with torch.cuda.device(self.device):
            self._shared = (groups, own, torch.empty(n, dtype=torch.uint8, device=self.device), first, prefix, set())

    def _sharing(self):
        """What share() was given last, kept for whatever this stream has queued, or a graph being captured, when share() is called again."""
        with torch.cuda.device(self.device):
            if not torch.cuda.is_current_stream_capturing():
                stream, seen = torch.cuda.current_stream(), self._shared[5]
                if stream.cuda_stream not in seen:                     # once per stream: it counts until the tensor is freed
                    for t in self._shared[2:5]:
                        t.record_stream(stream)
                    seen.add(stream.cuda_stream)
            elif all(self._shared is not s for s in self._captured):
                self._captured.append(self._shared)
        return self._shared[:3]

    def attend_shared(self, layer, q, scale=None, out=None, lse=None):
        """Attention of this step's rows over their group's prefix and everything their requests have cached."""
        if self._shared is None:
            raise ValueError("attend_shared without share")
        out = torch.empty_like(q) if out is None else out
        hq, ho = self._of_step(q, self.q_heads, "q"), self._of_step(out, self.q_heads, "out")
        groups, own, workspace = self._sharing()
        self._call(B.heisd_kv4_shared_attention, self.descs[layer], self.batch, groups, hq, ho, self._lse(lse),
                   self.head_dim ** -0.5 if scale is None else scale, self.max_new, own, workspace.data_ptr(), workspace.numel())
        return out

    def weigh(self, layer, q, lse, scale=None, decay=1.0):
        """Adds to the weight of every cached token (times decay) the attention that it receives from this step's rows, and begins the weights of
        this step's tokens (so no step that appends is left out); lse: what attend(), attend_shared() or chunk() of the same
        rows gave (prompt()'s is of keys as they are, not as they are held: weights are as far off as they).  Rows of requests that share a prefix count on its tokens, too:
        theirs is attend_shared()'s."""
        if self.weights is None:
            raise ValueError("weigh: made without weights")
        groups = self._sharing()[0] if self._shared is not None else None
        w = self.weights[layer].data_ptr()
        self._call(B.heisd_kv4_weigh, self.descs[layer], self.batch, groups, self._of_step(q, self.q_heads, "q"), self._lse(lse),
                   self.head_dim ** -0.5 if scale is None else scale, decay, w, w, self.max_len)      # not share()'s max_own: attend() goes as far

    def evict(self, keep, recent):
        """Cuts every request of more than keep[b] tokens (i32[max_batch], negative: it stays as it is) to keep[b], in every layer and head for itself: the last `recent`
        stay, and of the others those with the largest weights.  A request's tokens are those of the step begun last; of a request that this step left out, the
        cached_len that begin() was given; after fork(), what that returned.  Returns the lengths, i32[max_batch], which the next begin() takes as cached_len (the buffer is
        written again by the next evict() or fork())."""
        if self.weights is None:
            raise ValueError("evict: made without weights")
        w = self.weights.data_ptr()
        if keep.data_ptr() == self.lengths.data_ptr():
            keep = keep.clone()
        torch.where(self.seq_len >= 0, self.seq_len, self._cached, out=self._cached)
        self._call(B.heisd_kv4_evict, self.descs[0], len(self.descs), self.pools.shape[1], make_paged_batch(self.table, self._cached, None, 0),
                   _ints(keep, self.seq_len.shape, "keep", self.device), recent, w, w, self.lengths.data_ptr(), self.max_len)
        self._cached.copy_(self.lengths)
        torch.where(self.seq_len >= 0, self.lengths, self.seq_len, out=self.seq_len)
        return self.lengths

    def fork(self, parent, length, trim=False):
        """Request b goes on as a continuation of what was request parent[b] with its first length[parent[b]] tokens (i32[max_batch]; a parent outside
        0 .. max_batch - 1: it ends); trim: blocks behind those tokens are given back.  Between two steps.  Returns the lengths as evict() does; a request that got no blocks has -1."""
        shape, dev = self.seq_len.shape, self.device
        _ints(parent, shape, "parent", dev), _ints(length, shape, "length", dev)
        if length.data_ptr() == self.lengths.data_ptr():
            length = length.clone()
        self._call(B.heisd_paged_reorder, make_reorder_desc(self.block_size, self.n_blocks, parent, length, self.owned, self.table, self.lengths, self._owned,
                                                            self._table, self.copy_from, self.free_ids, self.free_count, self.free_count, trim))
        self._call(B.heisd_kv4_copy, self.descs[0], len(self.descs), self.pools.shape[1], make_paged_batch(self._table, self.lengths, None, 0),
                   self.copy_from.data_ptr(), None if self.weights is None else self.weights.data_ptr(), self.max_len)
        self.table.copy_(self._table)
        self.owned.copy_(self._owned)
        self.seq_len.fill_(-1)
        if self._cached is not None:
            self._cached.copy_(self.lengths)
        return self.lengths

    def prompt(self, q, k, v, scale=None, out=None, lse=None):
        """Causal attention of whole prompts over their own rows (nothing cached before them), as they are and not as they are held."""
        out = torch.empty_like(q) if out is None else out
        hq, ho = self._of_step(q, self.q_heads, "q"), self._of_step(out, self.q_heads, "out")
        hk, hv = self._of_step(k, self.kv_heads, "k"), self._of_step(v, self.kv_heads, "v")
        self._call(B.heisd_paged_prompt_attention, self.batch, hq, hk, hv, ho, self._lse(lse), self.head_dim,
                   self.head_dim ** -0.5 if scale is None else scale)
        return out

    def _chunk_rows(self, total, dtype):
        """[2, at least total, kv_heads, head_dim] for cached rows read back: a pair per dtype, of twice the size when it gets too small."""
        kv = self._kv.get(dtype)
        with torch.cuda.device(self.device):
            if kv is None or kv.shape[1] < total:
                rows = total if kv is None else max(total, min(2 * kv.shape[1], self.n_blocks * self.block_size))
                kv = self._kv[dtype] = None                        # the smaller one goes first
                kv = self._kv[dtype] = torch.empty((2, rows, self.kv_heads, self.head_dim), dtype=dtype, device=self.device)
            if not torch.cuda.is_current_stream_capturing():
                kv.record_stream(torch.cuda.current_stream())
            elif all(kv is not t for t in self._captured):         # the graph goes on reading and writing it, whatever comes after
                self._captured.append(kv)
        return kv

    def chunk(self, layer, q, total, scale=None, out=None, lse=None):
        """Causal attention of many rows per request over everything cached (total: at least the sum of the requests' lengths): the
        cached rows are read back once and multiplied as a prompt's."""
        out = torch.empty_like(q) if out is None else out
        hq, ho = self._of_step(q, self.q_heads, "q"), self._of_step(out, self.q_heads, "out")
        kv = self._chunk_rows(total, q.dtype)
        hk, hv = head_rows(kv[0]), head_rows(kv[1])
        self._call(B.heisd_kv4_gather, self.descs[layer], self.batch, self.cu_seq.data_ptr(), total, hk, hv)
        self._call(B.heisd_prompt_attention, hq, hk, hv, ho, self._lse(lse), self.cu_rows.data_ptr(),
                   self.cu_seq.data_ptr(), self.table.shape[0], self.rows, total, self.head_dim,
                   self.head_dim ** -0.5 if scale is None else scale, 1)
        return out


def beam_select(logits, beams, width, score, length=None, done=None, end_token=-1, length_power=0.0, parent=None, first=0, stride=0):
    """The `width` best continuations of every group of `beams` beams (heisd_beam_select): a dict of score, beam, token and, where they are given,
    length and done, [groups, width].  logits [groups * beams, vocab]; score f32, length and done i32 [groups * beams]; parent i32 takes, from entry
    first + group * stride on, which request every new beam continues, as PagedCache.fork() wants it."""
    if not logits.is_cuda or logits.dim() != 2 or beams < 1:
        raise ValueError("logits: expected [groups * beams, vocab] on a GPU, got %s on %s" % (tuple(logits.shape), logits.device))
    groups, dev = logits.shape[0] // beams, logits.device
    with torch.cuda.device(dev):
        out = {k: torch.empty((groups, width), dtype=torch.int32, device=dev)
               for k, given in (("beam", True), ("token", True), ("length", length is not None), ("done", done is not None)) if given}
        out["score"] = torch.empty((groups, width), device=dev)
        d = make_beam_desc(logits, beams, width, score, out["score"], out["beam"], out["token"], length, out.get("length"), done, out.get("done"),
                           end_token, length_power, parent, first, stride)
        n = B.heisd_beam_select_workspace_bytes(groups, beams, width, logits.shape[1])
        workspace = torch.empty(max(n, 1), dtype=torch.uint8, device=dev)
        rc = B.heisd_beam_select(d, workspace.data_ptr(), n, torch.cuda.current_stream(dev).cuda_stream)
    if rc != 0:
        raise RuntimeError("heisd_beam_select failed (%d): %s" % (rc, B.heisd_last_error(None)))
    return out
