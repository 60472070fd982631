"""Device-memory plumbing around the C ABI: uploads host arrays into torch
device tensors, fills the ABI structs with their addresses, allocates the
workspace and output buffers, and calls the library on torch's current
stream.  No arithmetic of the query happens here.

Inputs are plain host structures:
  tables = {"probe": {col: ndarray, "offsets": int64[n+1], "tokens": int32[nnz]},
            "build": {col: ndarray} or None, "prefix": int32[...]}
  model  = {"spec": <object with n_layers, d_model, ...>, "emb", "layers": [...],
            "final_norm", "lm_head"} with bf16 weights as uint16 bit patterns
  query  = <object with preds, labels, decision, agg, join, n_prefix, group_col,
            n_group_keys; AI_TRANSFORM by sampling: sampling = (temperature, top_k,
            top_p, min_p)>
"""
from __future__ import annotations

import ctypes as C

import numpy as np
import torch

from . import binding as B

_NP_DTYPE = {np.dtype(np.int8): B.AIQ_I8, np.dtype(np.int16): B.AIQ_I16, np.dtype(np.int32): B.AIQ_I32,
             np.dtype(np.float32): B.AIQ_F32}
_DECISION = {"binary_gt": B.AIQ_DECIDE_BINARY_GT, "argmax": B.AIQ_DECIDE_ARGMAX}
_AGG = {"count": B.AIQ_AGG_COUNT, "avg_label_count_by": B.AIQ_AGG_AVG_LABEL_COUNT_BY,
        "count_by_payload": B.AIQ_AGG_COUNT_BY_PAYLOAD, "sum_f32": B.AIQ_AGG_SUM_F32}
_LIST_KEYS = ("offsets", "tokens")
_TORCH_DTYPE = {torch.float32: B.AIQ_F32, torch.float16: B.AIQ_F16, torch.bfloat16: B.AIQ_BF16}


def _dev(a: np.ndarray, device) -> torch.Tensor:
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:   # bf16 bit patterns
        return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(a).to(device)


def _layers_opt(n_layers) -> int:
    # 0 asks for every layer; a request for zero layers is encoded as -1
    if n_layers is None:
        return 0
    return -1 if int(n_layers) == 0 else int(n_layers)


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


class DeviceModel:
    """Model weights resident in device memory plus the aiq_model struct.

    ``compute`` selects the projection type of a 16-bit model: "bf16" keeps the
    stored bf16 weights; "f16" uploads their fp16 images (exact except for
    |w| < 2**-14, which fp16 holds as subnormals) so that activations fed to
    the MFMA projections carry 10 mantissa bits instead of 7.  fp32 models
    are uploaded as they are."""

    def __init__(self, model: dict, device="cuda", compute: str | None = None):
        spec = model["spec"]
        self.spec = spec
        self.keep = []
        self.compute = "f32" if spec.dtype == "f32" else (compute or "f16")
        if self.compute not in ("f32", "bf16", "f16"):
            raise ValueError(compute)

        def up(a):
            t = _dev(a, device)
            if t.dtype == torch.bfloat16 and self.compute == "f16":   # fp16 images, converted by the library
                h = torch.empty(t.shape, dtype=torch.float16, device=t.device)
                B.aiq_convert_weights(t.data_ptr(), B.AIQ_BF16, h.data_ptr(), B.AIQ_F16, t.numel(),
                                      torch.cuda.current_stream(t.device).cuda_stream)
                t = h
            self.keep.append(t)
            return t

        self.emb = up(model["emb"])
        self.lm_head = up(model["lm_head"])
        self.final_norm = up(np.asarray(model["final_norm"], dtype=np.float32))
        L = len(model["layers"])
        self.layers = (B.aiq_layer * max(L, 1))()
        for i, lw in enumerate(model["layers"]):
            s = self.layers[i]
            s.attn_norm = _ptr(up(np.asarray(lw["attn_norm"], dtype=np.float32)))
            s.ffn_norm = _ptr(up(np.asarray(lw["ffn_norm"], dtype=np.float32)))
            for k in ("wq", "wk", "wv", "wo", "w_gate", "w_down"):
                setattr(s, k, _ptr(up(lw[k])))
            s.w_up = _ptr(up(lw["w_up"])) if "w_up" in lw else 0
        m = B.aiq_model()
        m.n_layers, m.d_model, m.n_heads = L, spec.d_model, spec.n_heads
        m.n_kv_heads, m.d_ff, m.vocab = spec.n_kv_heads, spec.d_ff, spec.vocab
        m.act = B.AIQ_ACT_SWIGLU if spec.act == "swiglu" else B.AIQ_ACT_GELU_ERF
        m.wdtype = {"f32": B.AIQ_F32, "bf16": B.AIQ_BF16, "f16": B.AIQ_F16}[self.compute]
        m.rope_theta, m.norm_eps = spec.rope_theta, spec.norm_eps
        m.emb, m.lm_head, m.final_norm = _ptr(self.emb), _ptr(self.lm_head), _ptr(self.final_norm)
        m.layers = C.cast(self.layers, C.POINTER(B.aiq_layer))
        self.struct = m


class DeviceTable:
    def __init__(self, cols: dict, device="cuda", with_list=True, max_list_len=None):
        self.names = [k for k in cols if k not in _LIST_KEYS]
        self.index = {k: i for i, k in enumerate(self.names)}
        self.tensors = {k: _dev(cols[k], device) for k in self.names}
        self.dtypes = {k: np.asarray(cols[k]).dtype for k in self.names}
        n = len(cols[self.names[0]]) if self.names else len(cols["offsets"]) - 1
        self.n_rows = n
        self.cols = (B.aiq_col * max(len(self.names), 1))()
        for i, k in enumerate(self.names):
            self.cols[i].data = _ptr(self.tensors[k])
            self.cols[i].dtype = _NP_DTYPE[self.dtypes[k]]
        t = B.aiq_table()
        t.n_rows, t.n_cols = n, len(self.names)
        t.cols = C.cast(self.cols, C.POINTER(B.aiq_col))
        if with_list:
            off = np.asarray(cols["offsets"], dtype=np.int64)
            self.offsets = _dev(off, device)
            t.list_offsets = _ptr(self.offsets)
            if "tokens" in cols:   # absent: offsets only (relational-only plans)
                tok = np.asarray(cols["tokens"], dtype=np.int32)
                self.tokens = _dev(tok if len(tok) else np.zeros(1, np.int32), device)
                t.list_tokens = _ptr(self.tokens)
            t.n_list_tokens = int(off[-1] - off[0])
            lens = np.diff(off)
            t.max_list_len = int(max_list_len if max_list_len is not None else max(1, lens.max(initial=1)))
        self.struct = t


def _pred(p, table: "DeviceTable") -> B.aiq_pred:
    s = B.aiq_pred()
    s.col = table.index[p.col]
    s.op = B.OPS[p.op]
    if table.dtypes[p.col].kind == "f":
        s.fk = float(p.k)
    else:
        s.k = int(p.k)
    vals = list(p.values)
    s.n_set = len(vals)
    for i, v in enumerate(vals):
        s.set[i] = int(v)
    return s


def make_query(query, probe: DeviceTable | None, build: DeviceTable | None, prefix) -> B.aiq_query:
    q = B.aiq_query()
    preds = list(getattr(query, "preds", ()))
    q.n_pred = len(preds)
    for i, p in enumerate(preds):
        q.preds[i] = _pred(p, probe)
    j = getattr(query, "join", None)
    if j is not None:
        q.join = 1
        q.probe_key_col = probe.index[j.probe_key]
        q.build_key_col = build.index[j.build_key]
        q.build_payload_col = build.index[j.payload]
        q.n_build_pred = len(j.build_preds)
        for i, p in enumerate(j.build_preds):
            q.build_preds[i] = _pred(p, build)
    n_prefix = int(getattr(query, "n_prefix", 0))
    q.n_prefix = n_prefix
    for i in range(n_prefix):
        q.prefix[i] = int(prefix[i])
    q.n_labels = len(query.labels)
    for i, l in enumerate(query.labels):
        q.label_ids[i] = int(l)
    q.decision = _DECISION[query.decision]
    q.agg = _AGG[query.agg]
    if getattr(query, "group_col", None):
        q.group_col = probe.index[query.group_col]
    q.n_group_keys = int(getattr(query, "n_group_keys", 0))
    q.gen_tokens = int(getattr(query, "gen_tokens", 0))
    q.eos_id = int(getattr(query, "eos_id", -1))
    q.pad_id = int(getattr(query, "pad_id", 0))
    like = tuple(getattr(query, "like", ()))
    q.n_like = len(like)
    for i, t in enumerate(like):
        q.like[i] = int(t)
    sm = getattr(query, "sampling", None)
    if sm is not None:
        q.sample = 1
        q.sampling.temperature, q.sampling.top_k = float(sm[0]), int(sm[1])
        q.sampling.top_p, q.sampling.min_p = float(sm[2]), float(sm[3])
    if getattr(query, "pair_key", None):
        q.pairs = 1
        q.pair_key_col = probe.index[query.pair_key]
        q.max_pairs = int(query.max_pairs)
    return q


class DeviceQuery:
    """A planned query over device-resident tables and weights.

    AI_TRANSFORM queries: ``kv_dtype`` "i8" keeps the keys and values that
    generation steps read in 8 bits (default 16); ``sample_u`` [probe rows,
    gen_tokens] holds the random numbers of a query that samples."""

    def __init__(self, tables: dict, model, query, device="cuda", chunk_tokens: int = 0,
                 n_layers: int | None = None, dmodel: DeviceModel | None = None, relational_only: bool = False,
                 want_sel: bool = True, share_prefix: bool = True, multipass_compact: bool = False,
                 full_last_layer: bool = False, kv_dtype: str = "f16", sample_u=None):
        if kv_dtype not in ("f16", "i8"):
            raise ValueError(kv_dtype)
        self.device = torch.device(device)
        self.query = query
        self.dm = dmodel if dmodel is not None else DeviceModel(model, device)
        self.probe = DeviceTable(tables["probe"], device)
        self.build = DeviceTable(tables["build"], device, with_list=False) if tables.get("build") is not None else None
        self.q = make_query(query, self.probe, self.build, tables.get("prefix", ()))
        if sample_u is not None:
            u = torch.as_tensor(sample_u, dtype=torch.float32).to(self.device).contiguous()
            if u.shape != (self.probe.n_rows, self.q.gen_tokens):
                raise ValueError(f"sample_u: [{self.probe.n_rows}, {self.q.gen_tokens}] wanted, got {tuple(u.shape)}")
            self.sample_u = u
            self.q.sample_u = _ptr(u)
        opts = B.aiq_plan_opts()
        opts.kv_dtype = B.AIQ_I8 if kv_dtype == "i8" else 0
        opts.chunk_tokens = int(chunk_tokens)
        opts.n_layers_override = _layers_opt(n_layers)
        opts.flags = (B.AIQ_PLAN_RELATIONAL_ONLY if relational_only else 0) | \
            (0 if share_prefix else B.AIQ_PLAN_UNSHARED_PREFIX) | \
            (B.AIQ_PLAN_MULTIPASS_COMPACT if multipass_compact else 0) | \
            (B.AIQ_PLAN_FULL_LAST_LAYER if full_last_layer else 0)
        self.plan = B.aiq_plan_create(self.dm.struct, self.probe.struct,
                                      self.build.struct if self.build else None, self.q, opts)
        self.ws_bytes = B.aiq_workspace_size(self.plan)
        self.ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=self.device)
        base = self.ws.data_ptr()
        self.ws_ptr = (base + 255) // 256 * 256
        n = self.probe.n_rows
        K = len(query.labels)
        dev = self.device
        self.pairs = bool(getattr(query, "pair_key", None))
        n = max(n, int(query.max_pairs)) if self.pairs else n   # outputs per row, or per pair
        self.scalars = torch.zeros(B.AIQ_N_SCALARS, dtype=torch.int64, device=dev)
        self.ids = torch.zeros(max(n, 1), dtype=torch.int32, device=dev)
        self.sel_ids = torch.zeros(max(n, 1), dtype=torch.int32, device=dev)
        self.sel_labels = torch.zeros(max(n, 1), dtype=torch.int32, device=dev)
        self.sel_logits = torch.zeros(max(n, 1) * K, dtype=torch.float32, device=dev)
        # dense keys: one group per key code; any int32 key (n_group_keys 0):
        # at most one group per probe row
        G = int(getattr(query, "n_group_keys", 0)) or n
        G = max(G, 1)
        self.grp_key = torch.zeros(G, dtype=torch.int32, device=dev)
        self.grp_count = torch.zeros(G, dtype=torch.int64, device=dev)
        self.grp_sum = torch.zeros(G, dtype=torch.int64, device=dev)
        self.grp_avg = torch.zeros(G, dtype=torch.float64, device=dev)
        self.sum_out = torch.zeros(1, dtype=torch.float64, device=dev)
        self.gen = int(getattr(query, "gen_tokens", 0))
        self.sel_gen = torch.zeros(max(n, 1) * max(self.gen, 1), dtype=torch.int32, device=dev)
        o = B.aiq_out()
        o.scalars, o.ids, o.ids_cap = _ptr(self.scalars), _ptr(self.ids), n
        o.sel_ids, o.sel_labels, o.sel_logits, o.sel_cap = (_ptr(self.sel_ids), _ptr(self.sel_labels),
                                                            _ptr(self.sel_logits), n if want_sel else 0)
        o.grp_key, o.grp_count, o.grp_sum, o.grp_avg = (_ptr(self.grp_key), _ptr(self.grp_count),
                                                        _ptr(self.grp_sum), _ptr(self.grp_avg))
        o.grp_cap = G
        o.sum_out = _ptr(self.sum_out)
        o.sel_gen = _ptr(self.sel_gen) if self.gen else None
        if self.pairs:
            self.pair_a = torch.zeros(n, dtype=torch.int32, device=dev)
            self.pair_b = torch.zeros(n, dtype=torch.int32, device=dev)
            self.cand_a = torch.zeros(n, dtype=torch.int32, device=dev)
            self.cand_b = torch.zeros(n, dtype=torch.int32, device=dev)
            o.pair_a, o.pair_b, o.cand_a, o.cand_b = (_ptr(self.pair_a), _ptr(self.pair_b), _ptr(self.cand_a),
                                                      _ptr(self.cand_b))
        self.out = o

    def run(self, trace=None, stream=None) -> None:
        s = stream if stream is not None else torch.cuda.current_stream(self.device)
        B.aiq_run(self.plan, self.ws_ptr, self.ws_bytes, self.out, trace, s.cuda_stream)

    def run_static(self, stream=None) -> None:
        """The relational-only plan through the entry point that allocates
        nothing (its scratch is the library's fixed device array)."""
        s = stream if stream is not None else torch.cuda.current_stream(self.device)
        B.aiq_run_relational_static(self.plan, self.out, s.cuda_stream)

    def results(self) -> dict:
        """Copies the outputs to the host (after the stream has been synchronised)."""
        sc = self.scalars.cpu().numpy()
        n_sel, n_kept, n_groups = int(sc[B.AIQ_S_SELECTED]), int(sc[B.AIQ_S_KEPT]), int(sc[B.AIQ_S_GROUPS])
        K = len(self.query.labels)
        r = {"scalars": sc, "status": int(sc[B.AIQ_S_STATUS]), "n_selected": n_sel, "count": n_kept,
             "n_tokens": int(sc[B.AIQ_S_TOKENS]),
             "kept_ids": self.ids[:n_kept].cpu().numpy().astype(np.int64),
             "sel_ids": self.sel_ids[:n_sel].cpu().numpy().astype(np.int64),
             "labels": self.sel_labels[:n_sel].cpu().numpy().astype(np.int64),
             "logits": self.sel_logits[:n_sel * K].cpu().numpy().reshape(n_sel, K)}
        if self.query.agg == "sum_f32":
            r["sum"] = float(self.sum_out.cpu().item())
        if self.gen:
            r["gen"] = self.sel_gen[:n_sel * self.gen].cpu().numpy().astype(np.int64).reshape(n_sel, self.gen)
        if self.pairs:   # labels / logits are per candidate pair; ids are kept pair numbers
            P = int(sc[B.AIQ_S_PAIRS])
            r.update(n_pairs=P, kept_pairs=r["kept_ids"],
                     pair_a=self.pair_a[:n_kept].cpu().numpy().astype(np.int64),
                     pair_b=self.pair_b[:n_kept].cpu().numpy().astype(np.int64),
                     cand_a=self.cand_a[:P].cpu().numpy().astype(np.int64),
                     cand_b=self.cand_b[:P].cpu().numpy().astype(np.int64),
                     labels=self.sel_labels[:P].cpu().numpy().astype(np.int64),
                     logits=self.sel_logits[:P * K].cpu().numpy().reshape(P, K))
        if self.query.agg in ("avg_label_count_by", "count_by_payload"):
            r["groups"] = (self.grp_key[:n_groups].cpu().numpy().astype(np.int64),
                           self.grp_count[:n_groups].cpu().numpy(), self.grp_sum[:n_groups].cpu().numpy(),
                           self.grp_avg[:n_groups].cpu().numpy())
        return r

    def close(self) -> None:
        if self.plan:
            B.aiq_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class DevicePrefill:
    """Prefill-only plan: runs the transformer on caller-packed sequences."""

    def __init__(self, model, labels=(1, 2), max_tokens: int = 4096, device="cuda",
                 n_layers: int | None = None, dmodel: DeviceModel | None = None, full_last_layer: bool = False):
        self.device = torch.device(device)
        self.dm = dmodel if dmodel is not None else DeviceModel(model, device)
        q = B.aiq_query()
        q.n_labels = len(labels)
        for i, l in enumerate(labels):
            q.label_ids[i] = int(l)
        q.decision = B.AIQ_DECIDE_BINARY_GT if len(labels) == 2 else B.AIQ_DECIDE_ARGMAX
        q.agg = B.AIQ_AGG_COUNT
        self.q = q
        self.K = len(labels)
        opts = B.aiq_plan_opts()
        opts.n_layers_override = _layers_opt(n_layers)
        opts.flags = B.AIQ_PLAN_FULL_LAST_LAYER if full_last_layer else 0
        self.plan = B.aiq_plan_create(self.dm.struct, None, None, q, opts)
        self.max_tokens = int(max_tokens)
        self.ws_bytes = B.aiq_prefill_workspace_size(self.plan, self.max_tokens)
        self.ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=self.device)
        self.ws_ptr = (self.ws.data_ptr() + 255) // 256 * 256

    def run(self, tok: torch.Tensor, cu: torch.Tensor, full_vocab: bool = False, stream=None) -> torch.Tensor:
        n_seq = cu.numel() - 1
        n_tok = tok.numel()
        width = self.dm.spec.vocab if full_vocab else self.K
        out = torch.empty(n_seq * width, dtype=torch.float32, device=self.device)
        s = stream if stream is not None else torch.cuda.current_stream(self.device)
        B.aiq_prefill_packed(self.plan, _ptr(tok), _ptr(cu), n_seq, n_tok,
                             B.AIQ_LOGITS_FULL_VOCAB if full_vocab else B.AIQ_LOGITS_LABELS,
                             _ptr(out), self.ws_ptr, self.ws_bytes, s.cuda_stream)
        return out.view(n_seq, width)

    def close(self) -> None:
        if self.plan:
            B.aiq_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _need(t: torch.Tensor, device, dtype, what: str) -> torch.Tensor:
    if t.device != device or t.dtype != dtype:
        raise ValueError(f"{what}: {dtype} on {device} wanted, got {t.dtype} on {t.device}")
    return t


class KvBatch:
    """The sequences of a call on a DeviceKvCache (see DeviceKvCache.batch), or on several: the caches of a model's layers, say."""

    def __init__(self, struct: B.aiq_kv_batch, keep: tuple, shape: tuple):
        self.struct = struct
        self.shape = shape    # K/V heads and head size of the cache that made it
        self.keep = keep      # the tensors that the struct points into
        self.device = keep[0].device
        self.n_rows = int(struct.n_rows)
        self.ws_bytes = {}    # attention workspace by query heads, for caches of the first one's shape; for others:
        self.ws_other = {}    # by (query heads, K/V heads, head size)

    def of(self, cache: "DeviceKvCache") -> B.aiq_kv_batch:
        """The struct, with the status word of the cache that a call is on."""
        if self.struct.status == cache.status.data_ptr():
            return self.struct
        b = B.aiq_kv_batch.from_buffer_copy(self.struct)
        b.status = _ptr(cache.status)
        return b


class DeviceKvCache:
    """Keys and values of many sequences in 8 bits, in blocks of 32 tokens with
    one scale per block and K/V head; the tokens of a last block that is not
    full yet are kept in 16 bits, one tail per sequence (include/aiq.h,
    aiq_kv_cache).  Rows are tensors [rows, heads, head_dim] of the cache's
    dtype whose heads lie next to each other (any row stride that is a multiple
    of 8: they may be columns of q|k|v rows)."""

    def __init__(self, n_blocks: int, n_tails: int, n_kv_heads: int, head_dim: int, dtype=torch.float16, device="cuda"):
        if dtype not in (torch.float16, torch.bfloat16):
            raise ValueError(f"keys and values are float16 or bfloat16, not {dtype}")
        self.device = _device(device)
        self.n_kv_heads, self.head_dim, self.dtype = int(n_kv_heads), int(head_dim), dtype
        nb, nt = int(n_blocks), int(n_tails)
        size = (nb, self.n_kv_heads, B.AIQ_KV_BLOCK * self.head_dim)
        # whole numbers of 0 (stored with 128 added), so that blocks that were never written hold zeros
        self.k = torch.full(size, 128, dtype=torch.uint8, device=self.device)
        self.v = torch.full(size, 128, dtype=torch.uint8, device=self.device)
        self.k_scale = torch.zeros(size[:2], dtype=torch.float32, device=self.device)
        self.v_scale = torch.zeros(size[:2], dtype=torch.float32, device=self.device)
        self.tail = torch.zeros((nt, 2, self.n_kv_heads, B.AIQ_KV_BLOCK, self.head_dim), dtype=dtype, device=self.device)
        self.status = torch.zeros(1, dtype=torch.int64, device=self.device)   # AIQ_DEV_KV_RANGE
        c = B.aiq_kv_cache()
        c.k, c.v, c.k_scale, c.v_scale, c.tail = (_ptr(t) for t in (self.k, self.v, self.k_scale, self.v_scale, self.tail))
        c.n_blocks, c.n_tails, c.n_kv_heads, c.head_dim, c.dtype = nb, nt, self.n_kv_heads, self.head_dim, _TORCH_DTYPE[dtype]
        self.struct = c

    def batch(self, length: torch.Tensor, blk_start: torch.Tensor, max_len: int, cu: torch.Tensor | None = None,
              n_rows: int | None = None, blk_ids: torch.Tensor | None = None,
              tail_ids: torch.Tensor | None = None) -> KvBatch:
        """Sequence i holds length[i] tokens once the call's rows cu[i] ..
        cu[i+1] are in (cu None: row i is its last token; length 0 is an empty
        slot), in the blocks blk_ids[blk_start[i] .. blk_start[i+1]] (None: the
        numbers themselves), with tail tail_ids[i] (None: i).  All int32
        tensors on the cache's device; they may change between calls, within
        max_len tokens and n_rows rows (None with cu: cu's last value is read
        back once, here).  The tensors are kept, not copied.  A batch may be used
        with other caches that have these blocks and tails, of any shape; each
        call sets the status of the cache that it is made on."""
        n = int(length.numel())
        for t, want, what in ((length, n, "length"), (blk_start, n + 1, "blk_start"), (cu, n + 1, "cu"),
                              (blk_ids, None, "blk_ids"), (tail_ids, n, "tail_ids")):
            if t is None:
                continue
            _need(t, self.device, torch.int32, what)
            if not t.is_contiguous() or (want is not None and t.numel() != want):
                raise ValueError(f"{what}: {want} contiguous values wanted, got {tuple(t.shape)}")
        if blk_ids is not None and not blk_ids.numel():   # (no address to tell it from None: one entry that is no block)
            blk_ids = torch.full((1,), -1, dtype=torch.int32, device=self.device)
        b = B.aiq_kv_batch()
        b.n_seq, b.max_len = n, int(max_len)
        b.n_rows = n if cu is None else int(cu[-1].item()) if n_rows is None else int(n_rows)
        b.len, b.cu, b.blk_start, b.blk_ids, b.tail_ids = (_ptr(t) for t in (length, cu, blk_start, blk_ids, tail_ids))
        b.n_blk_ids = 0 if blk_ids is None else blk_ids.numel()
        b.status = _ptr(self.status)
        return KvBatch(b, (length, blk_start, cu, blk_ids, tail_ids, self.status),
                       (self.n_kv_heads, self.head_dim))

    def _mine(self, batch: KvBatch) -> int:
        """The batch's rows; its tensors must be on the cache's device."""
        if batch.device != self.device:
            raise ValueError(f"batch: one on {self.device} wanted, got one on {batch.device}")
        return batch.n_rows

    def _rows(self, t: torch.Tensor, n_rows: int, heads: int | None, what: str) -> int:
        """Elements between rows of t [n_rows, heads, head_dim]."""
        shape = t.shape
        if t.device != self.device or t.dtype != self.dtype:
            raise ValueError(f"{what}: {self.dtype} on {self.device} wanted, got {t.dtype} on {t.device}")
        if len(shape) != 3 or shape[0] != n_rows or shape[2] != self.head_dim or (heads is not None and shape[1] != heads):
            raise ValueError(f"{what}: [{n_rows}, {heads or 'heads'}, {self.head_dim}] wanted, got {tuple(shape)}")
        row, head, one = t.stride()
        if n_rows and (one != 1 or (shape[1] > 1 and head != self.head_dim)):
            raise ValueError(f"{what}: a row's heads must lie next to each other (strides {t.stride()})")
        return row if n_rows > 1 else shape[1] * self.head_dim

    def write(self, batch: KvBatch, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """Appends the batch's rows."""
        n = self._mine(batch)
        ks, vs = (self._rows(t, n, self.n_kv_heads, w) for t, w in ((k, "k"), (v, "v")))
        with _on(self.device, stream) as s:
            B.aiq_kv_write(self.struct, batch.of(self), _ptr(k), ks, _ptr(v), vs, s)

    def read(self, batch: KvBatch, stream=None) -> tuple:
        """The batch's rows as the cache holds them: (k, v)."""
        n, w = self._mine(batch), self.n_kv_heads * self.head_dim
        with _on(self.device, stream) as s:
            k, v = (torch.empty((n, self.n_kv_heads, self.head_dim), dtype=self.dtype, device=self.device)
                    for _ in range(2))
            B.aiq_kv_read(self.struct, batch.of(self), _ptr(k), w, _ptr(v), w, s)
        return k, v

    def attend(self, batch: KvBatch, q: torch.Tensor, out: torch.Tensor | None = None,
               out_dtype: torch.dtype | None = None, stream=None) -> torch.Tensor:
        """Attention of the batch's rows q [rows, heads, head_dim] over the
        cache (their own tokens included), in out_dtype (default the cache's)."""
        qs = self._rows(q, self._mine(batch), None, "q")
        heads = q.shape[1]
        if out is not None and (out.shape != q.shape or not out.is_contiguous() or out.device != self.device):
            raise ValueError(f"out: contiguous {tuple(q.shape)} on {self.device} wanted")
        dtype = out.dtype if out is not None else out_dtype or self.dtype
        if dtype not in (torch.float16, torch.bfloat16):
            raise ValueError(f"out is float16 or bfloat16, not {dtype}")
        shape = (self.n_kv_heads, self.head_dim)
        sizes, key = (batch.ws_bytes, heads) if shape == batch.shape else (batch.ws_other, (heads, *shape))
        need = sizes.get(key)
        if need is None:
            need = sizes[key] = B.aiq_kv_attend_workspace_size(self.struct, batch.struct, heads)
        with _on(self.device, stream) as s:   # the workspace belongs to the stream that uses it
            if out is None:
                out = torch.empty(q.shape, dtype=dtype, device=self.device)
            ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
            B.aiq_kv_attend(self.struct, batch.of(self), _ptr(q), qs, heads, _ptr(out), heads * self.head_dim,
                            _TORCH_DTYPE[dtype], _ptr(ws), need, s)
        return out


class _on:
    """The device's given or current stream, current while tensors are
    allocated (they belong to the stream that uses them) and work is enqueued;
    `as` gives its handle."""

    def __init__(self, device: torch.device, stream):
        if stream is not None and stream.device != device:
            raise ValueError(f"stream: one of {device} wanted, got one of {stream.device}")
        self.device, self.stream = device, stream

    def __enter__(self) -> int:
        self.guards = ()
        if torch.cuda.current_device() != self.device.index:
            self.guards = (torch.cuda.device(self.device),)
        if self.stream is not None:
            self.guards += (torch.cuda.stream(self.stream),)
        for g in self.guards:
            g.__enter__()
        return (self.stream if self.stream is not None else torch.cuda.current_stream(self.device.index)).cuda_stream

    def __exit__(self, *e):
        for g in reversed(self.guards):
            g.__exit__(*e)


def _device(device) -> torch.device:
    d = torch.device(device)
    return torch.device(d.type, torch.cuda.current_device()) if d.type == "cuda" and d.index is None else d


def sample(logits: torch.Tensor, u: torch.Tensor | None, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0,
           min_p: float = 0.0, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The next token of each row of logits [rows, vocab] (float32, float16 or
    bfloat16; any row stride) with the random numbers u [rows] (float32 in
    [0, 1)): int32 [rows] (include/aiq.h, aiq_sample)."""
    if logits.dim() != 2 or logits.dtype not in _TORCH_DTYPE or logits.stride(1) != 1 and logits.numel():
        raise ValueError(f"logits: rows of float32, float16 or bfloat16 wanted, got {tuple(logits.shape)} {logits.dtype}")
    n, vocab = logits.shape
    dev = logits.device
    if dev.type != "cuda":
        raise ValueError("logits must be on a GPU")
    if u is not None:
        _need(u, dev, torch.float32, "u")
        if u.shape != (n,) or not u.is_contiguous():
            raise ValueError(f"u: {n} contiguous values wanted")
    if out is not None:
        _need(out, dev, torch.int32, "out")
        if out.shape != (n,) or not out.is_contiguous():
            raise ValueError(f"out: {n} contiguous values wanted")
    p = B.aiq_sampling()
    p.temperature, p.top_p, p.min_p, p.top_k = float(temperature), float(top_p), float(min_p), int(top_k)
    with _on(dev, stream) as s:
        if out is None:
            out = torch.empty(n, dtype=torch.int32, device=dev)
        B.aiq_sample(_ptr(logits), _TORCH_DTYPE[logits.dtype], logits.stride(0) if n > 1 else vocab, vocab, n, p, _ptr(u),
                     _ptr(out), s)
    return out
