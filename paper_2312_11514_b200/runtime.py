"""Device-memory plumbing around the C ABI: allocates the buffers a layer needs with torch
(pinned bundle store, window cache, workspace), creates the layer, and exposes the lists
inside the workspace as tensor views.  No arithmetic of the method lives here."""
from __future__ import annotations

import ctypes as C
import math
import struct
from typing import Dict, List, Optional, Sequence

import torch

from . import binding as B


class Layer:
    """One FFN layer: owns its torch buffers and the `lif_layer` handle."""

    def __init__(self, *, d_model: int, d_ff: int, rank: int, window_k: int, capacity: int,
                 host_bundles: torch.Tensor, bias_up: torch.Tensor,
                 pred_A: Optional[torch.Tensor] = None, pred_B: Optional[torch.Tensor] = None,
                 pred_c: Optional[torch.Tensor] = None,
                 bias_down: Optional[torch.Tensor] = None, n_streams: int = 1,
                 threshold_logit: float = 0.0, ffn_mode: int = 0, activation: int = 0,
                 activation_threshold: float = 0.0, budget_rows: int = 0, spec_keep: int = 0,
                 gate_mode: int = 0, gate: Optional[torch.Tensor] = None, append_first: int = 0,
                 staging_rows: int = 0, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2312_11514_b200 needs a CUDA device; there is no CPU path")
        self.device = torch.device(device)
        assert host_bundles.is_pinned() and host_bundles.dtype == torch.float16
        n_vec = 3 if gate_mode == B.GATE_BUNDLED else 2      # d_model-vectors per bundle
        # staging_rows > 0: the bundles live in a file and host_bundles is the staging buffer
        assert host_bundles.shape == (staging_rows or d_ff, n_vec * d_model) and host_bundles.is_contiguous()
        assert gate is None or (gate.shape == (d_ff, d_model) and gate.dtype == torch.float16
                                and gate.is_contiguous())
        self.d_model, self.d_ff, self.rank, self.capacity = d_model, d_ff, rank, capacity
        self.n_streams = n_streams
        self.keep = dict(host_bundles=host_bundles, pred_A=pred_A, pred_B=pred_B, pred_c=pred_c,
                         bias_up=bias_up, bias_down=bias_down, gate=gate)
        # One guard row past the cache and a guard block past the workspace, filled with a bit
        # pattern no kernel writes: `guards_intact()` tells whether anything ran past the end.
        self._cache_all = torch.zeros(capacity + 1, n_vec * d_model, dtype=torch.float16, device=self.device)
        self._cache_all[capacity].view(torch.int16).fill_(self._GUARD)
        self.cache = self._cache_all[:capacity]
        shape = dict(d_model=d_model, d_ff=d_ff, rank=rank, window_k=window_k, capacity=capacity,
                     n_streams=n_streams, threshold_logit=threshold_logit, ffn_mode=ffn_mode,
                     activation=activation, activation_threshold=activation_threshold,
                     budget_rows=budget_rows, spec_keep=spec_keep, gate_mode=gate_mode,
                     append_first=append_first, staging_rows=staging_rows)
        self.spec_keep, self.gate_mode = spec_keep, gate_mode
        nbytes = B.lif_workspace_bytes(B.make_desc(**shape))
        self._workspace_all = torch.zeros(nbytes + 256, dtype=torch.uint8, device=self.device)
        self._workspace_all[nbytes:].fill_(self._GUARD & 0xFF)
        self.workspace = self._workspace_all[:nbytes]
        with torch.cuda.device(self.device):
            self.handle = B.lif_create_layer(B.make_desc(
                **shape, host_bundles=host_bundles, pred_A=pred_A, pred_B=pred_B, pred_c=pred_c,
                bias_up=bias_up, bias_down=bias_down, gate=gate, cache=self.cache,
                workspace=self.workspace))
            torch.cuda.synchronize()   # the reset ran on the default stream
        self._lists = B.lif_get_lists(self.handle)
        self.counts = self._view("counts", B.CNT_LEN)

    _GUARD = 0x7B7B

    def guards_intact(self) -> bool:
        """True while the row after the cache and the block after the workspace still hold the
        pattern they were created with (synchronises)."""
        torch.cuda.synchronize(self.device)
        row_ok = bool((self._cache_all[self.capacity].view(torch.int16) == self._GUARD).all())
        ws_ok = bool((self._workspace_all[self.workspace.numel():] == (self._GUARD & 0xFF)).all())
        return row_ok and ws_ok

    def _view(self, name: str, n: int, dtype=torch.int32) -> torch.Tensor:
        off = getattr(self._lists, name) - self.workspace.data_ptr()
        size = n * torch.empty((), dtype=dtype).element_size()
        return self.workspace[off:off + size].view(dtype)

    def lists(self) -> Dict[str, object]:
        """Host copies of this step's lists and of the window state (synchronises)."""
        torch.cuda.synchronize(self.device)
        c = self.counts.cpu()
        na, ne, nm, nl, nh = (int(c[i]) for i in (B.CNT_N_ACTIVE, B.CNT_N_EVICT, B.CNT_N_MOVES,
                                                  B.CNT_N_LOAD, B.CNT_N_HITS))
        F, cap = self.d_ff, self.capacity
        out = {
            "active_idx": self._view("active_idx", F)[:na], "evict_ids": self._view("evict_ids", cap)[:ne],
            "move_src": self._view("move_src", cap)[:nm], "move_dst": self._view("move_dst", cap)[:nm],
            "load_ids": self._view("load_ids", cap)[:nl], "load_slots": self._view("load_slots", cap)[:nl],
            "active_slots": self._view("active_slots", F)[:na], "hit_slots": self._view("hit_slots", F)[:nh],
            "pointers": self._view("pointers", cap), "slot_of": self._view("slot_of", F),
            "last_active": self._view("last_active", F),
            "bias": self._view("bias", cap, torch.float16),
        }
        if self.spec_keep > 0:
            out["keep_token"] = self._view("keep_token", F, torch.int8)
        out = {k: v.cpu().numpy() for k, v in out.items()}
        out.update(num_used_before=int(c[B.CNT_NUM_USED_BEFORE]), num_kept=int(c[B.CNT_NUM_KEPT]),
                   num_used=int(c[B.CNT_NUM_USED]), step=int(c[B.CNT_STEP]), status=int(c[B.CNT_STATUS]),
                   k_eff=int(c[B.CNT_K_EFF]))
        return out

    def close(self) -> None:
        if getattr(self, "handle", None):
            intact = self.guards_intact()
            B.lif_destroy_layer(self.handle)
            self.handle = None
            if not intact:
                raise RuntimeError("a kernel wrote past the end of the cache or of the workspace")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def rope_frequencies(dims: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     context: int = 0, turns: Sequence[float] = (1.0, 32.0)) -> List[float]:
    """Radians per position of the ``dims / 2`` rotated pairs, base^(-2i / dims), for contexts
    ``factor`` times as long as ``context``, which the model was trained on:

    * ``"linear"``: every frequency divided by the factor;
    * ``"ntk"``: the base raised to base * factor^(dims / (dims - 2)): the lowest frequency is divided
      by the factor, the highest stays;
    * ``"by_parts"``: pairs with less than ``turns[0]`` turns in ``context`` positions divided by the
      factor, those with more than ``turns[1]`` as they are, a linear blend in between (the usual
      ``rope_scale`` beside it is 0.1 ln(factor) + 1)."""
    if dims < 2 or dims % 2 or not base > 0 or not factor >= 1:
        raise ValueError(f"rope_frequencies: dims={dims}, base={base}, factor={factor}")
    if scaling == "ntk":
        base = base * factor ** (dims / (dims - 2)) if dims > 2 else base
    elif scaling == "by_parts":
        if context < 1 or not turns[0] < turns[1]:
            raise ValueError("rope_frequencies: by_parts needs the trained context and turns[0] < turns[1]")
    elif scaling not in ("none", "linear"):
        raise ValueError(f"rope_frequencies: scaling {scaling!r}")
    out = []
    for i in range(dims // 2):
        f = base ** (-2.0 * i / dims)
        if scaling == "linear":
            f /= factor
        elif scaling == "by_parts":
            share = (context * f / (2 * math.pi) - turns[0]) / (turns[1] - turns[0])
            share = min(1.0, max(0.0, share))
            f = f * share + f / factor * (1.0 - share)
        out.append(f)
    return out


# lif_kv_rows and lif_kv_norms as bytes: a quarter of the time that ctypes takes to fill a structure
_ROWS, _NORMS = struct.Struct("=3q").pack, struct.Struct("=4q").pack


class KvCache:
    """A paged key-value cache for the attention between the FFN layers (include/lif_kv.h): owns its
    workspace (and the pool, unless ``pages`` is given) and the handle.  Tensors are checked here for
    device, type and shape; the calls run on ``stream``, by default the current stream of the cache's
    device, which has to be the current device (``stats`` and ``close`` see to it themselves; others
    raise LIF_ERR_STATE).  All calls of one cache are to be ordered (one stream, or events between streams),
    and tensors given stay until the call's stream is done with them.  An output
    that a call makes itself (``q_out``, ``out`` left out) is memory of the call's stream: on another
    stream it is to be used as any tensor of that stream is (an event, ``record_stream``).

    ``pages``: the pool, ``[n_layers][n_pages][2][n_kv_heads][page_tokens][head_dim]``; ``lens``,
    ``n_new``, ``table``, ``refs``: views of the tables on the device."""

    _TYPES = {torch.float16: B.TYPE_F16, torch.bfloat16: B.TYPE_BF16}

    def __init__(self, *, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, n_pages: int, max_seqs: int,
                 max_pages: Optional[int] = None, page_tokens: int = 64, max_new: int = 1, dtype=torch.float16,
                 window: int = 0, scale: Optional[float] = None, norm: int = B.NORM_NONE, norm_eps: float = 1e-5,
                 rope: int = B.ROPE_NONE, rope_dims: int = 0, rope_freq: Optional[Sequence[float]] = None,
                 rope_scale: float = 1.0, pages: Optional[torch.Tensor] = None, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2312_11514_b200 needs a CUDA device; there is no CPU path")
        if dtype not in self._TYPES:
            raise ValueError(f"KvCache: dtype {dtype} (float16 or bfloat16)")
        self.device = torch.device(device if pages is None else pages.device)
        self.dtype, self.max_seqs, self.max_new, self.norm = dtype, max_seqs, max_new, norm
        self.n_heads, self.n_kv_heads, self.head_dim, self.n_layers = n_heads, n_kv_heads, head_dim, n_layers
        self.max_pages = n_pages if max_pages is None else max_pages
        self._index = self.device.index if self.device.index is not None else torch.cuda.current_device()
        self._queries, self._keys = (max_seqs, max_new, n_heads, head_dim), (max_seqs, max_new, n_kv_heads, head_dim)
        self._places, self._table, self._head = (max_seqs,), (max_seqs, self.max_pages), (head_dim,)
        self._lib, self._both = B.lib(), max_seqs > 1 and max_new > 1
        shape = dict(n_layers=n_layers, n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim,
                     dtype=self._TYPES[dtype], page_tokens=page_tokens, n_pages=n_pages, max_seqs=max_seqs,
                     max_pages=self.max_pages, max_new=max_new, window=window, scale=scale or 0.0, norm=norm,
                     norm_eps=norm_eps, rope=rope, rope_dims=rope_dims if rope != B.ROPE_NONE else 0,
                     rope_scale=rope_scale)
        nbytes = B.lif_kv_workspace_bytes(B.make_kv_desc(**shape))
        pool = (n_layers, n_pages, 2, n_kv_heads, page_tokens, head_dim)
        if pages is None:
            pages = torch.zeros(pool, dtype=dtype, device=self.device)
        self._expect("pages", pages, pool)
        self.pages = pages
        freq = None
        if rope != B.ROPE_NONE:
            if rope_freq is None or len(rope_freq) != rope_dims // 2:
                raise ValueError(f"KvCache: rope_freq holds rope_dims / 2 = {rope_dims // 2} frequencies")
            freq = (C.c_double * len(rope_freq))(*rope_freq)
        # a guard block past the workspace, as for Layer
        self._workspace_all = torch.zeros(nbytes + 256, dtype=torch.uint8, device=self.device)
        self._workspace_all[nbytes:].fill_(self._GUARD)
        self.workspace = self._workspace_all[:nbytes]
        with torch.cuda.device(self.device):
            torch.cuda.synchronize()
            self.handle = B.lif_kv_create(B.make_kv_desc(**shape, rope_freq=freq, pages=pages, workspace=self.workspace))
        state = B.lif_kv_get_state(self.handle)
        view = lambda at, n: self.workspace[at - self.workspace.data_ptr():][:4 * n].view(torch.int32)
        self.counts = view(state.counts, B.KV_CNT_LEN)
        self.lens, self.n_new = view(state.lens, max_seqs), view(state.n_new, max_seqs)
        self.table = view(state.table, max_seqs * self.max_pages).view(max_seqs, self.max_pages)
        self.refs = view(state.refs, n_pages)

    _GUARD = 0x7B

    def _expect(self, name, t, shape, dtype=None, contiguous=True):
        # (a decode step makes several calls a layer: what is compared here is what torch answers fastest)
        if t.get_device() != self._index or t.dtype is not (dtype or self.dtype) or t.shape != shape or \
                (contiguous and not t.is_contiguous()):
            raise ValueError(f"KvCache: {name} is {tuple(t.shape)} {t.dtype} on {t.device}"
                             f"{'' if t.is_contiguous() else ', not contiguous'}; expected {tuple(shape)} "
                             f"{dtype or self.dtype} on {self.device}")

    def _ints(self, name, t, shape=None):
        if t is not None:
            self._expect(name, t, shape or self._places, torch.int32)
        return t

    def _on(self, stream):
        return torch._C._cuda_getCurrentRawStream(self._index) if stream is None else stream

    def _new(self, stream):
        # Memory of the stream that writes it: the current stream's may be a block that work pending there still uses.
        if stream is None:
            return torch.empty(self._queries, dtype=self.dtype, device=self.device)
        if not isinstance(stream, torch.cuda.Stream):
            at = B._stream(stream)
            stream = torch.cuda.ExternalStream(at, self.device) if at else torch.cuda.default_stream(self.device)
        with torch.cuda.stream(stream):
            return torch.empty(self._queries, dtype=self.dtype, device=self.device)

    def _rows(self, name, t, shape):
        if t.get_device() != self._index or t.dtype is not self.dtype or t.shape != shape:
            self._expect(name, t, shape, contiguous=False)
        places, tokens, step, element = t.stride()
        # places lie max_new tokens apart
        if element != 1 or (self._both and places != self.max_new * tokens):
            raise ValueError(f"KvCache: {name} has strides {t.stride()}; places have to lie max_new tokens apart, "
                             f"a head's elements beside each other")
        # a KvRows (torch leaves the stride of a dimension of one element undefined)
        if self.max_new == 1:
            tokens = places if self.max_seqs > 1 else 0
        return _ROWS(t.data_ptr(), tokens, step if shape[2] > 1 else 0)

    def reserve(self, n_new: torch.Tensor, stream=None) -> None:
        B.lif_kv_reserve(self.handle, self._ints("n_new", n_new), self._on(stream))

    def append(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_out: Optional[torch.Tensor] = None,
               norms: Optional[Sequence[Optional[torch.Tensor]]] = None, stream=None) -> torch.Tensor:
        """q ``[max_seqs][max_new][n_heads][head_dim]``, k and v with n_kv_heads; views into a fused
        projection's output are fine.  ``norms``: query weight, query bias, key weight, key bias.
        Returns the normed and rotated queries (rows of tokens that are not there are not written)."""
        index, dtype, head = self._index, self.dtype, self._head
        if q_out is None:
            q_out = self._new(stream)
        else:
            self._expect("q_out", q_out, self._queries)
        weights = None
        if self.norm and norms is not None:
            if len(norms) != 4:
                raise ValueError(f"KvCache: {len(norms)} norm tensors; expected query weight and bias, key weight and bias")
            at = []
            for t in norms:
                if t is None:
                    at.append(0)
                    continue
                if t.dtype is not dtype or t.get_device() != index or t.shape != head or not t.is_contiguous():
                    self._expect("norm weight", t, head)
                at.append(t.data_ptr())
            weights = _NORMS(*at)
        stream = torch._C._cuda_getCurrentRawStream(index) if stream is None else B._stream(stream)
        code = self._lib.lif_kv_append(self.handle, layer, self._rows("q", q, self._queries), self._rows("k", k, self._keys),
                                       self._rows("v", v, self._keys), weights, q_out.data_ptr(), stream)
        if code:
            raise B.LifError(code, "lif_kv_append")
        return q_out

    def attention(self, layer: int, q: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """q as `append` returns it; ``out`` of the same shape, in other memory.  Rows of tokens that are not
        there are not written: in an output made here they hold anything, NaN included, and are to be
        masked before sums over them."""
        self._expect("q", q, self._queries)
        if out is None:
            out = self._new(stream)
        else:
            self._expect("out", out, self._queries)
        stream = torch._C._cuda_getCurrentRawStream(self._index) if stream is None else B._stream(stream)
        code = self._lib.lif_kv_attention(self.handle, layer, q.data_ptr(), out.data_ptr(), stream)
        if code:
            raise B.LifError(code, "lif_kv_attention")
        return out

    def fork(self, src: Optional[torch.Tensor] = None, length: Optional[torch.Tensor] = None, stream=None) -> None:
        B.lif_kv_fork(self.handle, self._ints("src", src), self._ints("length", length), self._on(stream))

    def load(self, lens: torch.Tensor, table: torch.Tensor, n_new: Optional[torch.Tensor] = None, stream=None) -> None:
        B.lif_kv_load(self.handle, self._ints("lens", lens), self._ints("table", table, self._table),
                      self._ints("n_new", n_new), self._on(stream))

    def compact(self, stream=None) -> None:
        B.lif_kv_compact(self.handle, self._on(stream))

    def reset(self, stream=None) -> None:
        B.lif_kv_reset(self.handle, self._on(stream))

    def clear_status(self, stream=None) -> None:
        B.lif_kv_clear_status(self.handle, self._on(stream))

    def stats(self) -> Dict[str, int]:
        """Status, free pages, pages copied by the last call, calls refused (synchronises)."""
        with torch.cuda.device(self.device):
            c = B.lif_kv_get_stats(self.handle)
        return dict(status=c[B.KV_CNT_STATUS], free=c[B.KV_CNT_FREE], copies=c[B.KV_CNT_COPIES],
                    refused=c[B.KV_CNT_REFUSED])

    def close(self) -> None:
        if getattr(self, "handle", None):
            torch.cuda.synchronize(self.device)
            intact = bool((self._workspace_all[self.workspace.numel():] == self._GUARD).all())
            B.lif_kv_destroy(self.handle)
            self.handle = None
            if not intact:
                raise RuntimeError("a kernel wrote past the end of the workspace")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def pinned_store(d_ff: int, d_model: int, n_vec: int = 2) -> torch.Tensor:
    """Pinned (and, under unified addressing, device-mapped) host tensor for one layer's
    bundle store, fp16 [d_ff][n_vec*d_model] (n_vec = 3 when the gate row is bundled)."""
    return torch.empty(d_ff, n_vec * d_model, dtype=torch.float16, pin_memory=True)


def neuron_shard(d_ff: int, rank: int, world: int):
    """Ids [lo, hi) of the neurons that device ``rank`` of ``world`` owns when one layer's
    neurons are split over several devices: equal contiguous shares, each a multiple of 8
    (the layer description's rule for d_ff)."""
    if world < 1 or not 0 <= rank < world or d_ff % (8 * world):
        raise ValueError(f"d_ff={d_ff} does not split into {world} shares that are multiples of 8")
    per = d_ff // world
    return rank * per, (rank + 1) * per


def sum_partial_outputs(y: torch.Tensor, group=None) -> torch.Tensor:
    """The one exchange of a neuron-sharded layer-step: every device holds the FFN terms of its
    own neurons in ``y`` (fp32 ``[n_streams][d_model]``); afterwards every device holds their
    sum.  In place, on the current stream (NCCL) or on the host (gloo).  One device: no-op."""
    import torch.distributed as dist
    if dist.is_available() and dist.is_initialized() and dist.get_world_size(group) > 1:
        dist.all_reduce(y, op=dist.ReduceOp.SUM, group=group)
    return y


class PeerExchange:
    """The exchange of a neuron-sharded token over peer-mapped device memory instead of a
    library all-reduce.  Every rank writes its partial output of layer l into slot l of a
    buffer that all ranks of the group have mapped (torch symmetric memory: allocation and
    address exchange only); after a barrier across the ranks, ``lif_sum_peer_outputs`` reads
    all ranks' slots with plain loads and adds them in rank order, so every rank gets the same
    bits.  A slot is rewritten only in the next token, after ``end_token``'s barrier, so one
    barrier per layer is enough.  Call the methods with the compute stream current."""

    def __init__(self, n_layers: int, n_streams: int, d_model: int, device, group=None):
        import torch.distributed as dist
        import torch.distributed._symmetric_memory as symm
        group = group if group is not None else dist.group.WORLD
        self.partials = symm.empty(n_layers, n_streams, d_model, dtype=torch.float32,
                                   device=torch.device(device))
        self.handle = symm.rendezvous(self.partials, group)
        self.slot_bytes = n_streams * d_model * 4
        self.peer_ptrs = [int(p) for p in self.handle.buffer_ptrs]     # rank order
        assert self.peer_ptrs[self.handle.rank] == self.partials.data_ptr()

    def sum_layer(self, l: int, y: torch.Tensor, stream=None) -> None:
        """y = sum over ranks of slot l, once every rank's slot l is complete."""
        self.handle.barrier(channel=0)
        B.lif_sum_peer_outputs([p + l * self.slot_bytes for p in self.peer_ptrs], y, stream)

    def end_token(self) -> None:
        """No rank starts the next token (and rewrites its slots) while a peer still reads."""
        self.handle.barrier(channel=1)


def build_stack(cfg, device="cuda:0", n_layers: Optional[int] = None, capacity_margin: float = 8.0,
                ffn_mode: int = 0, gen_device=None, gate_mode: int = 0, activation: int = 0,
                activation_threshold: float = 0.0, append_first: int = 0,
                shard=None, bias_down: Optional[List[torch.Tensor]] = None) -> List[Layer]:
    """Generate the weights of a named synthetic configuration and create its layers.

    ``shard = (rank, world)`` keeps only this device's share of every layer's neurons (its rows
    of the bundle store, its predictor columns, offsets and biases, a window cache sized for its
    share): the layer's output is then the sum over devices of the outputs computed here
    (``sum_partial_outputs``).  ``bias_down`` (one fp16 ``[d_model]`` tensor per layer) is given
    to the first device only, so that the sum holds it once."""
    from . import workloads as W
    layers = []
    gen_device = gen_device or device
    n_vec = 3 if gate_mode == B.GATE_BUNDLED else 2
    for l in range(n_layers or cfg.n_layers):
        if shard is None:
            lo, hi = 0, cfg.d_ff
            store = pinned_store(cfg.d_ff, cfg.d_model, n_vec)
            w = W.make_layer(cfg, l, device=gen_device, bundles_out=store, gate_mode=gate_mode,
                             act_threshold=activation_threshold)
        else:
            lo, hi = neuron_shard(cfg.d_ff, *shard)
            w = W.slice_layer(W.make_layer(cfg, l, device=gen_device, gate_mode=gate_mode,
                                           act_threshold=activation_threshold), lo, hi)
            store = pinned_store(hi - lo, cfg.d_model, n_vec)
            store.copy_(w["bundles"])
        cap = min(hi - lo, W.window_capacity(cfg, w["p"], capacity_margin))
        dev = lambda t: None if t is None else t.to(device).contiguous()
        b_down = bias_down[l] if bias_down is not None and (shard is None or shard[0] == 0) else None
        layers.append(Layer(d_model=cfg.d_model, d_ff=hi - lo, rank=cfg.rank, window_k=cfg.window_k,
                            capacity=cap, host_bundles=store, pred_A=dev(w["A"]), pred_B=dev(w["B"]),
                            pred_c=dev(w["c"]), bias_up=dev(w["bias_up"]), bias_down=dev(b_down),
                            n_streams=cfg.n_streams,
                            ffn_mode=ffn_mode, gate_mode=gate_mode, gate=dev(w.get("gate")),
                            activation=activation, activation_threshold=activation_threshold,
                            append_first=append_first, device=device))
    return layers
