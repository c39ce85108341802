"""Harness helper around the C ABI: owns the torch tensors (device slab, pinned host adapters, device
inputs/outputs) that one synthetic workload needs and forwards every operation to liblora_mi355.
No arithmetic of the method happens here."""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

from . import binding as B
from .workloads import Workload


def _bf16_tensor(bits: np.ndarray, device=None, pin: bool = False) -> torch.Tensor:
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    if pin:
        t = t.pin_memory()
    if device is not None:
        t = t.to(device, non_blocking=False)
    return t.view(torch.bfloat16)


def pin_matrices(A: Sequence[np.ndarray], B: Sequence[np.ndarray], packed: bool) -> dict:
    """Page-locked host copies of an adapter's matrices (bf16 bits), A[k] / B[k] in the order the library takes them.
    packed: one buffer holding A[0], B[0], A[1], B[1], ... back to back (the order inside a slot: the load then
    moves whole runs); otherwise one buffer per matrix."""
    if not packed:
        A_t = [_bf16_tensor(m, pin=True) for m in A]
        B_t = [_bf16_tensor(m, pin=True) for m in B]
        return {"keep": A_t + B_t, "A_ptrs": [t.data_ptr() for t in A_t], "B_ptrs": [t.data_ptr() for t in B_t]}
    n_el = sum(a.size + b.size for a, b in zip(A, B))
    buf = torch.empty(n_el, dtype=torch.int16, pin_memory=True)
    view = buf.numpy()
    A_ptrs, B_ptrs, off = [], [], 0
    for a, b in zip(A, B):
        for m, ptrs in ((a, A_ptrs), (b, B_ptrs)):
            view[off:off + m.size] = np.ascontiguousarray(m).view(np.int16).reshape(-1)
            ptrs.append(buf.data_ptr() + 2 * off)
            off += m.size
    return {"keep": [buf], "A_ptrs": A_ptrs, "B_ptrs": B_ptrs}


def bf16_tensor_to_bits(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def packed_groups(w: Workload) -> List[List[int]]:
    """Projections a decoder layer computes from one input side by side: q|k|v and gate|up."""
    names = list(w.proj_names)
    groups, used = [], set()
    for fam in (("q", "k", "v"), ("gate", "up")):
        g = [names.index(nm) for nm in fam if nm in names]
        if len(g) > 1 and len({w.proj[p][0] for p in g}) == 1:
            groups.append(g)
            used.update(g)
    out = []
    for p in range(len(names)):
        if p in used:
            g = next(g for g in groups if p in g)
            if g[0] == p:
                out.append(g)
        else:
            out.append([p])
    return out


class Session:
    def __init__(self, w: Workload, path: int = B.LORA_PATH_AUTO, split_k: int = 0, device: str = "cuda:0",
                 max_tokens: Optional[int] = None, upload_inputs: bool = True, packed_host: bool = False,
                 n_pages: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("liblora_mi355 needs a GPU; there is no CPU path")
        self.w = w
        self.packed_host = packed_host
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.max_tokens = int(max_tokens or max(w.T, 1))
        cfg = B.make_config(w.proj, w.n_slots, w.max_rank, self.max_tokens, w.max_adapter_id, path=path,
                            split_k=split_k, n_pages=n_pages)
        nbytes = B.lora_slab_bytes(cfg)
        if nbytes == 0:
            raise B.LoraError(B.LORA_ERR_SHAPE, "lora_slab_bytes")
        self.slab = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        cfg.slab = self.slab.data_ptr()
        cfg.slab_bytes = nbytes
        self.cfg = cfg
        self.ctx = B.lora_create(cfg)
        self.pinned: Dict[int, dict] = {}
        self.seg: Optional[B.lora_segments] = None
        self.W: List[torch.Tensor] = []
        self.x: List[torch.Tensor] = []
        self.out: List[torch.Tensor] = []
        self.ids: Optional[torch.Tensor] = None
        self.bias: List[Optional[torch.Tensor]] = []
        if upload_inputs:
            self.upload_inputs()

    # ---- inputs ----
    def upload_inputs(self):
        w = self.w
        self.W = [_bf16_tensor(m, self.device) for m in w.W]
        self.x = [_bf16_tensor(m, self.device) for m in w.x]
        self.out = [torch.empty((w.T, d_out), dtype=torch.bfloat16, device=self.device) for (_, d_out) in w.proj]
        self.ids = torch.from_numpy(w.token_ids).to(self.device)
        self.bias = [None if w.bias_of(p) is None else _bf16_tensor(w.bias_of(p), self.device)
                     for p in range(len(w.proj))]
        for p, b in enumerate(self.bias):
            B.lora_set_bias(self.ctx, p, 0 if b is None else b.data_ptr())

    def pin_adapter(self, aid: int) -> dict:
        if aid not in self.pinned:
            a = self.w.adapters[aid]
            ent = {"adapter_id": aid, "rank": a.rank, "scale": a.scale, "slot": -1}
            if a.rank > 0:
                ent.update(pin_matrices(a.A, a.B, self.packed_host))
            self.pinned[aid] = ent
        return self.pinned[aid]

    # ---- the three hot calls ----
    def load(self, adapter_ids: Sequence[int], in_use: Sequence[int] = (), stream: Optional[torch.cuda.Stream] = None,
             slots: Optional[Sequence[int]] = None, chunk: int = 64):
        res = []
        ids = list(adapter_ids)
        s = (stream or torch.cuda.current_stream()).cuda_stream
        for i in range(0, len(ids), chunk):
            descs = []
            for k, aid in enumerate(ids[i:i + chunk]):
                d = dict(self.pin_adapter(aid))
                if slots is not None:
                    d["slot"] = int(slots[i + k])
                descs.append(d)
            res += B.lora_slots_load(self.ctx, descs, in_use, s)
        return res

    def bucket(self, ids: Optional[torch.Tensor] = None, mode: Optional[int] = None,
               stream: Optional[torch.cuda.Stream] = None) -> B.lora_segments:
        ids = self.ids if ids is None else ids
        mode = self.w.mode if mode is None else mode
        s = (stream or torch.cuda.current_stream()).cuda_stream
        self.seg = B.lora_bucket(self.ctx, ids.data_ptr() if ids.numel() else 0, int(ids.numel()), mode, s)
        return self.seg

    def forward(self, p: int, x: Optional[torch.Tensor] = None, W: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        x = self.x[p] if x is None else x
        W = self.W[p] if W is None else W
        out = self.out[p] if out is None else out
        s = (stream or torch.cuda.current_stream()).cuda_stream
        B.lora_layer_forward(self.ctx, p, x.data_ptr(), W.data_ptr(), self.seg, out.data_ptr(), s)
        return out

    def forward_group(self, ps: Sequence[int], stream: Optional[torch.cuda.Stream] = None) -> List[torch.Tensor]:
        s = (stream or torch.cuda.current_stream()).cuda_stream
        B.lora_layer_forward_group(self.ctx, list(ps), [self.x[p].data_ptr() for p in ps],
                                   [self.W[p].data_ptr() for p in ps], self.seg,
                                   [self.out[p].data_ptr() for p in ps], s)
        return [self.out[p] for p in ps]

    def forward_glu(self, p_gate: int, p_up: int, out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """silu(gate) * up of the two projections on the input of p_gate (lora_layer_forward_glu)."""
        if out is None:
            out = torch.empty((self.w.T, self.w.proj[p_gate][1]), dtype=torch.bfloat16, device=self.device)
        s = (stream or torch.cuda.current_stream()).cuda_stream
        B.lora_layer_forward_glu(self.ctx, p_gate, p_up, self.x[p_gate].data_ptr(), self.W[p_gate].data_ptr(),
                                 self.W[p_up].data_ptr(), self.seg, out.data_ptr(), s)
        return out

    def packed_groups(self) -> List[List[int]]:
        return packed_groups(self.w)

    def forward_all(self, packed: bool = True) -> None:
        """Every projection of the layer on the current segment map (q|k|v and gate|up as packed calls)."""
        if packed:
            for g in self.packed_groups():
                if len(g) == 1:
                    self.forward(g[0])
                else:
                    self.forward_group(g)
        else:
            for p in range(len(self.w.proj)):
                self.forward(p)

    def step(self, packed: bool = True) -> None:
        """One pass of the whole path: segment map + every projection."""
        self.bucket()
        self.forward_all(packed)

    # ---- read-back helpers ----
    def _i32_at(self, ptr: int, n: int) -> np.ndarray:
        off = ptr - self.slab.data_ptr()
        assert 0 <= off and off + 4 * n <= self.slab.numel()
        return self.slab[off:off + 4 * n].view(torch.int32).cpu().numpy()

    def read_segments(self):
        torch.cuda.synchronize()
        seg = self.seg
        n_seg = int(self._i32_at(seg.n_seg, 1)[0])
        perm = self._i32_at(seg.perm, seg.T) if seg.T else np.zeros(0, np.int32)
        return (perm, self._i32_at(seg.seg_start, n_seg + 1), self._i32_at(seg.seg_slot, n_seg) if n_seg else
                np.zeros(0, np.int32), n_seg)

    def id2slot(self) -> np.ndarray:
        return np.array([B.lora_slot_of(self.ctx, i) for i in range(self.w.max_adapter_id + 1)], dtype=np.int32)

    def close(self):
        if self.ctx:
            B.lora_destroy(self.ctx)
            self.ctx = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class ModelSession:
    """Whole-model harness: `layers` are the per-layer workloads of one step (workloads.model_layers), served by
    one context with n_layers layers: one slot table, one segment map per step, a slot holds an adapter's matrices
    of every layer.  Owns tensors and forwards to the C ABI; no arithmetic of the method happens here."""

    def __init__(self, layers: Sequence[Workload], path: int = B.LORA_PATH_AUTO, split_k: int = 0,
                 device: str = "cuda:0", n_slots: Optional[int] = None, packed_host: bool = True, n_pages: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("liblora_mi355 needs a GPU; there is no CPU path")
        self.layers = list(layers)
        self.packed_host = packed_host
        w = self.w = self.layers[0]
        for lw in self.layers:
            assert lw.proj == w.proj and np.array_equal(lw.token_ids, w.token_ids)
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        cfg = B.make_config(w.proj, n_slots or w.n_slots, w.max_rank, max(w.T, 1), w.max_adapter_id, path=path,
                            split_k=split_k, n_layers=len(self.layers), n_pages=n_pages)
        nbytes = B.lora_slab_bytes(cfg)
        if nbytes == 0:
            raise B.LoraError(B.LORA_ERR_SHAPE, "lora_slab_bytes")
        self.slab_bytes = nbytes
        self.slab = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        cfg.slab = self.slab.data_ptr()
        cfg.slab_bytes = nbytes
        self.cfg = cfg
        self.ctx = B.lora_create(cfg)
        self.W = [[_bf16_tensor(m, self.device) for m in lw.W] for lw in self.layers]
        self.x = [[_bf16_tensor(m, self.device) for m in lw.x] for lw in self.layers]
        self.out = [[torch.empty((w.T, d_out), dtype=torch.bfloat16, device=self.device) for (_, d_out) in w.proj]
                    for _ in self.layers]
        self.bias = [[None if lw.bias_of(p) is None else _bf16_tensor(lw.bias_of(p), self.device)
                      for p in range(len(w.proj))] for lw in self.layers]
        for l, row in enumerate(self.bias):
            for p, b in enumerate(row):
                if b is not None:
                    B.lora_set_bias(self.ctx, p, b.data_ptr(), layer=l)
        self.ids = torch.from_numpy(w.token_ids).to(self.device)
        self.groups = packed_groups(w)
        self._heads: Optional[List[torch.Tensor]] = None      # rotated queries and attention's result, if there is a cache
        self.pinned: Dict[int, dict] = {}
        self.seg: Optional[B.lora_segments] = None

    def pin_adapter(self, aid: int) -> dict:
        if aid not in self.pinned:
            a0 = self.w.adapters[aid]
            ent = {"adapter_id": aid, "rank": a0.rank, "scale": a0.scale, "slot": -1}
            if a0.rank > 0:
                # layer-major: every projection of layer 0, then of layer 1, ...
                ent.update(pin_matrices([m for lw in self.layers for m in lw.adapters[aid].A],
                                        [m for lw in self.layers for m in lw.adapters[aid].B], self.packed_host))
            self.pinned[aid] = ent
        return self.pinned[aid]

    def load(self, adapter_ids: Sequence[int], in_use: Sequence[int] = (), stream: Optional[torch.cuda.Stream] = None,
             chunk: int = 64):
        s = (stream or torch.cuda.current_stream()).cuda_stream
        ids, res = list(adapter_ids), []
        for i in range(0, len(ids), chunk):
            res += B.lora_slots_load(self.ctx, [dict(self.pin_adapter(a)) for a in ids[i:i + chunk]], in_use, s)
        return res

    def bucket(self, stream: Optional[torch.cuda.Stream] = None) -> B.lora_segments:
        s = (stream or torch.cuda.current_stream()).cuda_stream
        self.seg = B.lora_bucket(self.ctx, self.ids.data_ptr() if self.ids.numel() else 0, int(self.ids.numel()),
                                 self.w.mode, s)
        return self.seg

    def forward_layer(self, l: int, stream: Optional[torch.cuda.Stream] = None, without: Sequence[str] = ()) -> None:
        """Layer l's projections, apart from those named in `without`."""
        s = (stream or torch.cuda.current_stream()).cuda_stream
        for g in self.groups:
            if any(self.w.proj_names[p] in without for p in g):
                continue
            B.lora_model_forward_group(self.ctx, l, g, [self.x[l][p].data_ptr() for p in g],
                                       [self.W[l][p].data_ptr() for p in g], self.seg,
                                       [self.out[l][p].data_ptr() for p in g], s)

    def forward_glu(self, l: int, p_gate: int, p_up: int, out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """silu(gate) * up of layer l's two projections on the input of p_gate (lora_model_forward_glu)."""
        w = self.layers[l]
        if out is None:
            out = torch.empty((w.T, w.proj[p_gate][1]), dtype=torch.bfloat16, device=self.device)
        s = (stream or torch.cuda.current_stream()).cuda_stream
        B.lora_model_forward_glu(self.ctx, l, p_gate, p_up, self.x[l][p_gate].data_ptr(), self.W[l][p_gate].data_ptr(),
                                 self.W[l][p_up].data_ptr(), self.seg, out.data_ptr(), s)
        return out

    def forward_attention(self, l: int, cache: "KvCache", scale: Optional[float] = None,
                          stream: Optional[torch.cuda.Stream] = None, **rotation) -> torch.Tensor:
        """Layer l from the inputs of q, k and v to its o projection: q|k|v, their heads normed and rotated and the keys and values stored
        (`rotation`: inv_freq, q_norm, k_norm, eps, pairing of KvCache.store), attention over the cache, o on its result.
        The step is the latest cache.extend's, of as many token rows as the session's."""
        names = list(self.w.proj_names)
        q, k, v, o = (names.index(nm) for nm in ("q", "k", "v", "o"))
        if self.w.proj[q][1] != cache.q_width or self.w.proj[k][1] != cache.k_width or self.w.proj[v][1] != cache.k_width:
            raise ValueError("the cache's heads are not those of the q, k and v projections")
        if self._heads is None:
            self._heads = [_made(stream, (self.w.T, cache.q_width), self.device) for _ in range(2)]
        rotated, mixed = self._heads
        s = (stream or torch.cuda.current_stream()).cuda_stream
        out = self.out[l]
        B.lora_model_forward_group(self.ctx, l, [q, k, v], [self.x[l][p].data_ptr() for p in (q, k, v)],
                                   [self.W[l][p].data_ptr() for p in (q, k, v)], self.seg,
                                   [out[p].data_ptr() for p in (q, k, v)], s)
        cache.store(l, out[k], out[v], q=out[q], out=rotated, stream=stream, **rotation)
        cache.attend(l, rotated, scale, out=mixed, stream=stream)
        B.lora_model_forward_group(self.ctx, l, [o], [mixed.data_ptr()], [self.W[l][o].data_ptr()], self.seg,
                                   [out[o].data_ptr()], s)
        return out[o]

    def step(self, stream: Optional[torch.cuda.Stream] = None, cache: Optional["KvCache"] = None, **rotation) -> None:
        """One step of the whole model: one segment map, then every layer's projections; with a cache, attention over it
        between q|k|v and o (forward_attention)."""
        self.bucket(stream)
        for l in range(len(self.layers)):
            if cache is not None:
                self.forward_attention(l, cache, stream=stream, **rotation)
            self.forward_layer(l, stream, without=() if cache is None else ("q", "k", "v", "o"))

    def close(self):
        if self.ctx:
            B.lora_destroy(self.ctx)
            self.ctx = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- key/value cache in four bits ----
class _On:
    """The device as the current one, for as long as it is not already."""
    __slots__ = ("other",)

    def __init__(self, device: torch.device):
        self.other = None if torch._C._cuda_getDevice() == device.index else torch.cuda.device(device)

    def __enter__(self):
        if self.other is not None:
            self.other.__enter__()

    def __exit__(self, *e):
        if self.other is not None:
            self.other.__exit__(*e)


def _stream_of(stream: Optional[torch.cuda.Stream], device: torch.device) -> int:
    return torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream.cuda_stream


def _made(stream: Optional[torch.cuda.Stream], shape, device) -> torch.Tensor:
    """An output, out of the memory of the stream that will write it: another stream's may still have work on it."""
    if stream is None:
        return torch.empty(shape, dtype=torch.bfloat16, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=torch.bfloat16, device=device)


def _like(t: torch.Tensor, rows: int, width: int, stream: Optional[torch.cuda.Stream], device) -> torch.Tensor:
    """An output [rows, width] beside the operand t.  (Shorter for the host where t itself is dense.)"""
    if stream is None and t.is_contiguous() and t.shape == (rows, width):
        return torch.empty_like(t)
    return _made(stream, (rows, width), device)


def _rows(t: torch.Tensor, rows: int, width: int, device, what: str) -> int:
    """Stride in elements between the rows of a bf16 operand [rows, width] whose rows are contiguous; raises ValueError."""
    if t.dtype is not torch.bfloat16 or t.device != device or t.shape != (rows, width):
        raise ValueError(f"{what}: bf16 [{rows}, {width}] on {device} expected, not {t.dtype} {tuple(t.shape)} on {t.device}")
    stride, one = t.stride()
    if rows and (one != 1 or (rows > 1 and stride < width)):      # (strides of a tensor without elements say nothing)
        raise ValueError(f"{what}: the values of a row must lie next to each other, and rows must not overlap")
    return stride if rows > 1 else width


def _ints(t: torch.Tensor, n: int, device, what: str) -> int:
    """Address of a contiguous int32 operand [n] (0 if it is empty); raises ValueError."""
    if t.dtype is not torch.int32 or t.device != device or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous int32 [{n}] on {device} expected, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _weight(t: Optional[torch.Tensor], n: int, dtype, device, what: str) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not dtype or t.device != device or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous {dtype} [{n}] on {device} expected, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _heads(dim: int, device, inv_freq, q_norm, k_norm, eps: float, pairing: int, q=(None, 0), k=(None, 0), v=(None, 0),
           q_out=(None, 0), k_out=(None, 0)) -> B.lora_heads:
    """Each of q .. k_out: (address, stride)."""
    return B.lora_heads(q[0], k[0], v[0], q[1], k[1], v[1], q_out[0], k_out[0], q_out[1], k_out[1],
                        _weight(q_norm, dim, torch.bfloat16, device, "q_norm"), _weight(k_norm, dim, torch.bfloat16, device, "k_norm"),
                        eps, _weight(inv_freq, dim // 2, torch.float32, device, "inv_freq"), pairing)


def rotary_inv_freq(head_dim: int, base: float, device) -> torch.Tensor:
    """base^(-2 p / head_dim) for the pairs p of a head, as the rotation takes it (fp32)."""
    p = torch.arange(0, head_dim, 2, dtype=torch.float64)
    return (1.0 / base ** (p / head_dim)).to(torch.float32).to(device)


def head_norm_rotate(q: Optional[torch.Tensor], k: Optional[torch.Tensor], n_heads: int, n_kv_heads: int,
                     position: Optional[torch.Tensor], inv_freq: Optional[torch.Tensor] = None,
                     q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     pairing: int = B.LORA_ROTATE_HALVES, q_out: Optional[torch.Tensor] = None,
                     k_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Norm and rotation of q [T, n_heads * dim] and k [T, n_kv_heads * dim] (lora_head_norm_rotate); returns the outputs."""
    some, heads = (q, n_heads) if q is not None else (k, n_kv_heads)
    if some is None or some.dim() != 2 or heads < 1 or not some.is_cuda:
        raise ValueError("q or k: bf16 [T, heads * dim] on a GPU expected")
    if (q is None and q_out is not None) or (k is None and k_out is not None):
        raise ValueError("an output without its operand")
    T, device, dim = some.shape[0], some.device, some.shape[1] // heads
    with _On(device):
        at = {"q": (None, 0), "k": (None, 0), "q_out": (None, 0), "k_out": (None, 0)}
        if q is not None:
            q_out = _like(q, T, n_heads * dim, stream, device) if q_out is None else q_out
            at["q"] = q.data_ptr(), _rows(q, T, n_heads * dim, device, "q")
            at["q_out"] = q_out.data_ptr(), _rows(q_out, T, n_heads * dim, device, "q_out")
        if k is not None:
            k_out = _like(k, T, n_kv_heads * dim, stream, device) if k_out is None else k_out
            at["k"] = k.data_ptr(), _rows(k, T, n_kv_heads * dim, device, "k")
            at["k_out"] = k_out.data_ptr(), _rows(k_out, T, n_kv_heads * dim, device, "k_out")
        h = _heads(dim, device, inv_freq, q_norm, k_norm, eps, pairing, **at)
        if T:
            d_pos = 0 if position is None else _ints(position, T, device, "position")
            B.lora_head_norm_rotate(T, n_heads, n_kv_heads, dim, d_pos, h, _stream_of(stream, device))
    return q_out, k_out


class KvStep:
    """The step of a KvCache.extend: its arrays as tensors on the cache's memory, good until the cache's next extend or release."""

    def __init__(self, arrays: Dict[str, torch.Tensor], raw: B.lora_kv_step, n: int, T: int):
        self._arrays, self.raw, self.n, self.T = arrays, raw, n, T

    @property
    def start(self) -> torch.Tensor:
        return self._arrays["start"][:self.n + 1]

    @property
    def position(self) -> torch.Tensor:
        return self._arrays["position"][:self.T]

    @property
    def slot(self) -> torch.Tensor:
        return self._arrays["slot"][:self.T]

    @property
    def table(self) -> torch.Tensor:
        return self._arrays["table"]

    @property
    def held(self) -> torch.Tensor:
        return self._arrays["held"]


class KvCache:
    """Keys and values of the running sequences in four bits, for every decoder layer (lora_kv_*): owns the device memory
    and forwards to the C ABI.  No arithmetic of the method happens here."""

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, n_blocks: int, max_seqs: int,
                 max_seq_tokens: int, max_tokens: int, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("liblora_mi355 needs a GPU; there is no CPU path")
        self.kv = 0
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.n_layers, self.n_heads, self.n_kv_heads, self.head_dim = n_layers, n_heads, n_kv_heads, head_dim
        self.n_blocks, self.max_seqs, self.max_tokens = n_blocks, max_seqs, max_tokens
        self.q_width, self.k_width = n_heads * head_dim, n_kv_heads * head_dim
        cfg = B.make_kv_config(n_layers, n_heads, n_kv_heads, head_dim, n_blocks, max_seqs, max_seq_tokens, max_tokens)
        self.nbytes = B.lora_kv_slab_bytes(cfg)
        with _On(self.device):
            if self.nbytes:
                self.slab = torch.empty(self.nbytes, dtype=torch.uint8, device=self.device)
                cfg.slab, cfg.slab_bytes = self.slab.data_ptr(), self.nbytes
            self.kv = B.lora_kv_create(cfg)       # says what is wrong with a shape that has no slab
        self.step: Optional[KvStep] = None
        self._arrays: Dict[str, torch.Tensor] = {}

    def _view(self, ptr: int, n: int) -> torch.Tensor:
        off = int(ptr) - self.slab.data_ptr()
        assert 0 <= off and off + 4 * n <= self.slab.numel()
        return self.slab[off:off + 4 * n].view(torch.int32)

    def _current_step(self) -> KvStep:
        if self.step is None:
            raise ValueError("no step: call extend first")
        return self.step

    def extend(self, seq: torch.Tensor, length: torch.Tensor, new: torch.Tensor, T: int, max_new: Optional[int] = None,
               stream: Optional[torch.cuda.Stream] = None) -> KvStep:
        """Blocks and places for the next `new[i]` tokens of the sequences in rows `seq[i]`, which have `length[i]` tokens."""
        n = len(seq)
        d_seq, d_len, d_new = (_ints(t, n, self.device, what) for t, what in ((seq, "seq"), (length, "length"), (new, "new")))
        with _On(self.device):
            raw = B.lora_kv_extend(self.kv, n, d_seq, d_len, d_new, T, T if max_new is None else max_new, _stream_of(stream, self.device))
        if not self._arrays:                      # (the same memory for every step)
            self._arrays = {"start": self._view(raw.start, self.max_seqs + 1), "position": self._view(raw.position, self.max_tokens),
                            "slot": self._view(raw.slot, self.max_tokens), "held": self._view(raw.held, self.max_seqs),
                            "table": self._view(raw.table, self.max_seqs * raw.row_blocks).view(self.max_seqs, raw.row_blocks)}
        self.step = KvStep(self._arrays, raw, n, T)
        return self.step

    def release(self, seq: torch.Tensor, keep: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
        """Gives back the blocks of the rows `seq` behind their first `keep[i]` tokens (none are kept without `keep`)."""
        n = len(seq)
        d_seq = _ints(seq, n, self.device, "seq")
        d_keep = 0 if keep is None else _ints(keep, n, self.device, "keep")
        with _On(self.device):
            B.lora_kv_release(self.kv, n, d_seq, d_keep, _stream_of(stream, self.device))
        self.step = None

    def store(self, layer: int, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
              inv_freq: Optional[torch.Tensor] = None, q_norm: Optional[torch.Tensor] = None,
              k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, pairing: int = B.LORA_ROTATE_HALVES,
              out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> Optional[torch.Tensor]:
        """The step's keys (normed, rotated) and values into the layer's cache; returns the normed and rotated queries."""
        step, dev = self._current_step(), self.device
        T = step.T
        if q is None and out is not None:
            raise ValueError("out: there are no queries to put there")
        with _On(dev):
            at = {"k": (k.data_ptr(), _rows(k, T, self.k_width, dev, "k")), "v": (v.data_ptr(), _rows(v, T, self.k_width, dev, "v"))}
            if q is not None:
                out = _like(q, T, self.q_width, stream, dev) if out is None else out
                at["q"] = q.data_ptr(), _rows(q, T, self.q_width, dev, "q")
                at["q_out"] = out.data_ptr(), _rows(out, T, self.q_width, dev, "out")
            h = _heads(self.head_dim, dev, inv_freq, q_norm, k_norm, eps, pairing, **at)
            B.lora_kv_store(self.kv, layer, step.raw, h, _stream_of(stream, self.device))
        return out

    def attend(self, layer: int, q: torch.Tensor, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Attention of the step's tokens over the layer's cache; scale: 1 / sqrt(head_dim) unless given."""
        step, dev = self._current_step(), self.device
        T, w = step.T, self.q_width
        with _On(dev):
            out = _like(q, T, w, stream, dev) if out is None else out
            B.lora_kv_attend(self.kv, layer, step.raw, self.head_dim ** -0.5 if scale is None else scale, q.data_ptr(), out.data_ptr(),
                             _rows(q, T, w, dev, "q"), _rows(out, T, w, dev, "out"), _stream_of(stream, self.device))
        return out

    def read(self, layer: int, seq: torch.Tensor, position: torch.Tensor, stream: Optional[torch.cuda.Stream] = None):
        """Keys and values of the tokens (seq[i], position[i]) as the bf16 values that their codes stand for."""
        n, dev = len(seq), self.device
        with _On(dev):
            k, v = (_made(stream, (n, self.k_width), dev) for _ in range(2))
            if n:
                B.lora_kv_read(self.kv, layer, n, _ints(seq, n, dev, "seq"), _ints(position, n, dev, "position"), k.data_ptr(), v.data_ptr(),
                               _stream_of(stream, self.device))
        return k, v

    def poll(self, stream: Optional[torch.cuda.Stream] = None):
        """(status, flag word) since the last poll."""
        with _On(self.device):
            return B.lora_kv_poll_flags(self.kv, _stream_of(stream, self.device))

    def close(self):
        if self.kv:
            B.lora_kv_destroy(self.kv)
            self.kv = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
