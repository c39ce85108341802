"""Shared helpers for the tests of the cache in four bits (not collected by pytest)."""
import numpy as np
import torch

import oracle.kv as okv
from paper_2602_24044_amd import binding as B
from paper_2602_24044_amd.runtime import KvCache

HALF = 2.0 ** -8      # half a step of bf16, relative to the value
U32 = 2.0 ** -24      # half a step of fp32


def announce(msg):
    print(f"[gpu-case] {msg}", flush=True)


def i32(a):
    return torch.tensor([int(v) for v in a], dtype=torch.int32, device="cuda:0")


def bf16(rng, *shape, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).bfloat16()


def f64(t):
    return t.detach().double().cpu().numpy()


def attend_bound(out, size, top, n_keys, dim, split):
    """How far an element of the attention's output may be from the float64 result `out`; size: sum of the weights (which sum to 1)
    times |values|; top: the largest sum |q k| of a score, scaled; split: the largest max|q| sum |k| of a score, scaled.

    A score.  A query is taken as 2^n (a + b / 16) with a, b in e4m3 and 2^7 <= max|q| / 2^n < 2^8.  A bf16 value at or above 2^(n - 6) has its
    last bit at or above 2^(n - 13), and what a leaves over is at most half a step of a, so b, whose smallest step is 2^-9 / 16 = 2^-13,
    holds it exactly; a smaller value is off by half that step, 2^(n - 14) <= 2^-21 max|q|.  |a| + |b| / 16 <= (1 + 2 * 2^-4) |q|, so the 2 dim
    products in fp32 sum to within 2 dim U32 1.125 top; the factor scale * log2(e), its product and the difference from
    the running maximum are three roundings of at most 2 top: 6 U32 top.
    A weight is e^score (exp2 and rescalings: 8 U32, and U32 per rescaling, of which there is at most one per key), relative to
    itself, in the numerator and the denominator, and so is its rounding to bf16: with weights p (1 + d), |d| <= HALF,
    sum p (1 + d) v / sum p (1 + d) - out = sum p d (v - out) / sum p (1 + d), at most HALF (size + |out|) / (1 - HALF).
    Sums over the keys are fp32 (n_keys U32, twice), and the result is rounded once."""
    wiggle = 2 * ((2 * dim * 1.125 + 6) * U32 * top + 2.0 ** -21 * split) + 16 * U32 + 4 * n_keys * U32
    return (HALF / (1 - HALF) + wiggle * (1 + HALF)) * (size + np.abs(out)) + HALF * np.abs(out) * (1 + HALF) + 1e-38


class Model:
    """A cache and its plain counterpart, driven side by side."""

    def __init__(self, heads=4, kv=2, dim=64, n_blocks=64, max_seqs=8, max_seq_tokens=2048, max_tokens=512, layers=1, seed=0):
        self.kv = KvCache(layers, heads, kv, dim, n_blocks, max_seqs, max_seq_tokens, max_tokens)
        self.tables = okv.BlockTables(n_blocks, max_seqs, max_seq_tokens)
        self.heads, self.kvh, self.dim, self.layers = heads, kv, dim, layers
        self.rng = np.random.default_rng(seed)
        # what the cache must hold, by row: float64 [tokens, kv, dim]
        self.keys = [[np.zeros((0, kv, dim)) for _ in range(max_seqs)] for _ in range(layers)]
        self.values = [[np.zeros((0, kv, dim)) for _ in range(max_seqs)] for _ in range(layers)]

    def extend(self, seq, length, new, T=None, max_new=None):
        T = sum(max(0, v) for v in new) if T is None else T
        max_new = T if max_new is None else max_new
        s = self.kv.extend(i32(seq), i32(length), i32(new), T, max_new)
        start, position, slot = self.tables.extend(list(seq), list(length), list(new), T, max_new)
        assert s.start.cpu().tolist() == start
        rows = start[-1]
        assert s.position.cpu().tolist()[:rows] == position[:rows]
        assert s.slot.cpu().tolist()[:rows] == slot[:rows]
        assert np.array_equal(s.table.cpu().numpy(), self.tables.table())
        assert s.held.cpu().tolist() == [len(r) for r in self.tables.rows]
        self.seq, self.length, self.new, self.start, self.position = list(seq), list(length), list(new), start, position
        self.T = T
        return s

    def put(self, layer, k64, v64):
        """Records what the step's keys and values [T, kv, dim] (four-bit values) are."""
        for i, r in enumerate(self.seq):
            a, b = self.start[i], self.start[i + 1]
            if b > a and self.position[a] >= 0:
                for store, x in ((self.keys, k64), (self.values, v64)):
                    store[layer][r] = np.concatenate([store[layer][r][:self.length[i]], x[a:b]])

    def store(self, layer=0, k=None, v=None, **kw):
        """Random keys and values (or the given ones) of the step into the cache, without rotation unless asked for."""
        w = self.kvh * self.dim
        k = bf16(self.rng, self.T, w) if k is None else k
        v = bf16(self.rng, self.T, w) if v is None else v
        q = self.kv.store(layer, k.cuda(), v.cuda(), **kw)
        position = np.array(self.position)
        freq = kw.get("inv_freq")
        k64 = okv.norm_rotate(f64(k).reshape(self.T, self.kvh, self.dim), None if kw.get("k_norm") is None else f64(kw["k_norm"]), kw.get("eps", 1e-6),
                              position, None if freq is None else freq.cpu().numpy(), kw.get("pairing", 0) == B.LORA_ROTATE_NEIGHBOURS)
        with np.errstate(over="ignore"):
            self.put(layer, okv.four_bits(k64.astype(np.float32).astype(np.float64)), okv.four_bits(f64(v).reshape(self.T, self.kvh, self.dim)))
        return q

    def release(self, seq, keep=None):
        self.kv.release(i32(seq), None if keep is None else i32(keep))
        self.tables.release(list(seq), keep)
        assert np.array_equal(self.kv_table(), self.tables.table())

    def kv_table(self):
        return self.kv._arrays["table"].cpu().numpy()

    def fill(self, seq, length, layer=0, step=512):
        """Sequences of the given lengths, with random keys and values."""
        for r, n in zip(seq, length):
            for c in range(0, n, step):
                self.extend([r], [c], [min(step, n - c)])
                self.store(layer)

    def check_attend(self, layer=0, scale=None, q=None, out=None):
        """Attention of the current step's tokens against the definition; returns the output."""
        T, h, d = self.T, self.heads, self.dim
        q = bf16(self.rng, T, h * d) if q is None else q
        got = self.kv.attend(layer, q.cuda(), scale, out=out)
        torch.cuda.synchronize()
        scale = d ** -0.5 if scale is None else scale
        for i, r in enumerate(self.seq):
            a, b = self.start[i], self.start[i + 1]
            if a == b:
                continue
            y = f64(got[a:b]).reshape(b - a, h, d)
            if self.position[a] < 0:
                assert not y.any(), i
                continue
            keys, values = (x[layer][r][:self.length[i] + b - a] for x in (self.keys, self.values))
            ref, size, top = okv.attend(f64(q[a:b]).reshape(b - a, h, d), keys, values, self.length[i], scale)
            assert np.array_equal(np.isnan(y), np.isnan(ref)), i
            split = np.abs(scale) * np.abs(f64(q[a:b]).reshape(b - a, h, d)).max(axis=2, keepdims=True) * np.repeat(
                np.abs(keys).sum(axis=2).max(axis=0), h // self.kvh)[None, :, None]
            over = np.abs(y - ref) - attend_bound(ref, size, top, len(keys), d, split)
            assert not (over > 0).any(), (i, float(np.nanmax(over)), np.argwhere(over > 0)[:4].tolist())
        return got

    def close(self):
        self.kv.close()
