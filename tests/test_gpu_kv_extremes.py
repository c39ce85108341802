"""Norm, rotation and attention at the ends of the numbers' range, against float64."""
import numpy as np
import pytest
import torch

import oracle.kv as okv
import oracle.kv as okv
from kv_util import Model, announce, attend_bound, bf16, f64, i32
from paper_2602_24044_amd import binding as B
from paper_2602_24044_amd.runtime import head_norm_rotate, rotary_inv_freq
from test_gpu_kv_heads import _check as heads_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("rotate,neighbours", [(True, False), (True, True), (False, False)])
def test_norm_of_rows_at_every_scale(dim, eps, rotate, neighbours):
    """Rows from the smallest bf16 numbers (whose squares are none in 32 bits, and with eps = 0 all that there is) to the largest (whose
    squares' sum is infinite in 32 bits), side by side.  The bound is that of rows of ordinary size: it counts roundings relative to the values."""
    announce(f"norm at every scale dim={dim} eps={eps} rotate={rotate} neighbours={neighbours}")
    rng = np.random.default_rng(dim)
    T, heads, kv = 6, 66, 11
    rows = [bf16(rng, T, n, dim).float().clamp(-3.9, 3.9) for n in (heads, kv)]
    scale = torch.ldexp(torch.ones(T * heads), torch.arange(T * heads) % 259 - 133).reshape(T, heads, 1)      # 2^-133 .. 2^125
    q = (rows[0].double() * scale).float().bfloat16().reshape(T, heads * dim)
    k = (rows[1].double() * scale[:, ::6]).float().bfloat16().reshape(T, kv * dim)
    # (a row of the smallest numbers may have been rounded to zeros, which have no norm without an eps)
    for x in (q, k):
        x.view(T, -1, dim)[x.view(T, -1, dim).abs().amax(-1) == 0] = torch.tensor(2.0 ** -133).bfloat16()
    wq, wk = (bf16(rng, dim).cuda() + 1 for _ in range(2))
    freq, pos = (rotary_inv_freq(dim, 1e4, "cuda:0") if rotate else None), np.arange(T) * 1000
    dq, dk = q.cuda(), k.cuda()
    qo, ko = head_norm_rotate(dq, dk, heads, kv, i32(pos), freq, wq, wk, eps, int(neighbours))
    assert torch.isfinite(qo).all() and torch.isfinite(ko).all()
    heads_check(qo, q, wq, eps, pos, freq, neighbours, heads)
    heads_check(ko, k, wk, eps, pos, freq, neighbours, kv)
    head_norm_rotate(dq, None, heads, kv, i32(pos), freq, wq, None, eps, int(neighbours), q_out=dq)           # in place
    assert torch.equal(dq, qo)


def test_stored_queries_at_every_scale():
    """The same on the way into the cache, beside rows with a NaN, an infinity, and zeros."""
    heads, kv, dim = 130, 2, 128
    m = Model(heads, kv, dim, n_blocks=4, max_seqs=2, max_seq_tokens=128, max_tokens=8, seed=5)
    try:
        m.extend([1], [3 - 3], [3])
        scale = torch.ldexp(torch.ones(3 * heads), torch.arange(3 * heads) % 259 - 133).reshape(3, heads, 1)
        q = (bf16(m.rng, 3, heads, dim).double().clamp(-3.9, 3.9) * scale).float().bfloat16()
        q[q.abs().amax(-1) == 0] = torch.tensor(2.0 ** -133).bfloat16()
        freq, w = rotary_inv_freq(dim, 1e4, "cuda:0"), bf16(m.rng, dim).cuda() + 1
        kw = dict(inv_freq=freq, q_norm=w, k_norm=w, eps=0.0)
        k, v = bf16(m.rng, 3, kv * dim), bf16(m.rng, 3, kv * dim)
        out = m.store(0, k, v, q=q.reshape(3, -1).cuda(), **kw)
        assert torch.isfinite(out).all()
        heads_check(out, q.reshape(3, -1), w, 0.0, np.arange(3), freq, False, heads)
        odd = q.clone()
        odd[0, 5, 7], odd[1, 70, 3], odd[2, 9] = float("nan"), float("inf"), 0.0
        got = m.store(0, k, v, q=odd.reshape(3, -1).cuda(), **kw).view(3, heads, dim)
        assert got[0, 5].isnan().all() and got[1, 70].isnan().any() and got[2, 9].isnan().all()       # 0 / 0
        keep = torch.ones(3, heads, dtype=torch.bool)
        keep[0, 5] = keep[1, 70] = keep[2, 9] = False
        assert torch.equal(got[keep.cuda()], out.view(3, heads, dim)[keep.cuda()])
        assert m.kv.poll() == (B.LORA_OK, 0)
    finally:
        m.close()


@pytest.mark.parametrize("heads,kv,dim,past,new", [(8, 2, 64, 0, 1), (8, 2, 128, 70, 3), (4, 1, 128, 3000, 1), (16, 2, 64, 40, 30), (4, 1, 128, 40, 100),
                                                   (2, 1, 64, 3000, 200)])
@pytest.mark.parametrize("scale", [1.0, -1.0])
def test_scores_below_the_range(heads, kv, dim, past, new, scale):
    """Every score of the last head below -2^128: there is no weight to be had from them, which shows (a NaN or an infinity) instead of
    passing for zeros.  One tile, tiles cut along their keys and merged, tiles of few columns and of many."""
    announce(f"scores below the range {heads}/{kv}/{dim} {past}+{new} scale={scale}")
    m = Model(heads, kv, dim, n_blocks=64, max_seqs=3, max_seq_tokens=3500, max_tokens=4000, seed=past + new)
    try:
        n = past + new
        keys = bf16(m.rng, n, kv, dim)
        keys[:, -1] = -(keys[:, -1].abs() + 0.5) * 2.0 ** 60
        keys = keys.reshape(n, kv * dim)
        if past:
            m.extend([1], [0], [past])
            m.store(0, keys[:past])
        m.extend([1], [past], [new])
        m.store(0, keys[past:])
        q = bf16(m.rng, new, heads, dim)
        q[:, -(heads // kv):] *= 2.0 ** -60                    # (scores of ordinary size for the heads beside it)
        q[:, -1] = (bf16(m.rng, new, dim).abs() + 0.5) * 2.0 ** 70 * scale
        got = m.kv.attend(0, q.reshape(new, -1).cuda(), scale).view(new, heads, dim)
        # the other heads' are what they should be (a column's weights are rounded behind a maximum that its tile's other columns move: no
        # comparison bit for bit)
        q64, k64, v64 = f64(q), m.keys[0][1], m.values[0][1]
        with np.errstate(all="ignore"):
            ref, size, top = okv.attend(q64, k64, v64, past, scale)
        split = np.abs(q64).max(axis=2, keepdims=True) * np.repeat(np.abs(k64).sum(axis=2).max(axis=0), heads // kv)[None, :, None]
        over = np.abs(f64(got) - ref) - attend_bound(ref, size, top, n, dim, split)
        assert (over[:, :-1] <= 0).all(), float(over[:, :-1].max())
        assert not torch.isfinite(got[:, -1]).any()
    finally:
        m.close()


def test_a_score_below_the_range_beside_others_has_no_weight():
    """Where another key's score is a number, the weight of one below the range is zero, as it should be."""
    m = Model(2, 1, 64, n_blocks=64, max_seqs=3, max_seq_tokens=3500, max_tokens=4000)
    try:
        keys = bf16(m.rng, 3000, 64)
        keys[100:2700] = -(keys[100:2700].abs() + 0.5) * 2.0 ** 60
        keys[:100], keys[2700:] = keys[:100] * 2.0 ** -75, keys[2700:] * 2.0 ** -75
        m.extend([1], [0], [2990])
        m.store(0, keys[:2990])
        m.extend([1], [2990], [10])
        m.store(0, keys[2990:])
        q = (bf16(m.rng, 10, 128).float().abs() + 0.5) * 2.0 ** 70
        got = m.kv.attend(0, q.bfloat16().cuda(), 1.0)
        # what is left: keys 0 .. 99 and 2700 .. , attended by themselves in a second sequence
        left = torch.cat([torch.arange(100), torch.arange(2700, 3000)])
        values = m.values[0][1][left.numpy()]
        m.extend([2], [0], [390])
        m.store(0, keys[left[:390]], torch.from_numpy(values[:390].reshape(390, 64)).bfloat16())
        m.extend([2], [390], [10])
        m.store(0, keys[left[390:]], torch.from_numpy(values[390:].reshape(10, 64)).bfloat16())
        assert np.array_equal(m.values[0][2], values)          # (four-bit values are their own)
        want = m.check_attend(0, 1.0, q=q.bfloat16())
        # both round the same weights and the result once; the pieces' maxima differ, which shifts the weights' bits: two half steps of each
        size = np.abs(values[:, 0]).max()
        assert np.abs(f64(got) - f64(want)).max() <= 4 * 2.0 ** -8 * size
    finally:
        m.close()


@pytest.mark.parametrize("power", [20, 27, 33, 45, 80, 116])
@pytest.mark.parametrize("heads,kv,dim,past,new", [(4, 2, 64, 0, 1), (8, 2, 128, 70, 3), (1, 1, 128, 3000, 1), (4, 1, 128, 40, 100), (1, 1, 64, 3000, 200)])
def test_large_scores(heads, kv, dim, past, new, power):
    """Scores so large that their last bit stands for far more than a factor of two in the weights: one key takes all of the weight, and its
    value comes out.  The scores are sums of few products of few bits, so that they are exact, and one half apart or more."""
    announce(f"large scores 2^{power} {heads}/{kv}/{dim} {past}+{new}")
    m = Model(heads, kv, dim, n_blocks=64, max_seqs=3, max_seq_tokens=3500, max_tokens=4000, seed=past + new)
    try:
        n = past + new
        # two dimensions of a key count: a magnitude that the format holds exactly, and which token has the largest
        keys = torch.zeros(n, kv, dim)
        level = torch.from_numpy(m.rng.integers(0, 6, size=(n, kv)))
        keys[:, :, 1] = torch.tensor([0.5, 1.0, 1.5, 2.0, 3.0, 4.0])[level]
        best = int(m.rng.integers(0, past + 1))
        keys[best, :, 1] = 6.0                                 # seen by every token of the step
        keys = keys.reshape(n, kv * dim).bfloat16()
        values = bf16(m.rng, n, kv * dim)
        if past:
            m.extend([1], [0], [past])
            m.store(0, keys[:past], values[:past])
        m.extend([1], [past], [new])
        m.store(0, keys[past:], values[past:])
        for scale in (1.0, 0.7, -1.3, dim ** -0.5):
            q = torch.zeros(new, heads, dim)
            # (odd multiples: the product with scale * log2(e) is not exact, whichever side it is rounded to)
            q[:, :, 1] = float(np.sign(scale)) * (1 + torch.from_numpy(m.rng.integers(0, 128, size=(new, heads))) / 128) * 2.0 ** power
            got = f64(m.kv.attend(0, q.reshape(new, -1).bfloat16().cuda(), scale)).reshape(new, heads, dim)
            want = np.repeat(m.values[0][1][best], heads // kv, axis=0)
            assert np.array_equal(got, np.broadcast_to(want, got.shape)), (scale, float(np.nanmax(np.abs(got - want))))
    finally:
        m.close()
