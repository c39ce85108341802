"""Norm, rotation and attention at the ends of the numbers' range, against float64."""
import numpy as np
import pytest
import torch

import oracle.kv as okv
from kv_util import Model, announce, bf16, f64, i32
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
