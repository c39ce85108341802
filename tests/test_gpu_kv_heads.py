"""Norm and rotation of heads, and the way into the four-bit cache and out of it, against float64."""
import numpy as np
import pytest
import torch

import oracle.kv as okv
from kv_util import HALF, U32, Model, announce, bf16, f64, i32
from paper_2602_24044_amd import binding as B
from paper_2602_24044_amd.runtime import KvCache, head_norm_rotate, rotary_inv_freq

pytestmark = pytest.mark.gpu


def _check(got, x, weight, eps, position, freq, neighbours, heads):
    T = x.shape[0]
    x64 = f64(x).reshape(T, heads, -1)
    w64 = None if weight is None else f64(weight)
    ref = okv.norm_rotate(x64, w64, eps, position, None if freq is None else freq.cpu().numpy(), neighbours)
    u = np.abs(okv.norm_rotate(x64, w64, eps, position, None))
    dim = u.shape[-1]
    pair = u.reshape(T, heads, dim // 2, 2).sum(-1).repeat(2, -1) if neighbours else np.tile(u[..., :dim // 2] + u[..., dim // 2:], 2)
    # the norm: dim squares summed in fp32 (relative dim U32, halved by the root), a root, a division, two products; the rotation: cos and
    # sin rounded to fp32, two products and a sum; one rounding to bf16
    bound = (dim / 2 + 10) * U32 * pair * (1 + HALF) + HALF * np.abs(ref) + 1e-38
    err = np.abs(f64(got).reshape(ref.shape) - ref)
    assert (err <= bound).all(), float((err - bound).max())


@pytest.mark.parametrize("T", [1, 5, 1030])
@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 64), (7, 1, 128), (32, 8, 128)])
@pytest.mark.parametrize("norm,rotate,neighbours", [(False, True, False), (True, True, False), (True, True, True), (True, False, False),
                                                    (False, False, False)])
def test_norm_rotate(T, heads, kv, dim, norm, rotate, neighbours):
    announce(f"norm_rotate T={T} {heads}/{kv}/{dim} norm={norm} rotate={rotate} neighbours={neighbours}")
    rng = np.random.default_rng(T + heads)
    # rows of a wider buffer: q | k side by side
    buf = bf16(rng, T, (heads + kv) * dim + 16, std=3.0).cuda()
    q, k = buf[:, :heads * dim], buf[:, heads * dim:(heads + kv) * dim]
    if norm and T > 1:
        q[1] = 0
        k[1] *= 1e-3
    wq, wk = (bf16(rng, dim).cuda() + 1 for _ in range(2)) if norm else (None, None)
    freq = rotary_inv_freq(dim, 500000.0, "cuda:0") if rotate else None
    pos = rng.integers(0, 200000, size=T)
    pos[0] = 2 ** 24 - 1
    if T > 3:
        pos[2], pos[3] = 0, -17
    keep = buf.clone()
    qo, ko = head_norm_rotate(q, k, heads, kv, i32(pos), freq, wq, wk, 1e-5, B.LORA_ROTATE_NEIGHBOURS if neighbours else B.LORA_ROTATE_HALVES)
    assert torch.equal(buf, keep)
    _check(qo, q, wq, 1e-5, pos, freq, neighbours, heads)
    _check(ko, k, wk, 1e-5, pos, freq, neighbours, kv)
    # in place, and one of the two alone
    head_norm_rotate(q, None, heads, kv, i32(pos), freq, wq, None, 1e-5, int(neighbours), q_out=q)
    assert torch.equal(q, qo) and torch.equal(buf[:, heads * dim:], keep[:, heads * dim:])
    _, k2 = head_norm_rotate(None, k, heads, kv, i32(pos), freq, None, wk, 1e-5, int(neighbours))
    assert torch.equal(k2, ko)


def test_far_positions_and_frequencies_above_one():
    """Angles of 2^31 and more: their last bits count."""
    rng = np.random.default_rng(0)
    q = bf16(rng, 4, 64).cuda()
    pos = [2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, 99999999]
    freq = torch.linspace(0.1, 3.7, 32).cuda()
    qo, _ = head_norm_rotate(q, None, 1, 1, i32(pos), freq)
    _check(qo, q, None, 0, np.array(pos), freq, False, 1)


def test_what_is_not_finite_stays_in_its_head():
    rng = np.random.default_rng(1)
    q = bf16(rng, 3, 4 * 64).cuda()
    clean = q.clone()
    q[1, 70], q[1, 200] = float("nan"), float("inf")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda:0")
    args = (None, 4, 1, i32([1, 2, 3]), rotary_inv_freq(64, 1e4, "cuda:0"), w)
    a, b = head_norm_rotate(q, *args)[0], head_norm_rotate(clean, *args)[0]
    assert a[1, 64:128].isnan().all() and a[1, 192:].isnan().any()
    keep = torch.ones_like(a, dtype=torch.bool)
    keep[1, 64:128] = keep[1, 192:] = False
    assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 64), (7, 1, 128), (32, 8, 128)])
@pytest.mark.parametrize("norm,neighbours", [(False, False), (True, False), (True, True)])
def test_store_and_read(heads, kv, dim, norm, neighbours):
    """Codes equal to those of the float64 definition, in chunks that begin and end inside blocks; two layers apart."""
    announce(f"store {heads}/{kv}/{dim} norm={norm} neighbours={neighbours}")
    m = Model(heads, kv, dim, n_blocks=60, max_seqs=5, max_seq_tokens=1024, max_tokens=1200, layers=2, seed=heads)
    try:
        rng = m.rng
        kw = dict(inv_freq=rotary_inv_freq(dim, 1e6, "cuda:0"), eps=1e-6, pairing=int(neighbours))
        if norm:
            kw.update(q_norm=1 + bf16(rng, dim, std=0.1).cuda(), k_norm=1 + bf16(rng, dim, std=0.1).cuda())
        for seq, length, new in (([2, 0], [0, 0], [63, 1]), ([0, 2, 4], [1, 63, 0], [130, 2, 64]), ([4, 1, 2], [64, 0, 65], [1, 900, 37])):
            m.extend(seq, length, new)
            for layer in (0, 1):
                scale = torch.from_numpy(np.exp(3 * rng.standard_normal((m.T, 1))).astype(np.float32))
                k, v = ((bf16(rng, m.T, kv * dim).float() * scale).bfloat16() for _ in range(2))
                q = bf16(rng, m.T, heads * dim).cuda()
                out = m.store(layer, k, v, q=q, **kw)
                _check(out, q, kw.get("q_norm"), 1e-6, np.array(m.position), kw["inv_freq"], neighbours, heads)
        for layer in (1, 0):
            for r in range(5):
                n = len(m.keys[layer][r])
                if n:
                    ko, vo = m.kv.read(layer, i32([r] * n), i32(range(n)))
                    assert np.array_equal(f64(ko).reshape(n, kv, dim), m.keys[layer][r]), (layer, r)
                    assert np.array_equal(f64(vo).reshape(n, kv, dim), m.values[layer][r]), (layer, r)
        assert m.kv.poll() == (B.LORA_OK, 0)
    finally:
        m.close()


@pytest.mark.parametrize("heads,kv,dim", [(40, 20, 128), (17, 17, 128), (80, 40, 64), (300, 100, 64)])
@pytest.mark.parametrize("k_norm", [False, True])
def test_store_of_many_key_heads(heads, kv, dim, k_norm):
    """More rows on their way to the cache than a workgroup asks for at once; a norm of the keys alone."""
    m = Model(heads, kv, dim, n_blocks=4, max_seqs=2, max_seq_tokens=128, max_tokens=8, seed=kv)
    try:
        m.extend([1], [0], [3])
        freq = rotary_inv_freq(dim, 10000.0, "cuda:0")
        weight = bf16(m.rng, dim).cuda() if k_norm else None
        q = bf16(m.rng, 3, heads * dim).cuda()
        out = m.store(0, bf16(m.rng, 3, kv * dim), bf16(m.rng, 3, kv * dim), q=q, inv_freq=freq, k_norm=weight)
        _check(out, q, None, 1e-6, np.arange(3), freq, False, heads)
        ko, vo = m.kv.read(0, i32([1] * 3), i32(range(3)))
        assert np.array_equal(f64(ko).reshape(3, kv, dim), m.keys[0][1]) and np.array_equal(f64(vo).reshape(3, kv, dim), m.values[0][1])
    finally:
        m.close()


def test_store_of_borders_extremes_and_what_is_not_finite():
    m = Model(2, 1, 128, n_blocks=4, max_seqs=2, max_seq_tokens=128, max_tokens=128)
    try:
        x = torch.zeros(8, 128)
        x[0, :16] = torch.tensor([7, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -7.0])
        x[1] = x[0] * 2.0 ** 60
        x[2] = x[0] * 2.0 ** -97
        x[3] = x[0] * 2.0 ** -110
        x[4, 32:40] = torch.tensor([3.3e38, -3.3e38, 1e38, 1e30, 1, 2.0 ** -126, -0.0, 2e38])
        x[5, 64:] = 1e-40                                       # below the smallest normal number
        x[6, 100], x[6, 99], x[6, 98] = 7.0625, 1.0, 3.4
        m.extend([1], [0], [8])
        m.store(0, x.bfloat16(), x.flip(0).bfloat16())
        ko, vo = m.kv.read(0, i32([1] * 8), i32(range(8)))
        assert np.array_equal(f64(ko)[:, None], m.keys[0][1]) and np.array_equal(f64(vo)[:, None], m.values[0][1])
        assert m.kv.poll() == (B.LORA_OK, 0)
        x[7, :3] = torch.tensor([float("nan"), 2.0, 1.0])
        x[0, 40:42] = torch.tensor([float("-inf"), 5.0])
        m.store(0, x.bfloat16(), x.flip(0).bfloat16())
        ko, vo = m.kv.read(0, i32([1] * 8), i32(range(8)))
        assert torch.isfinite(ko).all() and torch.isfinite(vo).all()
        assert np.array_equal(f64(ko)[:, None], m.keys[0][1]) and np.array_equal(f64(vo)[:, None], m.values[0][1])
        assert m.kv.poll() == (B.LORA_ERR_NOT_FINITE, B.LORA_KV_FLAG_NOT_FINITE)
        assert m.kv.poll() == (B.LORA_OK, 0)
    finally:
        m.close()


def test_refused_and_padding_rows():
    """Rows of a refused request: zeros in the queries' output, nothing in the cache.  Rows behind the last request: left alone."""
    m = Model(4, 2, 64, n_blocks=8, max_seqs=3, max_seq_tokens=256, max_tokens=64)
    try:
        m.extend([0, 0, 1], [0, 0, 0], [3, 4, 2], T=20)
        before = m.kv.slab.clone()
        out = torch.full((20, 256), 7.0, dtype=torch.bfloat16, device="cuda:0")
        k, v = (bf16(m.rng, 20, 128) for _ in range(2))
        k[9:], v[9:] = float("nan"), float("nan")
        k[3:7] = float("nan")
        m.store(0, k, v, q=bf16(m.rng, 20, 256).cuda(), out=out)
        assert (out[9:] == 7.0).all() and (out[3:7] == 0).all() and (out[:3] != 7.0).any()
        used = sorted(set(b for r in m.tables.rows for b in r))
        part = m.kv.n_kv_heads * 68 * 64
        changed = (m.kv.slab != before).nonzero().flatten().cpu().numpy() // part
        assert set(changed.tolist()) == set(used)
        assert m.kv.poll()[1] == B.LORA_KV_FLAG_REFUSED
    finally:
        m.close()


def test_read_refusals():
    m = Model(4, 2, 64, n_blocks=8, max_seqs=3, max_seq_tokens=256, max_tokens=64)
    try:
        m.extend([1], [0], [64])
        m.store(0)
        for r, p in ((0, 0), (1, 64), (1, -1), (3, 0), (-1, 0), (1, 2 ** 31 - 1)):
            k, v = m.kv.read(0, i32([1, r]), i32([5, p]))
            assert not k[1].any() and not v[1].any() and np.array_equal(f64(k[0]).reshape(2, 64), m.keys[0][1][5]), (r, p)
            assert m.kv.poll() == (B.LORA_ERR_KV_REFUSED, B.LORA_KV_FLAG_REFUSED), (r, p)
    finally:
        m.close()


def test_host_refusals():
    kv = KvCache(2, 4, 2, 64, n_blocks=4, max_seqs=2, max_seq_tokens=128, max_tokens=16)
    try:
        bad = B.LORA_ERR_INVALID_ARG
        x = torch.zeros(4, 256, dtype=torch.bfloat16, device="cuda:0")
        k = x[:, :128]

        def status(fn):
            with pytest.raises(B.LoraError) as e:
                fn()
            return e.value.status

        for n, T, mx in ((3, 4, 4), (-1, 4, 4), (1, 17, 4), (1, -1, 4), (1, 4, -1)):
            assert status(lambda: B.lora_kv_extend(kv.kv, n, x.data_ptr(), x.data_ptr(), x.data_ptr(), T, mx)) == bad
        assert status(lambda: B.lora_kv_extend(kv.kv, 1, 0, x.data_ptr(), x.data_ptr(), 4, 4)) == bad
        with pytest.raises(ValueError):
            kv.attend(0, x)                                   # no step yet
        step = kv.extend(i32([0]), i32([0]), i32([4]), 4)
        assert status(lambda: kv.store(2, k, k)) == bad and status(lambda: kv.attend(-1, x)) == bad
        assert status(lambda: kv.attend(0, x, float("nan"))) == bad and status(lambda: kv.attend(0, x, out=x)) == bad
        assert status(lambda: kv.store(0, k, k, q=x, out=x[:, :], eps=-1.0)) == bad
        for wrong in (x[:3], x.float(), x[:, :128], x.t(), x.cpu(), x[:1].expand(4, 256)):
            with pytest.raises(ValueError):
                kv.attend(0, wrong)
        with pytest.raises(ValueError):
            kv.extend(i32([0]).long(), i32([0]), i32([4]), 4)
        kv.extend(i32([0]), i32([0]), i32([4]), 4)
        assert status(lambda: B.lora_kv_store(kv.kv, 0, step.raw, B.lora_heads(d_k=k.data_ptr(), d_v=k.data_ptr(), k_stride=256, v_stride=256))) == bad
        raw = kv.step.raw
        kv.release(i32([1]))
        assert status(lambda: B.lora_kv_attend(kv.kv, 0, raw, 1.0, x.data_ptr(), x.data_ptr() + 4096)) == bad
        assert kv.poll() == (B.LORA_OK, 0)
    finally:
        kv.close()
