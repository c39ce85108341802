"""Sizes at which attention's launches go round once more than their grid, or deal out their work in another order.  (What the cache holds is
read back from it: the way in and out has tests of its own.)"""
import numpy as np
import pytest
import torch

import oracle.kv as okv
from kv_util import announce, attend_bound, bf16, f64, i32
from paper_2602_24044_amd import binding as B
from paper_2602_24044_amd.runtime import KvCache

pytestmark = pytest.mark.gpu

CUS = 256


def _check(c, q, got, requests, heads_of):
    """requests: (row, first token row of the step, new tokens, tokens before) each, with the heads to look at."""
    group, dim = c.n_heads // c.n_kv_heads, c.head_dim
    for row, first, new, past in requests:
        keys, values = c.read(0, i32([row] * (past + new)), i32(range(past + new)))
        for h in heads_of(row):
            k64, v64 = (f64(t[:, h // group * dim:(h // group + 1) * dim])[:, None] for t in (keys, values))
            q64 = f64(q[first:first + new, h * dim:h * dim + dim])[:, None]
            ref, size, top = okv.attend(q64, k64, v64, past, dim ** -0.5)
            split = dim ** -0.5 * np.abs(q64).max(axis=2, keepdims=True) * np.abs(k64).sum(axis=2).max()
            y = f64(got[first:first + new, h * dim:h * dim + dim])[:, None]
            assert (np.abs(y - ref) <= attend_bound(ref, size, top, past + new, dim, split)).all(), (row, h)


def _fill(c, rng, rows, past, step):
    for r, n in zip(rows, past):
        for at in range(0, n, step):
            add = min(step, n - at)
            c.extend(i32([r]), i32([at]), i32([add]), add)
            c.store(0, bf16(rng, add, c.k_width).cuda(), bf16(rng, add, c.k_width).cuda())


@pytest.mark.parametrize("new,past", [(32, 2016), (20, 2028)])
def test_merges_of_many_pieces_go_round(new, past):
    """Columns of 16 pieces and more, one a workgroup, more of them than four a CU: a workgroup takes several, one behind the other."""
    announce(f"merges go round {past}+{new}")
    heads = kv = 64
    assert new * kv > 4 * CUS and past + new == 32 * 64        # two tiles of 32 blocks: 16 pieces of two each
    rng = np.random.default_rng(new)
    c = KvCache(1, heads, kv, 64, 120, 2, 4096, 2048)
    try:
        _fill(c, rng, [1], [past], 1024)
        c.extend(i32([1]), i32([past]), i32([new]), new)
        c.store(0, bf16(rng, new, c.k_width).cuda(), bf16(rng, new, c.k_width).cuda())
        q = bf16(rng, new, c.q_width).cuda()
        got = c.attend(0, q)
        _check(c, q, got, [(1, 0, new, past)], lambda r: (0, 13, 31, 47, 63))
        assert torch.equal(c.attend(0, q), got) and c.poll() == (B.LORA_OK, 0)
    finally:
        c.close()


@pytest.mark.parametrize("heads,kv,dim,new,past", [
    (32, 8, 128, [900, 1700, 40, 640, 1, 1300], [0, 0, 0, 0, 77, 0]),          # prompts of several tiles, in no order of their lengths
    (32, 8, 128, [2300], [0]),                                                 # one of them
    (8, 8, 64, [800, 2500, 3, 4800], [130, 0, 500, 64]),
])
def test_more_tiles_than_find_room_at_once(heads, kv, dim, new, past):
    """More workgroups of many columns than two a CU: the list in its own order."""
    announce(f"many tiles {heads}/{kv}/{dim} {new}")
    tiles = sum(-(-n * heads // kv // 128) for n in new if n * heads // kv > 64) * kv
    assert tiles > 2 * CUS
    rng = np.random.default_rng(sum(new))
    n = len(new)
    c = KvCache(1, heads, kv, dim, 200, 8, 5000, 8192)
    try:
        rows = list(range(n))[::-1]
        _fill(c, rng, rows, past, 1024)
        T = sum(new)
        c.extend(i32(rows), i32(past), i32(new), T + 3, max(new))
        c.store(0, bf16(rng, T + 3, c.k_width).cuda(), bf16(rng, T + 3, c.k_width).cuda())
        q = bf16(rng, T + 3, c.q_width).cuda()
        out = torch.full_like(q, 7.0)
        c.attend(0, q, out=out)
        first = np.concatenate([[0], np.cumsum(new)])[:-1].tolist()
        _check(c, q, out, list(zip(rows, first, new, past)), lambda r: (r % heads, heads - 1 - r % 4))
        assert (out[T:] == 7.0).all() and c.poll() == (B.LORA_OK, 0)
    finally:
        c.close()


@pytest.mark.parametrize("heads,kv", [(64, 64), (256, 4)])
def test_refused_rows_beyond_the_grid(heads, kv):
    """A refused request with more tiles than the launch has workgroups: every row of it is set to zero, and only those."""
    announce(f"refused rows beyond the grid {heads}/{kv}")
    rows = 2000
    assert rows * heads // kv // 16 * kv > (4 * 3 + 2048 // kv + 1) * kv
    rng = np.random.default_rng(kv)
    c = KvCache(1, heads, kv, 64, 20, 4, 1024, 4096)
    try:
        _fill(c, rng, [2], [70], 1024)
        c.extend(i32([2, -1, 3]), i32([70, 0, 0]), i32([2, rows, 1]), rows + 10, rows)
        T = rows + 10
        c.store(0, bf16(rng, T, c.k_width).cuda(), bf16(rng, T, c.k_width).cuda())
        q = bf16(rng, T, c.q_width).cuda()
        out = torch.full_like(q, float("nan"))
        c.attend(0, q, out=out)
        assert (out[2:2 + rows] == 0).all() and out[rows + 3:].isnan().all()
        _check(c, q, out, [(2, 0, 2, 70), (3, rows + 2, 1, 0)], lambda r: (0, heads // 2, heads - 1))
        assert c.poll() == (B.LORA_ERR_KV_REFUSED, B.LORA_KV_FLAG_REFUSED)
    finally:
        c.close()
