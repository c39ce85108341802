"""Attention over the cache in four bits against float64, with bounds counted in roundings (kv_util.attend_bound)."""
import numpy as np
import pytest
import torch

from kv_util import Model, announce, bf16, f64, i32
from paper_2602_24044_amd import binding as B

pytestmark = pytest.mark.gpu

LAYOUTS = [(8, 2, 64), (4, 4, 64), (32, 8, 128), (7, 1, 128), (16, 1, 128), (40, 2, 64), (33, 1, 128)]


@pytest.mark.parametrize("heads,kv,dim", LAYOUTS)
def test_mixed_step(heads, kv, dim):
    """One-token requests on every side of a block's end, chunks of prompts behind cached tokens and without, a request without new
    tokens, an empty past."""
    announce(f"attend {heads}/{kv}/{dim}")
    m = Model(heads, kv, dim, n_blocks=160, max_seqs=12, max_seq_tokens=2048, max_tokens=1024, seed=dim + heads)
    try:
        past = [0, 1, 62, 63, 64, 65, 127, 500, 90, 0, 300]
        new = [1, 1, 1, 1, 1, 2, 3, 1, 150, 131, 0]
        m.fill(range(11), past)
        m.extend(list(range(11)), past, new, T=sum(new) + 5)
        m.store(0)
        out = torch.full((m.T, heads * dim), 3.0, dtype=torch.bfloat16, device="cuda:0")
        q = bf16(m.rng, m.T, heads * dim)
        m.check_attend(0, q=q, out=out)
        assert (out[sum(new):] == 3.0).all()                   # rows behind the last request
        again = m.kv.attend(0, q.cuda())
        assert torch.equal(again[:sum(new)], out[:sum(new)])   # the same from call to call
    finally:
        m.close()


@pytest.mark.parametrize("heads,kv,dim,past,new", [(4, 1, 128, 9000, 1), (28, 4, 128, 5000, 3), (2, 2, 64, 20000, 1), (8, 1, 64, 6400, 100)])
def test_long_sequences_are_cut_and_merged(heads, kv, dim, past, new):
    announce(f"attend long {heads}/{kv}/{dim} {past}+{new}")
    m = Model(heads, kv, dim, n_blocks=400, max_seqs=3, max_seq_tokens=24000, max_tokens=4096, seed=past)
    try:
        m.fill([1], [past], step=4096)
        m.fill([2], [70])
        m.extend([2, 1], [70, past], [1, new])
        m.store(0)
        m.check_attend(0)
    finally:
        m.close()


@pytest.mark.parametrize("n", [1, 64, 65, 700])
def test_prompt_without_a_past(n):
    m = Model(8, 2, 128, n_blocks=40, max_seqs=2, max_seq_tokens=1024, max_tokens=1024, seed=n)
    try:
        m.extend([0], [0], [n])
        m.store(0)
        m.check_attend(0)
    finally:
        m.close()


def test_scales_and_large_scores():
    """Scores far apart: weights that vanish, a largest score that moves from block to block; no and negative scale."""
    m = Model(4, 1, 64, n_blocks=40, max_seqs=2, max_seq_tokens=1024, max_tokens=1024)
    try:
        m.extend([0], [0], [600])
        rise = torch.linspace(0.01, 8, 600)[:, None]
        m.store(0, (bf16(m.rng, 600, 64) * rise).bfloat16())
        for scale in (1.0, 0.0, -0.3, 1e-20):
            m.check_attend(0, scale)
    finally:
        m.close()


def test_queries_that_are_not_finite_stay_in_their_rows():
    m = Model(8, 2, 64, n_blocks=40, max_seqs=3, max_seq_tokens=1024, max_tokens=256)
    try:
        m.fill([0, 1], [130, 20])
        m.extend([0, 1], [130, 20], [40, 1])
        m.store(0)
        q = bf16(m.rng, 41, 512)
        clean = m.check_attend(0, q=q).clone()
        q[7, 64 * 3 + 5] = float("nan")
        q[40, 0] = float("nan")
        got = m.kv.attend(0, q.cuda())
        assert got[7, 192:256].isnan().all() and got[40, :64].isnan().all()
        got[7, 192:256], got[40, :64] = clean[7, 192:256], clean[40, :64]
        assert torch.equal(got, clean)
    finally:
        m.close()


def test_keys_and_values_that_are_not_finite_do_not_reach_earlier_tokens():
    """A NaN in a later token of the chunk: the tokens in front of it get what they would have got without it."""
    m = Model(8, 2, 64, n_blocks=40, max_seqs=3, max_seq_tokens=1024, max_tokens=256)
    try:
        m.extend([0], [0], [100])
        k, v = bf16(m.rng, 100, 128), bf16(m.rng, 100, 128)
        m.store(0, k, v)
        q = bf16(m.rng, 100, 512)
        clean = m.check_attend(0, q=q).clone()
        k[90, 3], v[90, 100], v[91, 0] = float("nan"), float("nan"), float("-inf")
        m.store(0, k, v)
        assert m.kv.poll()[0] == B.LORA_ERR_NOT_FINITE
        assert torch.equal(m.kv.attend(0, q.cuda())[:90], clean[:90])
    finally:
        m.close()


def test_refused_requests_get_zeros_and_disturb_nobody():
    m = Model(8, 2, 128, n_blocks=6, max_seqs=6, max_seq_tokens=512, max_tokens=512)
    try:
        m.fill([0], [70])
        m.extend([0, 9, 0, 1, 2], [70, 0, 70, 0, 0], [3, 40, 5, 100, 300])      # no such row, a row twice, no blocks left
        m.store(0)
        out = torch.full((m.T, 1024), float("nan"), dtype=torch.bfloat16, device="cuda:0")
        m.check_attend(0, out=out)
        assert m.kv.poll()[1] == B.LORA_KV_FLAG_REFUSED | B.LORA_KV_FLAG_EXHAUSTED
    finally:
        m.close()


def test_strided_queries_and_output():
    m = Model(8, 2, 64, n_blocks=40, max_seqs=3, max_seq_tokens=1024, max_tokens=256)
    try:
        m.fill([0, 1], [130, 20])
        m.extend([0, 1], [130, 20], [9, 1])
        m.store(0)
        wide = bf16(m.rng, 10, 520).cuda()
        q = wide[:, :512]
        out = torch.full((10, 768), 5.0, dtype=torch.bfloat16, device="cuda:0")
        m.check_attend(0, q=q, out=out[:, 128:640])
        assert (out[:, :128] == 5.0).all() and (out[:, 640:] == 5.0).all()
    finally:
        m.close()


def test_blocks_handed_on_hold_nothing_of_their_last_owner():
    """A sequence in blocks that another has left, whose last block still holds the other's tokens behind its own."""
    m = Model(4, 1, 128, n_blocks=3, max_seqs=2, max_seq_tokens=192, max_tokens=192)
    try:
        m.extend([0], [0], [192])
        m.store(0, (bf16(m.rng, 192, 128) * 1e30).bfloat16(), (bf16(m.rng, 192, 128) * 1e30).bfloat16())
        m.kv.release(i32([0]))
        m.tables.release([0])
        m.extend([1], [0], [3])
        m.store(0)
        m.check_attend(0)
        m.extend([1], [3], [62])
        m.store(0)
        m.check_attend(0)
    finally:
        m.close()


def test_cache_beyond_32_bit_offsets():
    """Blocks that start behind 4 GiB of the layer's memory."""
    n_blocks = 70000                                            # * 8 key heads * 8704 bytes = 4.9 GB
    m = Model(8, 8, 128, n_blocks=n_blocks, max_seqs=600, max_seq_tokens=9000, max_tokens=4096)
    try:
        # everything but the last blocks is taken
        rows = 500
        m.extend(list(range(rows)), [0] * rows, [1] * rows)
        first = rows
        for r in range(rows):
            take = min(140 - 1, n_blocks - 12 - first)
            if take <= 0:
                break
            # (the tables alone: lengths that the row then holds)
            for c in range(64, 64 * (take + 1), 4096):
                add = min(4096, 64 * (take + 1) - c)
                m.kv.extend(i32([r]), i32([c]), i32([add]), add)
                m.tables.extend([r], [c], [add], add, add)
            first += take
        m.extend([550], [0], [300])
        assert min(m.tables.rows[550]) > 65000
        m.store(0)
        ko, _ = m.kv.read(0, i32([550] * 300), i32(range(300)))
        assert np.array_equal(f64(ko).reshape(300, 8, 128), m.keys[0][550])
        m.check_attend(0)
    finally:
        m.close()
