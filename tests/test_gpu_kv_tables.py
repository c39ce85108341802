"""Block tables and slot maps built on the GPU against the plain ones: every value equal."""
import numpy as np
import pytest
import torch

from kv_util import Model, announce, i32
from paper_2602_24044_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(6))
def test_random_steps(seed):
    rng = np.random.default_rng(seed)
    n_blocks, seqs = [(40, 6), (64, 12), (33, 5), (2000, 70), (70000, 300), (31, 9)][seed]
    announce(f"tables seed={seed} blocks={n_blocks} rows={seqs}")
    m = Model(n_blocks=n_blocks, max_seqs=seqs, max_seq_tokens=640, max_tokens=4096)
    try:
        length = np.zeros(seqs, dtype=int)
        for _ in range(30):
            n = int(rng.integers(0, seqs + 1))
            seq = rng.permutation(seqs)[:n]
            new = rng.choice([0, 1, 1, 1, 2, 63, 64, 65, 200], size=n)
            m.tables.refused = m.tables.exhausted = False
            m.extend(seq.tolist(), length[seq].tolist(), new.tolist(), T=4096, max_new=int(rng.choice([200, 300])))
            for i, r in enumerate(seq):
                if m.start[i + 1] > m.start[i] and m.position[m.start[i]] >= 0:
                    length[r] += new[i]
            st, word = m.kv.poll()
            assert word == (B.LORA_KV_FLAG_REFUSED if m.tables.refused else 0) + (B.LORA_KV_FLAG_EXHAUSTED if m.tables.exhausted else 0)
            assert st == (B.LORA_ERR_KV_REFUSED if m.tables.refused else B.LORA_ERR_KV_EXHAUSTED if m.tables.exhausted else B.LORA_OK)
            gone = rng.permutation(seqs)[:int(rng.integers(0, seqs // 3 + 1))]
            if rng.random() < 0.5 or not len(gone):
                m.kv.release(i32(gone))
                m.tables.release(gone.tolist())
                length[gone] = 0
            else:                            # the same row twice: the smaller count of kept tokens holds
                gone = np.concatenate([gone, gone[:1]])
                keep = np.array([rng.integers(0, length[r] + 1) for r in gone])
                m.kv.release(i32(gone), i32(keep))
                m.tables.release(gone.tolist(), keep.tolist())
                for r, k in zip(gone, keep):
                    length[r] = min(length[r], k)
    finally:
        m.close()


@pytest.mark.parametrize("seq,length,new,T,max_new", [
    ([], [], [], 0, 0),                                       # an empty step
    ([], [], [], 50, 50),
    ([1], [0], [0], 0, 0),
    ([1], [0], [0], 8, 8),                                    # a request without new tokens
    ([3, 3, 2, 3], [0, 0, 0, 0], [5, 7, 9, 11], 40, 40),      # a row named more than once
    ([0, -1, 8, 1], [0, 0, 0, 0], [5, 7, 9, 11], 40, 40),     # rows that do not exist
    ([0, 1, 2], [0, -1, 1], [5, 7, 9], 40, 40),               # a negative length, tokens that are not there
    ([0, 1, 2], [0, 0, 0], [5, -7, 9], 40, 40),               # a negative count
    ([0, 1, 2], [0, 0, 0], [5, 17, 9], 40, 16),               # more than max_new
    ([0, 1, 2], [0, 0, 0], [5, 30, 9], 36, 36),               # more rows than the step has, and what comes behind them
    ([0, 1], [0, 0], [2 ** 31 - 1, 2 ** 31 - 1], 100, 100),
    ([0, 1], [2 ** 31 - 1, 0], [1, 1], 100, 100),
    ([0], [0], [1920], 2000, 2000),                           # the longest sequence, and one more
    ([0], [0], [1921], 2000, 2000),
    (list(range(8)), [0] * 8, [64, 300, 1, 65, 64, 1, 2, 3], 504, 504),   # the pool of 8 blocks runs out at the fourth
])
def test_single_steps(seq, length, new, T, max_new):
    announce(f"tables {seq} {length} {new} T={T} max_new={max_new}")
    m = Model(n_blocks=8 if len(seq) == 8 else 40, max_seqs=8, max_seq_tokens=1920, max_tokens=2000)
    try:
        m.extend(seq, length, new, T, max_new)
        again = m.kv.step.table.clone()
        m.extend(seq, length, new, T, max_new)                # the same once more changes nothing
        assert torch.equal(again, m.kv.step.table)
        assert m.kv.poll()[1] == m.tables.refused * B.LORA_KV_FLAG_REFUSED + m.tables.exhausted * B.LORA_KV_FLAG_EXHAUSTED
    finally:
        m.close()


def test_many_requests_and_a_full_bitmap():
    """More requests than a pass over them takes at once, blocks that are taken up to the last word of the bitmap."""
    n = 2500
    m = Model(n_blocks=2 * n + 7, max_seqs=n, max_seq_tokens=130, max_tokens=3 * n)
    try:
        rng = np.random.default_rng(3)
        seq = rng.permutation(n).tolist()
        m.extend(seq, [0] * n, rng.integers(0, 4, size=n).tolist(), T=3 * n)
        m.kv.release(i32(seq[::3]))
        m.tables.release(seq[::3])
        length = [0 if i % 3 == 0 else 1 for i in range(n)]
        m.extend(seq, [min(x, 64 * len(m.tables.rows[r])) for x, r in zip(length, seq)], [1 + 64 * (i % 2) * (i % 20 == 1) for i in range(n)], T=3 * n,
                 max_new=65)
    finally:
        m.close()


def test_release_refusals():
    m = Model(n_blocks=8, max_seqs=4)
    try:
        m.extend([0, 1], [0, 0], [100, 100])
        for seq, keep in (([4], None), ([-1], None), ([0], [-1])):
            m.kv.release(i32(seq), None if keep is None else i32(keep))
            m.tables.release(seq, keep)
            assert m.kv.poll() == (B.LORA_ERR_KV_REFUSED, B.LORA_KV_FLAG_REFUSED)
        m.kv.release(i32([]))
        m.extend([0, 1], [100, 100], [1, 1])
        assert m.kv.poll() == (B.LORA_OK, 0)
    finally:
        m.close()
