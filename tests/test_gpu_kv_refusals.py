"""Calls of the cache in four bits that name an output for which there is nothing."""
import pytest
import torch

from kv_util import Model
from paper_2602_24044_amd.runtime import head_norm_rotate

pytestmark = pytest.mark.gpu


def test_an_output_without_its_operand():
    m = Model(4, 2, 64, n_blocks=4, max_seqs=2, max_seq_tokens=128, max_tokens=16)
    try:
        m.extend([0], [0], [4])
        q, k = (torch.zeros(4, w, dtype=torch.bfloat16, device="cuda:0") for w in (256, 128))
        with pytest.raises(ValueError):
            m.kv.store(0, k, k, out=q)
        assert m.kv.store(0, k, k) is None and m.kv.store(0, k, k, q=q, out=q) is q
        for kw in ({"q": None, "k": k, "q_out": q}, {"q": q, "k": None, "k_out": k}):
            with pytest.raises(ValueError):
                head_norm_rotate(n_heads=4, n_kv_heads=2, position=None, **kw)
    finally:
        m.close()
