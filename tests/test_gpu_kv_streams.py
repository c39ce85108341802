"""The cache in four bits beside other streams' work: memory with a write still queued, captures that begin between its calls."""
import pytest
import torch

from kv_util import Model
from paper_2602_24044_amd import binding as B

pytestmark = pytest.mark.gpu

SHAPE = dict(heads=4, kv=2, dim=64, n_blocks=30, max_seqs=5, max_seq_tokens=640, max_tokens=256)


def test_cache_made_on_a_stream_with_a_write_queued():
    """Its memory is what another tensor has just left on that stream, with a write to it still waiting for its turn."""
    nbytes = B.lora_kv_slab_bytes(B.make_kv_config(1, SHAPE["heads"], SHAPE["kv"], SHAPE["dim"], *(SHAPE[k] for k in (
        "n_blocks", "max_seqs", "max_seq_tokens", "max_tokens"))))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        last = torch.empty(nbytes, dtype=torch.uint8, device="cuda:0")
        where = last.data_ptr()
        torch.cuda._sleep(20_000_000)                          # some milliseconds
        last.fill_(255)
        del last
        m = Model(**SHAPE)
    try:
        assert m.kv.slab.data_ptr() == where                   # (or the test shows nothing)
        torch.cuda.synchronize()
        tables, rest = m.kv.slab.cpu(), (m.kv.slab == 255).sum().item()
        assert rest == 4 * SHAPE["max_seqs"] * 10, rest        # the block table's -1, and nothing else
        assert not (tables != 0).logical_and(tables != 255).any()
        m.fill([3, 0], [70, 128])
        m.extend([3, 0], [70, 128], [3, 1])
        m.store(0)
        m.check_attend(0)
        assert m.kv.poll() == (B.LORA_OK, 0)
    finally:
        m.close()
