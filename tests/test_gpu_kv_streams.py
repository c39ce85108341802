"""The cache in four bits beside other streams' work: memory with a write still queued, captures that begin between its calls."""
import pytest
import torch

from kv_util import Model, bf16
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


def test_a_call_on_another_stream_inside_a_capture_is_refused():
    """The capture stays what it is: it ends, and its replays give what the eager call gives."""
    m = Model(**SHAPE)
    try:
        m.fill([2], [90])
        m.extend([2], [90], [7])
        m.store(0)
        q = bf16(m.rng, 7, 256)
        want = m.check_attend(0, q=q).clone()
        dq, out, other = q.cuda(), torch.zeros_like(want), torch.full_like(want, 3.0)
        side, third = torch.cuda.Stream(), torch.cuda.Stream()
        torch.cuda.synchronize()
        m.kv.attend(0, dq, out=out, stream=side)               # the latest call outside of a capture
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            m.kv.attend(0, dq, out=out, stream=side)
            with pytest.raises(B.LoraError) as e:
                m.kv.attend(0, dq, out=other, stream=third)
        assert e.value.status == B.LORA_ERR_INVALID_ARG
        for _ in range(3):
            out.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and (other == 3.0).all()
        m.kv.attend(0, dq, out=other, stream=third)
        torch.cuda.synchronize()
        assert torch.equal(other, want) and m.kv.poll() == (B.LORA_OK, 0)
    finally:
        m.close()
