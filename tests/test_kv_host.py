"""CPU-only checks of the cache in four bits: sizes, and calls that are refused before anything is enqueued."""
import ctypes

import pytest

from paper_2602_24044_amd import binding as B

GOOD = dict(n_layers=2, n_heads=8, n_kv_heads=2, head_dim=128, n_blocks=10, max_seqs=4, max_seq_tokens=1000, max_tokens=100)


def test_slab_holds_the_blocks():
    block = 2 * 68 * 128                     # key heads * (64 tokens * 2 * (64 + 4) bytes)
    small = B.lora_kv_slab_bytes(B.make_kv_config(**GOOD))
    more = B.lora_kv_slab_bytes(B.make_kv_config(**{**GOOD, "n_blocks": 1010}))
    assert 2 * 1000 * block <= more - small < 2 * 1000 * block + 8192


@pytest.mark.parametrize("key,value,status", [
    ("n_layers", 0, B.LORA_ERR_INVALID_ARG), ("n_layers", 257, B.LORA_ERR_INVALID_ARG),
    ("n_blocks", 0, B.LORA_ERR_INVALID_ARG), ("n_blocks", (1 << 20) + 1, B.LORA_ERR_INVALID_ARG),
    ("max_seqs", 0, B.LORA_ERR_INVALID_ARG), ("max_seqs", 8193, B.LORA_ERR_INVALID_ARG),
    ("max_seq_tokens", 0, B.LORA_ERR_INVALID_ARG), ("max_seq_tokens", (1 << 24) + 1, B.LORA_ERR_INVALID_ARG),
    ("max_tokens", 0, B.LORA_ERR_INVALID_ARG), ("max_tokens", (1 << 20) + 1, B.LORA_ERR_INVALID_ARG),
    ("n_heads", 7, B.LORA_ERR_SHAPE), ("n_heads", 1026, B.LORA_ERR_SHAPE), ("n_heads", 0, B.LORA_ERR_SHAPE),
    ("n_kv_heads", 0, B.LORA_ERR_SHAPE), ("n_kv_heads", -2, B.LORA_ERR_SHAPE), ("n_kv_heads", 16, B.LORA_ERR_SHAPE),
    ("head_dim", 96, B.LORA_ERR_SHAPE), ("head_dim", 256, B.LORA_ERR_SHAPE), ("head_dim", 0, B.LORA_ERR_SHAPE)])
def test_config_errors(key, value, status):
    cfg = B.make_kv_config(**{**GOOD, key: value}, slab_ptr=256, slab_bytes=1 << 40)
    assert B.lora_kv_slab_bytes(cfg) == 0
    with pytest.raises(B.LoraError) as e:
        B.lora_kv_create(cfg)
    assert e.value.status == status


def test_create_checks_the_slab():
    need = B.lora_kv_slab_bytes(B.make_kv_config(**GOOD))
    for ptr, size, status in ((0, need, B.LORA_ERR_INVALID_ARG), (128, need, B.LORA_ERR_INVALID_ARG), (256, need - 1, B.LORA_ERR_OOM)):
        with pytest.raises(B.LoraError) as e:
            B.lora_kv_create(B.make_kv_config(**GOOD, slab_ptr=ptr, slab_bytes=size))
        assert e.value.status == status


def test_null_handles_and_pointers():
    lib, n = B._lib, None
    step, heads = B.lora_kv_step(), B.lora_heads()
    h = ctypes.c_void_p()
    bad = B.LORA_ERR_INVALID_ARG
    assert lib.lora_kv_create(n, ctypes.byref(h)) == bad and lib.lora_kv_create(ctypes.byref(B.make_kv_config(**GOOD)), n) == bad
    assert lib.lora_kv_slab_bytes(n) == 0 and lib.lora_kv_destroy(n) == bad
    assert lib.lora_kv_extend(n, 0, n, n, n, 0, 0, ctypes.byref(step), n) == bad
    assert lib.lora_kv_release(n, 0, n, n, n) == bad
    assert lib.lora_kv_store(n, 0, ctypes.byref(step), ctypes.byref(heads), n) == bad
    assert lib.lora_kv_attend(n, 0, ctypes.byref(step), 1.0, n, 0, n, 0, n) == bad
    assert lib.lora_kv_read(n, 0, 0, n, n, n, n, n) == bad
    assert lib.lora_kv_poll_flags(n, n, n) == bad


def _heads(**kw):
    h = B.lora_heads(d_q=1 << 20, d_q_out=1 << 21, d_inv_freq=4096, eps=1e-6)
    for k, v in kw.items():
        setattr(h, k, v)
    return h


@pytest.mark.parametrize("kw", [
    dict(d_q=(1 << 20) + 8), dict(d_q_out=0), dict(d_q=0), dict(d_q=0, d_q_out=0), dict(q_stride=504), dict(q_stride=516), dict(q_stride=-512),
    dict(d_k=1 << 22), dict(d_k_out=1 << 22), dict(d_v=1 << 22), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(pairing=2), dict(pairing=-1), dict(d_q_norm=4104), dict(d_inv_freq=4098), dict(d_q_out=1 << 20, q_out_stride=1024)])
def test_rotate_argument_errors(kw):
    """8 heads of 64: a token is 512 values wide.  The addresses are never followed: the call ends on the host."""
    with pytest.raises(B.LoraError) as e:
        B.lora_head_norm_rotate(4, 8, 2, 64, 4096, _heads(**kw))
    assert e.value.status == B.LORA_ERR_INVALID_ARG


def test_rotate_sizes():
    for args, status in (((-1, 8, 2, 64, 4096), B.LORA_ERR_INVALID_ARG), (((1 << 20) + 1, 8, 2, 64, 4096), B.LORA_ERR_INVALID_ARG),
                         ((4, 8, 2, 64, 0), B.LORA_ERR_INVALID_ARG), ((4, 8, 2, 64, 4098), B.LORA_ERR_INVALID_ARG),
                         ((4, 8, 3, 64, 4096), B.LORA_ERR_SHAPE), ((4, 8, 0, 64, 4096), B.LORA_ERR_SHAPE),
                         ((4, 0, 0, 64, 4096), B.LORA_ERR_SHAPE), ((4, 8, 2, 80, 4096), B.LORA_ERR_SHAPE)):
        with pytest.raises(B.LoraError) as e:
            B.lora_head_norm_rotate(*args, _heads())
        assert e.value.status == status
    B.lora_head_norm_rotate(0, 8, 2, 64, 0, _heads())        # no token: nothing to do, also without a GPU


def test_status_strings():
    assert "refused" in B.lora_status_string(B.LORA_ERR_KV_REFUSED)
    assert "block" in B.lora_status_string(B.LORA_ERR_KV_EXHAUSTED)
    assert "finite" in B.lora_status_string(B.LORA_ERR_NOT_FINITE)


def test_cache_bytes():
    # two layers of three key heads of 64: a block of 64 tokens takes 2 * 3 * 64 * (64 + 4) bytes, 4.25 bits a value
    from paper_2602_24044_amd.model_step import cache_bytes
    r = cache_bytes(2, 3, 64, 65, slot_bytes=3 * 26112 - 1)
    assert r["four_bits"] == 2 * 26112 and 26112 * 8 == 2 * 3 * 2 * 64 * 64 * 4.25
    assert r["bf16"] == 65 * 2 * 3 * 2 * 64 * 2
    assert r["tokens_per_slot"] == 128                   # whole blocks


def test_operand_checks():
    """What the Python layer takes as rows of bf16 and as integers (no GPU needed for it)."""
    import numpy as np
    import torch

    from paper_2602_24044_amd.runtime import _ints, _rows
    cpu = torch.device("cpu")
    x = torch.zeros((6, 128), dtype=torch.bfloat16)
    assert _rows(x, 6, 128, cpu, "x") == 128 and _rows(x[:, :64], 6, 64, cpu, "x") == 128 and _rows(x[::2], 3, 128, cpu, "x") == 256
    assert _rows(x[:1], 1, 128, cpu, "x") == 128
    empty = torch.from_numpy(np.zeros((0, 128), dtype=np.float32)).bfloat16()
    assert empty.stride() == (0, 0) and _rows(empty, 0, 128, cpu, "x") == 128 and _rows(x[:0], 0, 128, cpu, "x") == 128
    for bad, width in ((x.float(), 128), (x[:5], 128), (x[:, :64], 128), (x[:, ::2], 64), (x[:1].expand(6, 128), 128), (x[0], 128)):
        with pytest.raises(ValueError):
            _rows(bad, 6, width, cpu, "x")
    n = torch.arange(6, dtype=torch.int32)
    assert _ints(n, 6, cpu, "n") == n.data_ptr()
    for bad in (n.long(), n[:5], torch.arange(12, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            _ints(bad, 6, cpu, "n")
