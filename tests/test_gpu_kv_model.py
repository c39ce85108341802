"""Attention over the cache inside a whole-model step: q|k|v and o with unmerged adapters around it."""
import numpy as np
import pytest
import torch

import oracle
import oracle.kv as okv
from gpu_util import TOL, announce, rel_err
from kv_util import Model, f64
from paper_2602_24044_amd import binding as B
from paper_2602_24044_amd import workloads as wl
from paper_2602_24044_amd.runtime import ModelSession, bf16_tensor_to_bits, rotary_inv_freq
from test_gpu_kv_heads import _check as heads_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("base,heads,kv", [(wl.qwen_decode(shrink=8, n_tokens=150), 7, 1), (wl.config2(shrink=8, n_tokens=150), 8, 2)])
def test_layers_with_attention(base, heads, kv):
    layers = wl.model_layers(base, 2)
    names, proj = list(base.proj_names), base.proj
    q, k, v, o = (names.index(nm) for nm in ("q", "k", "v", "o"))
    dim = proj[q][1] // heads
    announce(f"model step with attention {base.name} heads {heads}/{kv}/{dim} T={base.T}")
    assert proj[k][1] == kv * dim and proj[o][0] == heads * dim
    ms = ModelSession(layers)
    m = Model(heads, kv, dim, n_blocks=64, max_seqs=6, max_seq_tokens=512, max_tokens=256, layers=2)
    freq = rotary_inv_freq(dim, 10000.0, ms.device)
    try:
        ms.load(base.resident)
        ms.step()
        torch.cuda.synchronize()
        before = [[t.clone() for t in row] for row in ms.out]
        rows, past = [4, 0, 1, 2, 5], [0, 64, 200, 1, 63]
        new = [base.T - 40, 1, 36, 2, 1]
        for l in range(2):
            m.fill(rows, past, l)
        m.extend(rows, past, new)
        ms.bucket()
        position = np.array(m.position)
        ids = base.token_ids
        for l, lw in enumerate(layers):
            ms.forward_attention(l, m.kv, inv_freq=freq)
            torch.cuda.synchronize()
            for p in (q, k, v):
                assert torch.equal(ms.out[l][p], before[l][p])          # as without attention
            rotated, mixed = ms._heads
            heads_check(rotated, ms.out[l][q].cpu(), None, 1e-6, position, freq, False, heads)
            k64 = okv.norm_rotate(f64(ms.out[l][k]).reshape(m.T, kv, dim), None, 1e-6, position, freq.cpu().numpy())
            m.put(l, okv.four_bits(k64.astype(np.float32).astype(np.float64)), okv.four_bits(f64(ms.out[l][v]).reshape(m.T, kv, dim)))
            assert torch.equal(m.check_attend(l, q=rotated.cpu()), mixed)
            y_ref = oracle.project(bf16_tensor_to_bits(mixed), lw.W[o], ids, oracle.adapters_of(lw, o), bias=lw.bias_of(o))
            assert rel_err(bf16_tensor_to_bits(ms.out[l][o]), y_ref) <= TOL
        piecewise = [[t.clone() for t in row] for row in ms.out]
        m.extend(rows, past, new)
        ms.step(cache=m.kv, inv_freq=freq)
        torch.cuda.synchronize()
        for l in range(2):
            for p in range(len(proj)):
                assert torch.equal(ms.out[l][p], piecewise[l][p])
        assert m.kv.poll() == (B.LORA_OK, 0) and B.lora_poll_device_flags(ms.ctx) == (B.LORA_OK, 0)
        other = Model(heads, kv, 64 if dim == 128 else 128, n_blocks=4, max_seqs=1, max_seq_tokens=64, max_tokens=256, layers=2)
        with pytest.raises(ValueError):
            ms.forward_attention(0, other.kv)
        other.close()
    finally:
        ms.close()
        m.close()
