"""The cache's calls together, as a serving loop makes them: sequences that come, grow, take tokens back and end over several layers;
steps captured into a graph; streams; sizes at which the work is shared out differently."""
import numpy as np
import pytest
import torch

import oracle.kv as okv
from kv_util import Model, announce, attend_bound, bf16, f64, i32
from paper_2602_24044_amd import binding as B
from paper_2602_24044_amd.runtime import KvCache, head_norm_rotate, rotary_inv_freq

# (its bound: the queries' norm and rotation are fp32 sums, so a pair's difference is off relative to the pair)
from test_gpu_kv_heads import _check as heads_check  # noqa: E402

pytestmark = pytest.mark.gpu


def _layer(m, layer, freq, q_norm, k_norm, pairing):
    """One layer of the current step: store with norm and rotation, the queries against float64, attention with them."""
    q, k, v = bf16(m.rng, m.T, m.heads * m.dim), bf16(m.rng, m.T, m.kvh * m.dim), bf16(m.rng, m.T, m.kvh * m.dim)
    out = m.store(layer, k, v, q=q.cuda(), inv_freq=freq, q_norm=q_norm, k_norm=k_norm, eps=1e-5, pairing=pairing)
    rows = m.start[-1]
    position = np.array(m.position[:rows])
    heads_check(out[:rows], q[:rows], q_norm, 1e-5, position, freq, pairing == B.LORA_ROTATE_NEIGHBOURS, m.heads)
    m.check_attend(layer, q=out.cpu())


@pytest.mark.parametrize("heads,kv,dim,pairing", [(8, 2, 128, B.LORA_ROTATE_HALVES), (6, 3, 64, B.LORA_ROTATE_NEIGHBOURS)])
def test_a_serving_loop(heads, kv, dim, pairing):
    announce(f"serving loop {heads}/{kv}/{dim}")
    m = Model(heads, kv, dim, n_blocks=48, max_seqs=6, max_seq_tokens=640, max_tokens=640, layers=2, seed=3)
    freq = rotary_inv_freq(dim, 10000.0, "cuda:0")
    norms = [(bf16(m.rng, dim).cuda(), bf16(m.rng, dim).cuda()) for _ in range(2)]
    lens = {}
    try:
        rng = np.random.default_rng(11)
        for step in range(14):
            if step in (3, 8) and lens:                        # a sequence ends; its row is taken again later
                r = sorted(lens)[0]
                m.release([r])
                del lens[r]
            free = [r for r in range(6) if r not in lens]
            if free and step % 2 == 0:                         # a prompt, cut into chunks of at most 100
                lens[free[-1]] = 0
            rows = list(rng.permutation(sorted(lens)))
            new = [int(rng.integers(30, 100)) if lens[r] < 150 and rng.random() < 0.6 else int(rng.integers(1, 4)) for r in rows]
            m.extend(rows, [lens[r] for r in rows], new, T=sum(new) + int(rng.integers(0, 3)))
            for layer in range(2):
                _layer(m, layer, freq, *norms[layer], pairing)
            for r, n in zip(rows, new):
                lens[r] += n
            if step % 4 == 2:                                  # proposed tokens that were not taken: their blocks go back
                r = rows[-1]
                lens[r] = max(1, lens[r] - 2)
                m.release([r], [lens[r]])
        assert m.kv.poll() == (B.LORA_OK, 0)
    finally:
        m.close()


@pytest.mark.parametrize("max_new", [1, 40])
def test_captured_steps(max_new):
    """extend, store and attend of two layers in a graph whose lengths grow on the device, replayed with other tokens, other requests and
    rows behind the last one; each replay against float64 and against the same calls made eagerly."""
    announce(f"captured steps max_new={max_new}")
    n, T = 4, 4 * max_new + 3
    m = Model(8, 2, 128, n_blocks=40, max_seqs=6, max_seq_tokens=640, max_tokens=256, layers=2, seed=max_new)
    other = Model(4, 4, 64, n_blocks=20, max_seqs=2, max_seq_tokens=512, max_tokens=256, seed=9)
    try:
        lens = [0, 60, 63, 130]
        rows = [5, 1, 0, 3]
        for layer in range(2):
            m.fill(rows, lens, layer)
        seq, length, new = i32(rows), i32(lens), i32([1] * n)
        q, k, v = (torch.zeros((T, w), dtype=torch.bfloat16, device="cuda:0") for w in (1024, 256, 256))
        outs = [torch.zeros((T, 1024), dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]

        def calls():
            m.kv.extend(seq, length, new, T, max_new)
            for layer in range(2):
                m.kv.store(layer, k, v)
                m.kv.attend(layer, q, out=outs[layer])

        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            calls()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            calls()
            length.add_(new)
        other.extend([0], [0], [200])
        for rep in range(6):
            add = [int(x) for x in m.rng.integers(0, max_new + 1, size=n)] if rep else [1] * n
            if rep == 3:
                rows = [1, 5, 3, 0]                            # the same sequences in another order
                lens = [lens[1], lens[0], lens[3], lens[2]]
                seq.copy_(i32(rows))
                length.copy_(i32(lens))
            new.copy_(i32(add))
            kk, vv, qq = bf16(m.rng, T, 256), bf16(m.rng, T, 256), bf16(m.rng, T, 1024)
            for d, x in ((k, kk), (v, vv), (q, qq)):
                d.copy_(x)
            for o in outs:
                o.fill_(7.0)
            other.store(0)                                     # eager work of another cache in between
            other.check_attend(0)
            torch.cuda.synchronize()
            assert length.cpu().tolist() == lens
            g.replay()
            torch.cuda.synchronize()
            replayed = [o.clone() for o in outs]
            assert length.cpu().tolist() == [a + b for a, b in zip(lens, add)]
            length.copy_(i32(lens))
            m.extend(rows, lens, add, T, max_new)              # (again: nothing new)
            k4, v4 = (okv.four_bits(f64(x).reshape(T, 2, 128)) for x in (kk, vv))
            for layer in range(2):
                m.put(layer, k4, v4)
                eager = m.check_attend(layer, q=qq, out=torch.full_like(outs[0], 7.0))
                assert torch.equal(eager, replayed[layer]), (rep, layer)
            lens = [a + b for a, b in zip(lens, add)]
            length.copy_(i32(lens))
        assert m.kv.poll() == (B.LORA_OK, 0)
    finally:
        m.close()
        other.close()


def test_calls_on_other_streams_wait_for_each_other():
    """Every call on a stream of its own, with no event of the caller's between them; a second cache on the same streams."""
    m = Model(8, 2, 64, n_blocks=80, max_seqs=3, max_seq_tokens=2048, max_tokens=2048, seed=1)
    p = Model(4, 1, 128, n_blocks=80, max_seqs=3, max_seq_tokens=2048, max_tokens=2048, seed=2)
    streams = [torch.cuda.Stream() for _ in range(3)]
    try:
        for length, new in ((0, 1500), (1500, 1), (1501, 40)):
            q = [bf16(x.rng, new, x.heads * x.dim) for x in (m, p)]
            kv = [[bf16(x.rng, new, x.kvh * x.dim) for _ in range(2)] for x in (m, p)]
            dq, dkv = [t.cuda() for t in q], [[t.cuda() for t in two] for two in kv]
            out = [torch.zeros((new, x.heads * x.dim), dtype=torch.bfloat16, device="cuda:0") for x in (m, p)]
            d = i32([1]), i32([length]), i32([new])
            torch.cuda.synchronize()
            for i, x in enumerate((m, p)):
                x.kv.extend(*d, new, stream=streams[i])
                x.kv.store(0, *dkv[i], stream=streams[i + 1])
                x.kv.attend(0, dq[i], out=out[i], stream=streams[(i + 2) % 3])
            torch.cuda.synchronize()
            for i, x in enumerate((m, p)):
                x.extend([1], [length], [new])
                x.put(0, *(okv.four_bits(f64(t).reshape(new, x.kvh, x.dim)) for t in kv[i]))
                assert torch.equal(x.check_attend(0, q=q[i]), out[i])
    finally:
        m.close()
        p.close()


def test_outputs_come_from_the_stream_that_writes_them():
    """Memory given back on the current stream, which still has a write to it in its queue, is not an output of another stream."""
    m = Model(8, 2, 64, n_blocks=20, max_seqs=2, max_seq_tokens=512, max_tokens=256)
    side = torch.cuda.Stream()
    try:
        m.extend([0], [0], [200])
        m.store(0)
        q, k, v = (bf16(m.rng, 200, w).cuda() for w in (512, 128, 128))
        position, row = i32(range(200)), i32([0] * 200)
        calls = [lambda s: m.kv.attend(0, q, stream=s), lambda s: head_norm_rotate(q, k, 8, 2, None, stream=s)[0],
                 lambda s: head_norm_rotate(q, k, 8, 2, None, stream=s)[1], lambda s: m.kv.read(0, row, position, stream=s)[0],
                 lambda s: m.kv.store(0, k, v, q=q, stream=s)]
        for call in calls:
            want = call(None).clone()
            torch.cuda.synchronize()
            held = [torch.empty_like(want) for _ in range(4)]
            torch.cuda.synchronize()
            torch.cuda._sleep(20_000_000)                      # some milliseconds
            for t in held:
                t.fill_(7.0)
            del held, t
            got = call(side)
            torch.cuda.synchronize()
            assert torch.equal(got, want)
    finally:
        m.close()


def test_steps_of_nothing():
    m = Model(8, 2, 64, n_blocks=20, max_seqs=3, max_seq_tokens=512, max_tokens=64)
    try:
        m.fill([0, 1], [60, 64])
        for seq, length, new, T in (([], [], [], 0), ([0, 1], [60, 64], [0, 0], 0), ([], [], [], 9), ([0, 1], [60, 64], [0, 0], 9),
                                    ([2], [0], [0], 1)):
            m.extend(seq, length, new, T=T)
            q, k, v = (torch.randn(T, w, device="cuda:0").bfloat16() for w in (512, 128, 128))
            q_out, out = (torch.full((T, 512), 3.0, dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
            m.kv.store(0, k, v, q=q, out=q_out)
            m.kv.attend(0, q, out=out)
            assert (out == 3.0).all() and (q_out == 3.0).all()
        m.kv.release(i32([]))
        assert m.kv.read(0, i32([]), i32([]))[0].shape == (0, 128)
        k, _ = m.kv.read(0, i32([0] * 60), i32(range(60)))
        assert np.array_equal(f64(k).reshape(60, 2, 64), m.keys[0][0])
        assert m.kv.poll() == (B.LORA_OK, 0)
    finally:
        m.close()


def test_steps_that_have_ended_are_refused():
    m = Model(8, 2, 64, n_blocks=20, max_seqs=3, max_seq_tokens=512, max_tokens=64, layers=2)
    try:
        m.extend([0], [0], [5])
        k, v, q = (torch.zeros((5, w), dtype=torch.bfloat16, device="cuda:0") for w in (128, 128, 512))
        out, old = torch.empty_like(q), m.kv.step
        m.kv.extend(i32([0]), i32([0]), i32([5]), 5)
        new = m.kv.step
        h = B.lora_heads(d_k=k.data_ptr(), d_v=v.data_ptr(), eps=1e-6)

        def refused(call, *a):
            with pytest.raises(B.LoraError) as e:
                call(*a)
            assert e.value.status == B.LORA_ERR_INVALID_ARG

        refused(B.lora_kv_store, m.kv.kv, 0, old.raw, h, 0)
        refused(B.lora_kv_attend, m.kv.kv, 0, old.raw, 1.0, q.data_ptr(), out.data_ptr(), 0, 0, 0)
        for layer in (-1, 2):
            refused(B.lora_kv_store, m.kv.kv, layer, new.raw, h, 0)
            refused(B.lora_kv_attend, m.kv.kv, layer, new.raw, 1.0, q.data_ptr(), out.data_ptr(), 0, 0, 0)
        for scale in (float("nan"), float("inf")):
            refused(B.lora_kv_attend, m.kv.kv, 0, new.raw, scale, q.data_ptr(), out.data_ptr(), 0, 0, 0)
        for d_q, d_out, sq, so in ((0, out.data_ptr(), 0, 0), (q.data_ptr(), 0, 0, 0), (q.data_ptr(), q.data_ptr(), 0, 0),
                                   (q.data_ptr() + 2, out.data_ptr(), 0, 0), (q.data_ptr(), out.data_ptr() + 8, 0, 0),
                                   (q.data_ptr(), out.data_ptr(), 504, 0), (q.data_ptr(), out.data_ptr(), 0, 516)):
            refused(B.lora_kv_attend, m.kv.kv, 0, new.raw, 1.0, d_q, d_out, sq, so, 0)
        m.kv.release(i32([0]))
        refused(B.lora_kv_store, m.kv.kv, 0, new.raw, h, 0)
        refused(B.lora_kv_attend, m.kv.kv, 0, new.raw, 1.0, q.data_ptr(), out.data_ptr(), 0, 0, 0)
        for bad in (lambda: m.kv.attend(0, q), lambda: m.kv.store(0, k, v)):
            with pytest.raises(ValueError):
                bad()
    finally:
        m.close()


@pytest.mark.parametrize("heads,kv,past,new", [(8, 1, 300, 4), (8, 1, 300, 5), (1, 1, 500, 16), (1, 1, 500, 17),
                                               (1, 1, 500, 32), (1, 1, 500, 33), (8, 1, 300, 8), (8, 1, 300, 9), (1, 1, 500, 64),
                                               (1, 1, 500, 65), (1, 1, 500, 128), (1, 1, 500, 129), (1024, 1, 200, 2), (100, 1, 0, 1)])
def test_columns_on_both_sides_of_a_tile(heads, kv, past, new):
    """Queries of a request that just fill tiles of 16, 32, 64 and 128 columns, and one more; a thousand heads on one key head."""
    m = Model(heads, kv, 128, n_blocks=40, max_seqs=2, max_seq_tokens=1024, max_tokens=512, seed=new)
    try:
        m.fill([1], [past])
        m.extend([1], [past], [new])
        m.store(0)
        m.check_attend(0)
    finally:
        m.close()


@pytest.mark.parametrize("blocks", [2, 3, 4, 5, 8, 9, 30, 31, 32, 33, 60, 61, 64, 65])
@pytest.mark.parametrize("new", [1, 50])
def test_pieces_of_one_sequence(blocks, new):
    """Sequences of so many blocks that they just make another piece, and as many pieces as are merged another way."""
    m = Model(1, 1, 64, n_blocks=70, max_seqs=1, max_seq_tokens=70 * 64, max_tokens=70 * 64, seed=blocks)
    try:
        past = 64 * blocks - new
        m.fill([0], [past], step=70 * 64)
        m.extend([0], [past], [new])
        m.store(0)
        m.check_attend(0)
    finally:
        m.close()


@pytest.mark.parametrize("n,max_new", [(256, 1), (257, 1), (256, 5), (1500, 3)])
def test_many_requests(n, max_new):
    """Steps of so many requests that the plan takes them in other ways."""
    m = Model(2, 1, 64, n_blocks=2 * n, max_seqs=n + 10, max_seq_tokens=256, max_tokens=70 * n, seed=n)
    try:
        rows = [int(r) for r in m.rng.permutation(n + 10)[:n]]
        past = [int(x) for x in m.rng.choice([0, 1, 20, 63, 64], size=n, p=[0.3, 0.3, 0.3, 0.05, 0.05])]
        m.extend(rows, [0] * n, past)
        m.store(0)
        new = [int(x) for x in m.rng.integers(0, max_new + 1, size=n)]
        m.extend(rows, past, new, T=sum(new) + 1, max_new=max_new)
        m.store(0)
        m.check_attend(0)
        assert m.kv.poll() == (B.LORA_OK, 0)
    finally:
        m.close()


@pytest.mark.parametrize("new", [1, 129])
def test_pieces_of_many_blocks(new):
    """So much to read that a piece has more blocks than a wave holds the numbers of.  (What the cache holds is read back from it.)"""
    announce(f"pieces of many blocks, {new} new tokens")
    kv, dim, past = 64, 64, 66000
    w = kv * dim
    c = KvCache(1, kv, kv, dim, 2100, 2, 67000, 4096)
    try:
        gen = torch.Generator(device="cuda:0").manual_seed(new)

        def random(T):
            return torch.randn((T, w), device="cuda:0", generator=gen).bfloat16()

        for at in range(0, past, 4096):
            add = min(4096, past - at)
            for r in range(2):
                c.extend(i32([r]), i32([at]), i32([add]), add)
                c.store(0, random(add), random(add))
        c.extend(i32([1, 0]), i32([past, past - 700]), i32([new, 1]), new + 1, new)
        c.store(0, random(new + 1), random(new + 1))
        q = random(new + 1)
        got = c.attend(0, q)
        for r, first, n, length in ((1, 0, new, past), (0, new, 1, past - 700)):
            keys, values = c.read(0, i32([r] * (length + n)), i32(range(length + n)))
            for h in (0, 31, 63):
                cols = slice(h * dim, h * dim + dim)
                k64, v64, q64 = (f64(t[:, cols])[:, None] for t in (keys, values, q[first:first + n]))
                ref, size, top = okv.attend(q64, k64, v64, length, dim ** -0.5)
                split = dim ** -0.5 * np.abs(q64).max(axis=2, keepdims=True) * np.abs(k64).sum(axis=2).max()
                y = f64(got[first:first + n, cols])[:, None]
                assert (np.abs(y - ref) <= attend_bound(ref, size, top, length + n, dim, split)).all(), (r, h)
    finally:
        c.close()
