"""The operators between q|k|v and o of a decoder layer, as cases that can be timed and compared.

  plan     block tables and slot maps of a step, built on the GPU from the requests' lengths, behind the release of what the
           requests held beyond their cached tokens
  rotate   norms of queries and keys for each head (where the case has them) with the position rotation in the same pass
  store    the same on the way into the cache: queries rotated, keys rotated and rounded to four bits, values rounded to four
           bits; then the tokens' keys and values read back out of the cache, as a program that moves a sequence does
  attend   attention of a step's tokens over the cache held in four bits
  step     the three of a layer in a row: plan, store, attend

Head layouts are those of the projections in `workloads.py` at a head size of 128 (Llama-8B 32 query and 8 key heads, 70B 64
and 8, Qwen2.5-7B 28 and 4) and a small one with heads of 64.  Lengths are lognormal, like that file's.

Four bits: 32 values of a head share an exponent e, the smallest with max|x| <= 7 * 2^e (from -100 to 125), and each is
rounded (ties to the even code) to a magnitude of {0, .5, 1, 1.5, 2, 3, 4, 6} * 2^e with a sign.  A rotated key is rounded to
32 bits in front of that, and computed in 64: next to a border between two codes a last bit would decide.

Fields of a case
  op        as above
  shape     "8b", "70b", "qwen7b", "small"
  batch     "decode": `requests` sequences of lognormal length around `context`, `new` tokens each;  "prompts": prompts of
            lognormal lengths that add up to `tokens`, about 700 each;  "mixed": a chunk of `chunk` tokens behind `context` cached
            ones, and `requests` - 1 decoding sequences beside it
  limit     longest sequence
  norm      queries and keys have a norm for each head
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
BLOCK = 64
GROUP = 32
EPS = 1e-6
HEADS = {"8b": (32, 8, 128), "70b": (64, 8, 128), "qwen7b": (28, 4, 128), "small": (8, 2, 64)}
BASE = {"8b": 500000.0, "70b": 500000.0, "qwen7b": 1000000.0, "small": 10000.0}

_DEFAULT = {"shape": "8b", "batch": "decode", "requests": 1, "context": 512, "new": 1, "tokens": 0, "chunk": 0, "limit": 4096,
            "norm": False}


def _case(**kw):
    return {**_DEFAULT, **kw}


def listed():
    return [
        # one user's next token: the latency of the plan
        _case(name="plan_1", op="plan", context=900),
        # a full batch of prompts whose sequences are all new
        _case(name="plan_prompts_20462", op="plan", batch="prompts", tokens=20462),
        # one token of the small layout
        _case(name="rotate_1", op="rotate", shape="small"),
        # a prompt batch of a model with norms on its queries and keys; 28 heads are no power of two
        _case(name="rotate_prompts_4099_norm", op="rotate", shape="qwen7b", batch="prompts", tokens=4099, norm=True),
        # the headline decode batch on its way into the cache
        _case(name="store_256", op="store", requests=256),
        # a full prefill batch of the large layout, with norms
        _case(name="store_prompts_8190_norm", op="store", shape="70b", batch="prompts", tokens=8190, norm=True),
        # one user deep in a long context
        _case(name="attend_1_long", op="attend", context=131000, limit=131072),
        # the headline decode batch
        _case(name="attend_256", op="attend", requests=256, context=1024),
        # two tokens a request (one proposed), 28 heads over 4, an odd number of requests
        _case(name="attend_203_two_tokens", op="attend", shape="qwen7b", requests=203, context=1400, new=2, limit=8192),
        # a chunk of a long prompt beside decoding requests, the usual step of continuous batching
        _case(name="attend_mixed_2100", op="attend", batch="mixed", requests=201, chunk=1900, context=6100, limit=8192),
        # one long prompt
        _case(name="attend_prompt_8192", op="attend", batch="mixed", requests=1, chunk=8192, context=0, limit=8192),
        # a lightly loaded server: the operators of a layer in a row
        _case(name="step_32", op="step", requests=32, context=700),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "rotate", "store", "attend", "attend", "attend", "step"])
    shape = rng.choice(["8b", "70b", "qwen7b", "small"])
    batch = rng.choice(["decode", "decode", "prompts", "mixed"])
    norm = rng.random() < 0.4
    if batch == "prompts":
        return _case(op=op, shape=shape, batch=batch, tokens=_log_int(rng, 40, 6000 if op in ("attend", "step") else 8190), norm=norm)
    limit = rng.choice([2048, 4096, 8192])
    if batch == "mixed":
        chunk = _log_int(rng, 20, 1900)
        return _case(op=op, shape=shape, batch=batch, requests=_log_int(rng, 1, 200), chunk=chunk, context=rng.randint(0, limit - chunk),
                     limit=limit, norm=norm)
    if rng.random() < 0.2:
        return _case(op=op, shape=shape, requests=rng.randint(1, 3), context=_log_int(rng, 8000, 100000), new=rng.randint(1, 4), limit=131072,
                     norm=norm)
    return _case(op=op, shape=shape, requests=_log_int(rng, 1, 256), context=_log_int(rng, 16, 1600), new=rng.choice([1, 1, 1, 2, 4]),
                 limit=limit, norm=norm)


# ---- the batch of a case: host arithmetic, from the seed alone ----
def _batch(case, seed):
    """(tokens cached, new tokens) of every request, int64."""
    rng = np.random.default_rng([23, seed])
    lengths = lambda n, median, hi: np.clip(np.rint(np.exp(math.log(max(1, median)) + 0.8 * rng.standard_normal(n))), 0, hi).astype(np.int64)  # noqa: E731
    if case["batch"] == "prompts":
        share = np.maximum(lengths(max(1, case["tokens"] // 700), 512, case["limit"]), 16)
        new = np.clip(share * case["tokens"] // int(share.sum()), 1, case["limit"])
        while new.sum() < case["tokens"]:
            i = int(np.argmin(new))
            new[i] += min(case["tokens"] - int(new.sum()), case["limit"] - int(new[i]))
        return np.zeros(len(new), np.int64), new
    n = case["requests"]
    new = np.full(n, case["new"], np.int64)
    if n == 1 or case["limit"] > 100000:     # a length that the case names
        old = np.full(n, case["context"], np.int64) - np.arange(n) * (case["context"] // 7) - int(rng.integers(0, 65))
    else:
        old = lengths(n, case["context"] if case["batch"] == "decode" else 700, case["limit"] - case["new"])
    if case["batch"] == "mixed":
        new[0], old[0] = case["chunk"], case["context"]
    return np.clip(old, 0, case["limit"] - new), new


def _sizes(case, seed):
    heads, kv, dim = HEADS[case["shape"]]
    old, new = _batch(case, seed)
    held = -(-(old + new) // BLOCK)
    # beside the batch's sequences others sit in the pool, every second one of which has left: the free blocks are scattered
    others = np.array([1 + (7 * j + seed) % 13 for j in range(40)], np.int64)
    return {"heads": heads, "kv": kv, "dim": dim, "old": old, "new": new, "n": len(old), "T": int(new.sum()), "max_new": int(new.max()),
            "others": others, "rows": len(old) + len(others), "blocks_per_row": -(-case["limit"] // BLOCK),
            "blocks": int(held.sum() + others.sum()) + 37}


def _frequencies(case):
    dim = HEADS[case["shape"]][2]
    return (1.0 / BASE[case["shape"]] ** (np.arange(0, dim, 2, dtype=np.float64) / dim)).astype(np.float32)


def _inputs(case, seed):
    """What the case's calls work on, drawn on the GPU."""
    z = _sizes(case, seed)
    dev = torch.device(DEVICE)
    g = torch.Generator(device=dev)
    g.manual_seed(1000003 * seed + 77)
    randn = lambda *s: torch.randn(s, generator=g, device=dev)  # noqa: E731
    T, h, kv, d = z["T"], z["heads"], z["kv"], z["dim"]
    channel = torch.exp(0.4 * randn(kv, d))                                      # some channels of the keys are larger
    z["q"] = randn(T, h * d).bfloat16()
    z["k"] = (randn(T, kv, d) * channel).reshape(T, kv * d).bfloat16()
    z["v"] = randn(T, kv * d).bfloat16()
    z["freq"] = torch.from_numpy(_frequencies(case)).to(dev)
    z["q_norm"] = (1.0 + 0.1 * randn(d)).bfloat16() if case["norm"] else None
    z["k_norm"] = (1.0 + 0.1 * randn(d)).bfloat16() if case["norm"] else None
    z["old_t"], z["new_t"] = (torch.from_numpy(z[x].astype(np.int32)).to(dev) for x in ("old", "new"))
    z["row_t"] = torch.from_numpy(np.random.default_rng([29, seed]).permutation(z["rows"])[:z["n"]].astype(np.int32)).to(dev)
    if case["op"] in ("attend", "step"):
        C = int(z["old"].sum())
        z["k_old"] = (randn(C, kv, d) * channel).reshape(C, kv * d).bfloat16()    # what the cache holds already, by request
        z["v_old"] = randn(C, kv * d).bfloat16()
    return z


# ---- the operators in their plain form ----
def _quantise(x):
    """float32 [..., dim] -> (codes 0..15, biased exponents [..., dim / 32])."""
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    m, e = torch.frexp(g.abs().amax(-1))
    e = torch.where(m <= 0.875, e - 3, e - 2).clamp(-100, 125)
    e = torch.where(m == 0, -100, e)
    y = torch.ldexp(g.abs(), -e[..., None]).float()
    code = ((y > 0.25).byte() + (y >= 0.75).byte() + (y > 1.25).byte() + (y >= 1.75).byte() + (y > 2.5).byte() + (y >= 3.5).byte() + (y > 5).byte())
    code = code + 8 * (g < 0).byte()
    return code.reshape(x.shape), (e + 127).byte()


def _pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _values(packed, exponent):
    """float32 [..., dim] of packed codes [..., dim / 2] and biased exponents [..., dim / 32]."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device=packed.device)
    code = torch.stack([packed & 15, packed >> 4], -1).flatten(-2)
    x = table[code.int()].reshape(*code.shape[:-1], -1, GROUP)
    return torch.ldexp(x, (exponent.int() - 127)[..., None]).reshape(code.shape)


def _plain_release(st):
    keep = -(-st["old_t"].long() // BLOCK)
    rows, table = st["row_t"].long(), st["table"]
    mine = table[rows]
    gone = (torch.arange(table.shape[1], device=table.device)[None] >= keep[:, None]) & (mine >= 0)
    st["used"][mine[gone].long()] = False
    table[rows] = torch.where(gone, -1, mine)
    st["held"][rows] = torch.minimum(st["held"][rows], keep.int())


def _plain_extend(st):
    old, new, rows, table = st["old_t"].long(), st["new_t"].long(), st["row_t"].long(), st["table"]
    n, T = st["n"], st["T"]
    held = st["held"][rows].long()
    want = torch.maximum(-(-(old + new) // BLOCK), held)
    first = torch.cumsum(want - held, 0) - (want - held)
    free = torch.nonzero(~st["used"]).flatten()
    j = torch.arange(table.shape[1], device=table.device)[None]
    fresh = (j >= held[:, None]) & (j < want[:, None])
    at = free[(first[:, None] + j - held[:, None]).clamp(0, len(free) - 1)]
    table[rows] = torch.where(fresh, at.int(), table[rows])
    st["used"][at[fresh]] = True
    st["held"][rows] = want.int()
    start = torch.zeros(n + 1, dtype=torch.int32, device=table.device)
    start[1:] = torch.cumsum(new, 0).int()
    request = torch.repeat_interleave(torch.arange(n, device=table.device), new, output_size=T)
    position = old[request] + torch.arange(T, device=table.device) - start[request].long()
    slot = table[rows[request], position // BLOCK] * BLOCK + (position % BLOCK).int()
    return {"start": start, "position": position.int(), "slot": slot, "table": table, "held": st["held"]}


def _plain_rotate(x, heads, weight, position, freq, wide):
    """Norm (where there is a weight) and rotation of x [T, heads * dim]: in 64 bits where `wide`, in 32 otherwise, but for the
    angles."""
    T, dim = x.shape[0], x.shape[1] // heads
    x = x.reshape(T, heads, dim).to(torch.float64 if wide else torch.float32)
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.to(x.dtype)
    angle = (position.double()[:, None] * freq.double()[None])[:, None]
    c, s = torch.cos(angle).to(x.dtype), torch.sin(angle).to(x.dtype)
    a, b = x[..., :dim // 2], x[..., dim // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _plain_store(st):
    """Rotated queries; the tokens' keys and values go into the cache at their slots."""
    T, kv, d = st["T"], st["kv"], st["dim"]
    q = _plain_rotate(st["q"], st["heads"], st["q_norm"], st["position"], st["freq"], False).bfloat16().reshape(T, -1)
    k = _plain_rotate(st["k"], kv, st["k_norm"], st["position"], st["freq"], True).float()
    _plain_put(st, st["slot"].long(), k, st["v"].reshape(T, kv, d).float())
    return q


def _plain_put(st, slot, k, v):
    at, off = slot // BLOCK, slot % BLOCK
    code, e = _quantise(torch.stack([k, v], 1))                                  # [tokens, 2, kv, dim]
    st["codes"][at, :, :, off] = _pack(code)
    st["exponents"][at, :, :, off] = e


def _plain_read(st):
    at, off = st["slot"].long() // BLOCK, st["slot"].long() % BLOCK
    x = _values(st["codes"][at, :, :, off], st["exponents"][at, :, :, off]).bfloat16()
    return x[:, 0].reshape(st["T"], -1), x[:, 1].reshape(st["T"], -1)


def _plain_attend_some(st, q, requests, tokens, most):
    """Attention of the requests in `requests`, which hold `most` blocks or fewer; tokens [requests, new]: their rows (-1: none)."""
    new = tokens.shape[1]
    h, kv, d = st["heads"], st["kv"], st["dim"]
    n, G = requests.shape[0], h // kv
    old, count = st["old_t"].long()[requests], st["new_t"].long()[requests]
    blocks = st["table"][st["row_t"].long()[requests]].long()[:, :most]
    L = blocks.shape[1] * BLOCK
    x = _values(st["codes"][blocks.clamp(min=0)], st["exponents"][blocks.clamp(min=0)])   # [n, blocks, 2, kv, 64, dim]
    x = x.permute(2, 0, 3, 1, 4, 5).reshape(2, n, kv, L, d)
    rows = q[tokens.clamp(min=0)].float().reshape(n, new, kv, G, d).permute(0, 2, 1, 3, 4).reshape(n, kv, new * G, d)
    s = torch.matmul(rows, x[0].transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(d))
    last = old[:, None] + torch.arange(new, device=q.device)[None]
    seen = torch.arange(L, device=q.device)[None, None] <= last[..., None]       # [n, new, L]
    s = s.reshape(n, kv, new, G, L).masked_fill_(~seen[:, None, :, None], float("-inf"))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = (p / p.sum(-1, keepdim=True)).reshape(n, kv, new * G, L)
    o = torch.matmul(p, x[1]).reshape(n, kv, new, G, d).permute(0, 2, 1, 3, 4).reshape(n, new, h * d)
    return o[torch.arange(new, device=q.device)[None] < count[:, None]].bfloat16()


def _plain_attend(st, q):
    """Requests of many new tokens and of few, each kind padded to its longest."""
    parts = [_plain_attend_some(st, q, r, t, most) for r, t, most in st["kinds"]]
    return torch.cat(parts)[st["order"]]


# ---- a user's program ----
def _kinds(z):
    """The requests by kind (over or under 16 new tokens), with the rows of their tokens; and where each row's result is then."""
    start = np.concatenate([[0], np.cumsum(z["new"])])
    kinds, order = [], []
    for pick in (np.nonzero(z["new"] > 16)[0], np.nonzero(z["new"] <= 16)[0]):
        if not len(pick):
            continue
        tokens = np.full((len(pick), int(z["new"][pick].max())), -1, np.int64)
        for i, r in enumerate(pick):
            tokens[i, :z["new"][r]] = np.arange(start[r], start[r + 1])
        order.append(tokens[tokens >= 0])
        most = int((-(-(z["old"] + z["new"])[pick] // BLOCK)).max())
        kinds.append((torch.from_numpy(pick).to(DEVICE), torch.from_numpy(tokens).to(DEVICE), most))
    return kinds, torch.from_numpy(np.argsort(np.concatenate(order))).to(DEVICE)


def _prepare_plain(case, z):
    op, dev = case["op"], z["q"].device
    z["table"] = torch.full((z["rows"], z["blocks_per_row"]), -1, dtype=torch.int32, device=dev)
    z["held"] = torch.zeros(z["rows"], dtype=torch.int32, device=dev)
    z["used"] = torch.zeros(z["blocks"], dtype=torch.bool, device=dev)
    first = 0
    for j, (row, count) in enumerate(zip(z["other_rows"], z["others"])):
        if j % 2 == 0:
            z["table"][row, :count] = torch.arange(first, first + int(count), dtype=torch.int32, device=dev)
            z["held"][row] = int(count)
            z["used"][first:first + int(count)] = True
        first += int(count)
    # the blocks of the cached tokens first, then those of the step
    if int(z["old"].sum()):
        before = dict(z, new_t=z["old_t"], old_t=torch.zeros_like(z["old_t"]), T=int(z["old"].sum()))
        _plain_extend(before)
    made = _plain_extend(z)
    z["position"], z["slot"] = made["position"], made["slot"]
    if op in ("store", "attend", "step"):
        kv, d = z["kv"], z["dim"]
        z["codes"] = torch.zeros(z["blocks"], 2, kv, BLOCK, d // 2, dtype=torch.uint8, device=dev)
        z["exponents"] = torch.full((z["blocks"], 2, kv, BLOCK, d // GROUP), 127, dtype=torch.uint8, device=dev)
    if op in ("attend", "step"):
        C = int(z["old"].sum())
        request = torch.repeat_interleave(torch.arange(z["n"], device=dev), z["old_t"].long(), output_size=C)
        first = torch.cumsum(z["old_t"].long(), 0) - z["old_t"].long()
        position = torch.arange(C, device=dev) - first[request]
        slot = z["table"][z["row_t"].long()[request], position // BLOCK].long() * BLOCK + position % BLOCK
        for c in range(0, C, 65536):
            e = slice(c, min(C, c + 65536))
            _plain_put(z, slot[e], z["k_old"][e].reshape(-1, kv, d).float(), z["v_old"][e].reshape(-1, kv, d).float())
        if op == "attend":
            _plain_put(z, z["slot"].long(), z["k"].reshape(-1, kv, d).float(), z["v"].reshape(-1, kv, d).float())
        z["kinds"], z["order"] = _kinds(z)
    return z


def _prepare_own(case, z):
    from paper_2602_24044_amd.runtime import KvCache
    op = case["op"]
    if op == "rotate":
        z["position"] = _positions(z)
        return z
    C = int(z["old"].sum())
    most = max(1024, z["T"], min(C, 65536))
    kv = KvCache(n_layers=1, n_heads=z["heads"], n_kv_heads=z["kv"], head_dim=z["dim"], n_blocks=z["blocks"], max_seqs=z["rows"],
                 max_seq_tokens=case["limit"], max_tokens=most)
    z["cache"] = kv
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=z["q"].device)  # noqa: E731
    everyone = z["others"] * BLOCK
    for j, (row, count) in enumerate(zip(z["other_rows"], everyone)):
        kv.extend(i32([row]), i32([0]), i32([count]), int(count))
    kv.release(i32(z["other_rows"][1::2]))
    if C:
        # the cached tokens, request after request, in steps of at most `most` tokens
        for r, old in enumerate(z["old"]):
            for c in range(0, int(old), most):
                m = min(most, int(old) - c)
                kv.extend(z["row_t"][r:r + 1], i32([c]), i32([m]), m)
                if op in ("attend", "step"):
                    f = int(z["old"][:r].sum()) + c
                    kv.store(0, z["k_old"][f:f + m], z["v_old"][f:f + m])
    kv.extend(z["row_t"], z["old_t"], z["new_t"], z["T"], z["max_new"])
    if op == "attend":
        kv.store(0, z["k"], z["v"])
    z["position"] = _positions(z)
    z["row_of_token"] = torch.repeat_interleave(z["row_t"], z["new_t"].long(), output_size=z["T"])
    return z


def _positions(z):
    start = np.concatenate([[0], np.cumsum(z["new"])[:-1]])
    p = np.repeat(z["old"], z["new"]) + np.arange(z["T"]) - np.repeat(start, z["new"])
    return torch.from_numpy(p.astype(np.int32)).to(z["q"].device)


def prepare(case, seed):
    z = _inputs(case, seed)
    z["op"] = case["op"]
    taken = set(z["row_t"].cpu().tolist())
    z["other_rows"] = [r for r in range(z["rows"]) if r not in taken]
    z = _prepare_own(case, z) if own else _prepare_plain(case, z)
    z.pop("k_old", None)
    z.pop("v_old", None)
    return z


def run(st):
    op = st["op"]
    if own:
        return _run_own(st)
    if op == "plan":
        _plain_release(st)
        return _plain_extend(st)
    if op == "rotate":
        return {x: _plain_rotate(st[x], st[n], st[x + "_norm"], st["position"], st["freq"], False).bfloat16().reshape(st["T"], -1)
                for x, n in (("q", "heads"), ("k", "kv"))}
    if op == "store":
        q = _plain_store(st)
        k, v = _plain_read(st)
        return {"q": q, "k": k, "v": v}
    if op == "attend":
        return {"out": _plain_attend(st, st["q"])}
    made = _plain_extend(st)
    return {"out": _plain_attend(st, _plain_store(st)), "slot": made["slot"]}


def _run_own(st):
    op, kv = st["op"], st.get("cache")
    if op == "plan":
        kv.release(st["row_t"], st["old_t"])
        s = kv.extend(st["row_t"], st["old_t"], st["new_t"], st["T"], st["max_new"])
        return {"start": s.start, "position": s.position, "slot": s.slot, "table": s.table, "held": s.held}
    if op == "rotate":
        from paper_2602_24044_amd.runtime import head_norm_rotate
        q, k = head_norm_rotate(st["q"], st["k"], st["heads"], st["kv"], st["position"], st["freq"], q_norm=st["q_norm"], k_norm=st["k_norm"], eps=EPS)
        return {"q": q, "k": k}
    heads = {"inv_freq": st["freq"], "q_norm": st["q_norm"], "k_norm": st["k_norm"], "eps": EPS}
    if op == "store":
        q = kv.store(0, st["k"], st["v"], q=st["q"], **heads)
        k, v = kv.read(0, st["row_of_token"], st["position"])
        return {"q": q, "k": k, "v": v}
    if op == "attend":
        return {"out": kv.attend(0, st["q"])}
    s = kv.extend(st["row_t"], st["old_t"], st["new_t"], st["T"], st["max_new"])
    q = kv.store(0, st["k"], st["v"], q=st["q"], **heads)
    return {"out": kv.attend(0, q), "slot": s.slot}


# ---- what a pass cannot do without ----
def work(case):
    z = _sizes(case, 0)
    T, h, kv, d = z["T"], z["heads"], z["kv"], z["dim"]
    held = z["old"] + z["new"]
    token = kv * (d + d // 16)                                                   # keys and values of a token in the cache
    b = f = 0.0
    if case["op"] in ("plan", "step"):
        b += 12.0 * z["n"] + 8.0 * T + 4.0 * float(np.sum(-(-held // BLOCK) - -(-z["old"] // BLOCK))) + z["blocks"] / 8.0
        f += float(T)
    if case["op"] == "rotate":
        b += 4.0 * T * (h + kv) * d + 4.0 * T
        f += 3.0 * T * (h + kv) * d
    if case["op"] in ("store", "step"):
        b += 4.0 * T * h * d + 4.0 * T * kv * d + T * token
        f += 3.0 * T * (h + kv) * d
    if case["op"] == "store":
        b += T * token + 4.0 * T * kv * d
    if case["op"] in ("attend", "step"):
        b += 4.0 * T * h * d + float(held.sum()) * token
        f += 4.0 * h * d * float(np.sum(z["new"] * z["old"] + z["new"] * (z["new"] + 1) / 2.0))
    return {"bytes": b, "flops": f}


# ---- the definition in 64 bits, apart from the plain form ----
def _exact_four(x):
    """The values that four bits stand for; x: float64 [..., dim]."""
    g = x.reshape(-1, GROUP)
    top = g.abs().amax(1, keepdim=True)
    e = torch.ceil(torch.log2(top / 7.0)).clamp(-100, 125)
    e = e + (top > 7.0 * 2.0 ** e).double()          # log2 may be off by a last bit on either side of a power of two
    e = (e - (top <= 7.0 * 2.0 ** (e - 1)).double()).clamp(-100, 125)
    y = g.abs() / 2.0 ** e
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    y = (torch.round(y / step) * step).clamp(max=6.0)
    return (torch.sign(g) * y * 2.0 ** e).reshape(x.shape)


def _exact_rotate(x, heads, weight, position, freq):
    x = x.double().reshape(x.shape[0], heads, -1)
    if weight is not None:
        x = x / torch.sqrt(torch.mean(x * x, -1, keepdim=True) + EPS) * weight.double()
    half = x.shape[-1] // 2
    angle = position.double()[:, None, None] * freq.double()
    z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    if case["op"] == "plan":
        return None
    z = _inputs(case, seed)
    T, h, kv, d, old, new = z["T"], z["heads"], z["kv"], z["dim"], z["old"], z["new"]
    position = torch.cat([torch.arange(o, o + n) for o, n in zip(old.tolist(), new.tolist())]).to(DEVICE)
    if case["op"] == "attend":
        q = z["q"].double().reshape(T, h, d)
        k = _exact_four(z["k"].double().reshape(T, kv, d))
    else:
        q = _exact_rotate(z["q"], h, z["q_norm"], position, z["freq"])
        k = _exact_rotate(z["k"], kv, z["k_norm"], position, z["freq"])
        if case["op"] == "rotate":
            return {"q": q.reshape(T, -1), "k": k.reshape(T, -1)}
        k = _exact_four(k.float().double())          # a rotated key is rounded to 32 bits first
    v = _exact_four(z["v"].double().reshape(T, kv, d))
    if case["op"] == "store":
        return {"q": q.reshape(T, -1), "k": k.reshape(T, -1), "v": v.reshape(T, -1)}
    if case["op"] == "step":
        q = q.bfloat16().double()                    # attention reads the rotated queries as they are stored
    if float(np.sum((old + new) * new)) * h > 4e9:
        return None
    out = torch.empty(T, h, d, dtype=torch.float64, device=DEVICE)
    before, at = 0, 0
    for o, n in zip(old.tolist(), new.tolist()):
        past = [_exact_four(z[x][before:before + o].double().reshape(o, kv, d)) for x in ("k_old", "v_old")]
        keys, values = (torch.cat([p, c[at:at + n]]) for p, c in zip(past, (k, v)))
        hidden = torch.arange(o + n, device=DEVICE)[None] > torch.arange(o, o + n, device=DEVICE)[:, None]
        for i in range(h):
            s = torch.mm(q[at:at + n, i], keys[:, i // (h // kv)].T.contiguous()) / math.sqrt(d)
            s[hidden] = -math.inf
            out[at:at + n, i] = torch.mm(torch.softmax(s, -1), values[:, i // (h // kv)].contiguous())
        before, at = before + o, at + n
    out = out.reshape(T, -1)
    return {"out": out, "slot": None} if case["op"] == "step" else {"out": out}
