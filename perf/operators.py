"""The paged key-value cache and the attention over it, as measurable cases.

An engine behind the router keeps the keys and values of prompts in blocks ("pages") of a fixed number of
tokens; what the router calls a prefix hit is that the pages of a prompt's leading blocks are still there.
A case is a dict of plain values; ``op`` says which call it stands for:

  write    the new tokens' keys and values go into their pages, in 16 bits or as e4m3 with one power of
           two for each token and head
  read     tokens come back out of their pages in 16 bits
  prefill  the uncached tokens of several prompts attend to cached prefix and to one another, causally
  decode   one new token for every running request attends to everything before it

Pool layout ``[pages][kv heads][page tokens][head dim]``; a sequence's pages come from a table.  Lengths are
lognormal as in this repository's workloads (medians 1,000 and 20,000 tokens, cap 128,000, 512-token blocks,
4 to 64 slots) and fixed by the case; the values come from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


def _case(name, op, n, kv, *, new=0, heads=32, kv_heads=8, dim=128, dtype="bf16", store="bf16", page=512,
          sigma=0.8, lens=1):
    """`kv`: median of the tokens already cached; `new`: median of the new ones; `lens` draws the lengths."""
    c = {"op": op, "n": int(n), "kv": int(kv), "new": int(new), "heads": int(heads), "kv_heads": int(kv_heads),
         "dim": int(dim), "dtype": dtype, "store": store, "page": int(page), "sigma": float(sigma), "lens": int(lens)}
    return {"name": name, **c} if name else c


def listed():
    return [
        # a decode step's new tokens, one for each of 16 slots, quantised on the way in: latency counts
        _case("write 16 tokens e4m3", "write", 16, 1000, new=1, store="e4m3", sigma=1.0),
        # a batch of new turns of long conversations, stored as they are
        _case("write turns bf16", "write", 24, 20_000, new=1000),
        # the longest prompt a trace may hold, quantised
        _case("write 128000 tokens e4m3", "write", 1, 0, new=128_000, store="e4m3", sigma=0.0),
        # a short prompt in small pages and small heads
        _case("read short fp16", "read", 3, 0, new=333, heads=16, kv_heads=4, dim=64, dtype="fp16", store="fp16", page=16),
        # the cached prefixes of a full replica, to be moved or re-used in 16 bits
        _case("read prefixes e4m3", "read", 16, 0, new=20_000, store="e4m3"),
        # four slots of the smallest configuration
        _case("decode 4 slots short", "decode", 4, 1000, sigma=1.0),
        # sixteen slots of long conversations
        _case("decode 16 slots long", "decode", 16, 20_000),
        # 64 slots, the paper's concurrency limit, in 8 bits
        _case("decode 64 slots e4m3", "decode", 64, 20_000, store="e4m3"),
        # one conversation at the cap, few kv heads: only a split over its length fills the GPU
        _case("decode 1 slot longest", "decode", 1, 127_999, heads=16, kv_heads=2, dim=64, dtype="fp16", store="fp16", page=64, sigma=0.0),
        # first prompts of the multi-region configuration, packed
        _case("prefill first prompts", "prefill", 16, 0, new=1000, sigma=1.0),
        # a new turn on top of a long cached prefix, cache in 8 bits
        _case("prefill turn on prefix e4m3", "prefill", 2, 20_000, new=1000, store="e4m3"),
        # a first prompt of the long-context configuration, whole
        _case("prefill 20000 tokens", "prefill", 1, 0, new=20_000, sigma=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("write", "read", "decode", "prefill"))
    heads, kv_heads = rng.choice(((32, 8), (16, 2), (8, 8), (28, 4), (24, 8), (64, 8), (8, 1), (12, 6)))
    dtype = rng.choice(("bf16", "fp16"))
    store = rng.choice((dtype, "e4m3"))
    page = rng.choice((16, 32, 64, 128, 256, 512, 1024))
    n, dim = _log(rng, 1, 64), rng.choice((64, 128))
    room = 400_000 // n               # tokens a sequence may have on average
    kv = new = 0
    if op in ("write", "read"):
        new, kv = _log(rng, 1, min(room, 20_000)), rng.choice((0, _log(rng, 1, min(room, 20_000))))
    elif op == "decode":
        kv = _log(rng, 1, min(room, 20_000))
    else:
        n = _log(rng, 1, 16)
        new, kv = _log(rng, 1, 4000 // n + 40), rng.choice((0, _log(rng, 1, 20_000 // n)))
    return _case(None, op, n, kv, new=new, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, store=store,
                 page=page, sigma=rng.choice((0.0, 0.5, 0.8)), lens=rng.randrange(1 << 30))


def _lengths(case):
    """(new tokens, tokens in all) of every sequence."""
    r = random.Random(case["lens"])

    def one(median):
        return max(1, min(128_000, int(median * math.exp(case["sigma"] * r.gauss(0, 1))))) if median else 0

    cached = [one(case["kv"]) for _ in range(case["n"])]
    new = [1 if case["op"] == "decode" or case["new"] == 1 else one(case["new"]) for _ in cached]
    return new, [a + b for a, b in zip(cached, new)]


def prepare(case, seed):
    new, kv = _lengths(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    page, hk, d, store = case["page"], case["kv_heads"], case["dim"], _TYPES[case["store"]]
    need = [-(-x // page) for x in kv]
    pages = sum(need) + 3                                    # some pages of the pool belong to nobody
    order = torch.randperm(pages, device="cuda", generator=g, dtype=torch.int32)
    table = torch.full((len(kv), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = order[at:at + m]
        at += m
    shape = (pages, hk, page, d)

    def normal(shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) * scale

    s = {"case": dict(case), "new": new, "kv": kv, "scale": 1.0 / math.sqrt(d), "table": table,
         "cu": torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda"),
         "kv_len": torch.tensor(kv, dtype=torch.int32, device="cuda"), "k_exp": None, "v_exp": None}
    for x in ("k", "v"):
        if case["store"] == "e4m3":
            s[x] = normal(shape, 112.0).clamp_(-448, 448).to(store)
            s[x + "_exp"] = torch.randint(-9, -5, shape[:3], generator=g, device="cuda", dtype=torch.int8)
        else:
            s[x] = normal(shape).to(store)
    dtype, total = _TYPES[case["dtype"]], sum(new)
    if case["op"] == "write":                               # a row's size differs from token to token and head to head
        size = torch.exp(torch.randn((total, hk, 1), generator=g, device="cuda"))
        s["k_new"] = (normal((total, hk, d)) * size).to(dtype)
        s["v_new"] = (normal((total, hk, d)) * size.flip(0)).to(dtype)
    if case["op"] in ("decode", "prefill"):
        s["q"] = normal((total, case["heads"], d), 1.5).to(dtype)
    return s


def work(case):
    new, kv = _lengths(case)
    hk, h, d = case["kv_heads"], case["heads"], case["dim"]
    row = d + 1 if case["store"] == "e4m3" else 2 * d        # bytes of a stored row
    if case["op"] in ("write", "read"):
        return {"bytes": 2.0 * sum(new) * hk * (2 * d + row), "flops": 0}
    pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(new, kv))
    return {"bytes": 2.0 * sum(kv) * hk * row + 4.0 * sum(new) * h * d, "flops": 4.0 * pairs * h * d}


# ------------------------------------------------------------------------------- the two sides
def run(state):
    op = state["case"]["op"]
    if own:
        cache, batch = state.get("handle") or _handle(state)
        if op == "write":
            cache.write(batch, state["k_new"], state["v_new"])
            return _pool(state)
        if op == "read":
            return cache.read(batch, _TYPES[state["case"]["dtype"]])
        return (cache.decode if op == "decode" else cache.prefill)(batch, state["q"], state["scale"])
    return {"write": _write, "read": _read, "decode": _decode, "prefill": _prefill}[op](state)


def _handle(state):
    from paper_2602_11688_b200 import binding as gb
    cache = gb.GorgoKvCache(state["k"], state["v"], state["k_exp"], state["v_exp"])
    batch = gb.GorgoKvBatch(state["new"], state["kv"], state["table"], cu_new=state["cu"], kv_len=state["kv_len"])
    state["handle"] = cache, batch
    return state["handle"]


def _pool(state):
    return [state[x] for x in ("k", "v", "k_exp", "v_exp")]


# ------------------------------------------------------------------------------- plain forms
def _places(state):
    """Page and slot of every new token."""
    cu, page = state["cu"].long(), state["case"]["page"]
    t = torch.arange(sum(state["new"]), device="cuda")
    seq = torch.searchsorted(cu, t, right=True) - 1
    pos = state["kv_len"].long()[seq] - (cu[1:] - cu[:-1])[seq] + t - cu[seq]
    return state["table"][seq, pos // page].long(), pos % page


def _power(e):
    """2^e for each row, exactly: a power function may be off in its last bit, which moves ties."""
    return ((e.int() + 127) << 23).view(torch.float32)[..., None]


def _write(state):
    at, slot = _places(state)
    for x in ("k", "v"):
        rows = state[x + "_new"]
        if state[x + "_exp"] is None:
            state[x][at, :, slot] = rows
            continue
        rows = rows.float()
        part, e = torch.frexp(rows.abs().amax(-1))           # amax = part * 2^e, 0.5 <= part < 1
        e = torch.where(part > 0.875, e - 8, e - 9).clamp(min=-24)
        e = torch.where(part == 0, -24, e)
        state[x].view(torch.uint8)[at, :, slot] = (rows * _power(-e)).to(torch.float8_e4m3fn).view(torch.uint8)
        state[x + "_exp"][at, :, slot] = e.to(torch.int8)
    return _pool(state)


def _read(state):
    at, slot = _places(state)
    dtype, out = _TYPES[state["case"]["dtype"]], []
    for x in ("k", "v"):
        if state[x + "_exp"] is None:
            out.append(state[x][at, :, slot].to(dtype))
        else:
            rows = state[x].view(torch.uint8)[at, :, slot].view(torch.float8_e4m3fn).float()
            out.append((rows * _power(state[x + "_exp"][at, :, slot])).to(dtype))
    return out


def _rows(state, x, s):
    """Keys or values of one sequence in 32 bits, [kv heads][tokens][dim]."""
    m = -(-state["kv"][s] // state["case"]["page"])
    ids = state["table"][s, :m].long()
    rows = state[x].view(torch.uint8)[ids].view(torch.float8_e4m3fn).float() if state[x + "_exp"] is not None else state[x][ids].float()
    if state[x + "_exp"] is not None:
        rows = rows * _power(state[x + "_exp"][ids])
    return rows.transpose(0, 1).flatten(1, 2)[:, :state["kv"][s]]


def _attend(q, k, v, first, scale):
    """q [rows][heads][dim] at positions first, first + 1, ...; 32 bits."""
    n, h, d = q.shape
    hk = k.shape[0]
    z = torch.matmul(q.float().view(n, hk, h // hk, d).permute(1, 2, 0, 3).reshape(hk, -1, d), k.transpose(1, 2)) * scale
    z = z.view(hk, h // hk, n, -1)
    seen = torch.arange(k.shape[1], device="cuda") <= first + torch.arange(n, device="cuda")[:, None]
    z = z.masked_fill_(~seen, -math.inf)
    z = z.sub_(z.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(z.view(hk, -1, k.shape[1]), v) / z.sum(-1).view(hk, -1, 1)
    return o.view(hk, h // hk, n, d).permute(2, 0, 1, 3).reshape(n, h, d).to(q.dtype)


def _decode(state):
    q, scale = state["q"], state["scale"]
    return torch.cat([_attend(q[s:s + 1], _rows(state, "k", s), _rows(state, "v", s), kv - 1, scale)
                      for s, kv in enumerate(state["kv"])])


def _prefill(state):
    q, out, at = state["q"], [], 0
    for s, (n, kv) in enumerate(zip(state["new"], state["kv"])):
        k, v = _rows(state, "k", s), _rows(state, "v", s)
        for a in range(0, n, 1024):                          # as many rows as scores fit beside the rest
            b = min(n, a + 1024)
            out.append(_attend(q[at + a:at + b], k[:, :kv - n + b], v[:, :kv - n + b], kv - n + a, state["scale"]))
        at += n
    return torch.cat(out)


# ------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    d, page, hk = case["dim"], case["page"], case["kv_heads"]

    def place(i, j):                                         # flat row of the pool without the head
        return s["table"][i].long()[j // page] * hk * page + j % page

    where = [place(i, torch.arange(kv - n, kv, device="cuda")) for i, (n, kv) in enumerate(zip(s["new"], s["kv"]))]
    heads = torch.arange(hk, device="cuda") * page

    def values(x, rows):
        v = s[x].view(torch.uint8).view(-1, d)[rows].view(torch.float8_e4m3fn).double() if case["store"] == "e4m3" else s[x].view(-1, d)[rows].double()
        return v * torch.exp2(s[x + "_exp"].view(-1)[rows].double())[..., None] if case["store"] == "e4m3" else v

    if case["op"] == "read":
        rows = torch.cat(where)[:, None] + heads
        return [values("k", rows), values("v", rows)]
    if case["op"] == "write":
        rows = torch.cat(where)[:, None] + heads
        out = []
        for x in ("k", "v"):
            new = s[x + "_new"].double()
            if case["store"] == "e4m3":
                top = new.abs().amax(-1)
                e = (torch.round(torch.log2(top / 448)) - 1).clamp(min=-24)
                for _ in range(2):                           # a logarithm may be off in its last bit
                    e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
                y = new * torch.exp2(-e)[..., None]
                unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)   # distance of e4m3 values there
                new = torch.round(y / unit) * unit
            pool = torch.cat([c.double() for c in s[x].view(-1, d).split(1 << 20)])
            pool[rows] = new
            out.append(pool.view(s[x].shape))
        return out + [None, None]
    out, at = [], 0
    for i, (n, kv) in enumerate(zip(s["new"], s["kv"])):
        rows = place(i, torch.arange(kv, device="cuda"))
        q = s["q"][at:at + n].double()
        o = torch.empty_like(q)
        for h in range(case["heads"]):
            g = h // (case["heads"] // hk)
            k, v = values("k", rows + g * page), values("v", rows + g * page)
            for a in range(0, n, 4096):
                z = torch.einsum("nd,kd->nk", q[a:a + 4096, h], k) / math.sqrt(d)
                last = torch.arange(kv - n + a, kv - n + a + z.shape[0], device="cuda")
                z[torch.arange(kv, device="cuda")[None] > last[:, None]] = -math.inf
                o[a:a + 4096, h] = torch.einsum("nk,kd->nd", torch.exp(z - torch.logsumexp(z, 1, keepdim=True)), v)
        out.append(o)
        at += n
    return torch.cat(out)
