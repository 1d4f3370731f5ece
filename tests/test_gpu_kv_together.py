"""The cache's operators as an engine uses them: prompts, further turns on cached prefixes, decode steps and pages
that are given to another sequence, against one plain computation in 64 bits; the measured service model."""
import json

import numpy as np
import pytest
import torch

from tests.kv_util import BF16, E4M3, FP16, half_step, power, quantise

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,store", [(BF16, BF16), (FP16, E4M3), (BF16, E4M3)])
def test_a_conversation(dtype, store):
    from paper_2602_11688_b200 import binding as gb
    H, HK, D, page = 8, 2, 64, 32
    cache = gb.GorgoKvCache.empty(64, HK, D, store, page)
    for x in (cache.k, cache.v):                             # what other sequences left behind
        x.view(torch.uint8).fill_(0x7f)
    g = torch.Generator(device="cuda").manual_seed(5)
    free = list(np.random.default_rng(5).permutation(64))
    pages, kv = [[], [], []], [0, 0, 0]
    k_all, v_all = ([torch.zeros((0, HK, D), dtype=torch.float64, device="cuda") for _ in range(3)] for _ in "kv")

    def step(new, decode):
        for s, n in enumerate(new):
            kv[s] += n
            while len(pages[s]) * page < kv[s]:
                pages[s].append(int(free.pop()))
        table = torch.full((3, max(map(len, pages))), -1, dtype=torch.int32, device="cuda")
        for s, p in enumerate(pages):
            table[s, :len(p)] = torch.tensor(p, dtype=torch.int32)
        batch = gb.GorgoKvBatch(new, kv, table)
        rows = torch.randn((sum(new), H + 2 * HK, D), generator=g, device="cuda").to(dtype)
        q, k, v = rows[:, :H], rows[:, H:H + HK], rows[:, H + HK:]
        cache.write(batch, k, v)
        out = (cache.decode if decode else cache.prefill)(batch, q)
        batch.check()
        at = 0
        for s, n in enumerate(new):
            for kept, x in ((k_all, k), (v_all, v)):
                x = x[at:at + n].double()
                if store == E4M3 and n:
                    codes, e = quantise(x)
                    x = codes * power(e[..., None])
                kept[s] = torch.cat([kept[s], x])
            for i in range(n):
                seen = kv[s] - n + i + 1
                kk, vv = (x[s][:seen].repeat_interleave(H // HK, 1) for x in (k_all, v_all))
                p = torch.softmax(torch.einsum("hd,khd->hk", q[at + i].double(), kk) * D ** -0.5, 1)
                ref = torch.einsum("hk,khd->hd", p, vv)
                sizes = torch.einsum("hk,khd->hd", p, vv.abs())
                u = half_step(dtype)                         # P rounded, the output rounded; 2^-10 for 32-bit sums of scores and keys
                bound = sizes * (u + 2.0 ** -10) + ref.abs() * u + 2.0 ** -20
                assert ((out[at + i].double() - ref).abs() <= bound).all()
            at += n

    step([40, 130, 1], False)                                # first prompts
    for _ in range(5):
        step([1, 1, 1], True)
    step([70, 3, 200], False)                                # further turns on what is cached
    step([1, 1, 1], True)
    free.extend(pages[1])                                    # the second conversation is over, its pages go to a new one
    pages[1], kv[1] = [], 0
    k_all[1], v_all[1] = k_all[1][:0], v_all[1][:0]
    step([0, 150, 20], False)
    step([1, 1, 1], True)


def test_an_engine_layer_is_its_formula():
    """Prefill in two turns and a decode step of a whole layer against the same layer in 64 bits."""
    from paper_2602_11688_b200 import binding as gb
    from paper_2602_11688_b200 import service as S
    shape = S.EngineShape(2, 64, 96, 4, 2, 64)
    layer = S.EngineLayer(shape, 8, 64, "bf16")
    x = torch.randn((131, 64), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(BF16)
    table = torch.tensor([[5, 0, 7]], dtype=torch.int32, device="cuda")
    got = torch.cat([layer.prefill(gb.GorgoKvBatch([100], [100], table), x[:100]),
                     layer.prefill(gb.GorgoKvBatch([30], [130], table), x[100:130]),
                     layer.decode(gb.GorgoKvBatch([1], [131], table), x[130:])])
    w = {n: getattr(layer, n).double() for n in ("qkv", "out", "up", "down")}
    rows = (x.double() @ w["qkv"]).to(BF16).double().view(131, 8, 64)
    q, k, v = rows[:, :4], rows[:, 4:6].repeat_interleave(2, 1), rows[:, 6:].repeat_interleave(2, 1)
    z = torch.einsum("nhd,khd->hnk", q, k) / 8
    z = z.masked_fill(torch.ones((131, 131), device="cuda").triu(1).bool(), -torch.inf)
    a = x.double() + torch.einsum("hnk,khd->nhd", torch.softmax(z, 2), v).flatten(1) @ w["out"]
    gate, up = (a @ w["up"]).chunk(2, 1)
    ref = a + (torch.nn.functional.silu(gate) * up) @ w["down"]
    # eight roundings to bf16 (2^-8 each) on the way to a sum of terms of about the size of the result
    assert (got.double() - ref).norm() <= 8 * 2.0 ** -8 * ref.norm()


@pytest.mark.parametrize("kv_type", ["bf16", "e4m3"])
def test_the_tuner_measures_its_service_model(kv_type, capsys):
    from paper_2602_11688_b200 import tune
    tune.main(["--workload", "tiny", "--requests", "300", "--steps", "2", "--lam", "2", "--engine", "2x256x512x8x2x64",
               "--kv-type", kv_type])
    lines = [json.loads(x) for x in capsys.readouterr().out.splitlines()]
    s = lines[0]["service"]
    assert s["prefill_ms_per_token"] > 0 and s["tpot_ms"] > 0 and s["decode_slowdown"] >= 0
    assert s["cache_blocks"] > 0 and s["kv_budget_tokens"] == s["cache_blocks"] * 512
    assert len(s["prefill"]) > 0 and [b for b, _ in s["decode"]] == [1, 2, 4]
    table = lines[-1]["p95_ttft_ms_and_p95_e2e_ms"]
    assert "gorgo-tuned" in table and all(np.isfinite(v).all() and min(v) > 0 for v in table.values())


def test_the_measured_times_are_the_gpus(monkeypatch):
    """A host that takes its time between a layer's calls changes nothing: an engine replays a graph."""
    import time
    from paper_2602_11688_b200 import service as S
    from paper_2602_11688_b200 import workloads as W
    rest = S.EngineLayer._rest

    def slow(self, x, attended):
        time.sleep(0.01)
        return rest(self, x, attended)

    monkeypatch.setattr(S.EngineLayer, "_rest", slow)
    s = S.measure(W.make_workload("tiny", population=1, n_requests=300), S.EngineShape(1, 256, 512, 8, 2, 64), samples=2)
    assert all(t < 5.0 for _, t in s["decode"]) and all(t < 5.0 for *_, t in s["prefill"])
