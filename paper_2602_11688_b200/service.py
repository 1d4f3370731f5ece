"""The constants of the service model, measured on the GPU at hand.

The simulator takes an engine's times as five numbers: prefill time per uncached token, time per output
token, its growth with the number of busy slots, the blocks that a replica's cache holds and the tokens
that may run at once (the paper measures its engines, Section 4; it models prefill as the tokens that are
not cached, Eq. 1).  ``measure`` runs one layer of a decoder of a given shape on requests of the workload: their
uncached tokens on top of their cached prefix (``GorgoKvCache.write``, ``GorgoKvCache.prefill``), and decode
steps of one token per busy slot (``write``, ``decode``), with the cache in pages of the simulator's block
size.  Projections and feed-forward are plain library products over random weights; a layer's time counts
as often as the shape has layers.

    python -m paper_2602_11688_b200.tune --workload regions --engine 32x4096x14336x32x8x128 --kv-type e4m3
"""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np


@dataclass(frozen=True)
class EngineShape:
    layers: int
    hidden: int
    ffn: int
    heads: int
    kv_heads: int
    head_dim: int

    @classmethod
    def parse(cls, text: str) -> "EngineShape":
        """``LAYERSxHIDDENxFFNxHEADSxKV_HEADSxHEAD_DIM``"""
        parts = text.lower().split("x")
        if len(parts) != 6 or not all(p.isdigit() and int(p) > 0 for p in parts):
            raise ValueError(f"{text!r}: six positive numbers LAYERSxHIDDENxFFNxHEADSxKV_HEADSxHEAD_DIM")
        s = cls(*map(int, parts))
        if s.heads % s.kv_heads or s.heads // s.kv_heads > 128 or s.head_dim not in (64, 128) or s.hidden % 8:
            raise ValueError(f"{text!r}: heads a multiple of kv heads (at most 128 times), head_dim 64 or 128, "
                             "hidden a multiple of 8")
        return s

    def weight_bytes(self) -> int:
        """Bytes of all layers' weights in 16 bits."""
        qkv = self.hidden * (self.heads + 2 * self.kv_heads) * self.head_dim
        return 2 * self.layers * (qkv + self.heads * self.head_dim * self.hidden + 3 * self.hidden * self.ffn)

    def block_bytes(self, block_tokens: int, kv_type: str) -> int:
        """Bytes of one cache block over all layers, keys and values (and the e4m3 rows' powers of two)."""
        row = self.head_dim + 1 if kv_type == "e4m3" else 2 * self.head_dim
        return self.layers * 2 * self.kv_heads * block_tokens * row


class EngineLayer:
    """One decoder layer with random weights over a paged cache."""

    def __init__(self, shape: EngineShape, n_pages: int, block_tokens: int, kv_type: str = "bf16", device: int = 0,
                 seed: int = 0):
        import torch
        from . import binding as gb
        self.torch, self.shape = torch, shape
        self.device = torch.device("cuda", device)
        self.dtype = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.bfloat16}[kv_type]
        self.cache = gb.GorgoKvCache.empty(n_pages, shape.kv_heads, shape.head_dim,
                                           torch.float8_e4m3fn if kv_type == "e4m3" else self.dtype, block_tokens, device)
        g = torch.Generator(device=self.device).manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn((rows, cols), generator=g, device=self.device) * rows ** -0.5).to(self.dtype)

        s = shape
        self.qkv = weight(s.hidden, (s.heads + 2 * s.kv_heads) * s.head_dim)
        self.out = weight(s.heads * s.head_dim, s.hidden)
        self.up = weight(s.hidden, 2 * s.ffn)
        self.down = weight(s.ffn, s.hidden)

    def _project(self, batch, x):
        s = self.shape
        rows = (x @ self.qkv).view(x.shape[0], s.heads + 2 * s.kv_heads, s.head_dim)
        self.cache.write(batch, rows[:, s.heads:s.heads + s.kv_heads], rows[:, s.heads + s.kv_heads:])
        return rows[:, :s.heads]

    def _rest(self, x, attended):
        x = x + attended.flatten(1) @ self.out
        gate, up = (x @ self.up).chunk(2, dim=1)
        return x + (self.torch.nn.functional.silu(gate) * up) @ self.down

    def prefill(self, batch, x):
        """``x`` [new tokens, hidden]: the layer's output for the new tokens, whose keys and values are cached."""
        return self._rest(x, self.cache.prefill(batch, self._project(batch, x)))

    def decode(self, batch, x):
        """``x`` [sequences, hidden]: one more token of each sequence (``batch`` counts it as new)."""
        return self._rest(x, self.cache.decode(batch, self._project(batch, x)))


def requests_of(w, count: int, seed: int = 0):
    """(uncached tokens, all tokens) of ``count`` requests of a workload, as if the block lists of their session's
    previous turn were cached: what a router that follows the cache sees."""
    last, seen = {}, []
    ids, off = w.hash_ids, w.hash_off.astype(np.int64)
    for r in range(w.n_requests):
        mine = ids[off[r]:off[r + 1]]
        before = last.get(int(w.session[r]))
        hit = 0
        if before is not None:
            n = min(len(mine), len(before))
            differ = np.nonzero(mine[:n] != before[:n])[0]
            hit = n if differ.size == 0 else int(differ[0])
        last[int(w.session[r])] = mine
        tokens = int(w.input_tokens[r])
        uncached = tokens - min(hit * w.spec.block_tokens, tokens)
        if uncached:
            seen.append((uncached, tokens))
    rng = np.random.default_rng(seed)
    pick = rng.permutation(len(seen))[:count]
    return [seen[i] for i in pick]


def fit_prefill(uncached, ms) -> float:
    """Time per uncached token: least squares of ms = c * uncached."""
    u, t = np.asarray(uncached, np.float64), np.asarray(ms, np.float64)
    return float((u * t).sum() / (u * u).sum())


def fit_decode(busy, ms):
    """(tpot, decode slow-down): least squares of ms = tpot * (1 + slowdown * (busy - 1)), neither negative."""
    b, t = np.asarray(busy, np.float64) - 1.0, np.asarray(ms, np.float64)
    if len(b) == 1 or np.ptp(b) == 0:
        return float(t.mean()), 0.0
    slope = float(((b - b.mean()) * (t - t.mean())).sum() / ((b - b.mean()) ** 2).sum())
    at0 = float(t.mean() - slope * b.mean())
    if slope <= 0 or at0 <= 0:
        return float(t.mean()), 0.0
    return at0, slope / at0


def cache_and_budget(blocks: int, w):
    """(blocks of the prefix cache, tokens of requests that run) where there is memory for ``blocks`` blocks: prompts
    of running requests lie in the cache's blocks; their answers, up to the workload's longest in every slot,
    take the others."""
    answers = w.spec.slots * -(-int(w.output_tokens.max()) // w.spec.block_tokens)
    if blocks <= answers:
        raise ValueError("the weights leave no room for a cache block beside the running requests' answers")
    return blocks - answers, (blocks - answers) * w.spec.block_tokens


def measure(w, shape: EngineShape, kv_type: str = "bf16", *, device: int = 0, samples: int = 16, repeats: int = 5,
            memory_share: float = 0.9, seed: int = 0):
    """The service model's constants for workload ``w`` on an engine of ``shape``: a dict of
    ``prefill_ms_per_token``, ``tpot_ms``, ``decode_slowdown``, ``cache_blocks``, ``kv_budget_tokens`` and what
    they were fitted to.  The cache has what ``memory_share`` of the GPU's memory leaves beside the weights and the
    running requests' answers."""
    import torch
    from . import binding as gb
    block = w.spec.block_tokens
    blocks = int((torch.cuda.get_device_properties(device).total_memory * memory_share - shape.weight_bytes())
                 // shape.block_bytes(block, kv_type))
    blocks, budget = cache_and_budget(blocks, w)
    drawn = requests_of(w, max(samples, w.spec.slots), seed)
    if not drawn:
        raise ValueError("the workload has no request with uncached tokens")
    running = [drawn[i % len(drawn)][1] + 1 for i in range(w.spec.slots)]
    need = [-(-n // block) for n in running]
    layer = EngineLayer(shape, max(sum(need), max(-(-n // block) for _, n in drawn)), block, kv_type, device, seed)
    dev = layer.device
    g = torch.Generator(device=dev).manual_seed(seed + 1)

    def rows(n):
        return torch.randn((n, shape.hidden), generator=g, device=dev).to(layer.dtype)

    def table(need):
        t = torch.zeros((len(need), max(need)), dtype=torch.int32, device=dev)
        at = 0
        for s, n in enumerate(need):
            t[s, :n] = torch.arange(at, at + n, dtype=torch.int32, device=dev)
            at += n
        return t

    def ms(call, batch, x):
        """A layer as an engine runs it: replayed from a graph, its weights and cache out of the L2, where the other
        layers have been since."""
        call(batch, x)
        batch.check()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(batch, x)
        total = 0.0
        for _ in range(repeats):
            others.sum()                  # (read, as weights are: nothing is left to be written back)
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            begin.record()
            graph.replay()
            end.record()
            end.synchronize()
            total += begin.elapsed_time(end)
        batch.check()
        return total / repeats * shape.layers

    with torch.cuda.device(dev):
        others = torch.zeros(torch.cuda.get_device_properties(dev).L2_cache_size // 2, device=dev)   # twice the L2
        prefill = [(u, n, ms(layer.prefill, gb.GorgoKvBatch([u], [n], table([-(-n // block)])), rows(u)))
                   for u, n in drawn[:samples]]
        decode = []
        for b in sorted({1, max(1, w.spec.slots // 4), max(1, w.spec.slots // 2), w.spec.slots}):
            batch = gb.GorgoKvBatch([1] * b, running[:b], table(need[:b]))
            decode.append((b, ms(layer.decode, batch, rows(b))))
    tpot, slowdown = fit_decode(*zip(*decode))
    return {"prefill_ms_per_token": fit_prefill([u for u, _, _ in prefill], [t for _, _, t in prefill]),
            "tpot_ms": tpot, "decode_slowdown": slowdown, "cache_blocks": blocks,
            "kv_budget_tokens": budget, "prefill": prefill, "decode": decode}
