"""Inputs and the plain 64-bit implementation for the tests of the paged key-value cache."""
import numpy as np
import torch

BF16, FP16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def half_step(dtype):
    """Largest relative error of a rounding to `dtype`: half a step."""
    return torch.finfo(dtype).eps / 2


def table_for(kv, page, rng, spare=2, pad=2):
    """Random pages for sequences of kv[s] tokens: (int32 table with rubbish where nothing is needed, pages)."""
    need = [-(-x // page) for x in kv]
    order = rng.permutation(sum(need) + spare)
    table = rng.choice(np.array([-1, 1 << 30, -(1 << 31)]), size=(len(kv), max(need + [0]) + pad))
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = order[at:at + m]
        at += m
    return torch.tensor(table, dtype=torch.int32, device="cuda"), len(order)


def power(e):
    """2^e in 64 bits, exactly (a power function may be off in its last bit)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def quantise(x):
    """(codes, exponents) of the rows of x, by the definition, in 64 bits."""
    x = x.double()
    lost = ~torch.isfinite(x).all(-1, keepdim=True)         # such a row is NaN throughout, e = 0
    x = torch.where(lost, 448.0, x)
    top = x.abs().amax(-1).cpu().numpy()
    e = np.full(top.shape, -24)
    for _ in range(200):
        e = np.where(top > 448.0 * np.exp2(e.astype(np.float64)), e + 1, e)
    e = torch.tensor(e, device=x.device)
    y = x * power(-e[..., None])
    part, p = torch.frexp(y.abs())                          # |y| = part * 2^p, steps of 2^(p-4), 2^-9 at the low end
    step = power((p - 4).clamp(min=-9))
    return torch.where(lost, float("nan"), torch.round(y / step) * step), e


class Made:
    """A cache whose pools hold NaN wherever no sequence has a token, and what the sequences hold in 64 bits."""

    def __init__(self, seed, new, kv, *, heads=4, kv_heads=2, dim=64, dtype=BF16, store=None, page=64, q_scale=1.5):
        from paper_2602_11688_b200 import binding as gb
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        store = store or dtype
        self.new, self.kv, self.dtype, self.store, self.page = list(new), list(kv), dtype, store, page
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.table, n_pages = table_for(kv, page, rng)
        self.cache = gb.GorgoKvCache.empty(n_pages, kv_heads, dim, store, page)
        for pool in (self.cache.k, self.cache.v):
            if store == E4M3:
                pool.view(torch.uint8).fill_(0x7f)
            else:
                pool.fill_(float("nan"))
        self.batch = gb.GorgoKvBatch(new, kv, self.table)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.keys, self.values = [], []
        for s, n in enumerate(kv):
            for kept, pool, exps in ((self.keys, self.cache.k, self.cache.k_exp), (self.values, self.cache.v, self.cache.v_exp)):
                x = (rand(n, kv_heads, dim) * torch.exp(0.5 * rand(n, kv_heads, 1))).to(dtype)
                page_of, slot = self.where(s, torch.arange(n, device="cuda"))
                if store == E4M3:
                    codes, e = quantise(x) if n else (x.double(), torch.zeros((0, kv_heads), dtype=torch.int64, device="cuda"))
                    pool.view(torch.uint8)[page_of, :, slot] = codes.to(E4M3).view(torch.uint8)
                    exps[page_of, :, slot] = e.to(torch.int8)
                    kept.append(codes * power(e[..., None]))
                else:
                    pool[page_of, :, slot] = x
                    kept.append(x.double())
        self.q = (rand(sum(new), heads, dim) * q_scale).to(dtype)

    def where(self, s, j):
        return self.table[s].long()[j // self.page], j % self.page

    def row(self, s, q, seen, scale):
        """(out, lse, bound of the error of out for P rounded to the type) of one query row [heads][dim]."""
        d, group = self.dim, self.heads // self.kv_heads
        u = half_step(self.dtype)
        if seen <= 0:
            z = torch.zeros((self.heads, d), dtype=torch.float64, device="cuda")
            return z, torch.full((self.heads,), -np.inf, dtype=torch.float64, device="cuda"), z
        k = self.keys[s][:seen].repeat_interleave(group, 1)  # [seen][heads][dim]
        v = self.values[s][:seen].repeat_interleave(group, 1)
        z = torch.einsum("hd,khd->hk", q.double(), k) * scale
        p = torch.softmax(z, 1)
        # a score's error: `dim` products summed in 32 bits, each step off by at most 2^-22 of the sum of sizes (the
        # matrix unit cuts where it aligns), its product with the scale, the exponential (2^-21)
        far = torch.einsum("hd,khd->hk", q.double().abs(), k.abs()).amax(1) * abs(scale) * (d + 4) * 2.0 ** -22 + 2.0 ** -20
        out = torch.einsum("hk,khd->hd", p, v)
        sizes = torch.einsum("hk,khd->hd", p, v.abs())
        # fp16: P, at most 2^15, is a multiple of 2^-30 of its largest value or finer below its normal range
        few = seen * 2.0 ** -31 * v.abs().amax() if self.dtype == FP16 else 0.0
        # P rounded once (u), numerator and denominator each off by `far`, sums over the keys in 32 bits, the output's rounding
        keys = min(seen, 4096) * 2.0 ** -22
        bound = sizes * (u + 2 * far[:, None] + keys) * (1 + u) + out.abs() * u + 2.0 ** -24 * u + few
        return out, torch.logsumexp(z, 1), bound

    def expected(self, q, scale, decode):
        """Stacked (out, lse, bound) of all rows."""
        rows, at = [], 0
        for s, (n, kv) in enumerate(zip(self.new, self.kv)):
            for i in range(1 if decode else n):
                rows.append(self.row(s, q[s if decode else at + i], kv if decode else kv - n + i + 1, scale))
            at += n
        return [torch.stack([r[i] for r in rows]) for i in range(3)]


def check(out, lse, want, dtype):
    ref, ref_lse, bound = want
    assert torch.isfinite(out).all()
    off = (out.double() - ref).abs()
    worst = (off - bound).max().item()
    assert worst <= 0, (worst, off.max().item(), (off / bound.clamp(min=1e-30)).max().item())
    if lse is not None:
        none = torch.isinf(ref_lse)
        assert torch.equal(none, torch.isinf(lse)) and bool((lse[none] < 0).all())
        # the score's own error and 32-bit logarithms of sums
        assert ((lse.double() - ref_lse).abs()[~none] <= 2e-3 + 2.0 ** -20 * ref_lse[~none].abs()).all()
