"""Paged caches for the tests: seeded lists in a shuffled pool, the plain forms of the three operators in 64 bits, and the bounds that
the kernels' arithmetic allows."""
import math

import torch

from paper_2510_07651_b200 import api

D = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


def pow2(e):
    """2^e of whole numbers from -200 to 200, exactly."""
    table = torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64, device=e.device)
    return table[e.long() + 200]


def e4m3_64(x):
    """Rows in 64 bits -> (values of their codes before scaling, biased exponents): the smallest power of two with max|x| <= 448 times it,
    never below 2^-126; 4 significant bits from 2^-6 on, steps of 2^-9 below, ties to even.  Not finite: exponent 255, codes 0."""
    x = x.double()
    top = x.abs().amax(-1)
    fine = torch.isfinite(top)
    safe = torch.where(fine, top, 1.0)
    e = torch.full_like(top, -126.0)
    for k in range(-126, 121):                        # (no logarithm: the first power of two that is large enough)
        e = torch.where(safe > 448.0 * 2.0 ** k, k + 1.0, e)
    y = torch.where(fine[..., None], x, 0.0) / pow2(e)[..., None]
    step = torch.full_like(y, 2.0 ** -9)
    for k in range(-5, 9):
        step = torch.where(y.abs() >= 2.0 ** k, 2.0 ** (k - 3), step)
    return torch.round(y / step) * step, torch.where(fine, e + 127, 255.0).to(torch.uint8)


class Lists:
    """B x H lists of given lengths in pages of `P` tokens.  k, v: the rows' values in 64 bits (as the pages hold them), [B,H,N,d].
    Free places of the pool hold NaN (codes of all ones and scale 255 in 8 bits)."""

    def __init__(self, lens, H, P, pages="bf16", *, by_head=False, seed=0, spare_pages=3, k=None, v=None, dev="cuda", strided=False, spread=0.0):
        lens = torch.as_tensor(lens, dtype=torch.int32)
        B = lens.shape[0]
        g = torch.Generator().manual_seed(seed)
        self.B, self.H, self.P, self.pages, self.by_head = B, H, P, pages, by_head
        self.lens_bh = lens if lens.dim() == 2 else lens[:, None].expand(B, H)
        N = max(int(lens.max()), 1)
        self.N, self.max_pages = N, -(-N // P)
        rows = (B, H, N, D)
        self.k = (torch.randn(rows, generator=g) if k is None else k).double()
        self.v = (torch.randn(rows, generator=g) * torch.exp(0.5 * torch.randn(rows[:3] + (1,), generator=g)) if v is None else v).double()
        if spread:                                    # rows of very different magnitudes
            self.k *= torch.exp2(torch.randint(-3, 3, rows[:3] + (1,), generator=g).double())
            self.v *= torch.exp2(torch.randint(-int(spread), int(spread), rows[:3] + (1,), generator=g).double())
        heads, lists = (1, (B, H)) if by_head else (H, (B,))
        need = (lens if by_head else lens.view(B, -1).amax(1)).add(P - 1).div(P, rounding_mode="floor").expand(lists)
        n_pages = int(need.sum()) + spare_pages
        order = torch.randperm(n_pages, generator=g).to(torch.int32)
        table = torch.full(lists + (self.max_pages,), -1, dtype=torch.int32)
        at = 0
        for i in range(int(torch.tensor(lists).prod())):
            n = int(need.reshape(-1)[i])
            table.view(-1, self.max_pages)[i, :n] = order[at:at + n]
            at += n
        shape = (n_pages, heads, P, D)
        dt = TYPES[pages]
        pool, scales = [], []
        for name in ("k", "v"):
            x = getattr(self, name)
            if pages == "e4m3":
                codes, s = e4m3_64(x)
                setattr(self, name, torch.where((s == 255)[..., None], math.nan, codes * pow2(s.long() - 127)[..., None]))
                p = torch.full(shape, 255, dtype=torch.uint8)
                sc = torch.full(shape[:3], 255, dtype=torch.uint8)
                put, put_s = codes.float().to(dt).view(torch.uint8), s
            else:
                put = x.to(dt)
                setattr(self, name, put.double())
                p, sc, put_s = torch.full(shape, math.nan, dtype=dt), None, None
            for b in range(B):
                for h in range(H):
                    n = int(self.lens_bh[b, h])
                    t = torch.arange(n)
                    page = (table[b, h] if by_head else table[b])[t // P].long()
                    hp = 0 if by_head else h
                    p[page, hp, t % P] = put[b, h, :n]
                    if sc is not None:
                        sc[page, hp, t % P] = put_s[b, h, :n]
            p = p.view(dt) if pages == "e4m3" else p
            pool.append(p.to(dev))
            scales.append(None if sc is None else sc.to(dev))
        if strided:                                   # pages of a larger allocation: rows, heads and pages further apart than they are long
            wide = [torch.zeros((n_pages, heads + 1, P + 8, 160), dtype=torch.uint8 if pages == "e4m3" else dt, device=dev) for _ in range(2)]
            for w, p in zip(wide, pool):
                w[:, :heads, :P, :D] = p.view(w.dtype)
            pool = [w.view(dt)[:, :heads, :P, :D] for w in wide]
            if scales[0] is not None:
                ws = [torch.zeros((n_pages, heads + 1, P + 8), dtype=torch.uint8, device=dev) for _ in range(2)]
                for w, s in zip(ws, scales):
                    w[:, :heads, :P] = s
                scales = [w[:, :heads, :P] for w in ws]
        self.k, self.v = self.k.to(dev), self.v.to(dev)
        self.cache = api.PagedCache(pool[0], pool[1], table.to(dev), lens.to(dev), scales[0], scales[1])


def attention_64(q, L, *, q_lens=None, scale=None, causal=True):
    """(o, lse, bound on o's error, bound on lse's) in 64 bits over the lists' values; rows behind q_lens are NaN.  The bounds hold for logits summed in
    fp32 over 128 channels, weights rounded `p_bits` apart (see `check`), and do not count the rounding of o itself."""
    B, Hq, T, _ = q.shape
    G = Hq // L.H
    scale = scale or 1 / math.sqrt(D)
    o = torch.full((B, Hq, T, D), math.nan, dtype=torch.float64, device=q.device)
    lse, mean_abs, dz = (torch.full((B, Hq, T), math.nan, dtype=torch.float64, device=q.device) for _ in range(3))
    mean_abs = torch.full_like(o, math.nan)
    for b in range(B):
        m = T if q_lens is None else min(max(int(q_lens[b]), 0), T)
        for hq in range(Hq):
            h = hq // G
            n = int(L.lens_bh[b, h])
            k, v = L.k[b, h, :n], L.v[b, h, :n]
            qd = q[b, hq, :m].double()
            z = qd @ k.T * scale
            seen = (torch.arange(n, device=q.device) <= n - m + torch.arange(m, device=q.device)[:, None]) if causal else torch.ones((m, n), dtype=torch.bool, device=q.device)
            z = torch.where(seen, z, -math.inf)
            top = z.amax(-1, keepdim=True) if n else torch.full((m, 1), -math.inf, dtype=torch.float64, device=q.device)
            w = torch.exp(z - torch.where(torch.isneginf(top), 0.0, top))
            total = w.sum(-1, keepdim=True)
            p = w / torch.where(total == 0, 1.0, total)
            # tokens that a row does not see do not enter its sum, whatever they hold
            odd = ~torch.isfinite(v).all(-1)
            o[b, hq, :m] = p @ torch.where(odd[:, None], 0.0, v)
            for t in odd.nonzero()[:, 0].tolist():
                o[b, hq, :m] += torch.where(seen[:, t, None], p[:, t, None] * v[t], 0.0)
            mean_abs[b, hq, :m] = p @ torch.where(odd[:, None], 0.0, v).abs()
            lse[b, hq, :m] = (top + torch.log(total))[:, 0]
            spread = torch.where(seen, qd.abs() @ torch.nan_to_num(k, 0.0, 0.0, 0.0).abs().T * scale, 0.0)
            dz[b, hq, :m] = spread.amax(-1) if n else 0.0
    # a logit: 128 products summed in fp32 (136 roundings at most), its scaling and the subtraction of the reference; exp2 within 2^-22
    dz = dz * 140 * 2.0 ** -24 + 2.0 ** -21
    return o, lse, mean_abs, dz


def check(o, lse, q, L, *, weight_bits, q_lens=None, scale=None, causal=True, what=""):
    """o and lse against 64 bits.  weight_bits: weights are rounded to within 2^-weight_bits.  o is a quotient of two sums whose terms are off by a
    relative e = 2 dz + 2^-weight_bits + 2^-16 (running sums in fp32), so it is off by e (sum p|v| + |o|) <= 2 e sum p|v|, and by its own rounding."""
    want, want_lse, mean_abs, dz = attention_64(q, L, q_lens=q_lens, scale=scale, causal=causal)
    half_step = torch.finfo(o.dtype).eps / 2
    real = ~torch.isnan(mean_abs[..., 0])
    e = (2 * dz + 2.0 ** -weight_bits + 2.0 ** -16)[..., None]
    bound = 2 * e * mean_abs + half_step * want.abs() + 1e-30
    got = o.double()
    fine = torch.isfinite(want) & real[..., None]
    err = torch.where(fine, (got - want).abs() - bound, -1.0)
    assert (err <= 0).all(), f"{what}: {int((err > 0).sum())} of {err.numel()}, worst {float(err.max()):.3e}"
    odd = ~torch.isfinite(want) & real[..., None]
    assert torch.equal(torch.isnan(got[odd]), torch.isnan(want[odd])) and torch.equal(torch.nan_to_num(got[odd], nan=0.0), torch.nan_to_num(want[odd], nan=0.0)), what
    none = torch.isneginf(want_lse) & real
    assert (lse[none] == -math.inf).all() and (got[none] == 0).all(), what
    some = real & torch.isfinite(want_lse)
    lerr = torch.where(some, (lse.double() - want_lse).abs() - (dz + 2.0 ** -16 + 2.0 ** -23 * want_lse.abs()), -1.0)
    assert (lerr <= 0).all(), f"{what}: lse worst {float(lerr.max()):.3e}"
    return real
