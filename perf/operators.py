"""The paged cache as measurable cases: rows quantised as they are written into pages, read back from them, and attended to.

A KV list is held in pages of `P` tokens, in bf16, fp32 or e4m3 with one power-of-two scale per row (a byte, the biased exponent).
Lists belong to a sequence (a page then holds all KV heads) or, after an eviction with budgets of their own, to a KV head.
Every case goes through the public entry points of `paper_2510_07651_b200.api` where `own` is set, and is computed from elementary
operations otherwise.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128                                      # head_dim of every model shape the library takes


def listed():
    """The cases that stand for the operators; see the comments for what each is in real use."""
    return [
        # Decoding, 32 sequences: one new K and V row per KV head enters the 8-bit cache.  Latency counts.
        dict(name="write_token_e4m3", op="write", src="bf16", pages="e4m3", B=32, Hkv=8, T=1, N=4096, P=16, ragged=True, kept=0),
        # What follows a prompt's forward pass: four prompts of different lengths, 8-bit cache.
        dict(name="write_prompts_e4m3", op="write", src="bf16", pages="e4m3", B=4, Hkv=8, T=8191, N=8191, P=64, ragged=True, kept=0),
        # The rows that the selection kept of a 32k layer (2048 per head) move from the dense prefill cache into pages.
        dict(name="write_kept_e4m3", op="write", src="bf16", pages="e4m3", B=1, Hkv=8, T=32768, N=2048, P=32, ragged=False, kept=2048),
        # A few short bf16 lists read into an fp32 cache, for comparison with another implementation.
        dict(name="read_small_f32", op="read", dst="f32", pages="bf16", B=4, Hkv=2, N=1001, P=24, ragged=True),
        # A 32k layer held in 8 bits, read back for scoring.
        dict(name="read_e4m3_32k", op="read", dst="bf16", pages="e4m3", B=1, Hkv=8, N=32768, P=64, ragged=False),
        # Interactive decoding over a short (evicted) cache: the latency of one call.
        dict(name="attend_token_1k5", op="attend", pages="bf16", B=1, Hq=32, Hkv=8, T=1, N=1543, P=16, ragged=False, mixed=False, by_head=False),
        # Batched decoding over bf16 pages.
        dict(name="attend_token_b32", op="attend", pages="bf16", B=32, Hq=32, Hkv=8, T=1, N=8192, P=64, ragged=True, mixed=False, by_head=False),
        # Batched decoding after head-adaptive eviction, in 8 bits: every KV head has a list of its own length.
        dict(name="attend_heads_e4m3", op="attend", pages="e4m3", B=16, Hq=28, Hkv=4, T=1, N=8192, P=32, ragged=True, mixed=False, by_head=True),
        # A scheduler's batch: single tokens and chunks of a prompt together, in 8 bits.
        dict(name="attend_mixed_e4m3", op="attend", pages="e4m3", B=8, Hq=32, Hkv=8, T=256, N=16384, P=16, ragged=True, mixed=True, by_head=False),
        # A whole prompt of 4096 tokens.
        dict(name="attend_prompt_4k", op="attend", pages="bf16", B=1, Hq=32, Hkv=8, T=4096, N=4096, P=16, ragged=False, mixed=False, by_head=False),
        # The next 512 tokens of a 128k prompt.
        dict(name="attend_chunk_128k", op="attend", pages="bf16", B=1, Hq=28, Hkv=4, T=512, N=131072, P=128, ragged=False, mixed=False, by_head=False),
        # An fp32 cache, as for comparison with other implementations.
        dict(name="attend_fp32", op="attend", pages="f32", B=1, Hq=8, Hkv=2, T=16, N=2041, P=16, ragged=False, mixed=False, by_head=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


# (query heads, KV heads): no groups, the two model shapes of the benchmark, their tensor-parallel shares, eight queries per KV head
_HEADS = ((32, 32), (32, 8), (28, 4), (8, 2), (7, 1), (64, 8), (16, 8))
_PAGE = (16, 16, 24, 32, 64, 128)


def draw(rng):
    """One more case of the ranges above, sizes spread over their logarithm, odd ones among them."""
    op = rng.choice(("write", "read", "attend", "attend", "attend"))
    hq, hkv = rng.choice(_HEADS)
    page = rng.choice(_PAGE)
    batch = rng.choice((1, 1, 2, 4, 8, 32))
    rows = 1 << 18                                            # cached rows of a write or a read: the 32k layer's
    if op == "write":
        pages = rng.choice(("e4m3", "e4m3", "bf16"))
        src = rng.choice(("bf16", "bf16", "f32"))
        if rng.random() < 0.25:                               # the kept rows of a longer cache
            t = _log_int(rng, 512, rows // hkv)
            kept = max(1, t // rng.randint(4, 32))
            return dict(op=op, src=src, pages=pages, B=1, Hkv=hkv, T=t, N=kept, P=page, ragged=False, kept=kept)
        n = _log_int(rng, 64, rows // (batch * hkv))
        t = rng.choice((1, n, rng.randint(1, n)))
        return dict(op=op, src=src, pages=pages, B=batch, Hkv=hkv, T=t, N=n, P=page, ragged=batch > 1 and rng.random() < 0.5, kept=0)
    if op == "read":
        n = _log_int(rng, 64, rows // (batch * hkv))
        return dict(op=op, dst=rng.choice(("bf16", "f32")), pages=rng.choice(("e4m3", "e4m3", "bf16")), B=batch, Hkv=hkv, N=n, P=page,
                    ragged=batch > 1 and rng.random() < 0.5)
    pages = rng.choice(("bf16", "bf16", "e4m3", "e4m3", "e4m3", "f32"))
    if pages == "f32":
        hq, hkv = rng.choice(((4, 2), (8, 2), (7, 1)))
        t = _log_int(rng, 1, 32)
        return dict(op=op, pages=pages, B=1, Hq=hq, Hkv=hkv, T=t, N=max(t, _log_int(rng, 64, 8192)), P=page, ragged=False, mixed=False, by_head=False)
    few = rng.random() < 0.5
    if few:                                                   # decoding, with a few tokens at a time now and then
        t = rng.choice((1, 1, 1, 2, 4, rng.randint(2, 8)))
        n = _log_int(rng, 128, min(131072, (1 << 20) // (batch * hkv)))
    else:
        t = _log_int(rng, 8, 2048)
        batch = min(batch, max(1, 4096 // t))
        n = _log_int(rng, t, min(131072, (1 << 20) // (batch * hkv), (1 << 30) // (batch * hq * t)))
    return dict(op=op, pages=pages, B=batch, Hq=hq, Hkv=hkv, T=t, N=max(t, n), P=page, ragged=batch > 1 and rng.random() < 0.6,
                mixed=not few and batch > 1 and rng.random() < 0.5, by_head=few and rng.random() < 0.3)


_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


def _generator(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 64 + tag)
    return g


def _lengths(case, seed):
    """Lengths of the lists [B] (or [B,Hkv]): all N, or uniform between an eighth of the longest and the longest; the longest is there."""
    shape = (case["B"], case["Hkv"]) if case.get("by_head") else (case["B"],)
    if not case["ragged"]:
        return torch.full(shape, case["N"], dtype=torch.int32)
    g = torch.Generator().manual_seed(seed * 64 + 9)
    lens = torch.randint(max(case["N"] // 8, 1), case["N"] + 1, shape, generator=g, dtype=torch.int32)
    lens.view(-1)[seed % lens.numel()] = case["N"]
    return lens


def _table(lens, P, max_pages, seed):
    """Page lists: as many pages as a list needs, from a pool in random order, -1 behind them; and the pool's size, that of all lists at
    their longest."""
    need = (lens + P - 1) // P
    n_pages = need.numel() * max_pages + 1
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed * 64 + 10)).to(torch.int32)
    first = (torch.cumsum(need.view(-1), 0) - need.view(-1)).view(need.shape)
    j = torch.arange(max_pages)
    at = (first[..., None] + j).clamp(max=n_pages - 1)
    return torch.where(j < need[..., None], order[at], torch.tensor(-1, dtype=torch.int32)).contiguous().cuda(), n_pages


def _values(shape, g, lognormal):
    """Unit normal rows; values also with norms lognormal(0, 0.5)."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    return x * torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=g, device="cuda")).to(torch.bfloat16) if lognormal else x


def _exponents(x):
    """Biased exponent of every row's scale: the smallest power of two with max|x| <= 448 times it."""
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)
    s = (e - 9 + (m > 0.875) + 127).clamp(1, 254)
    return torch.where(top == 0, 1, torch.where(torch.isfinite(top), s, 255)).to(torch.uint8)


def _quantise(x):
    """Rows in 32 bits -> (e4m3 codes, scale exponents)."""
    s = _exponents(x)
    return (x * torch.exp2(127.0 - s.float())[..., None]).to(torch.float8_e4m3fn), s


def _pool(case, n_pages, seed):
    """Pages full of rows (those that no list uses hold what their last user left): k, v, k_scale, v_scale."""
    shape = (n_pages, 1 if case.get("by_head") else case["Hkv"], case["P"], D)
    k, v = _values(shape, _generator(seed, 2), False), _values(shape, _generator(seed, 3), True)
    if case["pages"] == "e4m3":
        (k, ks), (v, vs) = _quantise(k.float()), _quantise(v.float())
        return k, v, ks, vs
    return k.to(_TYPES[case["pages"]]), v.to(_TYPES[case["pages"]]), None, None


def prepare(case, seed):
    """What the caller holds before the call: the pool, the page lists and lengths, and the new rows, the queries or the outputs' buffers."""
    lens = _lengths(case, seed)
    P, N, B, H = case["P"], case["N"], case["B"], case["Hkv"]
    table, n_pages = _table(lens, P, -(-N // P), seed)
    k, v, ks, vs = _pool(case, n_pages, seed)
    st = dict(case=case, k=k, v=v, ks=ks, vs=vs, table=table, lens=lens.cuda())
    if case["op"] == "write":
        T = case["T"]
        dt = _TYPES[case["src"]]
        st["new_k"] = _values((B, H, T, D), _generator(seed, 5), False).to(dt)
        st["new_v"] = _values((B, H, T, D), _generator(seed, 6), True).to(dt)
        if case["kept"]:                                       # ascending indices, as the selection gives them
            pick = torch.rand((B, H, T), generator=_generator(seed, 7), device="cuda").topk(case["kept"], dim=-1).indices
            st["idx"], st["new_lens"] = pick.sort(-1).values.to(torch.int32), None
        else:                                                  # the last T tokens of every list (all of a shorter one)
            st["idx"], st["new_lens"] = None, st["lens"].clamp(max=T)
    elif case["op"] == "read":
        st["k_out"] = torch.zeros((B, H, N, D), dtype=_TYPES[case["dst"]], device="cuda")
        st["v_out"] = torch.zeros_like(st["k_out"])
    else:
        T, Hq = case["T"], case["Hq"]
        dt = torch.float32 if case["pages"] == "f32" else torch.bfloat16
        st["q"] = torch.randn((B, Hq, T, D), generator=_generator(seed, 1), device="cuda").to(dt)
        st["o"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros((B, Hq, T), device="cuda")
        q_lens = None
        if case["mixed"]:                                      # every other sequence decodes, the others bring a chunk
            q_lens = torch.full((B,), T, dtype=torch.int32)
            q_lens[seed % 2::2] = 1
        if case["ragged"] and T > 1:                           # no list is shorter than its new tokens
            short = lens.view(B, -1).amin(-1)
            q_lens = torch.minimum(q_lens if q_lens is not None else torch.full((B,), T, dtype=torch.int32), short)
        st["q_lens"] = q_lens.cuda() if q_lens is not None else None
    return st


# ---- the plain forms --------------------------------------------------------------------------------------------

def _rows(pages, scale, table):
    """The lists' rows in 32 bits, [B,Hkv,tokens,d]; entries of -1 read the first page (nothing sees them)."""
    at = table.clamp(min=0).long()
    eight = pages.dtype == torch.float8_e4m3fn
    x = pages.view(torch.uint8) if eight else pages
    if table.dim() == 3:                                       # a list per head
        x, s = x[:, 0][at], scale[:, 0][at] if eight else None
    else:
        x, s = x[at].transpose(1, 2), scale[at].transpose(1, 2) if eight else None
    x = x.reshape(x.shape[0], x.shape[1], -1, D)
    if not eight:
        return x.float()
    return x.contiguous().view(torch.float8_e4m3fn).float() * torch.exp2(s.reshape(x.shape[:3]).float() - 127.0)[..., None]


def _by_head(lens, H):
    return lens if lens.dim() == 2 else lens[:, None].expand(-1, H)


def _plain_attend(st):
    q, c = st["q"], st["case"]
    B, Hq, T, H = c["B"], c["Hq"], c["T"], c["Hkv"]
    k, v = _rows(st["k"], st["ks"], st["table"]), _rows(st["v"], st["vs"], st["table"])
    lens = _by_head(st["lens"], H)[:, :, None, None, None]
    n_new = (st["q_lens"] if st["q_lens"] is not None else torch.full((B,), T, dtype=torch.int32, device="cuda"))[:, None, None, None, None]
    i = torch.arange(T, device="cuda")[:, None]
    p = torch.arange(k.shape[2], device="cuda")
    s = (q.float().reshape(B, H, -1, D) @ k.transpose(2, 3)).view(B, H, Hq // H, T, -1) / math.sqrt(D)
    s = torch.where((p < lens) & (p <= lens - n_new + i) & (i < n_new), s, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    w = torch.exp(s - top)
    total = w.sum(-1, keepdim=True)
    o = (w.view(B, H, -1, k.shape[2]) @ v).view(B, H, Hq // H, T, D) / torch.where(total > 0, total, 1.0)
    real = (i < n_new).expand(B, H, Hq // H, T, 1).reshape(B, Hq, T, 1)
    lse = (top + torch.log(total)).view(B, Hq, T)
    return torch.where(real, o.reshape(B, Hq, T, D).to(q.dtype), st["o"]), torch.where(real[..., 0], lse, st["lse"])


def _plain_write(st):
    c = st["case"]
    H, P = c["Hkv"], c["P"]
    new_k, new_v = st["new_k"].float(), st["new_v"].float()
    if st["idx"] is not None:
        at = st["idx"].long()[..., None].expand(-1, -1, -1, D)
        new_k, new_v = new_k.gather(2, at), new_v.gather(2, at)
    S = new_k.shape[2]
    j = torch.arange(S, device="cuda")
    count = st["new_lens"][:, None, None] if st["new_lens"] is not None else S
    pos = (st["lens"][:, None, None] - count + j).expand(c["B"], H, S)
    page = st["table"].long().gather(1, (pos // P).clamp(0, st["table"].shape[1] - 1).reshape(c["B"], -1)).view(pos.shape)
    live = ((j < count) & (pos >= 0)).expand(pos.shape)
    b, h, r = live.nonzero(as_tuple=True)
    where = (page[b, h, r], h, (pos % P)[b, h, r].long())
    if c["pages"] != "e4m3":
        st["k"][where], st["v"][where] = new_k[b, h, r].to(st["k"].dtype), new_v[b, h, r].to(st["v"].dtype)
        return st["k"], st["v"]
    (kc, ks), (vc, vs) = _quantise(new_k[b, h, r]), _quantise(new_v[b, h, r])
    st["k"].view(torch.uint8)[where], st["v"].view(torch.uint8)[where] = kc.view(torch.uint8), vc.view(torch.uint8)
    st["ks"][where], st["vs"][where] = ks, vs
    return st["k"], st["v"], st["ks"], st["vs"]


def _plain_read(st):
    N = st["case"]["N"]
    live = (torch.arange(N, device="cuda") < st["lens"][:, None])[:, None, :, None]
    k, v = (_rows(x, s, st["table"])[:, :, :N] for x, s in ((st["k"], st["ks"]), (st["v"], st["vs"])))
    return torch.where(live, k.to(st["k_out"].dtype), st["k_out"]), torch.where(live, v.to(st["v_out"].dtype), st["v_out"])


def run(st):
    """One pass as a user's program makes it."""
    op = st["case"]["op"]
    if not own:
        return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[op](st)
    from paper_2510_07651_b200 import api

    cache = api.PagedCache(st["k"], st["v"], st["table"], st["lens"], st["ks"], st["vs"])
    if op == "write":
        api.obc_paged_write(cache, st["new_k"], st["new_v"], new_lens=st["new_lens"], idx=st["idx"])
        return (st["k"], st["v"]) if st["ks"] is None else (st["k"], st["v"], st["ks"], st["vs"])
    if op == "read":
        return api.obc_paged_read(cache, k_out=st["k_out"], v_out=st["v_out"])
    if "ws" not in st:                                         # a program that decodes keeps its workspace
        st["ws"] = torch.empty(api.obc_paged_attention_workspace(st["q"], cache), dtype=torch.uint8, device="cuda")
    return api.obc_paged_attention(st["q"], cache, q_lens=st["q_lens"], o=st["o"], lse=st["lse"], workspace=st["ws"])


def work(case):
    """Every row of the lists read or written once, with its scale; the queries and the outputs once; two contractions over the visible pairs."""
    es = {"f32": 4, "bf16": 2, "e4m3": 1}
    per_row = 2 * (D * es[case["pages"]] + (1 if case["pages"] == "e4m3" else 0))
    share = 9 / 16 if case["ragged"] else 1.0                 # mean length of a ragged batch
    lists = case["B"] * case["Hkv"]
    if case["op"] == "write":
        rows = lists * (case["kept"] or (case["T"] if case["T"] < case["N"] else case["N"] * share))
        return {"bytes": rows * (per_row + 2 * D * es[case["src"]] + (4 if case["kept"] else 0)), "flops": 0}
    if case["op"] == "read":
        return {"bytes": lists * case["N"] * share * (per_row + 2 * D * es[case["dst"]]), "flops": 0}
    n, T = case["N"] * share, case["T"]
    new = ([T] * (case["B"] - case["B"] // 2) + [1] * (case["B"] // 2)) if case["mixed"] else [T] * case["B"]
    new = [min(x, n) for x in new]
    pairs = sum(case["Hq"] * (x * n - x * (x - 1) / 2) for x in new)
    q = sum(new) * case["Hq"] * (2 * D * (4 if case["pages"] == "f32" else 2) + 4)
    return {"bytes": lists * n * per_row + q, "flops": 4 * D * pairs}


# ---- from the definitions, in 64 bits -----------------------------------------------------------------------------

def _e4m3_64(x):
    """Rows in 64 bits -> (what their e4m3 codes stand for before scaling, scale exponents): 1 + 3 bits from 2^-6 on, steps of 2^-9 below; ties to even."""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 448.0)).nan_to_num(neginf=-126.0)
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, torch.where(top <= 224.0 * torch.exp2(e), e - 1, e)).clamp(-126, 127)
    y = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, (e[..., 0] + 127).to(torch.uint8)


def _list_rows_64(st, name, b, h, n):
    """The n rows of list (b, h), one page after the other."""
    table, P = st["table"][b] if st["table"].dim() == 2 else st["table"][b, h], st["case"]["P"]
    hp = 0 if st["table"].dim() == 3 else h
    ids = table[: -(-n // P)].long()
    x = st[name].view(torch.uint8)[ids, hp].view(torch.float8_e4m3fn).double() if st[name].dtype == torch.float8_e4m3fn else st[name][ids, hp].double()
    if st[name + "s"] is not None:
        x = x * torch.pow(torch.tensor(2.0, dtype=torch.float64, device="cuda"), st[name + "s"][ids, hp].double() - 127)[..., None]
    return x.reshape(-1, D)[:n]


def exact(case, seed):
    st = prepare(case, seed)
    B, H, P = case["B"], case["Hkv"], case["P"]
    lens = _by_head(st["lens"], H).cpu()
    if case["op"] == "write":
        eight = case["pages"] == "e4m3"
        k, v = st["k"].double(), st["v"].double()
        for pages, scale, new in ((k, st["ks"], st["new_k"]), (v, st["vs"], st["new_v"])):
            for b in range(B):
                n_new = int(st["new_lens"][b]) if st["new_lens"] is not None else case["kept"]
                first = int(lens[b, 0]) - n_new
                pos = torch.arange(first, first + n_new, device="cuda")
                page = st["table"][b].long()[pos // P]
                for h in range(H):
                    rows = new[b, h][st["idx"][b, h].long() if st["idx"] is not None else slice(0, n_new)].double()
                    if eight:
                        rows, scale[page, h, pos % P] = _e4m3_64(rows)
                    pages[page, h, pos % P] = rows
        return (k, v, st["ks"], st["vs"]) if eight else (k, v)
    if case["op"] == "read":
        out = st["k_out"].double(), st["v_out"].double()
        for b in range(B):
            for h in range(H):
                n = int(lens[b, h])
                for x, name in zip(out, ("k", "v")):
                    x[b, h, :n] = _list_rows_64(st, name, b, h, n)
        return out
    o, lse = st["o"].double(), st["lse"].double()
    G, T = case["Hq"] // H, case["T"]
    for b in range(B):
        m = int(st["q_lens"][b]) if st["q_lens"] is not None else T
        for h in range(H):
            n = int(lens[b, h])
            k, v = _list_rows_64(st, "k", b, h, n), _list_rows_64(st, "v", b, h, n)
            hidden = torch.arange(n, device="cuda") > (n - m + torch.arange(m, device="cuda"))[:, None]
            for r in range(G):
                z = (st["q"][b, h * G + r, :m].double() @ k.T) / math.sqrt(D)
                z.masked_fill_(hidden, -math.inf)
                lse[b, h * G + r, :m] = torch.logsumexp(z, -1)
                o[b, h * G + r, :m] = torch.softmax(z, -1) @ v
    return o, lse
