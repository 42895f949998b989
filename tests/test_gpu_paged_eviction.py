"""What evict_to_pages leaves behind when it is refused, and replays of a captured step over lists of changing lengths."""
import pytest
import torch

from paper_2510_07651_b200 import api
from tests.paged_helpers import D, Lists, check

pytestmark = pytest.mark.gpu


def _rand(shape, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def _cache(B, H, pages, P, by_head, seed_lens=7):
    per = 12
    lists = (B, H) if by_head else (B,)
    n = per * B * (H if by_head else 1)
    k = torch.zeros((n, 1 if by_head else H, P, D), dtype=torch.uint8 if pages == "e4m3" else torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    s = (None, None)
    if pages == "e4m3":
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
        s = tuple(torch.ones(k.shape[:3], dtype=torch.uint8, device="cuda") for _ in range(2))
    table = torch.arange(n, dtype=torch.int32, device="cuda").view(*lists, per)
    return api.PagedCache(k, v, table, torch.full(lists, seed_lens, dtype=torch.int32, device="cuda"), *s)


@pytest.mark.parametrize("safeguard", [None, 0.2])
def test_a_refused_eviction_leaves_the_lengths_as_they_were(safeguard):
    B, Hq, H, N, W, budget = 2, 8, 4, 300, 16, 40
    q, k, v = _rand((B, Hq, W, D), 1), _rand((B, H, N, D), 2), _rand((B, H, N, D), 3)
    by_head = safeguard is not None
    for pages, bad in (("bf16", dict(P=12)), ("e4m3", dict(k_scale=None)), ("e4m3", dict(v_scale=torch.ones(3, dtype=torch.uint8, device="cuda"))), ("bf16", dict(k="shifted")),
                       ("bf16", dict(v="float")), ("bf16", dict(lens="batch")), ("bf16", dict(lens="long"))):
        cache = _cache(B, H, pages, bad.pop("P", 16), by_head)
        if bad.get("k") == "shifted":
            wide = torch.zeros(cache.k.shape[:3] + (D + 8,), dtype=cache.k.dtype, device="cuda")
            bad["k"] = wide[..., 4:4 + D]
        if bad.get("v") == "float":
            bad["v"] = cache.v.float()
        if bad.get("lens") == "batch":
            bad["lens"] = torch.full((B + 1, H) if by_head else (B + 1,), 7, dtype=torch.int32, device="cuda")
        if bad.get("lens") == "long":
            bad["lens"] = cache.lens.long()
        cache = cache._replace(**bad)
        with pytest.raises((ValueError, TypeError, api.ObcError)):
            api.evict_to_pages(q, k, v, cache, budget=budget, safeguard=safeguard)
        assert (cache.lens == 7).all(), bad


def test_lengths_that_share_memory_are_refused():
    B, Hq, H, N, W = 2, 8, 4, 300, 16
    q, k, v = _rand((B, Hq, W, D), 1), _rand((B, H, N, D), 2), _rand((B, H, N, D), 3)
    cache = _cache(B, H, "bf16", 16, False)
    cache = cache._replace(lens=torch.full((1,), 7, dtype=torch.int32, device="cuda").expand(B))
    with pytest.raises((ValueError, RuntimeError)):
        api.evict_to_pages(q, k, v, cache, budget=40)
    assert (cache.lens == 7).all() and (cache.k == 0).all()


@pytest.mark.parametrize("safeguard", [None, 0.2])
def test_a_captured_eviction(safeguard):
    """Replayed over other rows it leaves what an eager call leaves."""
    B, Hq, H, N, W, budget = 2, 8, 4, 160, 16, 40
    q, k, v = _rand((B, Hq, W, D), 1), _rand((B, H, N, D), 2), _rand((B, H, N, D), 3)
    caches = [_cache(B, H, "e4m3", 16, safeguard is not None) for _ in range(2)]
    api.evict_to_pages(q, k, v, caches[0], budget=budget, safeguard=safeguard)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        idx, scores = api.evict_to_pages(q, k, v, caches[0], budget=budget, safeguard=safeguard)
    q.copy_(_rand(q.shape, 4)); k.copy_(_rand(k.shape, 5)); v.copy_(_rand(v.shape, 6))
    g.replay()
    want_idx, want_scores = api.evict_to_pages(q, k, v, caches[1], budget=budget, safeguard=safeguard)
    assert torch.equal(idx, want_idx) and torch.equal(scores, want_scores) and torch.equal(caches[0].lens, caches[1].lens)
    for x, y in zip(api.obc_paged_read(caches[0]), api.obc_paged_read(caches[1])):
        assert torch.equal(x, y)


@pytest.mark.parametrize("T", [1, 24])
@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
def test_replays_over_lists_of_changing_lengths(pages, T):
    """A captured step whose lists (one of a few tokens, one that many CTAs share) grow and shrink between replays, so that the work is cut another way and
    other parts are merged every time."""
    L = Lists([9000, 40], 2, 16, pages, seed=3)
    q, kn, vn = _rand((2, 8, T, D), 1), _rand((2, 2, T, D), 2), _rand((2, 2, T, D), 3)
    o, lse = torch.empty_like(q), torch.empty((2, 8, T), device="cuda")
    ws = torch.empty(api.obc_paged_attention_workspace(q, L.cache), dtype=torch.uint8, device="cuda")
    # a pool without the fill of free places, and a full table for both lists
    table = torch.randperm(L.cache.k.shape[0] * 2, generator=torch.Generator().manual_seed(1)).int()[:1126].view(2, 563).cuda()
    pool = [torch.zeros((L.cache.k.shape[0] * 2,) + x.shape[1:], dtype=torch.uint8, device="cuda") if x.dtype != torch.bfloat16
            else torch.zeros((L.cache.k.shape[0] * 2,) + x.shape[1:], dtype=x.dtype, device="cuda") for x in (L.cache.k, L.cache.v)]
    scales = [torch.ones(pool[0].shape[:3], dtype=torch.uint8, device="cuda") if pages == "e4m3" else None for _ in range(2)]
    if pages == "e4m3":
        pool = [x.view(torch.float8_e4m3fn) for x in pool]
    cache = api.PagedCache(pool[0], pool[1], table, torch.tensor([9000, 9000], dtype=torch.int32, device="cuda"), scales[0], scales[1])
    api.obc_paged_write(cache, *(_rand((2, 2, 9000, D), s) for s in (5, 6)))

    def step():
        api.obc_paged_write(cache, kn, vn)
        api.obc_paged_attention(q, cache, o=o, lse=lse, workspace=ws)

    cache.lens.copy_(torch.tensor([9000, 40], dtype=torch.int32))
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t, lens in enumerate(([9000, 40], [40, 8999], [T, 700], [5000, 5001], [0, 9000])):
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(_rand(q.shape, 10 + t)); kn.copy_(_rand(kn.shape, 20 + t)); vn.copy_(_rand(vn.shape, 30 + t))
        g.replay()
        eager_o, eager_lse = api.obc_paged_attention(q, cache)
        assert torch.equal(o, eager_o) and torch.equal(lse, eager_lse)
        M = Lists(lens, 2, 16, pages, seed=1)
        kd, vd = api.obc_paged_read(cache, n_tokens=9000, dtype=torch.float32)
        M.k, M.v = kd.double(), vd.double()
        check(o, lse, q, M, weight_bits=8 if 4 * T > 16 else 15 if pages == "bf16" else 10.9)
    api.obc_score_status(ws)
