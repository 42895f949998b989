"""The paged-cache calls as they are used: a prompt evicted into pages and decoded from, scores from the attention over pages, captured and
replayed, on another stream, and two calls at once."""
import math

import pytest
import torch

from paper_2510_07651_b200 import api
from tests.paged_helpers import D, Lists, check

pytestmark = pytest.mark.gpu


def _rand(shape, seed, dt=torch.bfloat16):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dt)


def _pool(n_pages, heads, P, pages):
    if pages == "e4m3":
        k = torch.zeros((n_pages, heads, P, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        return k, k.clone(), torch.ones((n_pages, heads, P), dtype=torch.uint8, device="cuda"), torch.ones((n_pages, heads, P), dtype=torch.uint8, device="cuda")
    k = torch.zeros((n_pages, heads, P, D), dtype=torch.bfloat16, device="cuda")
    return k, torch.zeros_like(k), None, None


def _plain(q, k, v, lens, q_len):
    """Attention over dense caches in 64 bits: q [B,Hq,T,d], k, v [B,Hkv,N,d], lens [B,Hkv].

    What the calls may be off by: a weighted mean of v whose weights are off by a relative 2^-8 (one bf16) moves by at most 2 * 2^-8 max|v|, its own
    rounding to bf16 by 2^-8 max|v|: 3 * 2^-8 together, and less than 2 * 2^-8 with up to 16 rows per list (weights within 2^-11).  The log-sum-exp
    is off by what a logit is: 140 roundings in fp32 of sums of |q k| / sqrt(d), below 20 here: 140 * 2^-24 * 20 = 1.7e-4 at worst, if all went
    the same way; 1e-4 leaves a factor of ten over what they do."""
    B, Hq, T, _ = q.shape
    G = Hq // k.shape[1]
    o, lse = torch.zeros((B, Hq, T, D), dtype=torch.float64, device="cuda"), torch.zeros((B, Hq, T), dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(Hq):
            n = int(lens[b, h // G])
            z = q[b, h].double() @ k[b, h // G, :n].double().T / math.sqrt(D)
            z = torch.where(torch.arange(n, device="cuda") <= n - q_len + torch.arange(T, device="cuda")[:, None], z, -math.inf)
            lse[b, h] = torch.logsumexp(z, -1)
            o[b, h] = torch.softmax(z, -1) @ v[b, h // G, :n].double()
    return o, lse


def test_prompt_chunk_by_chunk_then_scored_evicted_and_decoded():
    """A prompt arrives in chunks: each is written into pages and attended to.  Its window's O and log-sum-exp give the scores of the cache read
    back, whose best tokens move into pages of 8 bits; decoding then appends to those."""
    B, Hq, H, N, P, W = 1, 8, 2, 700, 16, 32
    q, k, v = _rand((B, Hq, N, D), 1), _rand((B, H, N, D), 2), _rand((B, H, N, D), 3)
    lens = torch.zeros((B,), dtype=torch.int32, device="cuda")
    table = torch.randperm(60, generator=torch.Generator().manual_seed(4))[:48].int().view(1, 48).cuda()
    cache = api.PagedCache(*_pool(60, H, P, "bf16")[:2], table, lens)
    o, lse = torch.empty_like(q), torch.empty((B, Hq, N), device="cuda")
    at = 0
    for n in (300, 1, 256, 143):                               # chunks, a single token among them
        lens += n
        api.obc_paged_write(cache, k[:, :, at:at + n], v[:, :, at:at + n])
        oc, lc = api.obc_paged_attention(q[:, :, at:at + n], cache)
        o[:, :, at:at + n], lse[:, :, at:at + n] = oc, lc
        at += n
    kd, vd = api.obc_paged_read(cache, n_tokens=N)
    assert torch.equal(kd, k) and torch.equal(vd, v)
    want_o, want_lse = _plain(q, k, v, torch.full((B, H), N), N)
    assert (o.double() - want_o).abs().max() < 2.0 ** -8 * 3 * v.float().abs().max()      # weights and o in bf16
    assert (lse.double() - want_lse).abs().max() < 1e-4
    # the window's rows, as obc_score_given takes them: the scores of a recompute from the exact window attention
    window = slice(N - W, N)
    given = api.obc_score_given(q[:, :, window], kd, vd, o[:, :, window].contiguous(), lse[:, :, window].contiguous())
    exact = api.obc_score_given(q[:, :, window].contiguous(), k, v, want_o[:, :, window].float(), want_lse[:, :, window].float().contiguous())
    assert (given - exact).abs().max() <= 2e-2 * exact.abs().max()
    idx = api.obc_select(given[0], budget=100, n_recent=W, pool="max", pool_kernel=7)
    kept = api.PagedCache(*_pool(40, H, P, "e4m3")[:2], torch.arange(20, dtype=torch.int32, device="cuda").view(1, 20), torch.tensor([100], dtype=torch.int32, device="cuda"),
                          *_pool(40, H, P, "e4m3")[2:])
    api.obc_paged_write(kept, k, v, idx=idx)
    kk, vv = api.obc_compact(k, v, idx)
    back = api.obc_paged_read(kept, n_tokens=100)
    for x, y in zip(back, (kk, vv)):                           # 4 significant bits: off by half a step of 2^-3 at most, and by half of the smallest code
        assert ((x.double() - y.double()).abs() <= 2.0 ** -4 * y.double().abs() + 2.0 ** -10 * y.double().abs().amax(-1, keepdim=True)).all()
    for t in range(20):                                        # decoding: append a token, attend
        kept.lens.add_(1)
        kt, vt, qt = _rand((B, H, 1, D), 10 + t), _rand((B, H, 1, D), 40 + t), _rand((B, Hq, 1, D), 70 + t)
        api.obc_paged_write(kept, kt, vt)
        o1, l1 = api.obc_paged_attention(qt, kept)
        kd, vd = api.obc_paged_read(kept, n_tokens=101 + t, dtype=torch.float32)
        want_o, want_lse = _plain(qt, kd, vd, torch.full((B, H), 101 + t), 1)
        assert (o1.double() - want_o).abs().max() < 2.0 ** -8 * 2 * vd.abs().max() and (l1.double() - want_lse).abs().max() < 1e-4


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
@pytest.mark.parametrize("safeguard", [None, 0.2])
def test_evict_to_pages(pages, safeguard):
    """Score, select and move in one call: the lists hold the rows that evict_prefill and the adaptive selection keep, in their order."""
    B, Hq, H, N, W, P, budget = 2, 8, 4, 600, 16, 16, 96
    q, k, v = _rand((B, Hq, W, D), 1), _rand((B, H, N, D), 2), _rand((B, H, N, D), 3)
    by_head = safeguard is not None
    per = 38 if by_head else 6
    shape = (B, H, per) if by_head else (B, per)
    n_lists = B * H if by_head else B
    order = torch.randperm(n_lists * per, generator=torch.Generator().manual_seed(6)).int().view(shape).cuda()
    pool = _pool(n_lists * per, 1 if by_head else H, P, pages)
    cache = api.PagedCache(pool[0], pool[1], order, torch.zeros((B, H) if by_head else (B,), dtype=torch.int32, device="cuda"), pool[2], pool[3])
    idx, scores = api.evict_to_pages(q, k, v, cache, budget=budget, safeguard=safeguard, pool="max", pool_kernel=5)
    assert torch.equal(scores, api.obc_score(q, k, v))
    if by_head:
        want, counts = api.obc_select_adaptive(scores[0], budget=budget, safeguard=safeguard, idx_stride=600, n_recent=W, pool="max", pool_kernel=5)
        assert torch.equal(cache.lens, counts) and int(counts.sum()) == B * H * budget
    else:
        want = api.obc_select(scores[0], budget=budget, n_recent=W, pool="max", pool_kernel=5)
        assert (cache.lens == budget).all()
    assert torch.equal(idx, want)
    kd, vd = api.obc_paged_read(cache, n_tokens=608 if by_head else 96, dtype=torch.float32)
    for b in range(B):
        for h in range(H):
            n = int(cache.lens[b, h]) if by_head else budget
            for got, src in ((kd, k), (vd, v)):
                rows = src[b, h][want[b, h, :n].long()].double()
                tol = 0.0 if pages == "bf16" else 2.0 ** -4 * rows.abs() + 2.0 ** -10 * rows.abs().amax(-1, keepdim=True)
                assert ((got[b, h, :n].double() - rows).abs() <= tol).all() and (got[b, h, n:] == 0).all()


@pytest.mark.parametrize("lens_dims", [1, 2])
@pytest.mark.parametrize("safeguard", [None, 0.2])
def test_evict_to_pages_of_sequences_shorter_than_the_budget(safeguard, lens_dims):
    """Nothing is selected from such a sequence, so its lists are empty, whatever their pages held before; the others are as if alone."""
    if safeguard is not None and lens_dims == 1:
        pytest.skip("head-adaptive budgets have a length per head")
    B, Hq, H, N, W, P, budget = 3, 8, 4, 300, 16, 16, 96
    q, k, v = _rand((B, Hq, W, D), 1), _rand((B, H, N, D), 2), _rand((B, H, N, D), 3)
    seq_lens = torch.tensor([300, 95, 96], dtype=torch.int32, device="cuda")
    per = 19
    pool = _pool(B * H * per, 1, P, "bf16")
    pool[0].fill_(7.0); pool[1].fill_(7.0)
    table = torch.arange(B * H * per, dtype=torch.int32, device="cuda").view(B, H, per)
    lens = torch.zeros((B, H) if lens_dims == 2 else (B,), dtype=torch.int32, device="cuda")
    cache = api.PagedCache(pool[0], pool[1], table, lens)
    idx, _ = api.evict_to_pages(q, k, v, cache, budget=budget, seq_lens=seq_lens, safeguard=safeguard)
    got = cache.lens.view(B, -1)
    assert (idx[1] == -1).all() and (got[1] == 0).all()
    if safeguard is None:
        assert (got[0] == budget).all() and (got[2] == budget).all()
    else:
        assert int(got[0].sum()) == H * budget and int(got[2].sum()) == H * budget
    o, lse = api.obc_paged_attention(q[:, :, :1].contiguous(), cache)
    assert (o[1] == 0).all() and (lse[1] == -math.inf).all()
    assert torch.isfinite(lse[0]).all() and torch.isfinite(lse[2]).all()
    kd, _ = api.obc_paged_read(cache, n_tokens=per * P)
    for b in (0, 2):
        for h in range(H):
            n = int(got[b, h if lens_dims == 2 else 0])
            assert torch.equal(kd[b, h, :n], k[b, h][idx[b, h, :n].long()])


def test_evict_to_pages_refuses_what_the_lists_cannot_hold():
    q, k = _rand((1, 4, 8, D), 1), _rand((1, 2, 100, D), 2)
    cache = api.PagedCache(*_pool(4, 2, 16, "bf16")[:2], torch.arange(2, dtype=torch.int32, device="cuda").view(1, 2), torch.zeros(1, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="budget"):
        api.evict_to_pages(q, k, k, cache, budget=33)
    with pytest.raises(ValueError, match="list per head"):
        api.evict_to_pages(q, k, k, cache, budget=20, safeguard=0.2)


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
def test_captured_and_replayed(pages, T):
    """A decoding step (write, attend) as a graph: replays follow the lengths, the rows and the queries in their buffers."""
    L = Lists([300, 40], 2, 16, pages, seed=3)
    table = torch.arange(60, dtype=torch.int32, device="cuda").view(2, 30)
    pool = _pool(60, 2, 16, pages)
    cache = api.PagedCache(pool[0], pool[1], table, torch.tensor([T, T], dtype=torch.int32, device="cuda"), pool[2], pool[3])
    q, kn, vn = _rand((2, 8, T, D), 1), _rand((2, 2, T, D), 2), _rand((2, 2, T, D), 3)
    o, lse = torch.empty_like(q), torch.empty((2, 8, T), device="cuda")
    ws = torch.empty(api.obc_paged_attention_workspace(q, cache), dtype=torch.uint8, device="cuda")

    def step():
        api.obc_paged_write(cache, kn, vn)
        api.obc_paged_attention(q, cache, o=o, lse=lse, workspace=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t in range(5):
        cache.lens.add_(T)
        q.copy_(_rand(q.shape, 10 + t)); kn.copy_(_rand(kn.shape, 20 + t)); vn.copy_(_rand(vn.shape, 30 + t))
        g.replay()
        eager_o, eager_lse = api.obc_paged_attention(q, cache)
        assert torch.equal(o, eager_o) and torch.equal(lse, eager_lse)
        kd, vd = api.obc_paged_read(cache, n_tokens=T * 7, dtype=torch.float32)
        want, want_lse = _plain(q, kd, vd, cache.lens[:, None].expand(2, 2), T)
        assert (o.double() - want).abs().max() < 2.0 ** -8 * 3 * vd.abs().max() and (lse.double() - want_lse).abs().max() < 1e-4
    api.obc_score_status(ws)
    assert L is not None


def test_on_another_stream_and_two_at_once():
    """Calls on two streams, each with a workspace of its own, give what they give alone, bit for bit."""
    cases = [(Lists([900, 70], 2, 16, "bf16", seed=1), 1), (Lists([5000], 2, 64, "e4m3", seed=2), 1), (Lists([1200, 300], 2, 16, "bf16", seed=3), 200),
             (Lists([800], 2, 16, "f32", seed=4), 3)]
    alone, jobs = [], []
    for L, T in cases:
        q = _rand((L.B, 8, T, D), 5, torch.float32 if L.pages == "f32" else torch.bfloat16)
        o, lse = api.obc_paged_attention(q, L.cache)
        alone.append((o, lse))
        jobs.append((q, L.cache, torch.empty(api.obc_paged_attention_workspace(q, L.cache), dtype=torch.uint8, device="cuda"), torch.empty_like(o), torch.empty_like(lse)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for i, (q, cache, ws, o, lse) in enumerate(jobs):
            with torch.cuda.stream(streams[i % 2]):
                o.fill_(3.0)
                api.obc_paged_attention(q, cache, o=o, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    for (o, lse), (_, _, ws, o2, lse2) in zip(alone, jobs):
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_shared_prefix_pages():
    """Two lists that name the same pages for their first tokens and pages of their own behind them."""
    P, H = 16, 2
    L = Lists([64], H, P, "bf16", seed=1)
    k, v = L.cache.k, L.cache.v
    first = L.cache.table[0, :4]
    free = [i for i in range(k.shape[0]) if i not in first.tolist()]
    table = torch.stack([torch.cat([first, torch.tensor([free[0]], dtype=torch.int32, device="cuda")]), torch.cat([first, torch.tensor([free[1]], dtype=torch.int32, device="cuda")])])
    cache = api.PagedCache(k, v, table.contiguous(), torch.tensor([67, 65], dtype=torch.int32, device="cuda"))
    new = _rand((2, H, 3, D), 5)
    api.obc_paged_write(cache, new, -new, new_lens=torch.tensor([3, 1], dtype=torch.int32, device="cuda"))
    kd, vd = api.obc_paged_read(cache, n_tokens=67)
    assert torch.equal(kd[0, :, :64], kd[1, :, :64]) and torch.equal(kd[0, :, 64:67], new[0]) and torch.equal(kd[1, :, 64:65], new[1, :, :1])
    q = _rand((2, 4, 1, D), 6)
    o, lse = api.obc_paged_attention(q, cache)
    want, want_lse = _plain(q, kd, vd, torch.tensor([[67, 67], [65, 65]]), 1)
    assert (o.double() - want).abs().max() < 2.0 ** -8 * 2 * vd.float().abs().max() and (lse.double() - want_lse).abs().max() < 1e-4


def test_lse_may_be_left_out_of_the_c_call_and_outputs_are_made():
    L = Lists([70], 2, 16, "bf16", seed=2)
    q = _rand((1, 4, 1, D), 1)
    o, lse = api.obc_paged_attention(q, L.cache)
    assert o.shape == q.shape and o.dtype == q.dtype and lse.shape == (1, 4, 1)
    check(o, lse, q, L, weight_bits=15)


def test_refused_on_the_gpu():
    L = Lists([70], 2, 16, "bf16", seed=2)
    q = _rand((1, 4, 1, D), 1)
    with pytest.raises(api.ObcError) as e:
        api.obc_paged_attention(q.float(), L.cache)
    assert e.value.status == -3
    with pytest.raises(api.ObcError) as e:
        api.obc_paged_attention(q[:, :3], L.cache)
    assert e.value.status == -2
    with pytest.raises(api.ObcError) as e:
        api.obc_paged_attention(q, L.cache, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -5
    for bad in (dict(lens=L.cache.lens.long()), dict(table=L.cache.table.cpu()), dict(v=L.cache.v[:-1]), dict(k_scale=torch.zeros(1, dtype=torch.uint8, device="cuda")),
                dict(lens=torch.zeros((2,), dtype=torch.int32, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            api.obc_paged_attention(q, L.cache._replace(**bad))
    with pytest.raises(ValueError, match="o must be"):
        api.obc_paged_attention(q, L.cache, o=q[:, :2])
    with pytest.raises(ValueError, match="lse"):
        api.obc_paged_attention(q, L.cache, lse=torch.empty((1, 4, 1), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError, match="q_lens"):
        api.obc_paged_attention(q, L.cache, q_lens=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="both outputs"):
        api.obc_paged_read(L.cache, k_out=torch.empty((1, 2, 8, D), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError, match="idx"):
        api.obc_paged_write(L.cache, q[:, :2], q[:, :2], idx=torch.zeros((1, 2, 4), dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="new_lens"):
        api.obc_paged_write(L.cache, q[:, :2], q[:, :2], new_lens=torch.zeros(3, dtype=torch.int32, device="cuda"))


def test_extents_beyond_32_bits_are_refused():
    L = Lists([70], 2, 16, "bf16", seed=2)
    long = _rand((1, 2, 1, D), 1).expand(-1, -1, (1 << 32) + 1, -1)
    with pytest.raises(ValueError, match="32 bits"):
        api.obc_paged_attention(long, L.cache)
    with pytest.raises(ValueError, match="32 bits"):
        api.obc_paged_write(L.cache, long, long)
    with pytest.raises(ValueError, match="32 bits"):
        api.obc_paged_read(L.cache, k_out=long, v_out=long)
