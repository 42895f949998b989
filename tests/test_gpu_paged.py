"""Paged caches on the GPU (obc_paged_write, obc_paged_read, obc_paged_attention) against plain forms in 64 bits: rows and scales bit for
bit, attention within what its arithmetic allows (tests/paged_helpers.py)."""
import math

import pytest
import torch

from paper_2510_07651_b200 import api
from tests.paged_helpers import D, TYPES, Lists, check, e4m3_64, pow2

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ---- writing and reading ------------------------------------------------------------------------------------

def _values(cache, table_row, head, t, name):
    page = table_row[t // cache.k.shape[2]].long()
    x = getattr(cache, name)
    slot = t % cache.k.shape[2]
    if x.dtype == torch.float8_e4m3fn:
        codes = x.view(torch.uint8)[page, head, slot].view(torch.float8_e4m3fn).double()
        s = getattr(cache, name + "_scale")[page, head, slot].double()
        return torch.where((s == 255)[:, None], math.nan, codes * pow2(s.long() - 127)[:, None]), s
    return x[page, head, slot].double(), None


@pytest.mark.parametrize("pages", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("P,H,lens,news", [
    (16, 2, [40, 1, 17], [40, 1, 16]), (8, 1, [9], [1]), (24, 3, [50, 25], [7, 25]), (64, 4, [129, 64, 0], [128, 0, 0]),
    (16, 2, [5, 30], [9, 12]),                       # more rows than the list is long: the first ones are dropped
])
def test_write_and_read_back(pages, src, P, H, lens, news):
    L = Lists(lens, H, P, pages, seed=P)
    B, T = len(lens), max(max(news), 1)
    g = _gen(5)
    k, v = (torch.randn((B, H, T, D), generator=g, device="cuda").mul(3.0).to(TYPES[src]) for _ in range(2))
    before = [x.view(torch.uint8).clone() if x is not None else None for x in (L.cache.k, L.cache.v, L.cache.k_scale, L.cache.v_scale)]
    api.obc_paged_write(L.cache, k, v, new_lens=torch.tensor(news, dtype=torch.int32, device="cuda"))
    k_out, v_out = (torch.full((B, H, L.N + 2, D), 7.0, dtype=torch.float32, device="cuda") for _ in range(2))
    api.obc_paged_read(L.cache, k_out=k_out, v_out=v_out)
    written = torch.zeros(L.cache.k.shape[:3], dtype=torch.bool, device="cuda")
    for b in range(B):
        for h in range(H):
            n, m = lens[b], min(news[b], T)
            for name, new, old, out in (("k", k, L.k, k_out), ("v", v, L.v, v_out)):
                t = torch.arange(n, device="cuda")
                got, s = _values(L.cache, L.cache.table[b], h, t, name)
                want = old[b, h, :n].clone()
                first = n - m
                j0 = max(-first, 0)
                rows = new[b, h, j0:m].double()
                if pages == "e4m3":
                    codes, es = e4m3_64(rows)
                    assert torch.equal(s[first + j0:], es.double())
                    rows = codes * pow2(es.long() - 127)[:, None]
                else:
                    rows = rows.to(TYPES[pages]).double()
                want[first + j0:] = rows
                assert torch.equal(got, want), (b, h, name)
                assert torch.equal(out[b, h, :n].double(), want.float().double()) and (out[b, h, n:] == 7.0).all()
            t = torch.arange(max(n - m, 0), n, device="cuda")
            written[L.cache.table[b][t // P].long(), h, t % P] = True
    for x, y in zip((L.cache.k, L.cache.v, L.cache.k_scale, L.cache.v_scale), before):
        if x is not None:                              # nothing but the new rows was touched
            assert torch.equal(x.view(torch.uint8)[~written], y[~written])


@pytest.mark.parametrize("by_head", [False, True])
@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
def test_write_of_kept_rows_by_index(pages, by_head):
    lens = [[30, 17], [1, 0]] if by_head else [30, 30]
    L = Lists(lens, 2, 16, pages, by_head=by_head, seed=3)
    k, v = (torch.randn((2, 2, 100, D), generator=_gen(4), device="cuda").bfloat16() for _ in range(2))
    idx = torch.stack([torch.randperm(100, generator=torch.Generator().manual_seed(i))[:30].sort().values for i in range(4)]).view(2, 2, 30).int().cuda()
    idx[0, 0, 4] = -1; idx[0, 1, 3] = 100             # padding and an index that is not there: their places stay as they are
    api.obc_paged_write(L.cache, k, v, new_lens=L.cache.lens, idx=idx)
    out = api.obc_paged_read(L.cache, n_tokens=40, dtype=torch.float32)
    for b in range(2):
        for h in range(2):
            n = int(L.lens_bh[b, h])
            for new, old, got in ((k, L.k, out[0]), (v, L.v, out[1])):
                rows = new[b, h][idx[b, h, :n].clamp(0, 99).long()].double()
                if pages == "e4m3":
                    codes, es = e4m3_64(rows)
                    rows = codes * pow2(es.long() - 127)[:, None]
                live = (idx[b, h, :n] >= 0) & (idx[b, h, :n] < 100)
                assert torch.equal(got[b, h, :n].double(), torch.where(live[:, None], rows, old[b, h, :n]))
                assert (got[b, h, n:] == 0).all()     # outputs made by the call are zero behind the list


def test_rounding_into_8_bits():
    """Every scale, ties, the border between two scales, zeros, subnormal rows, infinities and NaN."""
    rows = torch.zeros((1, 1, 320, D), dtype=torch.float32)
    for e in range(-130, 120):
        rows[0, 0, e + 130, :64] = torch.linspace(-448, 448, 64) * 2.0 ** e
        rows[0, 0, e + 130, 64:] = torch.arange(64) * 2.0 ** (e - 10)             # subnormal codes and their ties
    rows[0, 0, 250, :] = torch.linspace(17, 19, D)                                # ties of 1/8 steps at 16..32
    rows[0, 0, 251, 0] = 448.0; rows[0, 0, 252, 0] = 448.0000305; rows[0, 0, 253, 0] = 224.0; rows[0, 0, 254, 0] = 3.4e38
    rows[0, 0, 255, 0] = 1e-45; rows[0, 0, 257, 3] = math.inf; rows[0, 0, 258, 9] = -math.inf; rows[0, 0, 259, 127] = math.nan
    rows[0, 0, 260:] = torch.randn((60, D), generator=torch.Generator().manual_seed(1))
    L = Lists([320], 1, 16, "e4m3", seed=1)
    api.obc_paged_write(L.cache, rows.cuda(), -rows.cuda())
    codes, es = e4m3_64(rows[0, 0].cuda())
    t = torch.arange(320, device="cuda")
    for name, sign in (("k", 1), ("v", -1)):
        got, s = _values(L.cache, L.cache.table[0], 0, t, name)
        assert torch.equal(s, es.double())
        want = torch.where((es == 255)[:, None], math.nan, sign * codes * pow2(es.long() - 127)[:, None])
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
        out = api.obc_paged_read(L.cache, n_tokens=320, dtype=torch.float32)[0 if name == "k" else 1][0, 0].double()
        assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(torch.nan_to_num(out), torch.nan_to_num(want.float().double()))


@pytest.mark.parametrize("pages", ["f32", "bf16", "e4m3"])
def test_pages_that_are_not_there(pages):
    """Page numbers outside the pool: read as zeros, never written; the rest of the list is not affected."""
    L = Lists([50], 2, 16, pages, seed=2)
    L.cache.table[0, 1] = L.cache.k.shape[0]
    L.cache.table[0, 2] = -5
    for x in (L.k, L.v):
        x[:, :, 16:48] = 0
    before = L.cache.k.view(torch.uint8).clone()
    k_out, v_out = api.obc_paged_read(L.cache, n_tokens=50, dtype=torch.float32)
    assert torch.equal(k_out.double(), L.k.float().double()) and torch.equal(v_out.double(), L.v.float().double())
    new = torch.randn((1, 2, 30, D), generator=_gen(1), device="cuda")
    api.obc_paged_write(L.cache, new[:, :, :28], new[:, :, :28], new_lens=torch.tensor([28], dtype=torch.int32, device="cuda"))
    page = int(L.cache.table[0, 3])
    keep = [i for i in range(L.cache.k.shape[0]) if i != page]
    assert torch.equal(L.cache.k.view(torch.uint8)[keep], before[keep])
    assert not torch.equal(L.cache.k.view(torch.uint8)[page], before[page])


# ---- attention -------------------------------------------------------------------------------------------------

def _attend(L, Hq, T, *, q_lens=None, causal=True, scale=0.0, seed=9, weight_bits=16, strided_q=False, what=""):
    dt = torch.float32 if L.pages == "f32" else torch.bfloat16
    q = torch.randn((L.B, Hq, T, D), generator=_gen(seed), device="cuda").to(dt)
    if strided_q:
        wide = torch.full((L.B, T, Hq + 1, D + 8), math.nan, dtype=dt, device="cuda")
        wide[:, :, :Hq, :D] = q.transpose(1, 2)
        q = wide[:, :, :Hq, :D].transpose(1, 2)
    o = torch.full((L.B, Hq, T, D), 5.0, dtype=dt, device="cuda")
    lse = torch.full((L.B, Hq, T), 5.0, device="cuda")
    ql = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32, device="cuda")
    ws = torch.full((api.obc_paged_attention_workspace(q, L.cache),), 255, dtype=torch.uint8, device="cuda")
    api.obc_paged_attention(q, L.cache, q_lens=ql, causal=causal, scale=scale, o=o, lse=lse, workspace=ws)
    api.obc_score_status(ws)
    real = check(o, lse, q, L, weight_bits=weight_bits, q_lens=q_lens, scale=scale or None, causal=causal, what=what)
    assert (o[~real] == 5.0).all() and (lse[~real] == 5.0).all()      # rows behind q_lens stay as they were
    return q, o, lse


# weights of up to 16 rows per list: fp32; two bf16 parts; fp16 (half a step of 2^-10, and 2^-25 of the largest where it is subnormal)
BITS = {"f32": 22, "bf16": 15, "e4m3": 10.9}
CHUNK_BITS = {"f32": 22, "bf16": 8, "e4m3": 8}       # of more rows: one bf16, off by half a step of 2^-7 at most


@pytest.mark.parametrize("pages", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("lens,Hq,H,P", [
    ([1], 1, 1, 16), ([2, 1], 4, 2, 8), ([127], 8, 1, 16), ([128], 4, 4, 32), ([129], 7, 1, 24), ([255, 300], 8, 2, 40),
    ([0, 5, 1000], 32, 8, 16), ([1543], 28, 4, 128), ([640, 17, 2049], 16, 1, 256), ([5000], 8, 8, 48),
])
def test_single_tokens(pages, lens, Hq, H, P):
    _attend(Lists(lens, H, P, pages, seed=len(lens)), Hq, 1, weight_bits=BITS[pages])


@pytest.mark.parametrize("pages", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("T,Hq,H", [(2, 4, 1), (3, 7, 1), (4, 8, 2), (5, 8, 4), (16, 1, 1), (9, 6, 2), (32, 1, 1), (4, 8, 1)])
@pytest.mark.parametrize("lens", [[33], [129, 64], [700]])
def test_few_rows(pages, T, Hq, H, lens):
    _attend(Lists(lens, H, 16, pages, seed=T), Hq, T, weight_bits=(BITS if Hq // H * T <= 16 else CHUNK_BITS)[pages])


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq", [8, 16])
def test_many_tiles_per_cta(pages, Hq):
    """Rings that go round many times, lists that end inside a run and lists that many CTAs share."""
    _attend(Lists([40000, 3, 9000, 130], 4, 64, pages, seed=1), Hq, 2, weight_bits=BITS[pages])
    _attend(Lists([1500] * 40, 8, 16, pages, seed=2), Hq, 1, weight_bits=BITS[pages])


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
@pytest.mark.parametrize("spread", [2, 12])
def test_rows_of_different_magnitude(pages, spread):
    _attend(Lists([400, 77], 2, 16, pages, seed=1, spread=spread), 8, 1, weight_bits=BITS[pages])


@pytest.mark.parametrize("pages", ["f32", "bf16", "e4m3"])
def test_lists_of_their_own_length_per_head(pages):
    lens = torch.randint(0, 900, (5, 4), generator=torch.Generator().manual_seed(8)).int()
    lens[0, 0], lens[1, 2] = 0, 1
    _attend(Lists(lens, 4, 32, pages, by_head=True, seed=4), 28, 1, weight_bits=BITS[pages])
    _attend(Lists(lens, 4, 32, pages, by_head=False, seed=4), 8, 3, weight_bits=BITS[pages])


@pytest.mark.parametrize("pages", ["f32", "bf16", "e4m3"])
def test_queries_without_tokens_and_padded_batches(pages):
    L = Lists([3, 0, 40, 200], 2, 8, pages, seed=6)
    _attend(L, 8, 4, q_lens=[4, 4, 0, 2], weight_bits=BITS[pages])     # more queries than tokens; an empty list; no queries
    _attend(L, 8, 4, q_lens=[9, -1, 1, 4], causal=False, scale=0.3, weight_bits=BITS[pages])


@pytest.mark.parametrize("pages", ["f32", "bf16", "e4m3"])
def test_strides(pages):
    _attend(Lists([150, 33], 2, 16, pages, seed=7, strided=True), 8, 2, strided_q=True, weight_bits=BITS[pages])
    _attend(Lists([[150, 20], [33, 64]], 2, 16, pages, by_head=True, seed=7, strided=True), 8, 2, weight_bits=BITS[pages])


@pytest.mark.parametrize("pages", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_infinities_and_nan_reach_only_the_queries_that_see_them(pages, what):
    g = torch.Generator().manual_seed(11)
    k, v = torch.randn((1, 2, 140, D), generator=g), torch.randn((1, 2, 140, D), generator=g)
    v[0, 0, 138, 5] = what                            # seen by the last two of four queries
    v[0, 1, 139, 77] = -what
    k[0, 1, 137] = math.nan                           # seen by the last three
    L = Lists([140], 2, 16, pages, seed=1, k=k, v=v)
    q = torch.randn((1, 4, 4, D), generator=_gen(3), device="cuda").to(torch.float32 if pages == "f32" else torch.bfloat16)
    o, lse = api.obc_paged_attention(q, L.cache)
    clean = Lists([140], 2, 16, pages, seed=1, k=torch.nan_to_num(k), v=torch.where(torch.isfinite(v), v, 0.0))
    oc, lc = api.obc_paged_attention(q, clean.cache)
    assert torch.equal(o[:, :2, :2], oc[:, :2, :2]) and torch.equal(o[:, 2:, 0], oc[:, 2:, 0]) and torch.equal(lse[:, 2:, 0], lc[:, 2:, 0])
    assert not torch.isfinite(o[:, :2, 2:, 5]).any()
    assert torch.isnan(o[:, 2:, 1:]).all() and torch.isnan(lse[:, 2:, 1:]).all()
    if pages != "e4m3":                               # (a row of 8 bits with one of them is NaN altogether)
        assert torch.isfinite(o[:, :2, :, :5]).all() and torch.isfinite(o[:, :2, :, 6:]).all()
    assert torch.isfinite(lse[:, :2]).all()


@pytest.mark.parametrize("pages", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("T,Hq,H", [(1, 8, 2), (2, 4, 1), (4, 8, 2), (40, 4, 2)])
def test_infinities_that_every_query_sees(pages, what, T, Hq, H):
    """They reach every output of their channel as the formula has it (an infinity stays one, whatever its weight's parts), and no other."""
    n = 700
    g = torch.Generator().manual_seed(12)
    k, v = torch.randn((1, H, n, D), generator=g), torch.randn((1, H, n, D), generator=g)
    for t, ch in ((0, 3), (131, 64), (350, 127), (513, 5)):
        v[0, :, t, ch] = what
    k[0, :, 350] *= 4                                 # (among its list's largest weights, and smallest)
    _attend(Lists([n], H, 16, pages, seed=2, k=k, v=v), Hq, T, weight_bits=(BITS if Hq // H * T <= 16 else CHUNK_BITS)[pages])


def test_long_list_behind_32_bits():
    """A pool of more than 2^32 elements; the list's pages lie at both of its ends."""
    P, H = 128, 2
    n_pages = (1 << 32) // (P * H * D) + 64
    k = torch.zeros((n_pages, H, P, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    L = Lists([1000], H, P, "bf16", seed=5)
    table = torch.tensor([[0, n_pages - 1, 1, n_pages - 2, n_pages - 3, 2, n_pages - 4, 3]], dtype=torch.int32, device="cuda")
    for i in range(8):
        k[table[0, i]] = L.cache.k[L.cache.table[0, i].long()]
        v[table[0, i]] = L.cache.v[L.cache.table[0, i].long()]
    L.cache = api.PagedCache(k, v, table, L.cache.lens)
    _attend(L, 8, 1, weight_bits=15)
    new = torch.randn((1, H, 300, D), generator=_gen(2), device="cuda").bfloat16()
    api.obc_paged_write(L.cache, new, new)
    ko, vo = api.obc_paged_read(L.cache, n_tokens=1000)
    assert torch.equal(ko[:, :, 700:], new) and torch.equal(vo[:, :, 700:], new)
    assert torch.equal(ko[:, :, :700].double(), L.k[:, :, :700])


# ---- chunks: more than 16 rows per list --------------------------------------------------------------------------

@pytest.mark.parametrize("pages", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("T,Hq,H,lens,P", [
    (33, 1, 1, [33], 16), (40, 4, 2, [100, 40], 8), (128, 1, 1, [128], 16), (129, 1, 1, [200], 24), (64, 8, 2, [700, 64, 129], 32), (37, 7, 1, [1000], 128),
    (256, 2, 2, [256], 16), (257, 1, 1, [1025], 40), (300, 4, 1, [300, 513], 64), (700, 2, 1, [701], 16), (5, 8, 1, [2000, 6], 16), (90, 28, 4, [90], 256),
])
@pytest.mark.parametrize("causal", [True, False])
def test_chunks(pages, T, Hq, H, lens, P, causal):
    _attend(Lists(lens, H, P, pages, seed=T), Hq, T, causal=causal, weight_bits=CHUNK_BITS[pages])


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
def test_long_chunks(pages):
    """Items that many CTAs share, items that one CTA finishes, and both in one run."""
    _attend(Lists([9000, 300], 2, 16, pages, seed=1), 8, 200, weight_bits=8)
    _attend(Lists([2500], 8, 64, pages, seed=2), 16, 900, weight_bits=8)
    _attend(Lists([700] * 20, 8, 16, pages, seed=3), 8, 100, weight_bits=8)


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
def test_chunks_of_a_padded_batch(pages):
    L = Lists([900, 1, 0, 260, 64, 500], 2, 16, pages, seed=6)
    _attend(L, 8, 260, q_lens=[260, 1, 0, 260, 100, 1], weight_bits=8)         # single tokens beside chunks; more queries than tokens
    _attend(L, 8, 260, q_lens=[1, 260, 260, 0, -3, 999], causal=False, scale=0.2, weight_bits=8)
    _attend(Lists([[150, 20], [33, 640]], 2, 16, pages, by_head=True, seed=7, strided=True), 8, 50, q_lens=[50, 33], strided_q=True, weight_bits=8)


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
@pytest.mark.parametrize("P", [16, 64])
def test_many_short_lists_in_chunks(pages, P):
    """More row tiles than CTAs, of one to four token tiles each, some without rows of the second warpgroup or any: every CTA goes through several lists."""
    g = torch.Generator().manual_seed(P)
    lens = torch.randint(1, 500, (24,), generator=g).tolist()
    q_lens = torch.randint(0, 81, (24,), generator=g).tolist()
    _attend(Lists(lens, 8, P, pages, seed=5), 32, 80, q_lens=q_lens, weight_bits=CHUNK_BITS[pages])


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq", [2, 8, 14, 32])
def test_single_tokens_beside_chunks(pages, Hq):
    """Lists of few rows, of the most that the kernel for few takes (and one more), and of many in one call, long and short ones of each."""
    q_lens = [1, 8, 100, 1, 9, 0, 2, 300, 1, 4]
    L = Lists([9000, 700, 800, 1, 64, 50, 3000, 300, 17, 4], 2, 16, pages, seed=Hq)
    _attend(L, Hq, 300, q_lens=q_lens, weight_bits=8)
    _attend(L, Hq, 300, q_lens=[1] * 10, weight_bits=8)
    _attend(L, Hq, 300, q_lens=[0] * 10, weight_bits=8)


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
@pytest.mark.parametrize("spread", [2, 12])
def test_chunks_of_different_magnitude(pages, spread):
    _attend(Lists([700, 77], 2, 16, pages, seed=1, spread=spread), 8, 60, weight_bits=8)


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
@pytest.mark.parametrize("what", [math.nan, math.inf])
@pytest.mark.parametrize("n,T", [(300, 100), (140, 140), (1100, 300)])
def test_infinities_and_nan_in_chunks(pages, what, n, T):
    """Rows of V that are not finite, at places that all, some and the last queries see, in tiles of one and of two warpgroups."""
    g = torch.Generator().manual_seed(n)
    k, v = torch.randn((1, 2, n, D), generator=g), torch.randn((1, 2, n, D), generator=g)
    first = n - T
    for t, ch in ((first + T // 2, 5), (first + T // 2 + 1, 6), (n - 1, 7), (first + 1, 8)):
        v[0, 0, t, ch] = what
    L = Lists([n], 2, 16, pages, seed=1, k=k, v=v)
    _attend(L, 4, T, weight_bits=8)
    k[0, 1, first + T // 3] = math.nan
    L = Lists([n], 2, 16, pages, seed=1, k=k, v=v)
    q = torch.randn((1, 4, T, D), generator=_gen(3), device="cuda").bfloat16()
    o, lse = api.obc_paged_attention(q, L.cache)
    assert torch.isfinite(o[:, 2:, :T // 3]).all() and torch.isnan(o[:, 2:, T // 3:]).all() and torch.isnan(lse[:, 2:, T // 3:]).all()
