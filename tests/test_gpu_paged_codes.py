"""Pages in 8 bits that something other than obc_paged_write filled: NaN codes (0x7f, 0xff) beside ordinary scales.  Reads and attention give them
one meaning: NaN in its channel for a NaN code, a row of NaN for scale 255, and neither reaches a query that does not see the row."""
import math

import pytest
import torch

from paper_2510_07651_b200 import api
from tests.paged_helpers import D, Lists, check

pytestmark = pytest.mark.gpu

SHAPES = [(1, 8, 2), (1, 16, 1), (4, 4, 2), (4, 8, 2), (40, 4, 2), (130, 4, 2)]      # T, Hq, Hkv: up to 8 and to 16 rows per list, and more


def _codes(L, name, h, t):
    """The codes and the scale byte's place of token t of list (0, h)."""
    page, slot = int(L.cache.table[0, t // L.P]), t % L.P
    return getattr(L.cache, name).view(torch.uint8)[page, h, slot], getattr(L.cache, name + "_scale")[page, h], slot


def _q(T, Hq, seed=3):
    return torch.randn((1, Hq, T, D), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


@pytest.mark.parametrize("code", [0x7f, 0xff])
@pytest.mark.parametrize("T,Hq,H", SHAPES)
def test_nan_codes_in_v_that_every_query_sees(code, T, Hq, H):
    n = 500
    L = Lists([n], H, 16, "e4m3", seed=1)
    for t, ch in ((3, 5), (200, 64), (n - T, 127)):
        row, _, _ = _codes(L, "v", 0, t)
        row[ch] = code
        L.v[0, 0, t, ch] = math.nan
    kd, vd = api.obc_paged_read(L.cache, n_tokens=n, dtype=torch.float32)
    assert torch.equal(torch.isnan(vd.double()), torch.isnan(L.v)) and torch.isfinite(kd).all()
    q = _q(T, Hq)
    o, lse = api.obc_paged_attention(q, L.cache)
    check(o, lse, q, L, weight_bits=8)
    odd = torch.isnan(o[0, :Hq // H])
    assert odd[..., [5, 64, 127]].all() and odd.sum() == 3 * T * (Hq // H) and torch.isfinite(lse).all() and torch.isfinite(o[0, Hq // H:]).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("what", ["code", "scale", "both"])
@pytest.mark.parametrize("T,Hq,H", [s for s in SHAPES if s[0] > 1])
def test_rows_of_v_reach_only_the_queries_that_see_them(what, T, Hq, H, causal):
    """A NaN code in one channel, or a row of NaN by its scale, in rows that some queries do not see."""
    n = 300 + T
    L = Lists([n], H, 16, "e4m3", seed=2)
    for t, ch in ((n - T // 2, 7), (n - 1, 120), (n - T + 1, 9)):
        row, scale, slot = _codes(L, "v", 0, t)
        if what != "scale":
            row[ch] = 0xff
            L.v[0, 0, t, ch] = math.nan
        if what == "scale" or (what == "both" and t == n - T // 2):
            scale[slot] = 255
            L.v[0, 0, t] = math.nan
    q = _q(T, Hq)
    o, lse = api.obc_paged_attention(q, L.cache, causal=causal)
    check(o, lse, q, L, weight_bits=8, causal=causal)
    assert torch.isfinite(lse).all()
    first = torch.isfinite(o[0, :Hq // H, 0])
    assert first.all() if causal else not first.all()


@pytest.mark.parametrize("what", ["code", "scale"])
@pytest.mark.parametrize("T,Hq,H", SHAPES)
def test_rows_of_k(what, T, Hq, H):
    """They make NaN of every query that sees them, and of no other."""
    n, t = 400, 400 - (T + 1) // 2
    L = Lists([n], H, 16, "e4m3", seed=4)
    row, scale, slot = _codes(L, "k", 0, t)
    if what == "code":
        row[77] = 0x7f
    else:
        scale[slot] = 255
    kd, _ = api.obc_paged_read(L.cache, n_tokens=n, dtype=torch.float32)
    assert torch.isnan(kd[0, 0, t, 77]) and int(torch.isnan(kd).sum()) == (1 if what == "code" else D)
    o, lse = api.obc_paged_attention(_q(T, Hq), L.cache)
    G, blind = Hq // H, T - (n - t)                   # queries before it
    assert torch.isnan(o[0, :G, blind:]).all() and torch.isnan(lse[0, :G, blind:]).all()
    assert torch.isfinite(o[0, :G, :blind]).all() and torch.isfinite(lse[0, :G, :blind]).all() and torch.isfinite(o[0, G:]).all()
