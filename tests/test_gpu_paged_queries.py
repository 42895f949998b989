"""Queries at the ends of their range."""
import math

import pytest
import torch

from paper_2510_07651_b200 import api
from tests.paged_helpers import D, TYPES, Lists, check

pytestmark = pytest.mark.gpu

SHAPES = [(1, 8, 2), (1, 16, 1), (4, 4, 2), (4, 8, 2), (40, 4, 2)]      # T, Hq, Hkv: up to 8 and to 16 rows per list, and more


@pytest.mark.parametrize("pages", list(TYPES))
@pytest.mark.parametrize("T,Hq,H", SHAPES)
@pytest.mark.parametrize("down", [100, 112, 113, 116, 118])
def test_tiny_queries_of_large_keys(pages, T, Hq, H, down):
    """Logits are ordinary."""
    n = 300
    g = torch.Generator().manual_seed(down)
    k, v = torch.randn((1, H, n, D), generator=g) * 2.0 ** down, torch.randn((1, H, n, D), generator=g)
    L = Lists([n], H, 16, pages, seed=6, k=k, v=v)
    q = (torch.randn((1, Hq, T, D), generator=g) * 2.0 ** -down).to("cuda", torch.float32 if pages == "f32" else torch.bfloat16)
    o, lse = api.obc_paged_attention(q, L.cache)
    check(o, lse, q, L, weight_bits=8)


@pytest.mark.parametrize("pages", list(TYPES))
@pytest.mark.parametrize("T,Hq,H", [s for s in SHAPES if s[2] == 2])
@pytest.mark.parametrize("large", [1.0, 1e6, 1e30])
def test_infinities_in_queries(pages, T, Hq, H, large):
    """Beside large values: a list whose keys have one sign in their channel gives logits of +inf alone (lse +inf, o NaN), of the other -inf alone (they weigh nothing)."""
    n = 300
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn((1, H, n, D), generator=g), torch.randn((1, H, n, D), generator=g)
    k[..., 9] = k[..., 9].abs() + 0.5
    k[:, 1, :, 9] *= -1
    q = torch.randn((1, Hq, T, D), generator=g)
    q[..., 20:40] *= large
    q[..., 9] = math.inf
    L = Lists([n], H, 16, pages, seed=1, k=k, v=v)
    o, lse = api.obc_paged_attention(q.to("cuda", torch.float32 if pages == "f32" else torch.bfloat16), L.cache)
    G = Hq // H
    assert (lse[:, :G] == math.inf).all() and torch.isnan(o[:, :G]).all()
    assert (lse[:, G:] == -math.inf).all() and (o[:, G:] == 0).all()
