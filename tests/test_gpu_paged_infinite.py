"""Keys with infinities: a logit of +inf gives a log-sum-exp of +inf (log of a sum that holds exp(inf)) and an o of NaN (inf - inf in its weight), a logit of -inf weighs
nothing; beside a NaN logit both are NaN."""
import math

import pytest
import torch

from paper_2510_07651_b200 import api
from tests.paged_helpers import D, Lists, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages", ["f32", "bf16"])
@pytest.mark.parametrize("T,Hq,H", [(1, 8, 2), (4, 4, 2), (4, 8, 2), (40, 4, 2)])
@pytest.mark.parametrize("n,at", [(90, (2,)), (700, (5, 400, 590)), (9000, (8000, 8100))])
def test_logits_of_infinity(pages, T, Hq, H, n, at):
    """Several such tokens in a list, in one CTA's part of it or in several."""
    g = torch.Generator().manual_seed(n)
    k, v = torch.randn((1, H, n, D), generator=g), torch.randn((1, H, n, D), generator=g)
    q = torch.randn((1, Hq, T, D), generator=g)
    q[..., 9] = q[..., 9].abs() + 0.5
    for t in at:
        k[0, 0, t, 9] = math.inf
        k[0, 1:, t, 9] = -math.inf
    L = Lists([n], H, 16, pages, seed=1, k=k, v=v)
    q = q.to("cuda", torch.float32 if pages == "f32" else torch.bfloat16)
    o, lse = api.obc_paged_attention(q, L.cache)
    G = Hq // H
    assert (lse[:, :G] == math.inf).all() and torch.isnan(o[:, :G]).all()
    assert torch.isfinite(lse[:, G:]).all() and torch.isfinite(o[:, G:]).all()
    # the others' rows are those of lists without the tokens that weigh nothing
    keep = [t for t in range(n) if t not in at]
    bits = {"f32": 22, "bf16": 15 if G * T <= 16 else 8}[pages]
    check(o[:, G:], lse[:, G:], q[:, G:], Lists([len(keep)], H - 1, 16, pages, seed=1, k=k[:, 1:, keep], v=v[:, 1:, keep]), weight_bits=bits)


@pytest.mark.parametrize("pages", ["f32", "bf16"])
@pytest.mark.parametrize("T,Hq,H", [(1, 8, 1), (4, 4, 1), (40, 4, 1)])
@pytest.mark.parametrize("far", [5, 3000])
def test_beside_nan(pages, T, Hq, H, far):
    g = torch.Generator().manual_seed(far)
    n = far + 400
    k, v = torch.randn((1, H, n, D), generator=g), torch.randn((1, H, n, D), generator=g)
    q = torch.randn((1, Hq, T, D), generator=g)
    q[..., 9] = q[..., 9].abs() + 0.5
    k[0, 0, 100, 9] = math.inf
    k[0, 0, 100 + far, 3] = math.nan
    L = Lists([n], H, 16, pages, seed=1, k=k, v=v)
    o, lse = api.obc_paged_attention(q.to("cuda", torch.float32 if pages == "f32" else torch.bfloat16), L.cache)
    assert torch.isnan(o).all() and torch.isnan(lse).all()
