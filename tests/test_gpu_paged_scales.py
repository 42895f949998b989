"""Scale bytes of 8-bit pages at both ends of their range, which single tokens, a few tokens, chunks and reads take alike."""
import pytest
import torch

from paper_2510_07651_b200 import api
from tests.paged_helpers import D, Lists, attention_64, check

pytestmark = pytest.mark.gpu

SHAPES = [(1, 8, 2), (1, 16, 1), (4, 4, 2), (4, 8, 2), (40, 4, 2), (130, 4, 2)]      # T, Hq, Hkv: up to 8 and to 16 rows per list, and more


def _q(T, Hq, seed=3):
    return torch.randn((1, Hq, T, D), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


@pytest.mark.parametrize("T,Hq,H", SHAPES)
@pytest.mark.parametrize("low", [0, 1])
def test_lists_of_the_smallest_scales(low, T, Hq, H):
    """Scale 0 is 2^-127.  All codes here are at least 16, so that every value is above fp32's smallest normal number and o is one, too; single bits of 2^-133, bf16's last,
    and sums that are cut off at 2^-126 may go."""
    n = 300
    L = Lists([n], H, 16, "e4m3", seed=5)
    codes = torch.randint(0x58, 0x7f, L.cache.v.shape, generator=torch.Generator().manual_seed(1), dtype=torch.uint8).cuda()      # 16 to 448
    L.cache.v.view(torch.uint8).copy_(codes)
    L.cache.v_scale.fill_(low)
    vd = api.obc_paged_read(L.cache, n_tokens=n, dtype=torch.float32)[1]
    at = L.cache.table[0].long()
    want = L.cache.v[at].float().double().permute(1, 0, 2, 3).reshape(1, H, -1, D)[:, :, :n] * 2.0 ** (low - 127)
    assert torch.equal(vd.double(), want)
    L.v = want
    q = _q(T, Hq)
    o, lse = api.obc_paged_attention(q, L.cache)
    assert (o.double() >= 15 * 2.0 ** (low - 127)).all()
    # weights within 2^-8 (sum p v is at most 448 * 2^(low - 127)), o's own rounding, and the steps named above
    ref = attention_64(q, L)[0]
    assert ((o.double() - ref).abs() <= 3 * 2.0 ** -8 * ref.abs() + 2.0 ** -126).all()


@pytest.mark.parametrize("T,Hq,H", SHAPES)
@pytest.mark.parametrize("up", [63, 80, 105])
def test_rows_of_large_scales(up, T, Hq, H):
    """Rows of K and V far beyond 2^60, and queries as small, so that logits are ordinary: scale bytes from 180 to 230."""
    n = 300
    g = torch.Generator().manual_seed(up)
    k, v = torch.randn((1, H, n, D), generator=g) * 2.0 ** up, torch.randn((1, H, n, D), generator=g) * 2.0 ** up
    L = Lists([n], H, 16, "e4m3", seed=6, k=k, v=v)
    assert int(L.cache.k_scale[L.cache.table[0, 0].long()].min()) > 110 + up
    q = (torch.randn((1, Hq, T, D), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") * 2.0 ** -up).bfloat16()
    o, lse = api.obc_paged_attention(q, L.cache)
    check(o, lse, q, L, weight_bits=8)
