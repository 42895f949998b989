"""Chunks over bf16 pages whose last row tile has rows for one warpgroup only, or whose warpgroups see different numbers of token tiles: the ring of operands
then holds some that an issuer releases without using them.  Large pages make the producers fast (few copies per operand)."""
import pytest
import torch

from paper_2510_07651_b200 import api
from tests.paged_helpers import D, Lists, check

pytestmark = pytest.mark.gpu


def _repeated(L, Hq, T, *, q_lens=None, causal=True, times=6):
    """Against 64 bits (weights are one bf16), and the same bits whenever the call is made again."""
    q = torch.randn((L.B, Hq, T, D), generator=torch.Generator(device="cuda").manual_seed(T), device="cuda").bfloat16()
    ql = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32, device="cuda")
    ws = torch.empty(api.obc_paged_attention_workspace(q, L.cache), dtype=torch.uint8, device="cuda")
    first = None
    for _ in range(times):
        o, lse = torch.full_like(q, 5.0), torch.full(q.shape[:3], 5.0, device="cuda")
        api.obc_paged_attention(q, L.cache, q_lens=ql, causal=causal, o=o, lse=lse, workspace=ws)
        api.obc_score_status(ws)
        if first is None:
            first = o, lse
            real = check(o, lse, q, L, weight_bits=8, q_lens=q_lens, causal=causal)
            assert (o[~real] == 5.0).all() and (lse[~real] == 5.0).all()
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
@pytest.mark.parametrize("P", [128, 256])
@pytest.mark.parametrize("T,Hq,H", [(96, 32, 8), (65, 32, 8), (130, 32, 8), (300, 8, 8)])
def test_row_tiles_for_one_warpgroup(pages, P, T, Hq, H):
    _repeated(Lists([500], H, P, pages, seed=1), Hq, T)
    _repeated(Lists([2000, 530], H, P, pages, seed=2), Hq, T)
    _repeated(Lists([640], H, P, pages, seed=3), Hq, T, causal=False)


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
@pytest.mark.parametrize("P", [16, 128])
def test_several_items_for_every_cta(pages, P):
    lens = torch.randint(500, 900, (24,), generator=torch.Generator().manual_seed(P)).tolist()
    _repeated(Lists(lens, 8, P, pages, seed=4), 32, 96, times=4)


@pytest.mark.parametrize("pages", ["bf16", "e4m3"])
def test_a_mixed_batch(pages):
    q_lens = [300, 1, 96, 1, 65, 130, 1, 0, 32, 64]
    _repeated(Lists([2000, 1800, 500, 640, 1300, 130, 3000, 700, 515, 900], 8, 128, pages, seed=5), 32, 300, q_lens=q_lens, times=4)
