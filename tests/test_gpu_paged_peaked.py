"""Attention whose weights lie far apart: one token's logit is many nats above all others', as that of a sequence's first token often is.  Where its row of V is
zero, o consists of the small weights alone, so that each of them has to keep its relative precision."""
import math

import pytest
import torch

from paper_2510_07651_b200 import api
from tests.paged_helpers import D, TYPES, Lists, check

pytestmark = pytest.mark.gpu

# a weight is off by at most (see `check`): fp32; two bf16 parts; fp16, half a step of 2^-10.  With more than 16 rows per list: one bf16, half a step of 2^-7
FEW, CHUNK = {"f32": 22, "bf16": 15, "e4m3": 10.9}, {"f32": 22, "bf16": 8, "e4m3": 8}


def peaked(pages, n, Hq, H, T, at, gap, v_row, P=16, causal=True, quiet_channel=False):
    """Channel 0 of every query is 8 and that of every key 0, but for token `at`: its logits are `gap` above what its other channels give.  v_row: what its row of V is
    multiplied by; quiet_channel: nothing but its channels 0 to 63 is set in that row."""
    g = torch.Generator().manual_seed(n + at)
    q = torch.randn((1, Hq, T, D), generator=g)
    k, v = torch.randn((1, H, n, D), generator=g), torch.randn((1, H, n, D), generator=g)
    q[..., 0] = 8.0
    k[..., 0] = 0.0
    k[:, :, at, 1:] = 0.0
    k[:, :, at, 0] = gap * math.sqrt(D) / 8
    v[:, :, at] *= v_row
    if quiet_channel:
        v[:, :, at, 64:] = 0.0
    L = Lists([n], H, P, pages, seed=1, k=k, v=v)
    q = q.to("cuda", torch.float32 if pages == "f32" else torch.bfloat16)
    o, lse = api.obc_paged_attention(q, L.cache, causal=causal)
    check(o, lse, q, L, weight_bits=(FEW if Hq // H * T <= 16 else CHUNK)[pages], causal=causal, what=f"{pages} {gap}")


@pytest.mark.parametrize("pages", list(TYPES))
@pytest.mark.parametrize("gap", [8, 14, 16, 18, 20, 30])
@pytest.mark.parametrize("v_row", [0.0, 1.0])
@pytest.mark.parametrize("T,Hq,H", [(1, 8, 1), (1, 16, 1), (4, 8, 2), (40, 4, 2)])
def test_the_first_token(pages, gap, v_row, T, Hq, H):
    peaked(pages, 4096, Hq, H, T, 0, gap, v_row)


@pytest.mark.parametrize("pages", list(TYPES))
@pytest.mark.parametrize("at", [2047, 4095])
@pytest.mark.parametrize("T,Hq,H", [(1, 8, 1), (4, 8, 2), (40, 4, 2)])
def test_a_token_in_the_middle_and_the_last(pages, at, T, Hq, H):
    """The softmax's reference moves late in the list, and the parts that CTAs merge are very unequal."""
    for gap in (10, 18):
        for v_row in (0.0, 1.0):
            peaked(pages, 4096, Hq, H, T, at, gap, v_row)
    peaked(pages, 4096, Hq, H, T, at, 18, 1.0, causal=False, P=64)


@pytest.mark.parametrize("pages", list(TYPES))
@pytest.mark.parametrize("v_row", [300.0, 2.0 ** 30])
def test_a_large_row_of_v_with_channels_of_zero(pages, v_row):
    """Its scale is far above the others', but half of the channels hold nothing of it."""
    for gap in (0, -12, 12):
        peaked(pages, 2000, 8, 1, 1, 0, gap, v_row, quiet_channel=True)
    peaked(pages, 2000, 8, 2, 40, 0, 12, v_row, quiet_channel=True)


@pytest.mark.parametrize("pages", list(TYPES))
@pytest.mark.parametrize("T", [1, 40])
def test_a_long_list(pages, T):
    """Many weights, each below 2^-25 of the largest, that together are not small."""
    peaked(pages, 60000, 4, 1, T, 5, 20, 0.0, P=64)
    peaked(pages, 60000, 4, 1, T, 5, 20, 1.0, P=64)
