"""obc_paged_read with outputs given: what n_tokens and dtype say has to agree with them (no GPU needed)."""
import pytest
import torch

from paper_2510_07651_b200 import api


def _cache():
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    return api.PagedCache(k, k, torch.zeros((1, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))


def test_contradictions_are_refused():
    out = torch.zeros((1, 2, 20, 128))
    with pytest.raises(ValueError, match="n_tokens"):
        api.obc_paged_read(_cache(), n_tokens=21, k_out=out, v_out=out.clone())
    with pytest.raises(ValueError, match="n_tokens"):
        api.obc_paged_read(_cache(), n_tokens=19, v_out=out.clone())
    with pytest.raises(ValueError, match="dtype"):
        api.obc_paged_read(_cache(), dtype=torch.bfloat16, k_out=out, v_out=out.clone())
    with pytest.raises(TypeError):
        api.obc_paged_read(_cache(), dtype=torch.float16, k_out=out, v_out=out.clone())


def test_what_agrees_goes_on_to_the_call():
    out = torch.zeros((1, 2, 20, 128))
    for kw in (dict(), dict(n_tokens=20), dict(dtype=torch.float32), dict(n_tokens=20, dtype=torch.float32)):
        with pytest.raises(ValueError, match="CUDA pages"):
            api.obc_paged_read(_cache(), k_out=out, v_out=out.clone(), **kw)
