"""Calls of the rotation that are too large are refused on the host, before anything is launched (the addresses here are nobody's)."""
import pytest
import torch

from paper_2411_17686_amd import ficoco as fc
from tests.test_gpu_cache_attention import ctx, i32  # noqa: F401

pytestmark = pytest.mark.gpu


def _rotation(B, n, H, H_kv, d):
    at = lambda i: (1 << 40) * (i + 1) * 256
    rows = (B * n * d, d, d)          # one token or one head: rows next to each other
    return fc._ROTATION.pack(B, H, H_kv, n, fc.BF16, fc.BF16, at(0), *rows, at(1) if H_kv else 0, *rows, at(2), *rows, at(3) if H_kv else 0, *rows, 0, 0, 0, 1, 0, 0)


@pytest.mark.parametrize("H", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 30])
def test_too_many_heads(ctx, H):  # noqa: F811
    d = 64
    rotary = fc.Rotary(d, fc.rotary_turns(d).cuda())
    assert fc.lib().ficoco_rotate(ctx._h, rotary.packed, _rotation(1, 1, H, 0, d), ctx.raw_stream()) == fc.EUNSUPPORTED
    c = fc.Cache.empty(1, 2, 16, 1, d, 1, 2)
    K = torch.zeros(1, 1, 1, d, dtype=torch.bfloat16, device="cuda")
    start = i32([0])
    tokens = fc._tokens(ctx, c, K, K.clone(), start, None, None)
    assert fc.lib().ficoco_cache_append_rotated(ctx._h, c._p, 0, rotary.packed, tokens, _rotation(1, 1, H, 0, d), ctx.raw_stream()) == fc.EUNSUPPORTED
    torch.cuda.synchronize()
    assert not bool(c.k.any()) and not bool(c.k_exp.any())
