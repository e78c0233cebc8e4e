"""Calls of the cache and its attention that the header allows and that lie at an edge of it."""
import pytest
import torch

from paper_2411_17686_amd import ficoco as fc
from tests.test_gpu_cache import i32
from tests.test_gpu_cache_attention import check, dense, filled

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = fc.Context(0)
    yield c
    c.close()


def rows(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


@pytest.mark.parametrize("byte", [0, 248, 254, 255])
@pytest.mark.parametrize("n_q,d", [(1, 64), (1, 128), (3, 128), (40, 64), (40, 128)])
@pytest.mark.parametrize("k_len,window,sinks", [(16, 0, 0), (65, 0, 0), (200, 20, 5), (200, 60, 20)])
def test_exponents_of_pages_that_nobody_sees_need_no_value(ctx, byte, n_q, d, k_len, window, sinks):
    """Pages of a prompt that are reserved and not yet written, or lie between the first tokens and the window."""
    n, P = 230, 16
    c = filled(ctx, [n], P, 2, d, seed=4)
    k, v = dense(ctx, c, 1, n)
    first = max(k_len - n_q, 0)                             # the lowest position; those below 0 see nothing
    near = max(first - window + 1, 0) if window else 0
    for at in range(-(-n // P)):
        keys = range(P * at, P * at + P)
        if not any(j < k_len and (j >= near or j < sinks) for j in keys):
            page = int(c.table[0, at])
            for x in "kv":
                getattr(c, x)[1, page] = 255
                getattr(c, x + "_exp")[1, page] = byte
    Q = rows(1, 1, 4, n_q, d)
    O = torch.full_like(Q, 7.0)
    fc.ficoco_cache_attention(ctx, c, 1, Q, O, fc.attention_workspace(c, Q, O, window=window, sinks=sinks), k_len=i32([k_len]), window=window, sinks=sinks)
    check(O, Q, k, v, [k_len], d ** -0.5, [k_len - n_q], [n_q], window, sinks, 2)
