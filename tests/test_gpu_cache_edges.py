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


@pytest.mark.parametrize("n_q,group,d", [(1, 4, 128), (2, 2, 64), (40, 2, 64), (70, 2, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 3)])
def test_more_queries_announced_than_given(ctx, n_q, group, d, window, sinks):
    """q_len beyond n_q counts as n_q, also where it decides the positions: the queries given are the last tokens."""
    lens, heads = [150, 90, 1200], 2
    c = filled(ctx, lens, 16, heads, d, seed=8)
    k, v = dense(ctx, c, 0, max(lens))
    Q = rows(2, 3, heads * group, n_q, d)
    q_len = i32([n_q + 1, n_q + 1000, 2 ** 31 - 1])
    O = torch.full_like(Q, 7.0)
    fc.ficoco_cache_attention(ctx, c, 0, Q, O, fc.attention_workspace(c, Q, O, window=window, sinks=sinks), q_len=q_len, window=window, sinks=sinks)
    check(O, Q, k, v, lens, d ** -0.5, [n - n_q for n in lens], [n_q] * 3, window, sinks, group)
    K, V = rows(3, 3, heads, 90, d), rows(4, 3, heads, 90, d)
    for K, V in ((K, V), tuple(torch.nn.functional.pad(t, (1, 2))[..., 1:-2] for t in (K, V))):       # (straight into LDS, and through registers)
        O = torch.full_like(Q, 7.0)
        fc.ficoco_window_attention(ctx, Q, K, V, O, q_len=q_len, window=window, sinks=sinks)
        check(O, Q, K.double().cpu().numpy(), V.double().cpu().numpy(), [90] * 3, d ** -0.5, [90 - n_q] * 3, [n_q] * 3, window, sinks, group)
