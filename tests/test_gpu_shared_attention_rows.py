"""Every row of large families of sequences that share pages against 64 bits, within the bound of tests/cache_ref.py (the reference computed on the device)."""
import pytest
import torch

from paper_2411_17686_amd import ficoco as fc
from tests.test_gpu_cache_attention import ctx  # noqa: F401
from tests.test_gpu_shared_attention import LARGE, family, queries, run

pytestmark = pytest.mark.gpu


def attention64(q, k, v, scale, pos, window, sinks):
    """cache_ref.attention() on the device: q [r][d] at positions pos [r], k and v [n][d], all float64.  The rows and the bound of the kernels' error."""
    n, d = k.shape
    j = torch.arange(n, device=q.device)[None]
    see = j <= pos[:, None]
    if window:
        see &= (j > pos[:, None] - window) | (j < sinks)
    logit = (scale * (q @ k.t())).masked_fill(~see, -torch.inf)
    w = torch.softmax(logit, 1)                            # (every row here sees a key)
    out = w @ v
    size = (scale * (q.abs() @ k.abs().t())).masked_fill(~see, 0.0).max(1).values
    delta = (d + 4) * 2.0 ** -24 * size + 2.0 ** -20
    return out, 2.0 ** -8 * out.abs() + (2.0 ** -8 + 2 * delta + n * 2.0 ** -24)[:, None] * (w @ v.abs()) * 1.01 + 1e-30


@pytest.mark.parametrize("case", LARGE, ids=str)
def test_every_row(ctx, case):  # noqa: F811
    prompt, tail, n, page, heads, g, d, n_q, window = case
    c, lens, group = family(ctx, page, heads, d, [(prompt, [prompt + tail + 3 * i for i in range(n)]), (prompt // 2, [prompt] * 3), (0, [prompt + 10])])
    B = len(lens)
    Q = queries(B, heads * g, n_q, d)
    K, V = (torch.zeros(B, heads, max(lens), d, device="cuda") for _ in range(2))
    fc.ficoco_cache_read(ctx, c, 1, K, V)
    outs = [run(ctx, c, Q, group, window=window, sinks=4, always=always) for always in (True, False)]
    for b in range(B):
        pos = torch.arange(lens[b] - n_q, lens[b], device="cuda").repeat(g)
        for h in range(heads):
            rows = slice(h * g, (h + 1) * g)
            want, bound = attention64(Q[b, rows].double().reshape(-1, d), K[b, h, :lens[b]].double(), V[b, h, :lens[b]].double(), d ** -0.5, pos, window, 4)
            for O in outs:
                assert bool(((O[b, rows].double().reshape(-1, d) - want).abs() <= bound).all()), (b, h)
