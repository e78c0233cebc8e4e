"""Keys rotated on their way into the pages: the same bytes as ficoco_rotate into single precision and ficoco_cache_append behind it."""
import pytest
import torch

from paper_2411_17686_amd import ficoco as fc
from tests.test_gpu_rotate import BF, F, H_, P_, ctx, i32, rotary, rows_of  # noqa: F401

pytestmark = pytest.mark.gpu


def caches(page, heads, d, slots, tokens, fill=0, layers=2):
    """Two equal caches whose slots have room for `tokens`, in pages out of order."""
    max_pages = -(-tokens // page)
    n_pages = slots * max_pages + 2
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(page + heads))[:slots * max_pages]
    made = []
    for _ in range(2):
        c = fc.Cache.empty(layers, n_pages, page, heads, d, slots, max_pages)
        c.k.fill_(fill)
        c.v.fill_(fill)
        c.table.copy_(order.view(slots, max_pages).int())
        made.append(c)
    return made


def two_steps(ctx, c, layer, r, Q, Qo, K, V, start, pos, n_new, seq):  # noqa: F811
    """The same by the two calls."""
    at = None if pos is None else pos
    rows = n_new
    Kf = torch.zeros(K.shape, dtype=F, device="cuda")
    own = None
    if pos is None:
        own = start
    fc.ficoco_rotate(ctx, r, None, K, None, Kf, pos=at, start=own, n_rows=rows)
    if Q is not None:
        ok = start >= 0
        if seq is not None:
            ok &= (seq >= 0) & (seq < c.table.shape[0])
        n = torch.full_like(start, K.shape[2]) if n_new is None else n_new
        fc.ficoco_rotate(ctx, r, Q, None, Qo, None, pos=at, start=own, n_rows=torch.where(ok, n, 0).int())
    fc.ficoco_cache_append(ctx, c, layer, Kf, V.float(), start, n_new=n_new, seq=seq)


def same(a, b):
    for x in ("k", "v", "k_exp", "v_exp", "table", "len", "refs"):
        assert torch.equal(getattr(a, x), getattr(b, x)), x


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d,rot,begin,layout", [(128, 128, 0, H_), (128, 64, 64, P_), (64, 64, 0, P_), (64, 32, 8, H_), (64, 16, 48, P_), (128, 0, 0, H_)])
@pytest.mark.parametrize("dtype,norm", [(BF, 1), (F, 0), (BF, 2)])
def test_prompts(ctx, page, d, rot, begin, layout, dtype, norm):  # noqa: F811
    B, n, H, Hk = 4, 150, 4, 2
    r = rotary(d, rot, norm, bias=norm == 2, layout=layout, rot_begin=begin, axes=3)
    a, b = caches(page, Hk, d, B, 200)
    x = rows_of(B, H + 2 * Hk, n, d, dtype, page + d)
    Q, K, V = x.split([H, Hk, Hk], 1)
    start, n_new = i32([0, 17, 50, 3]), i32([150, 90, 0, 1])
    pos = torch.randint(0, 5000, (3, B, n), dtype=torch.int32, device="cuda")
    Qa, Qb = (torch.full(Q.shape, 5.0, dtype=BF, device="cuda") for _ in range(2))
    for c in (a, b):        # what lies before the new tokens
        fc.ficoco_cache_append(ctx, c, 1, K[:, :, :60] * 0.4, V[:, :, :60] * 2, i32([0] * B))
    fc.ficoco_cache_append_rotated(ctx, a, 1, r, Q, Qa, K, V, start, pos=pos, n_new=n_new)
    two_steps(ctx, b, 1, r, Q, Qb, K, V, start, pos, n_new, None)
    same(a, b)
    assert torch.equal(Qa, Qb)


@pytest.mark.parametrize("page,d", [(16, 64), (32, 128), (64, 128), (128, 128), (128, 64)])
@pytest.mark.parametrize("dtype,norm,layout", [(BF, 1, H_), (F, 0, P_), (F, 2, H_)])
def test_single_tokens_over_whole_pages(ctx, page, d, dtype, norm, layout):  # noqa: F811
    """Louder and louder tokens: exponents rise at every step, of several blocks of a wavefront, at every place of a page."""
    B, H, Hk, steps = 3, 6, 3, page + 5
    r = rotary(d, d // 2, norm, layout=layout, rot_begin=d // 2 if layout else 0)
    a, b = caches(page, Hk, d, 5, steps)
    seq = i32([4, 0, 2])
    for i in range(steps):
        x = rows_of(B, H + 2 * Hk, 1, d, dtype, i) * (1.0 + 0.2 * i if i % 3 else 1.0)
        Q, K, V = x.split([H, Hk, Hk], 1)
        start = i32([i, i if i % 5 else -1, i])
        Qa, Qb = (torch.full(Q.shape, 5.0, dtype=Q.dtype, device="cuda") for _ in range(2))
        fc.ficoco_cache_append_rotated(ctx, a, 0, r, Q, Qa, K, V, start, seq=seq)
        two_steps(ctx, b, 0, r, Q, Qb, K, V, start, None, None, seq)
        assert torch.equal(Qa, Qb)
        if i % 11 == 0 or i == steps - 1:
            same(a, b)


def test_values_that_are_no_numbers(ctx):  # noqa: F811
    """Infinities and NaN, the largest numbers, zeros, denormals: as ficoco_cache_append has them."""
    r = rotary(64, 0)
    for n in (1, 20):
        a, b = caches(16, 2, 64, 3, 40)
        x = rows_of(3, 4, n, 64, F, 3)
        x[0, 0, 0, 0], x[0, 1, 0, 5], x[0, 2, 0, 0], x[0, 3, 0, 9] = float("inf"), float("nan"), -float("inf"), float("nan")
        x[1, :, 0] = 0
        x[2] *= 3e38 / x[2].abs().max()
        K, V = x.split([2, 2], 1)
        fc.ficoco_cache_append_rotated(ctx, a, 0, r, None, None, K, V, i32([0, 16, 1]))
        two_steps(ctx, b, 0, r, None, None, K, V, i32([0, 16, 1]), None, None, None)
        same(a, b)


def test_rows_that_are_left_out(ctx):  # noqa: F811
    """Slots out of range, positions without a page or behind the table, counts out of range: nothing else is touched."""
    r = rotary(128, 128, 1)
    for n in (1, 40):
        a, b = caches(32, 2, 128, 4, 70, fill=9)
        for c in (a, b):
            c.table[1, 0] = -1
            c.table[2, 1] = 1000
        x = rows_of(6, 8, n, 128, BF, n)
        Q, K, V = x.split([4, 2, 2], 1)
        seq, start, n_new = i32([0, 1, 2, 3, 4, -1]), i32([95, 0, 20, 96, 0, 0]), i32([n, n, n + 9, n, n, n])
        Qa, Qb = (torch.full(Q.shape, 5.0, dtype=BF, device="cuda") for _ in range(2))
        fc.ficoco_cache_append_rotated(ctx, a, 1, r, Q, Qa, K, V, start, n_new=n_new, seq=seq)
        two_steps(ctx, b, 1, r, Q, Qb, K, V, start, None, n_new, seq)
        same(a, b)
        assert torch.equal(Qa, Qb) and bool((Qa[4:] == 5).all())


def test_replayed(ctx):  # noqa: F811
    """Captured once, replayed over the places of a page."""
    r = rotary(64, 64, 1)
    a, b = caches(16, 2, 64, 3, 32)
    Q, K, V = (rows_of(3, h, 1, 64, BF, h) for h in (4, 2, 2))
    start, Qa, Qb = i32([0, 3, 9]), torch.zeros_like(Q), torch.zeros_like(Q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fc.ficoco_cache_append_rotated(ctx, a, 0, r, Q, Qa, K, V, start)
    for i in range(12):
        for t in (Q, K, V):
            t.mul_(1.1).add_(0.01)
        g.replay()
        torch.cuda.synchronize()
        two_steps(ctx, b, 0, r, Q, Qb, K, V, start, None, None, None)
        same(a, b)
        assert torch.equal(Qa, Qb)
        start.add_(1)


def test_in_place_queries_and_refusals(ctx):  # noqa: F811
    r = rotary(128, 128, 1)
    a, b = caches(64, 2, 128, 2, 64)
    x = rows_of(2, 8, 10, 128, BF, 5)
    Q, K, V = x.split([4, 2, 2], 1)
    want = torch.zeros_like(Q)
    two_steps(ctx, b, 0, r, Q, want, K, V, i32([0, 0]), None, None, None)
    fc.ficoco_cache_append_rotated(ctx, a, 0, r, Q, None, K, V, i32([0, 0]))
    same(a, b)
    assert torch.equal(Q, want)
    keep = [t.clone() for t in (a.k, a.v, a.k_exp)]
    for kw, code in ((dict(Q_out=x[:, 1:5]), fc.EINVAL), (dict(Q_out=x[:, 4:8]), fc.EINVAL), (dict(layer=2), fc.EINVAL),
                     (dict(rotary=rotary(64, 64)), fc.EINVAL), (dict(rotary=rotary(128, 120)), fc.EUNSUPPORTED),
                     (dict(rotary=rotary(128, 64, rot_begin=4)), fc.EUNSUPPORTED)):
        args = dict(layer=0, rotary=r, Q=Q, Q_out=None, K=K, V=V, start=i32([0, 0]))
        args.update(kw)
        with pytest.raises((fc.FicocoError, TypeError)) as e:
            fc.ficoco_cache_append_rotated(ctx, a, **args)
        assert not isinstance(e.value, fc.FicocoError) or e.value.code == code, kw
    with pytest.raises(TypeError):
        fc.ficoco_cache_append_rotated(ctx, a, 0, r, Q, None, None, V, i32([0, 0]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(keep, (a.k, a.v, a.k_exp)))
