"""Calls of the cache and its attention that the header allows and that lie at an edge of it."""
import numpy as np
import pytest
import torch

from paper_2411_17686_amd import ficoco as fc
from tests import cache_ref as R
from tests.test_gpu_cache import append, i32, pair, reserve, same
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_new", [1, 16])
def test_the_largest_numbers_stay_finite(ctx, monkeypatch, dtype, n_new):
    """From 248 * 2^120 on the nearest E4M3 number of a block with the largest byte (247) would be 2^128, infinity: 240 * 2^120 is the largest that a finite
    value is stored as there.  One token, a block of tokens, an exponent raised to 247, and blocks rewritten."""
    plain, most = R.encode, 240.0 * 2.0 ** 120
    monkeypatch.setattr(R, "encode", lambda x, e: plain(np.where(np.abs(x) < 2.0 ** 128, np.clip(x, -most, most), x) if e == 247 else x, e))
    g, h = pair(1, 20, 16, 1, 64, 4, 2)
    top, largest = torch.finfo(torch.float32).max, torch.finfo(torch.bfloat16).max
    K, V = (torch.randn(4, 1, 17, 64, generator=torch.Generator().manual_seed(s)) for s in (1, 2))
    K[0, 0, n_new - 1, 3], K[0, 0, n_new - 1, 4] = largest, -largest
    V[0, 0, n_new - 1, 5], V[0, 0, n_new - 1, 6] = -float("inf"), largest
    V[0, 0, n_new - 1, 7] = float("nan")
    K[1, 0, n_new - 1, :6] = torch.tensor([247.0, 248.0, 249.0, 255.0, -252.0, 231.0]) * 2.0 ** 120
    V[1, 0, 0] = 2.0 ** 119
    V[2, 0, n_new - 1, ::2] = 1.74 * 2.0 ** 127
    V[2, 0, 0, 1] = float("inf")                           # (byte 246: 448 is a finite number)
    K[3, 0, n_new - 1, 0] = 1.75 * 2.0 ** 127              # the largest value of a block with byte 246: 448 * 2^119
    if dtype == torch.float32:
        K[2, 0, n_new - 1, 9], V[3, 0, n_new - 1, 9] = top, -top
    K, V = K.to(dtype), V.to(dtype)
    seq = [0, 1, 2, 3]
    for first, stop in ((0, n_new), (n_new, 17)):          # (the second call finds pages begun, or begins the next one)
        start, at = reserve(ctx, g, h, seq, [stop - first] * 4)
        append(ctx, g, h, 0, K[:, :, first:stop], V[:, :, first:stop], at, [stop - first] * 4, seq)
        same(g, h)
    assert h.e["k"][0, h.table[0, 0], 0] == 247 and h.e["k"][0, h.table[3, 0], 0] == 246
    # a louder token raises a quiet page to the largest byte
    done = i32([0] * 4)
    keep = np.array([[0, 1, 2, 3, 5, 6, 7, 8]] * 4, np.int32)
    fc.ficoco_cache_compact(ctx, g, 0, 1, i32(seq), i32(seq), 4, 13, torch.from_numpy(keep).cuda(), done, fc.cache_workspace(g, 4))
    assert done.tolist() == h.compact([0], seq, seq, 4, 13, keep)
    same(g, h)
    for step in range(2):
        start, at = reserve(ctx, g, h, seq, [1] * 4)
        k1 = torch.full((4, 1, 1, 64), (1.0, float(largest))[step]).to(dtype)
        append(ctx, g, h, 0, k1, -k1, at, [1] * 4, seq)
        same(g, h)
    for dt in (torch.bfloat16, torch.float32):
        k, v = (torch.zeros(4, 1, 14, 64, dtype=dt, device="cuda") for _ in range(2))
        fc.ficoco_cache_read(ctx, g, 0, k, v)
        assert torch.isfinite(k).all()
        assert torch.isinf(v).nonzero().tolist() == ([[0, 0, 0, 5]] if n_new == 1 else [])      # (where an infinity was put, and stayed)


@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("layers,heads", [(1, 1), (3, 2)])
def test_fork_of_a_sequence_with_positions_that_have_no_page(ctx, whole, layers, heads):
    """What has no page in src has none in dst, in the pages that are shared and in those that are copied."""
    n, P, d = 90, 16, 64
    g, h = pair(layers, 60, P, heads, d, 6, 8)
    start, at = reserve(ctx, g, h, [0, 1, 2], [n] * 3)
    for layer in range(layers):
        K, V = (rows(10 * layer + i, 3, heads, n, d).cpu() for i in (1, 2))
        append(ctx, g, h, layer, K, V, at, [n] * 3, [0, 1, 2])
    for s, i, bad in ((0, 5, -1), (1, 0, -1), (1, 2, 60), (1, 5, 2 ** 31 - 1), (2, 1, -9)):
        h.refs[h.table[s, i]] -= 1
        h.table[s, i] = bad
    g.table.copy_(torch.from_numpy(h.table))
    g.refs.copy_(torch.from_numpy(h.refs))
    taken, src, dst = h.refs.copy(), [0, 1, 1, 2], [3, 4, 0, 5]      # (0 is not empty)
    done = i32([7] * 4)
    fc.ficoco_cache_fork(ctx, g, i32(src), i32(dst), done, whole=whole)
    # 0 is a dst of the call: entry 0 may not read it
    assert done.tolist() == [0, 1, 0, 1]
    table, refs = g.table.cpu().numpy(), g.refs.cpu().numpy()
    want = taken.copy()
    for s, t in ((1, 4), (2, 5)):
        assert int(g.len[t]) == n
        for i in range(6):
            p, q = h.table[s, i], table[t, i]
            if not 0 <= p < 60:
                assert not 0 <= q < 60
            elif i < 5 and not whole:
                assert p == q
                want[p] += 1
            else:
                assert taken[q] == 0
                want[q] += 1
                for x in "kv":
                    assert torch.equal(getattr(g, x)[:, q], getattr(g, x)[:, p]) and torch.equal(getattr(g, x + "_exp")[:, q], getattr(g, x + "_exp")[:, p])
    assert np.array_equal(refs, want) and (table[3] == -1).all() and np.array_equal(table[:3], h.table[:3])
    # attended to alike
    for n_q in (1, 40):
        Q = rows(3, 2, heads, n_q, d)
        out = [torch.zeros_like(Q) for _ in range(2)]
        for o, seq in zip(out, ([1, 2], [4, 5])):
            fc.ficoco_cache_attention(ctx, g, layers - 1, Q, o, fc.attention_workspace(g, Q, o), seq=i32(seq))
        assert torch.equal(*out) and out[0].any()
    fc.ficoco_cache_free(ctx, g, i32([0, 1, 2, 4, 5]))
    assert not g.refs.any() and (g.table < 0).all()


@pytest.mark.parametrize("n", [4, 9])                      # plans by 256 threads and by 1024
@pytest.mark.parametrize("in_place", [True, False])
def test_compact_of_a_sequence_with_positions_that_have_no_page(ctx, n, in_place):
    """A token that has no page cannot move: such a sequence is left as it is.  In the pages that are kept it changes nothing."""
    P, d, length, v, N = 16, 64, 100, 40, 30
    g, h = pair(2, 200, P, 2, d, 2 * n, 8)
    seq = list(range(n))
    start, at = reserve(ctx, g, h, seq, [length] * n)
    K, V = rows(1, n, 2, length, d).cpu(), rows(2, n, 2, length, d).cpu()
    for layer in (0, 1):
        append(ctx, g, h, layer, K, V, at, [length] * n, seq)
    for s, i, bad in ((0, 2, -1), (1, 6, 200), (2, 1, -1)):          # tokens 32 .. 47, the last page, a page in front of what moves
        h.refs[h.table[s, i]] -= 1
        h.table[s, i] = bad
    g.table.copy_(torch.from_numpy(h.table))
    g.refs.copy_(torch.from_numpy(h.refs))
    keep = np.tile(np.arange(3, 30, 2, dtype=np.int32), (n, 1))
    dst = seq if in_place else [n + s for s in seq]
    done = i32([7] * n)
    fc.ficoco_cache_compact(ctx, g, 0, 2, i32(seq), i32(dst), v, N, torch.from_numpy(keep).cuda(), done, fc.cache_workspace(g, n))
    assert done.tolist() == [0, 0] + [1] * (n - 2)
    ok = seq[2:]
    before = h.table[2].copy()
    h.table[2, 1] = h.n_pages - 1                          # (the model counts the pages kept: one that nobody has)
    h.refs[h.n_pages - 1] = 1
    assert h.compact([0, 1], ok, dst[2:], v, N, keep[2:]) == [1] * (n - 2)
    h.refs[h.n_pages - 1] = 0
    h.table[2, 1] = before[1]
    h.table[dst[2], 1] = before[1]
    same(g, h)


@pytest.mark.parametrize("in_place", [True, False])
def test_compact_drops_tokens_that_have_no_page(ctx, in_place):
    """Pages of which no token is preserved need not be there; the first and the last token of such a page preserved, they have to."""
    P, d, length, v, N, n = 16, 64, 85, 20, 65, 5              # the span ends with the sequence: tokens 20 .. 84, pages 1 .. 5
    g, h = pair(1, 60, P, 1, d, 2 * n, 8)
    seq = list(range(n))
    start, at = reserve(ctx, g, h, seq, [length] * n)
    K, V = rows(1, n, 1, length, d).cpu(), rows(2, n, 1, length, d).cpu()
    append(ctx, g, h, 0, K, V, at, [length] * n, seq)
    for s in seq:
        for i in (2, 3, 5):                                    # tokens 32 .. 63, 80 .. 84
            h.refs[h.table[s, i]] -= 1
            h.table[s, i] = -1
    g.table.copy_(torch.from_numpy(h.table))
    g.refs.copy_(torch.from_numpy(h.refs))
    keep = np.array([[21, 30, 64, 70], [21, 32, 64, 70], [21, 31, 63, 70], [22, 31, 64, 79], [22, 31, 64, 80]], np.int32) - v
    dst = seq if in_place else [n + s for s in seq]
    done = i32([7] * n)
    fc.ficoco_cache_compact(ctx, g, 0, 1, i32(seq), i32(dst), v, N, torch.from_numpy(keep).cuda(), done, fc.cache_workspace(g, n))
    assert done.tolist() == [1, 0, 0, 1, 0]
    spare = h.n_pages - 1                                      # (the model counts pages: one that nobody has)
    for s in (0, 3):
        for i in (2, 3, 5):
            h.table[s, i] = spare
            h.refs[spare] += 1
    assert h.compact([0], [0, 3], [dst[0], dst[3]], v, N, keep[[0, 3]]) == [1, 1]
    h.table[h.table == spare] = -1
    h.refs[spare] = 0
    same(g, h)


def test_outputs_and_workspaces_that_reach_into_the_cache_are_refused(ctx):
    c = fc.Cache.empty(1, 400, 16, 2, 64, 4, 100)
    start = i32([0, 0])
    fc.ficoco_cache_reserve(ctx, c, start, 20, seq=i32([0, 1]))
    K, V = rows(1, 2, 2, 20, 64), rows(2, 2, 2, 20, 64)
    fc.ficoco_cache_append(ctx, c, 0, K, V, start)
    names = ("k", "v", "k_exp", "v_exp", "table", "len", "refs")
    torch.cuda.synchronize()
    before = [getattr(c, name).clone() for name in names]
    Q, O = rows(3, 2, 4, 1, 64), torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16, device="cuda")
    ws, cws = fc.attention_workspace(c, Q, O), fc.cache_workspace(c, 2)
    keep, two, done = i32([[0, 1]] * 2), i32([0, 1]), i32([5, 5])

    def into(t, numel, dtype=torch.bfloat16):
        flat = t.view(-1).view(dtype)
        return flat[:numel] if flat.numel() >= numel else None

    def space(t, of):
        w = fc.Workspace(of.bytes, "cuda")
        w.ptr = -(-t.data_ptr() // 256) * 256
        return w

    calls = []
    for name in names:
        t = getattr(c, name)
        rows_of = into(t, 2 * 2 * 64)
        if rows_of is not None:
            out = rows_of.view(2, 2, 1, 64)
            calls += [lambda out=out: fc.ficoco_cache_read(ctx, c, 0, out, None), lambda out=out: fc.ficoco_cache_read(ctx, c, 0, None, out)]
        rows_of = into(t, 2 * 64)
        if rows_of is not None:
            out = rows_of.view(1, 2, 1, 64)
            calls.append(lambda out=out: fc.ficoco_cache_attention(ctx, c, 0, Q[:1, :2], out, ws))
        if t.numel() * t.element_size() >= 1024:
            calls += [lambda t=t: fc.ficoco_cache_attention(ctx, c, 0, Q, O, space(t, ws)),
                      lambda t=t: fc.ficoco_cache_compact(ctx, c, 0, 1, two, two, 0, 4, keep, done, space(t, cws))]
    big = fc.Workspace(ws.bytes, "cuda")
    calls.append(lambda: fc.ficoco_cache_attention(ctx, c, 0, big.t[big.ptr - big.t.data_ptr():][:1024].view(torch.bfloat16).view(2, 4, 1, 64), O, big))
    assert len(calls) > 20
    for i, call in enumerate(calls):
        with pytest.raises(fc.FicocoError) as err:
            call()
        assert err.value.code == fc.EINVAL, i
    torch.cuda.synchronize()
    for name, t in zip(names, before):
        assert torch.equal(getattr(c, name), t), name
    assert done.tolist() == [5, 5] and not O.any()


def test_calls_beyond_the_threads_of_a_launch_are_refused(ctx):
    """Along one axis a launch has less than 2^32 threads."""
    c = fc.Cache.empty(1, 4, 16, 1, 64, 2, 4)
    wide = rows(1, 1, 1, 1, 64).expand(1, 1, 1 << 30, 64)
    for n, refused in (((1 << 30) - 1, True), (1 << 30, True), (1 << 20, False)):
        call = lambda: fc.ficoco_cache_append(ctx, c, 0, wide[:, :, :n], wide[:, :, :n], i32([0]))
        if refused:
            with pytest.raises(fc.FicocoError) as err:
                call()
            assert err.value.code == fc.EUNSUPPORTED
        else:
            call()                                         # (positions that have no page: nothing to write)
    # 2^31 rows of queries, that many sequences freed, 2^29 tokens read: described, not there
    L, stream = fc.lib(), ctx.raw_stream()
    p = 1 << 40
    far = fc._ATTENTION.pack(1 << 16, 1, 1, 1 << 15, 0, 64, p, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 2 * p, 1 << 22, 1 << 21, 64, 0, 0, 0, 0, 0.1, 0, 0, 0)
    assert L.ficoco_window_attention(ctx._h, far, stream) == fc.EUNSUPPORTED
    ws = fc.Workspace(256, "cuda")
    assert L.ficoco_cache_attention(ctx._h, c._p, 0, far, ws.ptr, ws.bytes, stream) == fc.EUNSUPPORTED
    assert L.ficoco_cache_free(ctx._h, c._p, 1 << 24, None, stream) == fc.EUNSUPPORTED
    tokens = fc._TOKENS.pack(1, 1 << 29, fc.BF16, 0, 0, 0, p, 0, 1 << 40, 1 << 40, 64, 0, 0, 0)
    assert L.ficoco_cache_read(ctx._h, c._p, 0, tokens, stream) == fc.EUNSUPPORTED
    torch.cuda.synchronize()
    assert not c.k.any() and not c.refs.any() and not c.len.any()
