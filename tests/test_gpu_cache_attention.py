"""Attention over the pages and over dense prompts against 64 bits, within the bound derived in tests/cache_ref.py."""
import numpy as np
import pytest
import torch

from paper_2411_17686_amd import ficoco as fc
from tests import cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = fc.Context(0)
    yield c
    c.close()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def filled(ctx, lens, page, heads, d, seed=0, slots=None, spare=1):
    """A cache whose slot s holds lens[s] tokens in pages out of order; what no token fills is NaN."""
    slots = slots or len(lens)
    max_pages = -(-max(lens) // page) + spare
    n_pages = sum(-(-n // page) for n in lens) + 3
    c = fc.Cache.empty(2, n_pages, page, heads, d, slots, max_pages)
    c.k.fill_(127)
    c.v.fill_(127)
    order = np.random.RandomState(seed).permutation(n_pages)
    table = np.full((slots, max_pages), -1, np.int32)
    at = 0
    for s, n in enumerate(lens):
        m = -(-n // page)
        table[s, :m] = order[at:at + m]
        at += m
    c.table.copy_(torch.from_numpy(table))
    c.len.copy_(torch.tensor(list(lens) + [0] * (slots - len(lens)), dtype=torch.int32))
    g = torch.Generator(device="cuda").manual_seed(seed)
    n_max = max(max(lens), 1)
    for layer in (0, 1):
        k, v = (torch.randn(len(lens), heads, n_max, d, generator=g, device="cuda") * 2.0 ** torch.randint(-1, 2, (len(lens), heads, n_max, 1), generator=g, device="cuda")
                for _ in range(2))
        fc.ficoco_cache_append(ctx, c, layer, k, v, i32([0] * len(lens)), n_new=i32(lens))
    return c


def dense(ctx, c, layer, n):
    """What the pages hold, float64 [slots][heads][n][d]."""
    S = c.table.shape[0]
    k, v = (torch.zeros(S, c.c.heads, max(n, 1), c.c.d_head, device="cuda") for _ in range(2))
    fc.ficoco_cache_read(ctx, c, layer, k, v)
    return [np.nan_to_num(t.double().cpu().numpy()) for t in (k, v)]


def check(out, Q, k, v, lens, scale, starts, q_lens, window, sinks, group, have=None, before=None):
    """out, Q: [B][H][n_q][d]; k, v: float64 [B][heads][n][d]."""
    B, H, n_q, d = Q.shape
    got, q64 = out.double().cpu().numpy(), Q.double().cpu().numpy()
    for b in range(B):
        for h in range(H):
            n = max(lens[b], 0)
            pos = starts[b] + np.arange(max(q_lens[b], 0))
            want, bound = R.attention(q64[b, h, :len(pos)], k[b, h // group, :n], v[b, h // group, :n], scale, pos, window, sinks,
                                      None if have is None else have[b][:n])
            diff = np.abs(got[b, h, :len(pos)] - want)
            assert (diff <= bound).all(), (b, h, float(np.nanmax(diff / bound)), np.argwhere(~(diff <= bound))[:4].tolist())
            if before is not None:
                assert np.array_equal(got[b, h, len(pos):], np.full((n_q - len(pos), d), before))


FEW = [  # lens, page, heads, group, d, n_q, window, sinks, max_len
    ([1], 16, 1, 1, 64, 1, 0, 0, 0),
    ([0, 1, 15, 16, 17, 31, 32, 33], 16, 2, 1, 128, 1, 0, 0, 0),
    ([63, 64, 65, 127, 128, 129], 64, 1, 8, 128, 1, 0, 0, 0),
    ([300, 7, 511], 32, 2, 7, 64, 1, 0, 0, 0),
    ([1000, 3, 517], 128, 2, 4, 128, 1, 0, 0, 0),
    ([700, 40, 1], 64, 3, 4, 128, 4, 0, 0, 0),
    ([5, 33, 2], 16, 1, 2, 64, 8, 0, 0, 0),            # more queries than tokens: rows that see nothing
    ([900, 130, 20], 32, 2, 4, 128, 1, 100, 4, 0),
    ([900, 130, 20], 16, 2, 4, 64, 3, 33, 0, 0),
    ([900, 130, 20], 64, 2, 1, 64, 2, 1, 35, 0),
    ([900, 700, 64], 64, 1, 16, 128, 1, 640, 70, 0),
    ([9000, 5000], 64, 2, 4, 128, 1, 0, 0, 9000),      # cut over many workgroups
    ([9000, 12, 4097], 16, 1, 3, 64, 5, 0, 0, 0),
    ([9000, 5000], 32, 1, 2, 128, 1, 3000, 17, 64),    # a hint that is too small
]


@pytest.mark.parametrize("case", FEW, ids=str)
def test_few_rows(ctx, case):
    _run(ctx, *case)


MANY = [
    ([200, 70, 17], 64, 1, 1, 64, 17, 0, 0, 0),
    ([129, 64, 1, 0], 16, 2, 4, 128, 64, 0, 0, 0),
    ([640, 300, 33], 32, 2, 7, 128, 33, 0, 0, 0),
    ([1500, 900], 128, 1, 4, 64, 200, 0, 0, 0),
    ([1500, 900], 64, 2, 2, 128, 65, 0, 0, 1500),
    ([700, 130, 50], 64, 2, 3, 128, 130, 100, 4, 0),
    ([700, 130, 50], 16, 1, 1, 64, 300, 64, 0, 0),
    ([2000, 1999], 32, 1, 2, 128, 40, 1, 200, 0),
    ([5000], 64, 1, 4, 128, 64, 0, 0, 0),
]


@pytest.mark.parametrize("case", MANY, ids=str)
def test_many_rows(ctx, case):
    _run(ctx, *case)


def _run(ctx, lens, page, heads, group, d, n_q, window, sinks, max_len):
    c = filled(ctx, lens, page, heads, d, seed=len(lens) + n_q)
    B = len(lens)
    g = torch.Generator(device="cuda").manual_seed(n_q)
    Q = (torch.randn(B, heads * group, n_q, d, generator=g, device="cuda") * 2).to(torch.bfloat16)
    O = torch.full_like(Q, 77.0)
    ws = fc.attention_workspace(c, Q, O, window=window, sinks=sinks, max_len=max_len)
    ws.t.fill_(255)
    fc.ficoco_cache_attention(ctx, c, 1, Q, O, ws, window=window, sinks=sinks, max_len=max_len)
    k, v = dense(ctx, c, 1, max(lens))
    check(O, Q, k, v, lens, d ** -0.5, [n - n_q for n in lens], [n_q] * B, window, sinks, group)


@pytest.mark.parametrize("n_q,group", [(1, 4), (3, 2), (70, 2)])
def test_ragged_queries_slots_and_strides(ctx, n_q, group):
    """Sequences by slot (one out of range, one named twice), fewer queries than n_q, given positions and lengths, rows apart."""
    lens = [500, 90, 260, 31]
    c = filled(ctx, lens, 32, 2, 64, seed=5)
    seq, B = [2, 0, 9, 2, 3, -1, 1], 7
    q_len = [min(n_q, x) for x in (n_q, max(1, n_q - 1), n_q, 0, n_q + 5, 1, -2)]
    k_len = [260, 1000, 50, 100, 31, 10, 40]
    q_start = [200, 480, 5, 7, -2, 3, 39]
    H = 2 * group
    g = torch.Generator(device="cuda").manual_seed(1)
    base = torch.randn(B, n_q, H, 3, 67, generator=g, device="cuda").to(torch.bfloat16)
    Q = base[..., 1, 1:65].transpose(1, 2)
    out = torch.full((B, n_q, H, 71), 9.0, dtype=torch.bfloat16, device="cuda")
    O = out[..., 3:67].transpose(1, 2)
    ws = fc.attention_workspace(c, Q, O)
    fc.ficoco_cache_attention(ctx, c, 0, Q, O, ws, scale=0.3, q_len=i32(q_len), k_len=i32(k_len), q_start=i32(q_start), seq=i32(seq))
    k, v = dense(ctx, c, 0, 500)
    keys = [min(kl, lens[s]) if 0 <= s < 4 else 0 for s, kl in zip(seq, k_len)]
    idx = [s if 0 <= s < 4 else 0 for s in seq]
    check(O, Q, k[idx], v[idx], keys, 0.3, q_start, q_len, 0, 0, group, before=9.0)
    assert (out[..., :3] == 9).all() and (out[..., 67:] == 9).all()


@pytest.mark.parametrize("n_q", [1, 40])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 20)])
def test_positions_without_a_page_hold_no_key(ctx, n_q, window, sinks):
    lens = [400, 400]
    c = filled(ctx, lens, 16, 1, 128, seed=3)
    have = np.ones((2, 400), bool)
    for s, at, p in ((0, 0, -1), (0, 17, -1), (0, 20, c.c.n_pages), (1, 24, 2147483647), (1, 1, -7)):
        c.table[s, at] = p
        have[s, 16 * at:16 * at + 16] = False
    g = torch.Generator(device="cuda").manual_seed(1)
    Q = torch.randn(2, 2, n_q, 128, generator=g, device="cuda").to(torch.bfloat16)
    O = torch.zeros_like(Q)
    fc.ficoco_cache_attention(ctx, c, 0, Q, O, fc.attention_workspace(c, Q, O), window=window, sinks=sinks)
    k, v = dense(ctx, c, 0, 400)
    check(O, Q, k, v, lens, 128 ** -0.5, [400 - n_q] * 2, [n_q] * 2, window, sinks, 2, have=have)


@pytest.mark.parametrize("n_q", [1, 20])
def test_what_nobody_sees_may_hold_anything(ctx, n_q):
    """NaN keys and values outside the window, and in the first tokens' block behind them."""
    c = filled(ctx, [600], 32, 1, 64, seed=9)
    k, v = dense(ctx, c, 0, 600)
    bad = torch.full((1, 1, 400, 64), float("nan"), device="cuda")
    fc.ficoco_cache_append(ctx, c, 0, bad, bad, i32([37]))
    g = torch.Generator(device="cuda").manual_seed(1)
    Q = torch.randn(1, 2, n_q, 64, generator=g, device="cuda").to(torch.bfloat16)
    O = torch.zeros_like(Q)
    # (the append took the exponents of the begun and the left page along: read them again)
    k2, v2 = dense(ctx, c, 0, 600)
    fc.ficoco_cache_attention(ctx, c, 0, Q, O, fc.attention_workspace(c, Q, O), window=100, sinks=37)
    check(O, Q, k2, v2, [600], 0.125, [600 - n_q], [n_q], 100, 37, 2)


@pytest.mark.parametrize("n_q", [1, 24])
def test_large_logits_and_growing_maxima(ctx, n_q):
    """Keys whose logits grow along the sequence by hundreds, and one row whose largest comes first."""
    n, d = 700, 64
    c = fc.Cache.empty(1, 12, 64, 1, d, 1, 12)
    start = i32([0])
    fc.ficoco_cache_reserve(ctx, c, start, n)
    ramp = torch.linspace(0, 1, n).view(1, 1, n, 1)
    K = (torch.ones(1, 1, n, d) * ramp * 30).cuda()
    K[0, 0, 0] = 40.0
    V = torch.randn(1, 1, n, d, generator=torch.Generator().manual_seed(2)).cuda()
    fc.ficoco_cache_append(ctx, c, 0, K, V, start)
    Q = torch.ones(1, 2, n_q, d).cuda()
    Q[:, 1] = -1
    Q[0, 0, 0, ::2] = 3
    Q = Q.to(torch.bfloat16)
    O = torch.zeros_like(Q)
    fc.ficoco_cache_attention(ctx, c, 0, Q, O, fc.attention_workspace(c, Q, O), scale=1.0)
    k, v = dense(ctx, c, 0, n)
    check(O, Q, k, v, [n], 1.0, [n - n_q], [n_q], 0, 0, 2)


WINDOW = [  # B, H_kv, group, d, n_q, n_k, window, sinks, q_len, k_len
    (1, 1, 1, 64, 1, 1, 0, 0, None, None),
    (2, 2, 1, 128, 64, 64, 0, 0, None, None),
    (2, 1, 4, 64, 129, 129, 16, 0, None, None),
    (1, 2, 7, 128, 300, 300, 100, 35, None, None),
    (3, 1, 2, 128, 200, 200, 64, 4, [200, 1, 77], [200, 1, 77]),
    (2, 1, 3, 64, 50, 400, 0, 0, None, None),           # the last tokens of longer sequences
    (2, 1, 3, 128, 50, 400, 37, 70, [50, 20], [400, 333]),
    (2, 2, 1, 64, 90, 20, 0, 0, None, None),            # more queries than keys
    (2, 1, 1, 128, 33, 100, 1, 0, [33, 0], [100, 0]),
    (1, 1, 1, 64, 700, 700, 1, 1, None, None),
    (1, 1, 2, 128, 1000, 1000, 1000, 0, None, None),
]


@pytest.mark.parametrize("aligned", [True, False])      # rows of 16-byte chunks go straight into LDS, others through registers
@pytest.mark.parametrize("case", WINDOW, ids=str)
def test_window_attention(ctx, case, aligned):
    B, heads, group, d, n_q, n_k, window, sinks, q_len, k_len = case
    g = torch.Generator(device="cuda").manual_seed(n_q)
    H = heads * group
    qkv = torch.randn(B, max(n_q, n_k), H + 2 * heads, d + 8 if aligned else d + 3, generator=g, device="cuda").to(torch.bfloat16)
    qkv = qkv[..., 8:d + 8] if aligned else qkv[..., 1:d + 1]
    Q = qkv[:, :n_q, :H].transpose(1, 2)
    K, V = qkv[:, :n_k, H:H + heads].transpose(1, 2), qkv[:, :n_k, H + heads:].transpose(1, 2)
    O = torch.full((B, n_q, H, d), 5.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    kl, ql = k_len or [n_k] * B, q_len or [n_q] * B
    k64, v64 = K.double().cpu().numpy(), V.double().cpu().numpy()
    for b in range(B):                                  # behind a sequence's end there may be anything
        K[b, :, kl[b]:] = float("nan")
        V[b, :, kl[b]:] = float("nan")
    fc.ficoco_window_attention(ctx, Q, K, V, O, window=window, sinks=sinks, q_len=None if q_len is None else i32(q_len),
                               k_len=None if k_len is None else i32(k_len))
    check(O, Q, k64, v64, kl, d ** -0.5, [a - b for a, b in zip(kl, ql)], ql, window, sinks, group, before=5.0)


def test_window_attention_given_positions(ctx):
    g = torch.Generator(device="cuda").manual_seed(4)
    Q, K, V = (torch.randn(3, 2, n, 64, generator=g, device="cuda").to(torch.bfloat16) for n in (70, 150, 150))
    O = torch.zeros_like(Q)
    starts = [0, 100, -30]
    fc.ficoco_window_attention(ctx, Q, K, V, O, q_start=i32(starts), window=40, sinks=3)
    check(O, Q, K.double().cpu().numpy(), V.double().cpu().numpy(), [150] * 3, 0.125, starts, [70] * 3, 40, 3, 1)
