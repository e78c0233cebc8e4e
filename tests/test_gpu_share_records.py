"""The plan of sequences that share pages as the device writes it, record by record (tests/share_records.py), and the attention by plans whose workgroups go on with another tile."""
import random

import numpy as np
import pytest
import torch

from paper_2411_17686_amd import ficoco as fc
from tests.share_records import Records, up
from tests.test_gpu_cache_attention import check, ctx, dense, i32  # noqa: F401
from tests.test_gpu_shared_attention import family, queries

pytestmark = pytest.mark.gpu


def plan(ctx, c, B, H, n_q, groups, window=0, sinks=0, max_len=0, always=True, **arrays):  # noqa: F811
    share = fc.Share(c, B, H, n_q, window=window, sinks=sinks, max_len=max_len)
    share.plan.t.fill_(255)
    share.ws.t.fill_(255)
    fc.ficoco_cache_share(ctx, c, share, group=i32(groups), always=always, **arrays)
    return share, Records(share, c.c.heads, max_len, c.c.max_pages * c.c.page_size)


@pytest.mark.parametrize("seed", range(24))
def test_records_of_drawn_tables(ctx, seed):  # noqa: F811
    """Tables alone: a plan reads nothing else.  Families of all sizes, slots named twice or not at all, fewer queries than n_q and none, windows."""
    r = random.Random(seed)
    for _ in range(6):
        g, n_q, page = r.choice([1, 2, 4, 7]), int(2 ** (r.random() * 6.5)), r.choice([16, 32, 64, 128])
        B = r.choice([1, 2, 5, 16, 17, 40, 150, 600]) if n_q * g < 64 else r.choice([1, 3, 16, 30])
        heads = r.choice([1, 2, 8, 32, 200, 600] if B < 20 else [1, 2, 8, 32])
        longest = int(2 ** r.uniform(4, 14 if B < 100 else 11))
        n_seqs, width = max(1, B - r.randint(0, 2)), up(longest, page) + 1
        prompts = [[r.randrange(10 ** 6) for _ in range(width)] for _ in range(r.choice([1, 1, 2, 5]))]
        table, lens = np.zeros((n_seqs, width), np.int32), []
        for s in range(n_seqs):
            p, n = r.choice(prompts), r.choice([0, width, r.randint(0, width), r.randint(0, width)])
            table[s] = p[:n] + [r.randrange(10 ** 6) for _ in range(width - n)]
            lens.append(r.choice([longest, r.randint(0, longest), r.randint(max(0, longest - 40), longest)]))
        c = fc.Cache.empty(1, 1, page, heads, 64, n_seqs, width)
        c.table.copy_(torch.from_numpy(table))
        c.len.copy_(torch.tensor(lens, dtype=torch.int32))
        slots = [r.choice([b, b, b, r.randint(-1, n_seqs)]) for b in range(B)]
        ok = [0 <= s < n_seqs for s in slots]
        names = [r.choice([0, 0, 0, b % 3 if B > 2 else 0, b, -1, B]) if r.random() < 0.8 else 0 for b in range(B)]
        q_lens = [r.choice([n_q, n_q, n_q + 1, r.randint(-1, n_q)]) for _ in range(B)]
        window = r.choice([0, 0, 1, 100, longest])
        sinks = r.choice([0, 4, 70]) if window else 0
        arrays = dict(seq=i32(slots), q_len=i32(q_lens))
        keys = [lens[s] if o else 0 for s, o in zip(slots, ok)]
        queries_ = [min(max(q, 0), n_q) for q in q_lens]
        starts = [k - q for k, q in zip(keys, queries_)]
        if r.random() < 0.3:
            starts = [r.randint(-5, longest + 5) for _ in range(B)]
            arrays["q_start"] = i32(starts)
        max_len = r.choice([0, 0, longest, 64])
        print(seed, dict(B=B, heads=heads, g=g, n_q=n_q, page=page, longest=longest, window=window, sinks=sinks, max_len=max_len), flush=True)
        _, rec = plan(ctx, c, B, heads * g, n_q, names, window, sinks, max_len, **arrays)
        taken = [x if 0 <= x < B and o else -1 for x, o in zip(names, ok)]
        rec.verify(table, page, keys, starts, queries_, [s if o else 0 for s, o in zip(slots, ok)], taken, window, sinks)


FEW, MANY = 1, 0
CHAINS = [  # families, page, heads, query heads a head, d, n_q, window, sinks; what one workgroup takes after what (16 rows straight from memory, 128 through LDS)
    ([(2100, [2160]), (1100, [2600, 2601, 2602])], 128, 4, 2, 128, 48, 0, 0, {(FEW, FEW), (FEW, MANY), (MANY, FEW), (MANY, MANY)}),
    ([(700, [760]), (1100, [1160]), (1100, [1160, 1161])], 64, 4, 4, 128, 20, 0, 0, {(FEW, FEW), (MANY, FEW), (MANY, MANY)}),
    ([(1100, [1160, 1161]), (700, [760])], 16, 4, 4, 64, 33, 0, 0, {(FEW, FEW), (FEW, MANY), (MANY, MANY)}),
    ([(1100, [2600, 2601])], 32, 4, 4, 64, 20, 0, 0, {(MANY, MANY)}),
    ([(2100, [2160 + i for i in range(3)]), (1100, [2600 + i for i in range(8)])], 32, 32, 1, 64, 33, 0, 0, {(MANY, MANY)}),
    ([(700, [760]), (1100, [2600 + i for i in range(8)]), (2100, [3600 + i for i in range(24)])], 64, 8, 4, 128, 1, 0, 0, {(FEW, FEW), (FEW, MANY), (MANY, FEW)}),
    ([(2100, [2160]), (1100, [2600, 2601, 2602])], 128, 4, 2, 128, 48, 1800, 600, {(FEW, FEW), (FEW, MANY), (MANY, FEW), (MANY, MANY)}),
]


@pytest.mark.parametrize("case", CHAINS, ids=str)
def test_workgroups_that_go_on_with_another_tile(ctx, case):  # noqa: F811
    families, page, heads, g, d, n_q, window, sinks, pairs = case
    c, lens, groups = family(ctx, page, heads, d, families)
    B, H = len(lens), heads * g
    share, rec = plan(ctx, c, B, H, n_q, groups, window, sinks)
    starts, slots = [n - n_q for n in lens], list(range(B))
    chained = rec.verify(c.table.cpu().numpy(), page, lens, starts, [n_q] * B, slots, groups, window, sinks)
    assert pairs <= set(chained), set(chained)
    Q = queries(B, H, n_q, d)
    outs = []
    for layer in (1, 0, 1):
        O = torch.full_like(Q, 77.0)
        fc.ficoco_cache_shared_attention(ctx, c, layer, share, Q, O)
        outs.append(O)
    assert torch.equal(outs[0], outs[2])
    for layer in (0, 1):
        k, v = dense(ctx, c, layer, max(lens))
        check(outs[1 - layer], Q, k, v, lens, d ** -0.5, starts, [n_q] * B, window, sinks, g)
