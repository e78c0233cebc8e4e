"""How the blocks of sequences that share pages are cut over workgroups, on the host: the rule of share.hip as a model, held against the sizes that the library gives for plan and workspace.  Every block of
every tile is taken once, by the workgroup whose part the join expects, and nothing lies behind the end of the plan or of the workspace."""
import ctypes as C
import random
from bisect import bisect_right

import pytest

from paper_2411_17686_amd import ficoco as fc
from tests.test_cache_abi import _attention, _cache

LEAST, MOST, FEW_WORK = 4, 512, 2100
ENTRY, MEMBER, OWNER, ITEM = 96, 16, 64, 96          # bytes of a plan's records


def up(a, b):
    return -(-a // b)


def sizes(B, heads, group, n_q, d, max_pages, page, max_len):
    """Items of the plan, and rows of parts in the workspace."""
    c = _cache(heads=heads, d_head=d, page_size=page, max_pages=max_pages)
    a = _attention(B=B, H=heads * group, n_q=n_q, d_head=d, max_len=max_len)
    plan, ws = C.c_size_t(), C.c_size_t()
    rc = fc.lib().ficoco_cache_share_bytes(C.byref(c), C.byref(a), C.byref(plan), C.byref(ws))
    if rc == fc.EUNSUPPORTED and B * heads * group * n_q > 1 << 20:          # (more rows than a launch takes)
        return None
    assert rc == fc.OK
    items = (plan.value - 256 - sum(up(n, 256) * 256 for n in (B * ENTRY, B * MEMBER, 2 * B * OWNER))) // ITEM
    return items, ws.value // (heads * (4 * d + 8))


def cut(case, r):
    B, heads, R, longest = case["B"], case["heads"], case["n_q"] * case["group"], up(case["longest"], case["page"]) * case["page"]
    few = up(R, 16)
    own_tile = 16 if few <= 1 or (few <= 4 and B * heads * few <= (1024 if few <= 3 else 512)) else 128
    pieces = max(1, min(max(1, MOST // heads), B * up(R, own_tile) * up(longest, 256)))
    room = sizes(B, heads, case["group"], case["n_q"], case["d"], longest // case["page"], case["page"], 0)
    if room is None:
        return
    most_items, most_parts = room
    blocks = lambda: r.choice([r.randint(0, up(longest, 64)), r.randint(0, 4), up(longest, 64)])
    names = [r.randrange(case["groups"]) if case["groups"] and r.random() < 0.9 else -1 for _ in range(B)]
    members = {}
    for b, x in enumerate(names):
        if x >= 0:
            members.setdefault(x, []).append(b)
    own = [(up(case["group"] * r.choice([case["n_q"], case["n_q"], r.randint(0, case["n_q"])]), own_tile), blocks(), min(R, own_tile)) for _ in range(B)]
    common = [(0, 0, 0)] * B
    shared = set()
    for m in members.values():
        n = blocks()
        if len(m) > 1 and n:
            rows = len(m) * R
            small, large = up(rows, 16), up(rows, 128)
            tile = 16 if 3 * small <= 8 * large or (3 * small - 8 * large) * n * heads < FEW_WORK else 128
            common[m[0]] = (up(rows, tile), n, min(rows, tile))
            shared.update(m)
    owners = [o for pair in zip(common, own) for o in pair]
    unit = max(LEAST, (sum(t * n for t, n, _ in owners) + pieces - 1) // pieces)
    larger = unit + max(unit // 8, 5)
    whole = lambda u: sum(t * up(n, u) for t, n, _ in owners if n > u)
    apart = whole(unit) <= pieces or whole(larger) <= pieces
    if whole(unit) > pieces and apart:
        unit = larger
    at, cuts, items, parts, starts, counts, records = 0, 0, 0, 0, [], [], []
    for i, (t, n, rows) in enumerate(owners):
        is_cut = n > unit
        room = n // unit + 2 if is_cut else 1
        stride = up(n, unit) * unit if apart else n
        starts.append(at)
        counts.append(cuts)
        direct = i % 2 == 1 and i // 2 not in shared and not is_cut
        records.append((t, n, is_cut, room, stride))
        if is_cut:
            at, cuts = at + t * stride, cuts + t
        else:
            items += t
        parts += 0 if direct else t * room * rows
    assert cuts <= pieces and 2 * pieces + items <= most_items and parts <= most_parts, (cuts, pieces, items, most_items, parts, most_parts)
    assert at <= pieces * unit
    taken = {}
    for w in range(pieces):
        if w * unit >= at:
            break
        i = bisect_right(starts, w * unit) - 1
        t, n, is_cut, room, stride = records[i]
        tile, i0 = divmod(w * unit - starts[i], stride)
        assert is_cut and tile < t and i0 < n
        i1, piece, after = min(i0 + unit, n), w - (starts[i] + tile * stride) // unit, counts[i] + tile + 1
        assert 0 <= piece < room
        taken.setdefault((i, tile), []).append((piece, i0, i1))
        if not apart and i1 - i0 < unit and after < cuts:          # goes on with the next tile
            i = bisect_right(counts, after) - 1
            t, n, is_cut, room, stride = records[i]
            behind = (starts[i] + (after - counts[i]) * n) % unit
            assert is_cut and behind and unit - behind <= n and i1 - i0 == behind
            taken.setdefault((i, after - counts[i]), []).append((0, 0, unit - behind))
    for i, (t, n, is_cut, room, stride) in enumerate(records):
        for tile in range(t if is_cut else 0):
            first = starts[i] + tile * stride
            count = (first + n - 1) // unit - first // unit + 1
            got = sorted(taken[i, tile])
            assert [p for p, _, _ in got] == list(range(count)) and count <= room
            assert got[0][1] == 0 and got[-1][2] == n and all(x[2] == y[1] for x, y in zip(got, got[1:]))


@pytest.mark.parametrize("seed", range(8))
def test_every_block_is_taken_once(seed):
    r = random.Random(seed)
    for _ in range(120):
        B = int(2 ** (r.random() * 10))
        cut(dict(B=B, heads=r.choice([1, 2, 4, 8, 32, 600]), group=r.choice([1, 2, 4, 7]), n_q=int(2 ** (r.random() * 7)), d=r.choice([64, 128]), page=r.choice([16, 64, 128]),
                 longest=int(2 ** (r.random() * 16)), groups=r.choice([0, 1, 1, 2, max(1, B // 3), B])), r)


def test_sizes_that_are_refused():
    call = lambda c, a: fc.lib().ficoco_cache_share_bytes(C.byref(c), C.byref(a), C.byref(C.c_size_t()), C.byref(C.c_size_t()))
    assert call(_cache(), _attention(B=1024)) == fc.OK
    for c, a, code in ((_cache(), _attention(B=1025), fc.EUNSUPPORTED), (_cache(), _attention(H=6), fc.EINVAL), (_cache(page_size=48), _attention(), fc.EUNSUPPORTED),
                       (_cache(), _attention(n_q=1 << 28), fc.EUNSUPPORTED), (_cache(), _attention(window=-1), fc.EINVAL)):
        assert call(c, a) == code
    assert fc.lib().ficoco_cache_share_bytes(None, None, None, None) == fc.EINVAL
    assert fc.lib().ficoco_cache_share(None, None, None, None, 0, None, 0, None) == fc.EINVAL
    assert fc.lib().ficoco_cache_shared_attention(None, None, 0, None, None, 0, None, 0, None) == fc.EINVAL
