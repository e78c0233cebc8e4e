"""The records of a plan of sequences that share pages, as the device leaves them, and what has to hold for them: every block of every tile is taken once, by an item whose part of
the result has rows of its own, and the join reads the parts that were written."""
import numpy as np

KEYS, TILE = 64, 128                 # keys of a block; rows of a tile where there are many (else 16)

_OWNER = [(n, "<i4") for n in ("owner", "slot", "from", "keys", "lo", "hi", "rows", "few", "blocks", "tiles", "part", "part_rows", "part_pieces", "cut", "stride", "pad")]
OWNER = np.dtype(_OWNER)
ITEM = np.dtype(_OWNER + [(n, "<i4") for n in ("tile", "i0", "i1", "part_at", "next", "pad1", "pad2", "pad3")])
_PARTS = [("at", "<f8")] + [(n, "<i4") for n in ("blocks", "part", "rows", "pieces", "tile", "cut", "stride", "pad")]
ENTRY = np.dtype([("own", _PARTS), ("group", _PARTS), ("queries", "<i4"), ("direct", "<i4"), ("row0", "<i4"), ("pad", "<i4")])
MEMBER = np.dtype([(n, "<i4") for n in ("b", "first", "queries", "pad")])
assert (OWNER.itemsize, ITEM.itemsize, ENTRY.itemsize, MEMBER.itemsize) == (64, 96, 96, 16)


def up(a, b):
    return -(-a // b)


class Records:
    def __init__(self, share, heads, max_len, room):
        """share: an fc.Share with a plan; heads: key / value heads; room: tokens that a row of the table holds."""
        B, H, n_q, d = share.shape
        self.B, self.heads, self.R, self.group = B, heads, n_q * (H // heads), H // heads
        at = share.plan.ptr - share.plan.t.data_ptr()
        raw = share.plan.t[at:at + share.plan.bytes].cpu().numpy()
        self.unit = int(raw[8:12].view("<i4")[0])
        at = 256
        for name, dtype, n in (("entries", ENTRY, B), ("members", MEMBER, B), ("owners", OWNER, 2 * B)):
            setattr(self, name, raw[at:at + n * dtype.itemsize].view(dtype))
            at += up(n * dtype.itemsize, 256) * 256
        self.items = raw[at:at + (len(raw) - at) // ITEM.itemsize * ITEM.itemsize].view(ITEM)
        few = up(self.R, 16)
        self.own_tile = 16 if few <= 1 or (few <= 4 and B * heads * few <= (1024 if few <= 3 else 512)) else TILE
        longest = min(room, max_len) if max_len else room
        self.pieces = max(1, min(max(1, 512 // heads), B * up(self.R, self.own_tile) * up(longest, 256)))
        # which of `owners` a record's owner is
        self.index = {b: 2 * b + 1 for b in range(B)}
        self.index.update({int(self.owners[i]["owner"]): i for i in range(0, 2 * B, 2) if self.owners[i]["tiles"] > 0})
        assert len(self.index) == B + int((self.owners["tiles"][::2] > 0).sum())
        self.part_rows = share.ws.bytes // (heads * (4 * d + 8))           # that the workspace has room for

    def live(self):
        """(number, item) of all that have work, where workgroups begin and where they go on, and the pairs (few, few) of items that one workgroup takes one after the other."""
        found, chained, begun = [], [], list(range(self.pieces)) + list(range(2 * self.pieces, len(self.items)))
        for i in begun:
            it = self.items[i]
            if it["owner"] == -1:
                continue
            found.append((i, it))
            if it["next"] >= 0:
                n = int(it["next"])
                assert self.pieces <= n < 2 * self.pieces and i < self.pieces
                after = self.items[n]
                assert after["owner"] != -1 and after["next"] == -1
                found.append((n, after))
                chained.append((int(it["few"]), int(after["few"])))
        assert len({i for i, _ in found}) == len(found)          # nothing is taken twice
        return found, chained

    def verify(self, table, page, lens, starts, q_lens, slots, groups, window, sinks):
        """Against the row of the table, keys, first position and queries of each entry; groups: who is taken together (-1: for itself).  Returns the pairs of live()."""
        B, R = self.B, self.R
        # ---- what is common
        first, members = {}, {}
        for b in range(B):
            if groups[b] >= 0 and q_lens[b] > 0:
                members.setdefault(groups[b], []).append(b)
        held = {}
        for m in members.values():
            n = min(lens[b] // page for b in m)
            while not all(np.array_equal(table[slots[b], :n], table[slots[m[0]], :n]) for b in m):
                n = int(next(np.nonzero(table[slots[b], :n] != table[slots[m[0]], :n])[0][0] for b in m if not np.array_equal(table[slots[b], :n], table[slots[m[0]], :n])))
            if len(m) > 1:
                held[m[0]] = n * page // KEYS * KEYS
            first.update({b: m[0] for b in m})

        def seen(lo, hi, keys, begin):
            """Blocks from `begin` on of which a query at lo .. hi sees a key."""
            j = np.arange(begin, max(begin, min(keys, hi + 1)))
            j = j[(j > lo - window) | (j < sinks)] if window else j
            return len(set((j // KEYS).tolist()))

        for b in range(B):
            own, shared = self.owners[2 * b + 1], held.get(first.get(b, -1), 0)
            assert (own["owner"], own["from"], own["keys"], own["rows"], own["slot"]) == (b, shared, lens[b], q_lens[b] * self.group, slots[b])
            assert own["tiles"] == up(int(own["rows"]), self.own_tile) and bool(own["few"]) == (self.own_tile == 16)
            if own["rows"]:
                assert (own["lo"], own["hi"]) == (starts[b], starts[b] + q_lens[b] - 1)
                assert 0 <= own["blocks"] - seen(int(own["lo"]), int(own["hi"]), lens[b], shared) <= 1
            all_, e = self.owners[2 * b], self.entries[b]
            assert e["queries"] == q_lens[b]
            if held.get(b, 0) > 0:
                m = members[groups[b]]
                lo, hi = min(starts[x] for x in m), max(starts[x] + q_lens[x] - 1 for x in m)
                assert (all_["from"], all_["keys"], all_["rows"], all_["lo"], all_["hi"], all_["slot"]) == (0, held[b], len(m) * R, lo, hi, slots[b])
                assert all_["tiles"] == up(len(m) * R, 16 if all_["few"] else TILE) and 0 <= all_["blocks"] - seen(lo, hi, held[b], 0) <= 1
                at = -2 - int(all_["owner"])
                assert [tuple(x)[:3] for x in self.members[at:at + len(m)]] == [(x, starts[x], q_lens[x]) for x in m]
                assert [int(self.entries[x]["row0"]) for x in m] == [i * R for i in range(len(m))]
            else:
                assert all_["tiles"] == 0
            assert (e["group"]["pieces"] > 0) == (shared > 0)

        # ---- every block of every tile once
        taken, rows = {}, []
        found, chained = self.live()
        for _, it in found:
            i = self.index[int(it["owner"])]
            o = self.owners[i]
            assert all(it[n] == o[n] for n in OWNER.names if n != "pad") and 0 <= it["tile"] < o["tiles"]
            taken.setdefault((i, int(it["tile"])), []).append((int(it["i0"]), min(int(it["i1"]), int(o["blocks"])), int(it["part_at"])))
            if it["part_at"] >= 0:
                rows.append((int(it["part_at"]), int(it["part_at"] + o["part_rows"])))
            else:
                assert o["part"] == -1 and not o["cut"]
        rows.sort()
        assert all(x[1] <= y[0] for x, y in zip(rows, rows[1:])) and (not rows or (rows[0][0] >= 0 and rows[-1][1] <= self.part_rows))
        for i, o in enumerate(self.owners):
            for t in range(o["tiles"]):
                got = sorted(taken.pop((i, t)))
                assert got[0][0] == 0 and got[-1][1] == o["blocks"] and all(x[1] == y[0] for x, y in zip(got, got[1:])) and (len(got) == 1 or all(x[0] < x[1] for x in got)), (i, t, got)
                taken[i, t, "parts"] = [p for _, _, p in got]
        assert all(len(k) == 3 for k in taken)

        # ---- the join reads what is written
        for b in range(B):
            e = self.entries[b]
            for which, i in (("own", 2 * b + 1), ("group", 2 * first.get(b, b))):
                p, o = e[which], self.owners[i]
                if e["direct"] or not q_lens[b] or p["pieces"] == 0:
                    continue
                assert p["part"] >= 0 and p["rows"] == o["part_rows"]
                for r in range(0 if which == "own" else int(e["row0"]), (0 if which == "own" else int(e["row0"])) + q_lens[b] * self.group):
                    t, count = r // int(p["tile"]), 1
                    if p["cut"]:
                        begin = int(p["at"]) + t * int(p["stride"])
                        count = (begin + int(p["blocks"]) - 1) // self.unit - begin // self.unit + 1
                    assert r - t * p["tile"] < p["rows"]
                    assert [int(p["part"] + (t * p["pieces"] + j) * p["rows"]) for j in range(count)] == taken[i, t, "parts"], (b, which, r)
            assert not e["direct"] or (e["own"]["part"] == -1 and e["group"]["pieces"] == 0)
        return chained
