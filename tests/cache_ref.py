"""The decoder's cache and its attention as plain statements: numpy integers for the pages, float64 for the values.
Nothing here comes from the library."""
import numpy as np
import torch

E4M3 = np.array([float(v) for v in torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).float()])


def exponent(block):
    """The byte of a block: the smallest e >= 17 with max|x| <= 448 * 2^(e - 127) over the finite values."""
    a = np.abs(np.asarray(block, np.float64))
    a = a[np.isfinite(a)]
    top = a.max() if a.size else 0.0
    e = 17
    while top > 448.0 * 2.0 ** (e - 127):
        e += 1
    return e


_GRID = E4M3[:127]                       # 0 .. 448 ascending


def encode(x, e):
    """The E4M3 byte nearest to x * 2^(127 - e), ties to the even byte."""
    y = np.asarray(x, np.float64) * 2.0 ** (127 - e)
    a = np.minimum(np.abs(y), 448.0)
    a0 = np.where(np.isnan(a), 0.0, a)
    hi = np.clip(np.searchsorted(_GRID, a0), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a0 - _GRID[lo], _GRID[hi] - a0
    b = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(y), 127, b + 128 * np.signbit(y)).astype(np.uint8)


class Cache:
    """The host's model of a cache."""

    def __init__(self, layers, n_pages, page, heads, d, n_seqs, max_pages):
        self.P, self.n_pages, self.max_pages, self.layers, self.heads, self.d = page, n_pages, max_pages, layers, heads, d
        self.q = {x: np.zeros((layers, n_pages, heads, page, d), np.uint8) for x in "kv"}
        self.e = {x: np.zeros((layers, n_pages, heads), np.uint8) for x in "kv"}
        self.table = np.full((n_seqs, max_pages), -1, np.int32)
        self.len = np.zeros(n_seqs, np.int32)
        self.refs = np.zeros(n_pages, np.int32)

    def pages(self, n):
        return -(-n // self.P)

    def ok(self, s):
        return 0 <= s < len(self.len)

    def serve(self, needs):
        """Free pages for entries in order, None for those that are not served."""
        free = [int(p) for p in np.nonzero(self.refs == 0)[0]]
        got, short = [], False
        for n in needs:
            if n == 0:
                got.append([])
            elif short or n > len(free):
                short = True
                got.append(None)
            else:
                got.append(free[:n])
                free = free[n:]
        return got

    def reserve(self, seq, n_new):
        seen, want, ok = set(), [], []
        for s, n in zip(seq, n_new):
            good = self.ok(s) and s not in seen and n >= 0 and self.len[s] + n <= self.max_pages * self.P
            if self.ok(s):
                seen.add(s)
            ok.append(good)
            want.append(self.pages(self.len[s] + n) - self.pages(self.len[s]) if good else 0)
        start = []
        for s, n, good, got in zip(seq, n_new, ok, self.serve(want)):
            if not good or got is None:
                start.append(-1)
                continue
            have = self.pages(self.len[s])
            self.table[s, have:have + len(got)] = got
            self.refs[got] = 1
            start.append(int(self.len[s]))
            self.len[s] += n
        return start

    def append(self, layer, K, V, start, n_new, seq):
        """K, V: [n][heads][n_max][d] float64."""
        for b, s in enumerate(seq):
            if not self.ok(s) or start[b] < 0:
                continue
            t, stop = start[b], start[b] + n_new[b]
            while t < stop:
                till = min(stop, (t // self.P + 1) * self.P)
                at = t // self.P
                p = self.table[s, at] if at < self.max_pages else -1
                if 0 <= p < self.n_pages:
                    for x, T in (("k", K), ("v", V)):
                        for h in range(self.heads):
                            new = T[b, h, t - start[b]:till - start[b]]
                            q, old = self.q[x][layer, p, h], int(self.e[x][layer, p, h])
                            e = exponent(new)
                            lo = t % self.P
                            if lo:
                                e = max(e, old)
                                if e != old:
                                    q[:lo] = encode(E4M3[q[:lo]] * 2.0 ** (old - 127), e)
                            q[lo:lo + till - t] = encode(new, e)
                            self.e[x][layer, p, h] = e
                t = till

    def values(self, x, layer, s, t):
        """[heads][d] of one token, zeros where it has no page."""
        at = t // self.P
        p = self.table[s, at] if self.ok(s) and at < self.max_pages else -1
        if not 0 <= p < self.n_pages:
            return np.zeros((self.heads, self.d))
        return E4M3[self.q[x][layer, p, :, t % self.P]] * 2.0 ** (self.e[x][layer, p].astype(np.float64) - 127)[:, None]

    def fork(self, src, dst, whole):
        seen, want, ok = set(), [], []
        targets = {d for d in dst if self.ok(d)}
        for s, d in zip(src, dst):
            good = self.ok(s) and self.ok(d) and d not in seen and s not in targets and self.len[d] == 0
            if self.ok(d):
                seen.add(d)
            ok.append(good)
            want.append(self.pages(self.len[s]) - (0 if whole else self.len[s] // self.P) if good else 0)
        done = []
        for s, d, good, got in zip(src, dst, ok, self.serve(want)):
            done.append(int(good and got is not None))
            if not done[-1]:
                continue
            pages = self.pages(self.len[s])
            shared = pages - len(got)
            self.table[d, :shared] = self.table[s, :shared]
            np.add.at(self.refs, self.table[s, :shared], 1)
            for i, p in enumerate(got):
                self.table[d, shared + i] = p
                self.refs[p] = 1
                for x in "kv":
                    self.q[x][:, p] = self.q[x][:, self.table[s, shared + i]]
                    self.e[x][:, p] = self.e[x][:, self.table[s, shared + i]]
            self.len[d] = self.len[s]
        return done

    def compact(self, layers, src, dst, v, N, keep):
        seen, want, ok, plans = set(), [], [], []
        targets = {d for d in dst if self.ok(d)}
        for b, (s, d) in enumerate(zip(src, dst)):
            good = (self.ok(s) and self.ok(d) and d not in seen and (s == d or s not in targets) and self.len[s] >= v + N
                    and (s == d or self.len[d] == 0))
            if self.ok(d):
                seen.add(d)
            tokens, same = [], 0
            if good:
                tokens = list(range(v)) + [v + int(k) for k in keep[b]] + list(range(v + N, self.len[s]))
                first = next((i for i, t in enumerate(tokens) if i != t), len(tokens))
                same = first // self.P
                if s == d and len(tokens) == self.len[s]:
                    same = self.pages(len(tokens))
            ok.append(good)
            want.append(self.pages(len(tokens)) - same if good else 0)
            plans.append((tokens, same))
        got = self.serve(want)
        old = self.table.copy()
        for s, d, good, new, (tokens, same) in zip(src, dst, ok, got, plans):
            if not good or new is None:
                continue
            if s == d:
                for i in range(same, self.pages(self.len[s])):
                    self.refs[old[s, i]] -= 1
                    self.table[s, i] = -1
            else:
                self.table[d, :same] = old[s, :same]
                np.add.at(self.refs, old[s, :same], 1)
            for i, p in enumerate(new):
                self.table[d, same + i] = p
                self.refs[p] = 1
                at = tokens[(same + i) * self.P:(same + i + 1) * self.P]
                for x in "kv":
                    for l in layers:
                        for h in range(self.heads):
                            val = np.stack([E4M3[self.q[x][l, old[s, t // self.P], h, t % self.P]] *
                                            2.0 ** (float(self.e[x][l, old[s, t // self.P], h]) - 127) for t in at])
                            e = exponent(val)
                            self.q[x][l, p, h, :len(at)] = encode(val, e)
                            self.e[x][l, p, h] = e
            self.len[d] = len(tokens)
        return [int(g and n is not None) for g, n in zip(ok, got)]

    def free(self, seq):
        for s in seq:
            if self.ok(s):
                for p in self.table[s]:
                    if 0 <= p < self.n_pages:
                        self.refs[p] -= 1
                self.table[s] = -1
                self.len[s] = 0


def attention(q, k, v, scale, pos, window, sinks, have=None):
    """One query head in float64: q [r][d] at positions pos [r], k and v [n][d].  Returns the rows, and the bound of the kernels'
    error: the result is rounded to bfloat16 (half a step: 2^-8 of it); so is each weight (2^-8 of sum w|v|); a logit is a sum of d
    exact products in single precision, each addition off by 2^-24 of the magnitudes so far, and enters the weight and the sum of
    the weights; exponential, scaling and the sums of n terms are single precision too."""
    n, d = k.shape
    j = np.arange(n)
    see = j[None, :] <= np.asarray(pos)[:, None]
    if window:
        see &= (j[None, :] > np.asarray(pos)[:, None] - window) | (j[None, :] < sinks)
    if have is not None:
        see &= have[None, :]
    if n == 0:
        return np.zeros((len(pos), d)), np.zeros((len(pos), d))
    logit = np.where(see, scale * (q @ np.where(np.isfinite(k), k, 0.0).T), -np.inf)
    top = np.max(logit, axis=1, initial=-1e300)
    w = np.exp(logit - top[:, None])
    total = w.sum(1)
    some = total > 0
    w = np.where(some[:, None], w / np.where(some, total, 1.0)[:, None], 0.0)
    vv = np.where(np.isfinite(v), v, 0.0)
    out = w @ vv
    size = scale * (np.abs(q) @ np.abs(np.where(np.isfinite(k), k, 0.0)).T)
    delta = (d + 4) * 2.0 ** -24 * np.max(np.where(see, size, 0.0), axis=1) + 2.0 ** -20
    bound = 2.0 ** -8 * np.abs(out) + ((2.0 ** -8 + 2 * delta + n * 2.0 ** -24)[:, None] if np.ndim(delta) else 0) * (w @ np.abs(vv)) * 1.01 + 1e-30
    return out, bound
