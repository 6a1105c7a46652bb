"""Plain restatements, in 64 bits and with Python lists, of what the calls on a growing cache do (for the tests)."""
import math

import torch

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def frequencies(dim, base=10000.0, scaling="none", factor=1.0, original=0, low=1.0, high=4.0):
    """(frequencies, magnitude) from the definitions."""
    if scaling == "ntk":
        base = base * factor ** (dim / (dim - 2))
    out = []
    for i in range(dim // 2):
        f = base ** (-2 * i / dim)
        if scaling == "linear":
            f /= factor
        elif scaling == "llama3":
            turns = original * f / (2 * math.pi)
            if turns <= low:
                f /= factor
            elif turns < high:
                s = (turns - low) / (high - low)
                f = s * f + (1 - s) * f / factor
        elif scaling == "yarn":
            pair = lambda t: dim * math.log(original / (t * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
            lo, hi = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), dim - 1)
            s = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f = (1 - s) * f + s * f / factor
        out.append(f)
    return out, 0.1 * math.log(factor) + 1 if scaling == "yarn" else 1.0


def rotate(x, positions, freq, magnitude, layout, inverse=False):
    """x [..., tokens, d] -> (turned rows, |x| + |y| of each element's pair times the magnitude), float64."""
    r = 2 * len(freq)
    angle = positions.double()[..., None] * torch.tensor(freq, dtype=torch.float64)
    angle = -angle if inverse else angle
    y, size = x.double().clone(), x.double().abs()
    a, b = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    p, q = x.double()[..., a], x.double()[..., b]
    y[..., a] = magnitude * (p * angle.cos() - q * angle.sin())
    y[..., b] = magnitude * (q * angle.cos() + p * angle.sin())
    both = abs(magnitude) * (p.abs() + q.abs())
    size[..., a], size[..., b] = both, both
    return y, size


def assert_rotated(got, want, size, what=""):
    """The angle is off by at most 2 pi 2^-26 (half a turn rounded to fp32), sine and cosine by an ulp, 2^-24 each; magnitude,
    its products with them and the two products of the pair round four times more: 4.1e-7 of |x| + |y|; then one rounding to
    the type (of what it is given: a little more than half a step of the exact value)."""
    bound = 4.1e-7 * size + 1.001 * HALF_STEP[got.dtype] * want.abs() + 3.1e-8 * (got.dtype == torch.float16)
    bad = (got.double() - want).abs() > bound
    assert not bad.any(), "%s: %d of %d rotated elements are off, worst %g" % (what, int(bad.sum()), bad.numel(), float(((got.double() - want).abs() - bound).max()))


def attend(q, k, v, *, positions=None, q_position=None, scale=None, softcap=0.0, slopes=None, window=0, prefix=0):
    """q [group][d], k, v [rows][d] of one head -> (out, lse, sum of weights times |v|), float64; rows that are not seen left out."""
    keep = torch.ones(k.shape[0], dtype=torch.bool)
    if q_position is not None:
        far = q_position - positions.long()
        keep = far >= 0
        if window:
            keep &= (far < window) | (positions < prefix)
    k, v = k[keep].double(), v[keep].double()
    if k.shape[0] == 0:
        zero = torch.zeros(q.shape, dtype=torch.float64)
        return zero, torch.full((q.shape[0],), -math.inf, dtype=torch.float64), zero
    x = q.double() @ k.T * (scale if scale else 1 / math.sqrt(q.shape[1]))
    if softcap:
        x = softcap * torch.tanh(x / softcap)
    if slopes is not None:
        x = x - slopes.double()[:, None] * far[keep].double()
    w = torch.softmax(x, -1)
    return w @ v, torch.logsumexp(x, -1), w @ v.abs()


class ListCache:
    """The tables of a cache as Python lists, and the page calls on them."""

    def __init__(self, tables, lens, refs, page):
        self.tables, self.lens, self.refs, self.page = tables.tolist(), lens.tolist(), refs.tolist(), page
        self.max_pages = tables.shape[3]
        self.heads = tables.shape[2]

    def pages(self, n):
        return -(-n // self.page)

    def fork(self, parents, add):
        """-> (granted, copies [(source page, page, rows)]) or None if the call cannot be met (nothing changes)."""
        layers, batch = len(self.lens), len(self.lens[0])
        if any(p < -1 or p >= batch for p in parents):
            return None
        refs = list(self.refs)
        kept, counts = [], []
        for l in range(layers):
            for b in range(batch):
                children = [c for c, p in enumerate(parents) if p == b]
                n, full = self.lens[l][b], self.lens[l][b] // self.page
                for h in range(self.heads):
                    for j, page in enumerate(self.tables[l][b][h][:self.pages(n)]):
                        refs[page] += (len(children) if j < full else min(1, len(children))) - 1
        free = [i for i, r in enumerate(refs) if r == 0]
        tables, lens, copies, taken = [], [], [], 0
        for l in range(layers):
            tables.append([])
            lens.append([])
            for c, p in enumerate(parents):
                more = max(0, add[l][c])
                old = self.lens[l][p] if p >= 0 else 0
                n, full, part = old + more, old // self.page, old % self.page
                if self.pages(n) > self.max_pages:
                    return None
                first = c == parents.index(p) or p < 0
                rows = []
                for h in range(self.heads):
                    row = list(self.tables[l][p][h][:full + (1 if part and first else 0)]) if p >= 0 else []
                    while len(row) < self.pages(n):
                        if taken >= len(free):
                            return None
                        if part and not first and len(row) == full:
                            copies.append((self.tables[l][p][h][full], free[taken], part))
                        row.append(free[taken])
                        refs[free[taken]] = 1
                        taken += 1
                    rows.append(row)
                tables[l].append(rows)
                lens[l].append(n)
                counts.append(more)
        self.tables, self.lens, self.refs = tables, lens, refs
        return counts, copies

    def compact(self):
        """-> (pages in use, moves [(source page, page)])."""
        used = sum(r > 0 for r in self.refs)
        holes = [i for i, r in enumerate(self.refs) if r == 0 and i < used]
        movers = [i for i, r in enumerate(self.refs) if r > 0 and i >= used]
        place = dict(zip(movers, holes))
        for l, row in enumerate(self.tables):
            for b, heads in enumerate(row):
                for h, pages in enumerate(heads):
                    n = self.pages(self.lens[l][b])
                    heads[h] = [place.get(p, p) for p in pages[:n]]
        for s, t in place.items():
            self.refs[t], self.refs[s] = self.refs[s], 0
        return used, list(place.items())

    def check(self, tables, lens, refs):
        """Device tensors against the lists; table entries behind a sequence's last page are not looked at."""
        assert lens.tolist() == self.lens
        assert refs.tolist() == self.refs
        got = tables.tolist()
        for l, row in enumerate(self.tables):
            for b, heads in enumerate(row):
                for h, pages in enumerate(heads):
                    n = self.pages(self.lens[l][b])
                    assert got[l][b][h][:n] == pages[:n], (l, b, h)

    def row(self, l, b, h, r):
        return self.tables[l][b][h][r // self.page] * self.page + r % self.page
