"""Plain fp64 checkers of the token policy's operators (test infrastructure only): attention over a paged cache, the pages'
life, adjusted logits and draws.  Everything is written from the definitions in the C header, one row and one page at a time."""
import numpy as np

from . import philox

STREAM_TOKEN = 2


# ---------------------------------------------------------------- 8-bit codes

def e4m3_values():
    """The 256 values of the 8-bit format with 4 bits of exponent (bias 7) and 3 of fraction: no infinities, S.1111.111 is NaN."""
    out = np.empty(256)
    for b in range(256):
        s, e, m = b >> 7, b >> 3 & 15, b & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[b] = np.nan if e == 15 and m == 7 else -v if s else v
    return out


def to_e4m3(x):
    """Codes of the nearest values, ties to the even code, limited to +-448; NaN is 0x7F of either sign."""
    x = np.asarray(x, dtype=np.float64)
    grid = e4m3_values()[:127]                          # ascending, 0 .. 448
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(grid, np.where(np.isnan(a), 0.0, a)), 1, 126)
    lo = hi - 1
    up = grid[hi] - a < a - grid[lo]
    tie = grid[hi] - a == a - grid[lo]
    code = np.where(up | (tie & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isnan(x), 127, code) | np.where(np.signbit(x), 128, 0)
    return code.astype(np.uint8)


# ---------------------------------------------------------------- attention

def tokens_of(pool, row, n, page, values):
    """Tokens 0 .. n-1 of a table row: [heads, n, hd] in fp64; pool [pages, heads, page, hd], or the transposed values'."""
    out = []
    for j in range(-(-n // page)):
        p = np.asarray(pool[row[j]], dtype=np.float64)
        out.append(np.swapaxes(p, 1, 2) if values else p)
    return np.concatenate(out, axis=1)[:, :n]


def attention(q, k, v, scale):
    """q [heads_q, hd], k, v [heads, n, hd] -> out [heads_q, hd], lse [heads_q], largest sum of |q k| scale (for error bounds)."""
    heads_q, group = q.shape[0], q.shape[0] // k.shape[0]
    out, lse, size = np.zeros(q.shape), np.full(heads_q, -np.inf), 0.0
    for h in range(heads_q):
        if k.shape[1]:
            s = scale * (k[h // group] @ q[h])
            size = max(size, abs(scale) * float(np.max(np.abs(k[h // group]) @ np.abs(q[h]))))
            p = np.exp(s - s.max())
            out[h] = p @ v[h // group] / p.sum()
            lse[h] = s.max() + np.log(p.sum())
    return out, lse, size


# ---------------------------------------------------------------- pages

class Pages:
    """Reference counts and rows of pages; `data[p]` names what page p holds."""

    def __init__(self, n_pages, page, width):
        self.page, self.width = page, width
        self.refs = [0] * n_pages
        self.rows, self.lens = [], []
        self.moves = []                                 # (from, to) of page copies, in order
        self.status = 0

    def _pages(self, n):
        return -(-n // self.page)

    def reserve(self, add):
        free = [p for p, c in enumerate(self.refs) if c == 0]
        wanted = 0
        for r, m in enumerate(add):
            if m < 0:
                self.status |= 8
                continue
            if self.lens[r] + m > self.width * self.page:
                self.status |= 4
                continue
            need = self._pages(self.lens[r] + m) - self._pages(self.lens[r])
            got = free[wanted:wanted + need]
            wanted += need
            if len(got) < need:
                self.status |= 4
                continue
            for p in got:
                self.refs[p] = 1
            self.rows[r] = self.rows[r] + got
            self.lens[r] += m

    def select(self, src):
        free = [p for p, c in enumerate(self.refs) if c == 0]
        seen, rows, lens = set(), [], []
        refs = list(self.refs)
        for s in src:
            if not 0 <= s < len(self.rows):
                self.status |= 0 if s == -1 else 8
                rows.append([])
                lens.append(0)
                continue
            row, n = list(self.rows[s]), self.lens[s]
            if s in seen:
                for p in row[:n // self.page]:
                    refs[p] += 1
                if n % self.page:
                    if free:
                        new = free.pop(0)
                        refs[new] = 1
                        self.moves.append((row[-1], new))
                        row[-1] = new
                    else:
                        self.status |= 4
                        row.pop()
                        n = n // self.page * self.page
            seen.add(s)
            rows.append(row)
            lens.append(n)
        for s, row in enumerate(self.rows):
            if s not in seen:
                for p in row:
                    refs[p] -= 1
        self.rows, self.lens, self.refs = rows, lens, refs

    def compact(self):
        live = sum(c > 0 for c in self.refs)
        goes = dict(zip([p for p in range(live, len(self.refs)) if self.refs[p]], [p for p in range(live) if not self.refs[p]]))
        for old, new in goes.items():
            self.moves.append((old, new))
            self.refs[new], self.refs[old] = self.refs[old], 0
        self.rows = [[goes.get(p, p) for p in row] for row in self.rows]

    def table(self):
        return np.array([row + [-1] * (self.width - len(row)) for row in self.rows], dtype=np.int32).reshape(len(self.rows), self.width)


# ---------------------------------------------------------------- logits and draws

def adjusted(x, prompt, output, rep, freq, pres, bias, allowed):
    """One row; bias: [(id, value)], of equal ids the first counts; allowed: boolean [vocab] or None."""
    z = np.array(x, dtype=np.float64)
    V = len(z)
    c = np.zeros(V)
    for t in output:
        if 0 <= t < V:
            c[t] += 1
    seen = c > 0
    for t in prompt:
        if 0 <= t < V:
            seen[t] = True
    with np.errstate(invalid="ignore"):
        z[seen] = np.where(z[seen] > 0, z[seen] / rep, z[seen] * rep)
        z = z - freq * c - pres * (c > 0)
    done = set()
    for i, b in bias:
        if i not in done and 0 <= i < V:
            z[i] += b
        done.add(i)
    if allowed is not None:
        z[~allowed] = -np.inf
    return z


def scores(z, temperature, seed, step, row_id):
    """(scores whose arg-max is the token, y)."""
    if temperature == 0:
        return z, z
    n = philox.uint32_words(seed, STREAM_TOKEN, row_id, step, len(z)).astype(np.float64)
    w = np.minimum((n + 0.5) / 2.0 ** 32, 1 - 2.0 ** -24)
    y = z / temperature
    return y - np.log(-np.log1p(-w)), y


def log_softmax_at(y, token):
    top = y.max()
    return y[token] - top - np.log(np.exp(y - top).sum())
