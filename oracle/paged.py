"""A KV cache in pages in plain 64-bit arithmetic and lists: the plan of a step, attention of a ragged batch, verification of drafted tokens."""
import numpy as np


class Pages:
    """Tables and the stack of free pages as the plan keeps them."""

    def __init__(self, B, P, max_len, n_pages, free):
        self.P, self.max_len, self.W = P, max_len, -(-max_len // P)
        self.lists, self.n_pages = [[] for _ in range(B)], n_pages
        self.stack, self.behind = list(free), list(free) + [-1] * (n_pages - len(free))

    def plan(self, length, add, T):
        """start, end, slot, pos of a step; the state goes on."""
        B = len(self.lists)
        valid = [n >= 0 and a >= 0 and n + a <= self.max_len for n, a in zip(length, add)]
        want = [-(-(n + a) // self.P) if ok else len(pages) for n, a, ok, pages in zip(length, add, valid, self.lists)]
        given = []
        for pages, w in zip(self.lists, want):
            given += pages[w:]
            del pages[w:]
        self.stack += given[::-1]
        self.behind[:len(self.stack)] = self.stack
        left, room, start, end, slot, pos = len(self.stack), T, [0], [], [], []
        for b in range(B):
            need, rows = max(0, want[b] - len(self.lists[b])), add[b] if valid[b] else 0
            left, room = left - need, room - rows
            if (need and left < 0) or (rows and room < 0):
                need = rows = 0
            self.lists[b] += [self.stack.pop() for _ in range(need)]
            for p in range(length[b], length[b] + rows):
                pos.append(p)
                slot.append(self.lists[b][p // self.P] * self.P + p % self.P)
            start.append(start[-1] + rows)
            end.append(length[b] + rows)
        rest = [-1] * (T - len(pos))
        return np.array(start), np.array(end), np.array(slot + rest), np.array(pos + rest)

    def table(self):
        return np.array([pages + [-1] * (self.W - len(pages)) for pages in self.lists]).reshape(len(self.lists), self.W)


def attention(q, K, V, first, window=0, sinks=0, there=None):
    """q [S, Hq, Dh] at positions first ... over K, V [Hkv, n, Dh], n >= first + S; there [n]: positions that exist.  The result, zero where nothing is seen, and for every element the weighted mean of
    |V|, for every row the largest sum of |q k| / sqrt(Dh)."""
    S, Hq, Dh = q.shape
    G = Hq // K.shape[0]
    out, mean, most = np.zeros((S, Hq, Dh)), np.zeros((S, Hq, Dh)), np.zeros((S, Hq))
    for t in range(S):
        p = first + t
        see = np.arange(p + 1)
        if window:
            see = see[(see > p - window) | (see < sinks)]
        if there is not None:
            see = see[there[see]]
        for h in range(Hq):
            k, v = K[h // G, see], V[h // G, see]
            with np.errstate(invalid="ignore", over="ignore"):
                s = k @ q[t, h] / np.sqrt(Dh)
                if not len(see) or s.max() == -np.inf:
                    continue
                w = np.exp(s - s.max())
                out[t, h] = (w[:, None] * v).sum(0) / w.sum()
                mean[t, h] = (w[:, None] * np.abs(v)).sum(0) / w.sum()
                most[t, h] = (np.abs(k) @ np.abs(q[t, h])).max() / np.sqrt(Dh)
    return out, mean, most


def rows(start, T):
    """(first row, rows) of each sequence of a verification: none where they do not lie in [0, T), or begin before the start of a sequence before it (of those in [0, T])."""
    out, highest = [], 0
    for s, e in zip(start, start[1:]):
        out.append((int(s), int(e - s) if highest <= s < e <= T else 0))
        if 0 <= s <= T:
            highest = max(highest, s)
    return out


def softmax(x, t):
    """Of logits at a temperature; those of -inf and NaN are 0, and all are where there are no others."""
    x = np.asarray(x, np.float64)
    real = x > -np.inf
    if not real.any():
        return np.zeros(len(x))
    top = x[real].max()
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(~real, 0.0, np.where(x == top, 1.0, np.exp((x - top) / t) if top < np.inf else 0.0))
    return w / w.sum()


def likeliest(x):
    x = np.asarray(x, np.float64)
    return int(np.argmax(np.where(np.isnan(x), -np.inf, x)))


def draw(w, u):
    sums = np.cumsum(w)
    return int(np.searchsorted(sums, min(max(float(u), 0.0), 1 - 2.0 ** -24) * sums[-1], side="right"))


def verify(x, y, drafted, u, u_draw, temperature=1.0):
    """One sequence: x [n, V] logits of the target, y [n, V] or None of the draft, drafted [n - 1] tokens, u [n].  The tokens it goes on with."""
    out, n, V = [], len(x), x.shape[1]
    for i in range(n):
        last = i == n - 1
        if not temperature > 0:
            out.append(likeliest(x[i]))
            if last or drafted[i] != out[-1] or not (np.asarray(x[i]) > -np.inf).any():             # (a row of nothing takes no token)
                return out
            continue
        p = softmax(x[i], temperature)
        if not last:
            d = int(drafted[i])
            q = softmax(y[i], temperature) if y is not None else (np.arange(V) == d).astype(float)
            if 0 <= d < V and min(max(float(u[i]), 0.0), 1.0) * q[d] < p[d]:
                out.append(d)
                continue
            rest = np.maximum(p - q, 0.0)
            p = rest if rest.sum() > 0 else p
        out.append(draw(p, u_draw) if p.any() else 0)
        return out
