"""Plain 64-bit forms of the paged cache's operators, row by row, for the tests."""
import math

import numpy as np
import torch


def keys_of_row(table, length, ps, n_pages, S, pos, spans):
    """Tokens of a row per part: [(slot or None for the window, token numbers)], tokens without a page left out."""
    c = pos // S
    parts = [(k, range(j * S, (j + 1) * S)) for k, j in enumerate(spans) if 0 <= j < c] + [(None, range(c * S, pos + 1))]
    return [(k, [t for t in ts if t < length and 0 <= table[t // ps] < n_pages]) for k, ts in parts]


def attention(K, V, tables, lens, seqs, cu, Q, idx, scores, S, scale, L=None):
    """O, LSE and A = sum p |v| (what a relative error of the weights is multiplied by), all float64; None rows stay NaN.
    K, V: [n_pages, Hkv, ps, D]; everything on the CPU."""
    n_pages, Hkv, ps, D = K.shape
    Hq, T, _ = Q.shape
    G = Hq // Hkv
    K, V, Q = (x.double().numpy() for x in (K, V, Q))
    tables, lens = tables.numpy(), lens.numpy()
    O, A = np.full((Hq, T, D), np.nan), np.full((Hq, T, D), np.nan)
    LSE = np.full((Hq, T), np.nan)
    cap = tables.shape[1] * ps
    for b, s in enumerate(seqs):
        for r in range(cu[b], cu[b + 1]):
            for h in range(Hq):
                O[h, r] = A[h, r] = 0
                LSE[h, r] = -math.inf
                if not 0 <= s < len(lens):
                    continue
                length = min(int(lens[s]), cap)
                pos = length - (cu[b + 1] - r)
                if pos < 0 or pos >= length or (L and pos >= L):
                    continue
                spans = [] if idx is None else idx[h, r].tolist()
                out = []
                for k, ts in keys_of_row(tables[s], length, ps, n_pages, S, pos, spans):
                    ts = np.array(ts, dtype=np.int64)
                    page, at = tables[s][ts // ps], ts % ps
                    out.append((k, (K[page, h // G, at] @ Q[h, r]) * scale, V[page, h // G, at]))
                if scores is None or len(out) == 1:
                    groups = [(1.0, out)]
                else:
                    g = np.array([scores[h, r, k].item() for k, _, _ in out[:-1]], dtype=np.float64)
                    a = np.exp(g - g.max())
                    groups = [(w, [part, out[-1]]) for w, part in zip(a / a.sum(), out[:-1])]
                for w, parts in groups:
                    z, v = np.concatenate([p[1] for p in parts]), np.concatenate([p[2] for p in parts])
                    if not len(z):
                        continue
                    m = z.max()
                    p = np.exp(z - m)
                    O[h, r] += w * (p @ v) / p.sum()
                    A[h, r] += w * (p @ np.abs(v)) / p.sum()
                    LSE[h, r] = m + math.log(p.sum())
    return O, LSE, A


class Pages:
    """The page bookkeeping, one step after the other."""

    def __init__(self, cache):
        self.ps, self.K, self.V = cache.page_size, cache.K.double().cpu(), cache.V.double().cpu()
        self.tables, self.lens, self.refs = cache.tables.tolist(), cache.lens.tolist(), cache.refs.tolist()

    def agrees(self, cache):
        assert cache.tables.tolist() == self.tables
        assert cache.lens.tolist() == self.lens
        assert cache.refs.tolist() == self.refs
        assert torch.equal(cache.K.double().cpu(), self.K) and torch.equal(cache.V.double().cpu(), self.V)

    def free_pages(self):
        return [p for p, r in enumerate(self.refs) if r <= 0]

    def extend(self, seqs, cu):
        free, ok, ran_out, seen = self.free_pages(), [], False, set()
        cap = len(self.tables[0]) * self.ps
        for i, s in enumerate(seqs):
            n = cu[i + 1] - cu[i]
            good = 0 <= s < len(self.lens) and s not in seen and n >= 0 and self.lens[s] >= 0 and self.lens[s] + n <= cap
            seen.add(s)
            if good:
                have = -(-self.lens[s] // self.ps)
                need = -(-(self.lens[s] + n) // self.ps) - have
                ran_out = ran_out or need > len(free)
                good = need == 0 or not ran_out
            if good:
                for k in range(need):
                    page = free.pop(0)
                    self.tables[s][have + k] = page
                    self.refs[page] = 1
                self.lens[s] += n
            ok.append(int(good))
        return ok

    def fork(self, src, dst):
        free, ok, seen, before = self.free_pages(), [], set(), list(self.lens)
        for s, d in zip(src, dst):
            good = 0 <= d < len(before) and d not in seen and 0 <= s < len(before) and s != d and before[d] == 0 and before[s] >= 0
            seen.add(d)
            if good:
                full, part = divmod(before[s], self.ps)
                good = not part or len(free) > 0
            if good:
                for k in range(full):
                    self.tables[d][k] = self.tables[s][k]
                    self.refs[self.tables[s][k]] += 1
                if part:
                    page, old = free.pop(0), self.tables[s][full]
                    self.tables[d][full] = page
                    self.refs[page] = 1
                    for x in (self.K, self.V):
                        x[..., page, :, :part, :] = x[..., old, :, :part, :]
                self.lens[d] = before[s]
            ok.append(int(good))
        return ok

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < len(self.lens):
                for page in self.tables[s]:
                    if 0 <= page < len(self.refs):
                        self.refs[page] -= 1
                self.tables[s] = [-1] * len(self.tables[s])
                self.lens[s] = 0

    def compact(self):
        used = [r > 0 for r in self.refs]
        n = sum(used)
        new = [p if u else -1 for p, u in enumerate(used)]
        for hole, page in zip([p for p in range(n) if not used[p]], [p for p in range(n, len(used)) if used[p]]):
            new[page] = hole
            self.refs[hole], self.refs[page] = self.refs[page], 0
            for x in (self.K, self.V):
                x[..., hole, :, :, :] = x[..., page, :, :, :]
        self.tables = [[new[p] if 0 <= p < len(used) else p for p in t] for t in self.tables]
        return new
