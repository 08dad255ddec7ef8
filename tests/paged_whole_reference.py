"""Span-attention over pages in plain 64-bit steps, a chunk and head at a time and on the tensors' device, for tests of calls that row by row
would take too long."""
import math

import torch

from tests import fp4_reference as fp4


def values(cache, tensor, layer=0):
    """float64 [n_pages, Hkv, ps, D] of the cache's K or V."""
    x = getattr(cache, tensor)
    x = x[layer] if x.dim() == (4 if cache.fp4 else 5) else x
    if not cache.fp4:
        return x.double()
    ps, D = cache.page_size, cache.D
    codes, scales = x[..., :ps * (D // 2)], x[..., ps * (D // 2):ps * (D // 2 + D // 32)].double()
    sizes = torch.tensor([s * v for s in (1.0, -1.0) for v in fp4.SIZES], dtype=torch.float64, device=x.device)
    v = sizes[torch.stack([codes & 15, codes >> 4], -1).long()].view(*x.shape[:-1], ps, D)
    power = torch.where(scales == 255, math.nan, torch.exp2(scales - 127))
    return v * power.view(*x.shape[:-1], ps, D // 32).repeat_interleave(32, -1)


def weighed(z, on, v):
    """Softmax of the scores z [n, t] over what is `on`, times the values v [t, D], and times their magnitudes; log-sum-exp [n]."""
    z = torch.where(on, z, -math.inf)
    m = z.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), 0.0, m)
    p = torch.exp(z - m)
    s = p.sum(-1, keepdim=True)
    w = p / torch.where(s == 0, 1.0, s)
    bad = torch.isnan(v)
    clean = torch.where(bad, 0.0, v)
    spoilt = on.double() @ bad.double() > 0   # (a value that is not finite spoils the rows that attend it, and no other)
    o, a = (torch.where(spoilt, math.nan, w @ x) for x in (clean, clean.abs()))
    return o, a, (m + torch.log(s)).squeeze(-1)


def attention(cache, seqs, cu, Q, idx, scores, S, scale=None, L=None, layer=0):
    """O, A = sum p |v| (what a relative error of the weights is multiplied by) [Hq, T, D] and LSE [Hq, T], float64; rows of no chunk are left
    at 7.  Spans of a row are distinct, or empty slots."""
    K, V = (values(cache, name, layer) for name in "KV")
    n_pages, Hkv, ps, D = K.shape
    Hq, T, _ = Q.shape
    dev, scale = Q.device, scale or 1 / math.sqrt(D)
    O, A, LSE = (torch.full(shape, 7.0, dtype=torch.float64, device=dev) for shape in (Q.shape, Q.shape, (Hq, T)))
    lens = cache.lens.tolist()
    for s, r0, r1 in zip(seqs, cu, cu[1:]):
        if r1 == r0:
            continue
        n, t = r1 - r0, torch.arange(max(lens[s], 1), device=dev)
        page = cache.tables[s].long()[t // ps]
        here = (page >= 0) & (page < n_pages)
        page = torch.where(here, page, 0)
        pos = torch.arange(n, device=dev)[:, None] + lens[s] - n
        rows = (pos >= 0) & (pos < (L or 1 << 31))
        window = here & rows & (t // S == pos // S) & (t <= pos)
        for h in range(Hq):
            k, v = (x[page, h // (Hq // Hkv), t % ps] for x in (K, V))
            z = (Q[h, r0:r1].double() @ k.T) * scale
            lists = torch.full((n, 1), -1, device=dev) if idx is None else idx[h, r0:r1].long()
            lists = torch.where((lists >= 0) & (lists < pos // S) & rows, lists, -1)
            if scores is None or idx is None:
                on = window.clone()
                for j in lists.T:
                    on |= here & (t // S == j[:, None])
                O[h, r0:r1], A[h, r0:r1], LSE[h, r0:r1] = weighed(z, on, v)
                continue
            gate = torch.where(lists >= 0, scores[h, r0:r1].double(), -math.inf)
            none = (lists < 0).all(-1, keepdim=True)
            gate = torch.softmax(torch.where(none, 0.0, gate), -1)
            gate = torch.where(none, 0.0, gate)
            o, a, LSE[h, r0:r1] = weighed(z, window, v)
            O[h, r0:r1], A[h, r0:r1] = (torch.where(none, x, 0.0) for x in (o, a))
            for j, g in zip(lists.T, gate.T):
                if bool((j >= 0).any()):
                    o, a, _ = weighed(z, window | (here & (t // S == j[:, None]) & (j[:, None] >= 0)), v)
                    used = j[:, None] >= 0
                    O[h, r0:r1] += torch.where(used, g[:, None] * o, 0.0)
                    A[h, r0:r1] += torch.where(used, g[:, None] * a, 0.0)
    return O, A, LSE
