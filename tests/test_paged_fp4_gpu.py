"""A paged cache held in 4 bits against plain 64-bit forms.

What is held is defined bit by bit: codes, scales and rows that are read back are compared for equality.  Attention's tolerances are those
of the other caches on the values that the codes stand for, which bf16 and fp32 hold exactly: fp32, below 1e-4 for values of unit
variance, at most 6; bf16, the output's rounding (2^-8 |O|), weights rounded once (2^-8 of sum p |v|), partial outputs to
11 bits of their largest element (2^-11 max |V|), beside the fp32 part."""
import math

import numpy as np
import pytest
import torch

from paper_2601_18401_amd import binding as B
from tests import fp4_reference as fp4
from tests import paged_reference as ref
from tests.test_paged_gpu import CASES, choose, i32

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def make_cache(g, Ls, ps, Hkv, D, dtype, layers=1, spare=3, width=1, gap=0):
    """Sequences of Ls tokens in pages of random order.  Whatever no sequence holds is NaN, the gaps between parts are 0xA5."""
    need = sum(-(-L // ps) for L in Ls)
    n_pages, max_pages, size = need + spare, max(-(-max(Ls) // ps), 1) + width, B.PageCache.page_bytes(ps, D)
    wide = [torch.full((layers, n_pages, Hkv, size + gap), 0xA5, dtype=torch.uint8) for _ in range(2)]
    K, V = (x.narrow(3, 0, size) for x in wide)
    for x in (K, V):
        x[...] = 255
    order = torch.randperm(n_pages, generator=g).tolist()
    tables = torch.full((len(Ls), max_pages), -1, dtype=torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32)
    for s, L in enumerate(Ls):
        for k in range(-(-L // ps)):
            page = order.pop()
            tables[s, k] = page
            refs[page] = 1
            n = min(ps, L - k * ps)
            for x in (K, V):
                codes, scales = fp4.encode(torch.randn((layers * Hkv * n, D), generator=g).double().numpy())
                at = ps * (D // 2)
                x[:, page, :, : n * (D // 2)] = torch.from_numpy(fp4.pack(codes)).view(layers, Hkv, -1)
                x[:, page, :, at:at + n * (D // 32)] = torch.from_numpy(scales).view(layers, Hkv, -1)
    K, V = (x.to(DEV).narrow(3, 0, size) for x in wide)
    return B.PageCache(K, V, tables.to(DEV), i32(Ls), refs.to(DEV), page_size=ps, D=D, dtype=dtype)


def check(cache, seqs, cu, Q, idx, scores, S, O, LSE=None, scale=None, layer=0, L=None):
    torch.cuda.synchronize()
    K, V = (fp4.values(x if x.dim() == 3 else x[layer], cache.page_size, cache.D) for x in (cache.K, cache.V))
    scale = scale or 1 / math.sqrt(cache.D)
    with np.errstate(invalid="ignore"):
        wO, wL, A = ref.attention(K, V, cache.tables.cpu(), cache.lens.cpu(), seqs, cu, Q.cpu(), None if idx is None else idx.cpu(),
                                  None if scores is None else scores.cpu(), S, scale, L)
    live = ~np.isnan(wL)
    got = O.double().cpu().numpy()
    assert np.isfinite(got[live]).all()
    big = float(np.nanmax(A)) if live.any() else 0.0
    tol = 1e-4 + (0 if cache.dtype == F32 else 2.0 ** -8 * (np.abs(wO) + A) + 2.0 ** -11 * max(6.0, big))
    off = np.abs(got - wO) - tol
    assert (off[live] <= 0).all(), float(off[live].max())
    if LSE is not None:
        lse = LSE.double().cpu().numpy()
        assert np.array_equal(np.isinf(lse[live]), np.isinf(wL[live]))
        fin = live & np.isfinite(wL)
        assert (np.abs(lse[fin] - wL[fin]) <= 1e-4).all()
    return live


# ---- written, read back
def awkward_rows(g, shape, dtype):
    """Rows whose blocks are ordinary, far apart, on the borders between codes, zero, tiny, huge, not finite."""
    x = torch.randn(shape, generator=g).double()
    blocks = x.view(-1, 32)
    n = blocks.shape[0]
    kind = torch.arange(n) % 12
    blocks[kind == 1] *= 2.0 ** torch.randint(-60, 60, (int((kind == 1).sum()), 1), generator=g).double()
    halves = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.0, 6.875])
    sign = torch.where(torch.rand(blocks.shape, generator=g) < 0.5, -1.0, 1.0).double()
    blocks[kind == 2] = (halves[torch.randint(0, 10, blocks.shape, generator=g)] * sign)[kind == 2]
    blocks[kind == 3] = 0.0
    blocks[kind == 4] *= 2.0 ** -128
    blocks[kind == 5] *= 2.0 ** -133
    blocks[kind == 6] = (torch.randint(0, 256, blocks.shape, generator=g).double() / 256 * 2.0 ** 127.9 * sign)[kind == 6]
    blocks[kind == 7] = blocks[kind == 7].clamp(-1.7, 1.7)
    blocks[kind == 7, 5] = torch.tensor([1.75, 1.7421875, -3.5, 7.0]).double().repeat(n)[: int((kind == 7).sum())]
    for k, bad in ((8, math.nan), (9, math.inf), (10, -math.inf)):
        where = (torch.randperm(n, generator=g) < n // 8) & (kind == k)
        blocks[where, 17] = bad
    return x.to(dtype)


def check_bytes(cache, before, written, layer=0):
    """written: {(tensor, page, head, place): float64 row}; everything else as it was."""
    torch.cuda.synchronize()
    ps, D = cache.page_size, cache.D
    for name in ("K", "V"):
        want, got = before[name].copy(), getattr(cache, name).cpu().numpy()
        codes, scales = fp4.parts(want[layer], ps, D)
        keys = [k for k in written if k[0] == name]
        if keys:
            c, s = fp4.encode(np.stack([written[k] for k in keys]))
            for (_, page, head, at), cc, ss in zip(keys, fp4.pack(c), s):
                first = ps * (D // 2) + at * (D // 32)
                want[layer, page, head, at * (D // 2):(at + 1) * (D // 2)] = cc
                want[layer, page, head, first:first + D // 32] = ss
        assert np.array_equal(got, want), (name, np.argwhere(got != want)[:5])


ROWS = [
    # dtype Hkv D   ps  chunks          lengths          layers gap token-major rows
    (BF16, 2, 128, 64, [1], [1], 1, 0, False),
    (BF16, 4, 64, 16, [1, 1, 1], [15, 16, 17], 2, 32, True),
    (BF16, 2, 128, 48, [5, 0, 1, 130], [300, 20, 97, 130], 1, 16, False),
    (BF16, 1, 64, 9, [70], [400], 3, 0, True),
    (BF16, 3, 128, 1, [40], [40], 1, 0, False),
    (F32, 4, 128, 16, [1, 37], [500, 200], 1, 48, True),
    (F32, 2, 64, 7, [64, 3], [333, 3], 2, 0, False),
    (F32, 1, 128, 100, [257], [300], 1, 0, True),
]


@pytest.mark.parametrize("case", ROWS, ids=lambda c: "-".join(str(v) for v in c[1:]).replace(" ", ""))
def test_rows_are_rounded_as_defined_and_read_back(case):
    dtype, Hkv, D, ps, ns, Ls, layers, gap, token_major = case
    g = torch.Generator().manual_seed(Ls[0] + D)
    cache = make_cache(g, Ls, ps, Hkv, D, dtype, layers=layers, gap=gap)
    T, cu, layer = sum(ns), [sum(ns[:b]) for b in range(len(ns) + 1)], layers - 1
    rows = [awkward_rows(g, (T, Hkv, D), dtype).transpose(0, 1) if token_major else awkward_rows(g, (Hkv, T, D), dtype) for _ in range(2)]
    K, V = (r.to(DEV) for r in rows)
    before = {n: getattr(cache, n).cpu().numpy().copy() for n in ("K", "V")}
    seqs = list(range(len(Ls)))
    B.sl_paged_append(cache, i32(seqs), i32(cu), K, V, layer=layer)
    written, tables = {}, cache.tables.cpu()
    for b, s in enumerate(seqs):
        for r in range(cu[b], cu[b + 1]):
            t = Ls[s] - (cu[b + 1] - r)
            for h in range(Hkv):
                for name, x in zip("KV", rows):
                    written[name, int(tables[s, t // ps]), h, t % ps] = x[h, r].double().numpy()
    check_bytes(cache, before, written, layer)
    got = B.sl_paged_read(cache, i32(seqs), i32(cu), T, layer=layer)
    for x, y in zip(rows, got):
        want = torch.from_numpy(fp4.hold(x.double().numpy().reshape(-1, D))).view(Hkv, T, D)
        assert torch.equal(torch.isnan(y.cpu()), torch.isnan(want)) and torch.equal(y.double().cpu().nan_to_num(0.0), want.nan_to_num(0.0))
    # all of every sequence, and the caller's own tensors, tokens first
    whole = [sum(Ls[:b]) for b in range(len(Ls) + 1)]
    out = tuple(torch.empty((whole[-1], Hkv, D), dtype=dtype, device=DEV).transpose(0, 1) for _ in range(2))
    assert B.sl_paged_read(cache, i32(seqs), i32(whole), whole[-1], layer=layer, out=out) is out
    for name, y in zip(("K", "V"), out):
        v = fp4.values(getattr(cache, name)[layer], ps, D)
        for s, L in enumerate(Ls):
            t = torch.arange(L)
            want = v[tables[s, t // ps].long(), :, t % ps].transpose(0, 1)
            x = y[:, whole[s]:whole[s + 1]].double().cpu()
            assert torch.equal(torch.isnan(x), torch.isnan(want)) and torch.equal(x.nan_to_num(0.0), want.nan_to_num(0.0))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("held", ["4 bits", "rows"])
def test_read_passes_over_what_has_no_token(dtype, held):
    """Missing pages and numbers that name none, sequences out of range, chunks longer than the sequence: zeros.  Rows of nobody stay."""
    g = torch.Generator().manual_seed(6)
    Ls, ps = [60, 40, 25], 16
    if held == "rows":
        from tests.test_paged_gpu import make_cache as make
        cache = make(g, Ls, ps, 2, 64, dtype, token_major=True)
    else:
        cache = make_cache(g, Ls, ps, 2, 64, dtype)
    cache.tables[0, 1] = -1
    cache.tables[0, 2] = 1 << 20
    seqs, ns, first = [0, 99, 1, -1, 2, 1], [60, 3, 50, 2, 25, 1], 4
    cu = [first + sum(ns[:b]) for b in range(len(ns) + 1)]
    T = cu[-1] + 3
    out = tuple(torch.full((2, T, 64), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    B.sl_paged_read(cache, i32(seqs), i32(cu), T, out=out)
    torch.cuda.synchronize()
    tables = cache.tables.cpu()
    for x, y in zip((cache.K, cache.V), out):
        v = fp4.values(x[0], ps, 64) if held == "4 bits" else x[0].cpu().double()
        want = torch.full((2, T, 64), 7.0).double()
        want[:, cu[0]:cu[-1]] = 0
        for b, (s, n) in enumerate(zip(seqs, ns)):
            for r in range(n):
                t = Ls[s] - n + r if 0 <= s < 3 else -1
                if t >= 0 and 0 <= tables[s, t // ps] < v.shape[0]:
                    want[:, cu[b] + r] = v[int(tables[s, t // ps]), :, t % ps]
        assert torch.equal(y.double().cpu(), want)


def test_shared_and_missing_pages_are_not_written():
    g = torch.Generator().manual_seed(8)
    cache = make_cache(g, [50, 64, 64], 16, 2, 128, BF16)
    cache.refs[int(cache.tables[1, 3])] = 2
    cache.tables[2, 3] = -1
    before = {n: getattr(cache, n).cpu().numpy().copy() for n in ("K", "V")}
    new = torch.randn((2, 43, 128), generator=g).to(BF16).to(DEV)
    seqs, cu = [1, 2, -1, 99, 0], [3, 13, 20, 25, 30, 40]
    B.sl_paged_append(cache, i32(seqs), i32(cu), new, new)
    written = {(n, int(cache.tables[0, t // 16]), h, t % 16): new[h, 30 + k].double().cpu().numpy()
               for n in "KV" for h in range(2) for k, t in enumerate(range(40, 50))}
    check_bytes(cache, before, written)


@pytest.mark.parametrize("dtype,D,ps,S", [(BF16, 128, 16, 24), (BF16, 64, 7, 7), (F32, 128, 64, 100), (F32, 64, 9, 1)])
def test_span_keys(dtype, D, ps, S):
    g = torch.Generator().manual_seed(S)
    Ls, ns = [200, 37, 120, 5], [200, 1, 30, 0]
    cache = make_cache(g, Ls, ps, 2, D, dtype, layers=2)
    Ks = torch.full((4, 2, 210 // S, D), 7.0, dtype=dtype, device=DEV)
    cu = [sum(ns[:b]) for b in range(5)]
    B.sl_paged_span_keys(cache, i32([0, 1, 2, 3]), i32(cu), Ks, S, layer=1)
    want = torch.full(Ks.shape, 7.0).double()
    v = fp4.values(cache.K[1], ps, D)
    for s in range(4):
        for j in range((Ls[s] - ns[s]) // S, min(Ls[s] // S, Ks.shape[2])):
            if ns[s]:
                t = j * S + S - 1
                want[s, :, j] = v[int(cache.tables[s, t // ps]), :, t % ps]
    assert torch.equal(Ks.double().cpu(), want)


# ---- attention
@pytest.mark.parametrize("form", ["joint", "gated"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c[1:]).replace(" ", ""))
def test_attention(case, form):
    dtype, Hq, Hkv, D, ps, S, topk, ns, Ls, gap = case
    g = torch.Generator().manual_seed(len(Ls) * 1000 + Ls[0])
    cache = make_cache(g, Ls, ps, Hkv, D, dtype, gap=16 * gap)
    T = sum(ns)
    cu = [sum(ns[:b]) for b in range(len(ns) + 1)]
    Q = torch.randn((T, Hq, D), generator=g).to(dtype).to(DEV).transpose(0, 1)
    idx = choose(g, Hq, T, topk, max(Ls) // S + 1)
    scores = torch.randn(idx.shape, generator=g).to(DEV) * 2
    seqs = list(range(len(Ls)))
    if form == "joint":
        O, LSE = B.sl_paged_span_attention(cache, i32(seqs), i32(cu), Q, idx, S)
        check(cache, seqs, cu, Q, idx, None, S, O, LSE)
    else:
        O = B.sl_paged_span_attention_combined(cache, i32(seqs), i32(cu), Q, idx, scores, S, L=max(Ls))
        check(cache, seqs, cu, Q, idx, scores, S, O)


@pytest.mark.parametrize("Hq,Hkv,D,ps,S,topk,ns,Ls", [
    (32, 4, 128, 32, 4, 32, [1] * 20, list(range(380, 420, 2))),       # two spans and three a workgroup, pages of many spans
    (32, 4, 64, 24, 3, 32, [1] * 32, list(range(300, 364, 2))),        # pages that end anywhere
    (16, 2, 128, 16, 70, 16, [1] * 64, [9 * 70 + k for k in range(64)]),   # spans that begin and end inside 32 tokens
    (32, 4, 64, 64, 1, 32, [5] * 8, [500, 430, 480, 9, 5, 511, 450, 500]),   # spans of one token, columns of several rows
])
def test_several_spans_a_workgroup(Hq, Hkv, D, ps, S, topk, ns, Ls):
    """More lists than workgroups that the chip holds: one takes several slots of a row, with the codes of the next one on their way."""
    g = torch.Generator().manual_seed(S)
    cache = make_cache(g, Ls, ps, Hkv, D, BF16)
    cu = [sum(ns[:b]) for b in range(len(ns) + 1)]
    Q = torch.randn((Hq, cu[-1], D), generator=g).to(BF16).to(DEV)
    idx = choose(g, Hq, cu[-1], topk, max(Ls) // S + 1)
    idx[:, ::3] = idx[:1, ::3]      # heads that share their spans
    scores = torch.randn(idx.shape, generator=g).to(DEV)
    seqs = list(range(len(Ls)))
    O, LSE = B.sl_paged_span_attention(cache, i32(seqs), i32(cu), Q, idx, S, L=max(Ls))
    check(cache, seqs, cu, Q, idx, None, S, O, LSE)
    O = B.sl_paged_span_attention_combined(cache, i32(seqs), i32(cu), Q, idx, scores, S, L=max(Ls))
    check(cache, seqs, cu, Q, idx, scores, S, O)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,ps,ns,Ls", [
    (BF16, 8, 2, 128, 64, [1, 1], [1500, 3]), (BF16, 8, 1, 64, 20, [4, 1, 7], [900, 513, 7]), (BF16, 4, 4, 128, 32, [200], [200]),
    (BF16, 12, 4, 128, 64, [150, 1, 64], [900, 64, 65]), (F32, 4, 2, 64, 16, [100, 3], [100, 600]), (BF16, 2, 1, 64, 64, [300, 129], [300, 640]),
    (BF16, 5, 5, 128, 16, [257], [300]), (F32, 3, 1, 128, 64, [1], [3000]), (F32, 8, 2, 128, 32, [150, 70], [200, 70]),
    (F32, 2, 1, 64, 10, [130], [400]), (BF16, 4, 1, 128, 37, [300], [333]), (BF16, 8, 2, 64, 70, [2, 1], [600, 71]),
    (BF16, 8, 1, 64, 16, [40], [2300]), (F32, 8, 4, 128, 16, [1, 1, 2], [1, 33, 700])])
def test_dense(dtype, Hq, Hkv, D, ps, ns, Ls):
    """No spans and S beyond every length: causal attention over all of the sequence."""
    g = torch.Generator().manual_seed(sum(Ls))
    cache = make_cache(g, Ls, ps, Hkv, D, dtype, layers=2)
    cu = [sum(ns[:b]) for b in range(len(ns) + 1)]
    Q = torch.randn((Hq, sum(ns), D), generator=g).to(dtype).to(DEV)
    O, LSE = B.sl_paged_span_attention(cache, i32(list(range(len(Ls)))), i32(cu), Q, None, (1 << 31) - 1, layer=1, L=max(Ls), scale=0.1)
    check(cache, list(range(len(Ls))), cu, Q, None, None, (1 << 31) - 1, O, LSE, scale=0.1, layer=1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("topk,S,n", [(3, 40, 6), (0, 4000, 6), (3, 40, 150), (0, 4000, 150)])
def test_rows_without_tokens_and_rows_of_nobody(dtype, topk, S, n):
    """Missing pages (all of a row's among them), sequence numbers out of range, chunks longer than the sequence, positions
    from L on, the same sequence twice, rows before the first chunk and behind the last, a lengths entry beyond the table."""
    g = torch.Generator().manual_seed(5)
    cache = make_cache(g, [300, 200, 160, 30, 250], 16, 2, 64, dtype)
    cache.tables[0, 3:7] = -1
    cache.tables[0, 9] = 1 << 20
    cache.tables[1, :] = -1          # nothing left at all
    cache.tables[1, 5] = -7
    for x in (cache.K, cache.V):     # the rest of sequence 4's last page, which its lengths entry makes tokens
        x[0, int(cache.tables[4, 250 // 16])] = torch.where(x[0, int(cache.tables[4, 250 // 16])] == 255, 126, x[0, int(cache.tables[4, 250 // 16])])
    cache.lens[4] = 1 << 30          # more than the table holds: its whole table
    seqs = [0, 1, 99, 2, -1, 3, 0, 4]
    ns = [n, 3, 2, 4, 1, 40, 2, 2]
    first, behind = 5, 7
    cu = [first + sum(ns[:b]) for b in range(len(ns) + 1)]
    T = cu[-1] + behind
    Q = torch.randn((4, T, 64), generator=g).to(dtype).to(DEV)
    idx = choose(g, 4, T, topk, 8) if topk else None
    scores = torch.randn((4, T, topk), generator=g).to(DEV) if topk else None
    for L in (0, 290):
        out = torch.full(Q.shape, 7.0, dtype=dtype, device=DEV), torch.full(Q.shape[:2], 7.0, device=DEV)
        O, LSE = B.sl_paged_span_attention(cache, i32(seqs), i32(cu), Q, idx, S, L=L, out=out)
        live = check(cache, seqs, cu, Q, idx, None, S, O, LSE, L=L)
        assert bool((O[:, torch.tensor(~live[0], device=DEV)] == 7).all()) and int((~live[0]).sum()) == first + behind
        if topk:
            out = torch.full(Q.shape, 7.0, dtype=dtype, device=DEV)
            B.sl_paged_span_attention_combined(cache, i32(seqs), i32(cu), Q, idx, scores, S, L=L, out=out)
            check(cache, seqs, cu, Q, idx, scores, S, out, L=L)
            assert bool((out[:, torch.tensor(~live[0], device=DEV)] == 7).all())


@pytest.mark.parametrize("dtype,n,ps,Hq", [(BF16, 3, 32, 4), (BF16, 130, 32, 4), (BF16, 130, 27, 4), (F32, 130, 32, 4), (F32, 3, 32, 4),
                                           (F32, 270, 27, 4), (BF16, 150, 32, 32), (F32, 200, 16, 32)])
@pytest.mark.parametrize("tensor", ["K", "V"])
def test_blocks_that_are_not_finite_where_some_rows_attend(tensor, dtype, n, ps, Hq):
    """A block held as NaN makes those rows NaN that attend its token (its 32 channels, or, of a key, all), and no other."""
    g = torch.Generator().manual_seed(n)
    L, S = 400, 50
    cache = make_cache(g, [L], ps, 2, 128, dtype)
    bad = [L - 2, 120]  # one of the new tokens, and one in span 2
    changed = getattr(cache, tensor).clone()
    for t in bad:
        changed[0, int(cache.tables[0, t // ps]), :, ps * 64 + t % ps * 4 + 1] = 255
    K, V = (changed, cache.V) if tensor == "K" else (cache.K, changed)
    spoilt = B.PageCache(K, V, cache.tables, cache.lens, cache.refs, page_size=ps, D=128, dtype=dtype)
    Q = torch.randn((Hq, n, 128), generator=g).to(dtype).to(DEV)
    idx = torch.tensor([[[0, 2], [0, 1]][(h + r) % 2] for h in range(Hq) for r in range(n)], dtype=torch.int32, device=DEV).view(Hq, n, 2)
    zeros = torch.zeros(idx.shape, device=DEV)
    seqs, cu = i32([0]), i32([0, n])
    calls = [(lambda c: B.sl_paged_span_attention(c, seqs, cu, Q, idx, S)[0], S), (lambda c: B.sl_paged_span_attention_combined(c, seqs, cu, Q, idx, zeros, S), S),
             (lambda c: B.sl_paged_span_attention(c, seqs, cu, Q, None, 10 * L)[0], 10 * L)]
    for call, S in calls:
        x, w = call(spoilt).double().cpu(), call(cache).double().cpu()
        for h in range(Hq):
            for r in range(n):
                pos = L - n + r
                if any((t // S == pos // S and t <= pos) or (t // S < pos // S and t // S in idx[h, r].tolist()) for t in bad):
                    where = slice(32, 64) if tensor == "V" else slice(None)
                    assert bool(torch.isnan(x[h, r, where]).all())
                    x[h, r, where] = w[h, r, where]
        # (the two may take different kernels: two roundings each of outputs below 6)
        assert float((x - w).abs().max()) <= (2.0 ** -7 * 6 if dtype == BF16 else 1e-4)


@pytest.mark.parametrize("held", ["4 bits", "rows"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,topk", [(1, 0), (3, 0), (160, 0), (3, 2), (160, 2)])
def test_a_key_that_is_nan_before_tokens_that_a_row_does_not_attend(n, topk, dtype, held):
    """The last tokens that a row attends are NaN, what its tile goes on with is masked for it: the row is NaN all the same."""
    from tests.test_paged_gpu import make_cache as make_rows
    g = torch.Generator().manual_seed(n)
    L, ps = 2000, 32
    cache = make_cache(g, [L], ps, 1, 64, dtype) if held == "4 bits" else make_rows(g, [L], ps, 1, 64, dtype)
    bad = L - n  # the first new token: every row attends it, the first one as its last
    if held == "4 bits":
        cache.K[0, int(cache.tables[0, bad // ps]), :, ps * 32 + bad % ps * 2] = 255
    else:
        cache.K[0, int(cache.tables[0, bad // ps]), :, bad % ps, 3] = math.nan
    Q = torch.randn((2, n, 64), generator=g).to(dtype).to(DEV)
    idx = torch.tensor([0, 3], dtype=torch.int32, device=DEV).expand(2, n, 2).contiguous() if topk else None
    S = 500 if topk else 4000
    O, LSE = B.sl_paged_span_attention(cache, i32([0]), i32([0, n]), Q, idx, S)
    assert bool(torch.isnan(O).all()) and bool(torch.isnan(LSE).all())
    if topk:
        O = B.sl_paged_span_attention_combined(cache, i32([0]), i32([0, n]), Q, idx, torch.zeros(idx.shape, device=DEV), S)
        assert bool(torch.isnan(O).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_results_do_not_change_from_run_to_run(dtype):
    g = torch.Generator().manual_seed(23)
    cache = make_cache(g, [3000], 64, 2, 128, dtype)
    Q = torch.randn((8, 900, 128), generator=g).to(dtype).to(DEV)
    for idx, S in ((choose(g, 8, 900, 4, 40), 64), (None, 3000)):
        want = None
        for _ in range(6):
            got = B.sl_paged_span_attention(cache, i32([0]), i32([0, 900]), Q, idx, S)
            want = want or got
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_two_captured_graphs_and_eager_calls_between():
    """A step (append, read, attention) in each graph: replays in any order, with eager calls of the other between them."""
    g = torch.Generator().manual_seed(24)
    cache = make_cache(g, [2000, 700], 64, 2, 128, BF16)
    jobs = []
    for seq, n, topk in ((0, 200, 4), (1, 1, 3)):
        Q = torch.randn((8, n, 128), generator=g).to(BF16).to(DEV)
        K, V = (torch.randn((2, n, 128), generator=g).to(BF16).to(DEV) for _ in range(2))
        idx, cu, seqs = choose(g, 8, n, topk, 20), i32([0, n]), i32([seq])

        def job(Q=Q, K=K, V=V, idx=idx, cu=cu, seqs=seqs, n=n):
            B.sl_paged_append(cache, seqs, cu, K, V)
            return (*B.sl_paged_read(cache, seqs, cu, n), *B.sl_paged_span_attention(cache, seqs, cu, Q, idx, 64))

        jobs.append(job)
    want = [tuple(x.clone() for x in job()) for job in jobs]
    graphs, outs = [], []
    for job in jobs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(job())
        graphs.append(graph)
    for k in (0, 1, 1, 0, 1, 0, 0):
        for x in outs[k]:
            x.zero_()
        cache.K[:, cache.tables[0, 31].long()] = 0   # (the graph of sequence 0 writes it again, whole)
        graphs[k].replay()
        jobs[1 - k]()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[k], want[k]))


def test_work_on_a_stream_of_its_own():
    g = torch.Generator().manual_seed(31)
    cache = make_cache(g, [900], 32, 2, 64, BF16)
    Q = torch.randn((4, 5, 64), generator=g).to(BF16).to(DEV)
    K, V = (torch.randn((2, 5, 64), generator=g).to(BF16).to(DEV) for _ in range(2))
    seqs, cu = i32([0]), i32([0, 5])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.sl_paged_append(cache, seqs, cu, K, V)
        O, LSE = B.sl_paged_span_attention(cache, seqs, cu, Q, None, 2000)
        k, _ = B.sl_paged_read(cache, seqs, cu, 5)
    torch.cuda.current_stream().wait_stream(side)
    check(cache, [0], [0, 5], Q, None, None, 2000, O, LSE)
    assert torch.equal(k.double().cpu(), torch.from_numpy(fp4.hold(K.double().cpu().numpy().reshape(-1, 64))).view(2, 5, 64))


@pytest.mark.parametrize("topk", [0, 8])
@pytest.mark.parametrize("cu,rows", [([0, 512] * 50 + [512], 512), ([0, 4] * 6 + [4], 4), ([300, 20, 512, -40, 512, 1 << 30, 7], 512),
                                     ([0, -5, 1 << 30, 3, 512], 512)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_out_of_order_stay_inside_the_arrays(cu, rows, topk, dtype):
    """cu_rows that decrease name rows twice, or rows that are none: results may be anything, what lies around them stays."""
    g = torch.Generator().manual_seed(25)
    cache = make_cache(g, [1600, 300], 64, 1, 64, dtype)
    n = len(cu) - 1
    seqs, cu = i32([0] * (n - 1) + [1]), i32(cu)
    Q = torch.randn((16, rows, 64), generator=g).to(dtype).to(DEV)
    idx = choose(g, 16, rows, topk, 18) if topk else None
    S = 80 if topk else 10000
    tables, lens, refs = cache.tables.clone(), cache.lens.clone(), cache.refs.clone()
    a = B.SlPagedAttention(16, S, topk, 0.0, 0, 0, 0, 0)
    b = cache.batch(seqs, cu, rows, 1600)
    need = B.load().sl_paged_attention_workspace_bytes(cache.record, b, a)
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device=DEV)   # (every float in it is NaN)
    O = torch.full((Q.numel() + 2048,), 7.0, dtype=dtype, device=DEV)
    LSE = torch.full((16 * rows + 2048,), 7.0, device=DEV)
    for _ in range(2):
        st = B.load().sl_paged_span_attention(cache.record, b, a, Q.data_ptr(), None if idx is None else idx.data_ptr(), O.data_ptr() + 2048,
                                              LSE.data_ptr() + 4096, ws.data_ptr(), need, cache.stream())
        assert st == 0
        torch.cuda.synchronize()
        edge = 2048 // O.element_size()
        assert bool((ws[need:] == 0xFF).all()) and bool((O[:edge] == 7).all()) and bool((O[edge + Q.numel():] == 7).all())
        assert bool((LSE[:1024] == 7).all()) and bool((LSE[1024 + 16 * rows:] == 7).all())
    new = torch.randn((1, rows, 64), generator=g).to(dtype).to(DEV)
    out = tuple(torch.full((1, rows + 16, 64), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    st = B.load().sl_paged_read(cache.record, b, out[0].data_ptr(), out[1].data_ptr(), rows * 64, 64, cache.stream())
    assert st == 0
    B.sl_paged_append(cache, seqs, cu, new, new)
    B.sl_paged_span_keys(cache, seqs, cu, torch.empty((2, 1, 20, 64), dtype=dtype, device=DEV), 80)
    torch.cuda.synchronize()
    assert all(bool((x[:, rows:] == 7).all()) for x in out)
    assert torch.equal(cache.tables, tables) and torch.equal(cache.lens, lens) and torch.equal(cache.refs, refs)


# ---- pages
@pytest.mark.parametrize("D,ps,layers,gap", [(128, 16, 2, 0), (64, 7, 1, 16), (64, 33, 2, 0), (128, 5, 1, 32)])
def test_pages_are_forked_and_compacted_with_their_scales(D, ps, layers, gap):
    g = torch.Generator().manual_seed(ps)
    Ls = [5 * ps + 3, 2 * ps, 1, 4 * ps - 1, 0, 0, 0]
    cache = make_cache(g, Ls, ps, 2, D, BF16, layers=layers, gap=gap, spare=6, width=2)
    lens = [L for L in Ls]

    def held():
        torch.cuda.synchronize()
        out, tables = [], cache.tables.cpu()
        for x in (cache.K, cache.V):
            codes, scales = fp4.parts(x.cpu().contiguous().numpy(), ps, D)
            for s, L in enumerate(lens):
                for t in range(L):
                    page = int(tables[s, t // ps])
                    out.append((s, t, codes[:, page, :, t % ps].tobytes(), scales[:, page, :, t % ps].tobytes()))
        return out

    before = held()
    rows = {(s, t, n): (c, sc) for n in (0, 1) for s, t, c, sc in before[n * len(before) // 2:(n + 1) * len(before) // 2]}
    assert B.sl_pages_fork(cache, i32([0, 3, 0]), i32([4, 5, 6])).tolist() == [1, 1, 1]
    lens[4], lens[5], lens[6] = Ls[0], Ls[3], Ls[0]
    after = held()
    for n in (0, 1):
        for s, t, c, sc in after[n * len(after) // 2:(n + 1) * len(after) // 2]:
            assert (c, sc) == rows[{4: 0, 5: 3, 6: 0}.get(s, s), t, n]
    B.sl_pages_free(cache, i32([0, 2]))
    lens[0] = lens[2] = 0
    want = held()
    B.sl_pages_compact(cache)
    assert held() == want
    used = int((cache.refs > 0).sum())
    assert int(cache.tables.max()) == used - 1 and bool((cache.refs[:used] > 0).all())


def test_a_run_of_steps():
    """An empty cache, prompts, a fork, single tokens with routed spans, an end: as a serving program goes."""
    g = torch.Generator().manual_seed(40)
    Hq, Hkv, D, S, ps, topk = 8, 2, 128, 32, 24, 3
    cache = B.PageCache.empty(60, ps, Hkv, D, n_seqs=4, max_pages=20, fp4=True)
    assert cache.K.dtype == torch.uint8 and cache.dtype == BF16
    Ks = torch.zeros((4, Hkv, 15, D), dtype=BF16, device=DEV)
    rows = {s: torch.zeros((2, Hkv, 0, D), dtype=torch.float64) for s in range(4)}

    def step(seqs, ns):
        cu = [sum(ns[:b]) for b in range(len(ns) + 1)]
        s32, c32 = i32(seqs), i32(cu)
        K, V = (torch.randn((Hkv, cu[-1], D), generator=g).to(BF16) for _ in range(2))
        ok = B.sl_pages_extend(cache, s32, c32)
        assert ok.tolist() == [1] * len(seqs)
        s32 = B.sl_pages_served(cache, s32, ok)
        B.sl_paged_append(cache, s32, c32, K.to(DEV), V.to(DEV))
        B.sl_paged_span_keys(cache, s32, c32, Ks, S)
        for b, s in enumerate(seqs):
            new = torch.stack([torch.from_numpy(fp4.hold(x[:, cu[b]:cu[b + 1]].double().numpy().reshape(-1, D))).view(Hkv, -1, D) for x in (K, V)])
            rows[s] = torch.cat([rows[s], new], 2)
        Q = torch.randn((Hq, cu[-1], D), generator=g).to(BF16).to(DEV)
        idx = torch.full((Hq, cu[-1], topk), -1, dtype=torch.int32, device=DEV)
        scores = torch.zeros(idx.shape, device=DEV)
        for b, s in enumerate(seqs):
            pos, at = rows[s].shape[2] - ns[b], slice(cu[b], cu[b + 1])
            idx[:, at], scores[:, at] = B.sl_span_search_prefill(Q[:, at], None, Ks[s], S, topk, q_pos0=pos, want_scores=True)
        longest = max(rows[s].shape[2] for s in seqs)
        O, LSE = B.sl_paged_span_attention(cache, s32, c32, Q, idx, S, L=longest)
        check(cache, seqs, cu, Q, idx, None, S, O, LSE)
        O = B.sl_paged_span_attention_combined(cache, s32, c32, Q, idx, scores, S, L=longest)
        check(cache, seqs, cu, Q, idx, scores, S, O)
        for s in seqs:
            n = rows[s].shape[2]
            got = B.sl_paged_read(cache, i32([s]), i32([0, n]), n)
            assert torch.equal(torch.stack(got).double().cpu(), rows[s])
            done = n // S
            assert torch.equal(Ks[s, :, :done].double().cpu(), rows[s][0][:, S - 1::S][:, :done])

    step([0, 1], [100, 150])
    step([0, 1], [1, 1])
    assert B.sl_pages_fork(cache, i32([1]), i32([2])).tolist() == [1]
    rows[2] = rows[1]
    B.sl_paged_span_keys(cache, i32([2]), i32([0, 151]), Ks, S)
    step([2, 0, 1], [5, 1, 1])
    B.sl_pages_free(cache, i32([1]))
    rows[1] = rows[1][:, :, :0]
    B.sl_pages_compact(cache)
    step([0, 2], [1, 40])
    step([1, 2, 0], [33, 1, 2])


def test_offsets_beyond_32_bits():
    """Pages whose bytes lie beyond 2^32: written, read, attended."""
    Hkv, ps, D = 8, 64, 128
    n_pages = (1 << 32) // (Hkv * B.PageCache.page_bytes(ps, D)) + 200
    cache = B.PageCache.empty(n_pages, ps, Hkv, D, n_seqs=1, max_pages=4, fp4=True)
    g = torch.Generator().manual_seed(50)
    pages = [n_pages - 1, 5, n_pages - 90]
    cache.tables[0, :3] = i32(pages)
    cache.refs[pages] = 1
    cache.lens[0] = n = 170
    K, V = (torch.randn((Hkv, n, D), generator=g).to(BF16) for _ in range(2))
    seqs, cu = i32([0]), i32([0, n])
    B.sl_paged_append(cache, seqs, cu, K.to(DEV), V.to(DEV))
    got = B.sl_paged_read(cache, seqs, cu, n)
    want = [torch.from_numpy(fp4.hold(x.double().numpy().reshape(-1, D))).view(Hkv, n, D) for x in (K, V)]
    assert all(torch.equal(a.double().cpu(), b) for a, b in zip(got, want))
    small = B.PageCache(cache.K[:, pages].contiguous(), cache.V[:, pages].contiguous(), i32([[0, 1, 2, -1]]), cache.lens, i32([1, 1, 1]),
                        page_size=ps, D=D, dtype=BF16)
    for m in (2, n):
        Q = torch.randn((16, m, D), generator=g).to(BF16).to(DEV)
        a, b = (B.sl_paged_span_attention(c, seqs, i32([0, m]), Q, None, 1000) for c in (cache, small))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
