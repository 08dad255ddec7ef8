"""The paged cache's operators against plain 64-bit forms.

Tolerances.  fp32: a score is a sum of 128 products in about nine roundings of 2^-24 each, relative to sum |q k| (about 100) / sqrt(D):
6e-6, twice that on a weight, times |v| up to 5, plus the exponential's 2^-22: below 1e-4.  bf16: the output is rounded
(2^-8 |O|), weights may be rounded once (2^-8 of A = sum p |v|), partial outputs to 11 bits of their largest element
(2^-11 max |V|): all of that beside the fp32 part."""
import math
import random

import numpy as np
import pytest
import torch

from paper_2601_18401_amd import binding as B
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def make_cache(g, Ls, ps, Hkv, D, dtype, token_major=False, layers=1, spare=3, width=1, std=1.0):
    """Sequences of Ls tokens in pages of random order.  Whatever no sequence holds is NaN."""
    need = sum(-(-L // ps) for L in Ls)
    n_pages, max_pages = need + spare, max(-(-max(Ls) // ps), 1) + width
    shape = (layers, n_pages, ps, Hkv, D) if token_major else (layers, n_pages, Hkv, ps, D)
    K, V = (torch.full(shape, math.nan, dtype=dtype, device=DEV) for _ in range(2))
    if token_major:
        K, V = K.transpose(2, 3), V.transpose(2, 3)
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
                x[:, page, :, :n] = (torch.randn((layers, Hkv, n, D), generator=g) * std).to(dtype).to(DEV)
    return B.PageCache(K, V, tables.to(DEV), i32(Ls), refs.to(DEV))


def choose(g, Hq, T, topk, spans):
    """Random distinct spans, some beyond the candidates, and empty slots among them."""
    idx = torch.stack([torch.stack([torch.randperm(max(spans, topk), generator=g)[:topk] for _ in range(T)]) for _ in range(Hq)])
    idx[torch.rand(idx.shape, generator=g) < 0.15] = -1
    return idx.to(torch.int32).to(DEV)


def check(cache, seqs, cu, Q, idx, scores, S, O, LSE=None, scale=None, layer=0, L=None):
    torch.cuda.synchronize()
    K, V = (x[layer] if x.dim() == 5 else x for x in (cache.K.cpu(), cache.V.cpu()))
    scale = scale or 1 / math.sqrt(cache.D)
    with np.errstate(invalid="ignore"):
        wO, wL, A = ref.attention(K, V, cache.tables.cpu(), cache.lens.cpu(), seqs, cu, Q.cpu(), None if idx is None else idx.cpu(),
                                  None if scores is None else scores.cpu(), S, scale, L)
    live = ~np.isnan(wL)
    got = O.double().cpu().numpy()
    assert np.isfinite(got[live]).all()
    big = float(np.nanmax(A)) if live.any() else 0.0
    tol = 1e-4 + (0 if cache.dtype == F32 else 2.0 ** -8 * (np.abs(wO) + A) + 2.0 ** -11 * max(5.0, big))
    off = np.abs(got - wO) - tol
    assert (off[live] <= 0).all(), float(off[live].max())
    if LSE is not None:
        lse = LSE.double().cpu().numpy()
        assert np.array_equal(np.isinf(lse[live]), np.isinf(wL[live]))
        fin = live & np.isfinite(wL)
        assert (np.abs(lse[fin] - wL[fin]) <= 1e-4).all()
    return live


CASES = [
    # dtype Hq Hkv D   ps   S    topk chunks                 lengths                 token-major
    (BF16, 8, 2, 128, 64, 64, 4, [1], [1], False),            # the first token of all
    (BF16, 8, 2, 128, 64, 64, 4, [1], [1000], False),
    (BF16, 4, 4, 64, 16, 40, 3, [1, 1, 1], [39, 40, 41], True),   # around a span's end
    (BF16, 6, 2, 128, 48, 96, 2, [5, 0, 1, 130], [300, 20, 97, 130], False),   # a chunk of none; pages that end inside a tile
    (BF16, 3, 1, 64, 9, 33, 5, [70], [400], True),
    (BF16, 16, 2, 128, 128, 256, 8, [33, 200], [700, 1300], False),
    (BF16, 64, 1, 64, 32, 100, 2, [3, 9], [250, 130], False),    # 64 heads on one
    (F32, 4, 2, 128, 16, 64, 4, [1, 37], [500, 200], True),
    (F32, 4, 4, 64, 7, 50, 8, [64], [333], False),
    (F32, 2, 1, 64, 1, 5, 32, [20], [64], False),             # pages of one token, all spans asked for
    (BF16, 2, 2, 128, 1, 3, 1, [17], [17], False),
    (BF16, 8, 2, 128, 50, 96, 4, [160, 77], [420, 300], False),   # buckets, pages of no multiple of 16
    (BF16, 6, 2, 64, 21, 64, 3, [300], [300], True),
    (BF16, 8, 1, 128, 100, 1000, 2, [7], [2500], False),      # spans that cross many pages, a few rows
    (F32, 6, 2, 128, 64, 48, 3, [200, 90], [300, 260], False),    # buckets in fp32
    (F32, 4, 4, 64, 13, 40, 2, [250], [250], True),
    (F32, 4, 2, 64, 32, 20, 2, [1] * 150 + [0, 3] + [1] * 120, list(range(3, 275)), False),   # many sequences of one token each
    (BF16, 4, 2, 64, 32, 20, 2, [1] * 150 + [0, 3] + [1] * 120, list(range(3, 275)), False),
    (BF16, 32, 4, 64, 16, 24, 3, [90, 50], [200, 60], False),     # more than 4096 rows and heads
    (BF16, 32, 4, 128, 16, 24, 7, [90, 50], [200, 60], True),
    (BF16, 32, 8, 64, 16, 4, 32, [140], [300], False),
    (BF16, 32, 8, 128, 32, 4, 1, [150], [3000], False),
    (BF16, 32, 1, 64, 16, 1, 8, [160], [13000], False),          # more spans than are counted in LDS
    (F32, 32, 4, 64, 16, 48, 3, [90, 60], [300, 110], False),
    (F32, 32, 4, 128, 16, 48, 9, [90, 60], [500, 70], False),
    (F32, 32, 8, 128, 16, 16, 32, [140], [700], False),
]


@pytest.mark.parametrize("form", ["joint", "gated"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c[1:]).replace(" ", ""))
def test_attention(case, form):
    dtype, Hq, Hkv, D, ps, S, topk, ns, Ls, token_major = case
    g = torch.Generator().manual_seed(len(Ls) * 1000 + Ls[0])
    cache = make_cache(g, Ls, ps, Hkv, D, dtype, token_major)
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


@pytest.mark.parametrize("dtype,Hq,Hkv,D,ps,ns,Ls", [
    (BF16, 8, 2, 128, 64, [1, 1], [1500, 3]), (BF16, 8, 1, 64, 20, [4, 1, 7], [900, 513, 7]), (BF16, 4, 4, 128, 32, [200], [200]),
    (BF16, 12, 4, 128, 64, [150, 1, 64], [900, 64, 65]), (F32, 4, 2, 64, 16, [100, 3], [100, 600]), (BF16, 2, 1, 64, 64, [300, 129], [300, 640]),
    (BF16, 5, 5, 128, 16, [257], [300]), (F32, 3, 1, 128, 64, [1], [3000]), (F32, 8, 2, 128, 32, [150, 70], [200, 70]),
    (F32, 2, 1, 64, 10, [130], [400]), (BF16, 4, 1, 128, 37, [300], [333]), (BF16, 8, 2, 64, 70, [2, 1], [600, 71]),
    (BF16, 8, 1, 64, 16, [40], [2300])])
def test_dense(dtype, Hq, Hkv, D, ps, ns, Ls):
    """No spans and S beyond every length: causal attention over all of the sequence."""
    g = torch.Generator().manual_seed(sum(Ls))
    cache = make_cache(g, Ls, ps, Hkv, D, dtype)
    cu = [sum(ns[:b]) for b in range(len(ns) + 1)]
    Q = torch.randn((Hq, sum(ns), D), generator=g).to(dtype).to(DEV)
    O, LSE = B.sl_paged_span_attention(cache, i32(list(range(len(Ls)))), i32(cu), Q, None, (1 << 31) - 1, L=max(Ls), scale=0.1)
    check(cache, list(range(len(Ls))), cu, Q, None, None, (1 << 31) - 1, O, LSE, scale=0.1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("topk,S,n", [(3, 40, 6), (0, 4000, 6), (3, 40, 150), (0, 4000, 150)])
def test_rows_without_tokens_and_rows_of_nobody(dtype, topk, S, n):
    """Missing pages (all of a row's among them), sequence numbers out of range, chunks longer than the sequence, positions
    from L on, the same sequence twice, rows before the first chunk and behind the last, a lengths entry beyond the table."""
    g = torch.Generator().manual_seed(5)
    Ls = [300, 200, 160, 30, 250]
    cache = make_cache(g, Ls, 16, 2, 64, dtype)
    cache.tables[0, 3:7] = -1
    cache.tables[0, 9] = 1 << 20
    cache.tables[1, :] = -1          # nothing left at all
    cache.tables[1, 5] = -7
    cache.lens[4] = 1 << 30          # more than the table holds: its whole table
    seqs = [0, 1, 99, 2, -1, 3, 0, 4]
    ns = [n, 3, 2, 4, 1, 40, 2, 2]
    first, behind = 5, 7
    cu = [first + sum(ns[:b]) for b in range(len(ns) + 1)]
    T = cu[-1] + behind
    Q = torch.randn((4, T, 64), generator=g).to(dtype).to(DEV)
    idx = choose(g, 4, T, topk, 8) if topk else None
    scores = torch.randn((4, T, topk), generator=g).to(DEV) if topk else None
    K, V = cache.K.clone(), cache.V.clone()
    cache.K.nan_to_num_(0.5)  # (sequence 4 names no page behind its own: what remains is unread)
    cache.V.nan_to_num_(0.5)
    for L in (0, 290):
        out = torch.full(Q.shape, 7.0, dtype=dtype, device=DEV), torch.full(Q.shape[:2], 7.0, device=DEV)
        O, LSE = B.sl_paged_span_attention(cache, i32(seqs), i32(cu), Q, idx, S, L=L, out=out)
        assert O is out[0]
        live = check(cache, seqs, cu, Q, idx, None, S, O, LSE, L=L)
        assert bool((O[:, torch.tensor(~live[0], device=DEV)] == 7).all()) and int((~live[0]).sum()) == first + behind
        if topk:
            out = torch.full(Q.shape, 7.0, dtype=dtype, device=DEV)
            B.sl_paged_span_attention_combined(cache, i32(seqs), i32(cu), Q, idx, scores, S, L=L, out=out)
            check(cache, seqs, cu, Q, idx, scores, S, out, L=L)
            assert bool((out[:, torch.tensor(~live[0], device=DEV)] == 7).all())
    cache.K.copy_(K)
    cache.V.copy_(V)


@pytest.mark.parametrize("dtype,n,ps,Hq", [(BF16, 3, 32, 4), (BF16, 130, 32, 4), (BF16, 130, 27, 4), (F32, 130, 32, 4), (F32, 3, 32, 4),
                                           (F32, 270, 27, 4), (BF16, 150, 32, 32), (F32, 200, 16, 32)])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_not_finite_where_some_rows_attend(what, dtype, n, ps, Hq):
    """A token that is not finite makes those rows not finite that attend it, as the formula has it, and no other: rows
    before it, rows whose spans leave it out."""
    g = torch.Generator().manual_seed(n)
    L, S = 400, 50
    cache = make_cache(g, [L], ps, 2, 128, dtype)
    bad = [L - 2, 120]  # one of the new tokens, and one in span 2
    clean_V = cache.V.clone()
    for t in bad:
        cache.V[0, int(cache.tables[0, t // ps]), :, t % ps, 5] = what
        clean_V[0, int(cache.tables[0, t // ps]), :, t % ps, 5] = 0
    clean = B.PageCache(cache.K, clean_V, cache.tables, cache.lens, cache.refs)
    Q = torch.randn((Hq, n, 128), generator=g).to(dtype).to(DEV)
    idx = torch.tensor([[[0, 2], [0, 1]][(h + r) % 2] for h in range(Hq) for r in range(n)], dtype=torch.int32, device=DEV).view(Hq, n, 2)
    zeros = torch.zeros(idx.shape, device=DEV)
    seqs, cu = i32([0]), i32([0, n])
    calls = [(lambda c: B.sl_paged_span_attention(c, seqs, cu, Q, idx, S)[0], S), (lambda c: B.sl_paged_span_attention_combined(c, seqs, cu, Q, idx, zeros, S), S),
             (lambda c: B.sl_paged_span_attention(c, seqs, cu, Q, None, 10 * L)[0], 10 * L)]
    for call, S in calls:
        x, w = call(cache).double().cpu(), call(clean).double().cpu()
        for h in range(Hq):
            for r in range(n):
                pos = L - n + r
                hit = any((t // S == pos // S and t <= pos) or (t // S < pos // S and t // S in idx[h, r].tolist()) for t in bad)
                if hit:
                    assert torch.isnan(x[h, r, 5]) if math.isnan(what) else x[h, r, 5].item() == what
                    x[h, r, 5] = w[h, r, 5]
        # (the two may take different kernels: two roundings each of outputs below 5)
        assert float((x - w).abs().max()) <= (2.0 ** -7 * 5 if dtype == BF16 else 1e-4)
    LSE, want = (B.sl_paged_span_attention(c, seqs, cu, Q, idx, 50)[1] for c in (cache, clean))
    assert float((LSE - want).abs().max()) <= 1e-4


def test_scores_that_are_not_finite_are_masked_like_others():
    """Keys that are not finite, behind every row's position or in spans that nobody lists, change nothing."""
    g = torch.Generator().manual_seed(21)
    for dtype, n in ((BF16, 2), (BF16, 140), (F32, 140), (F32, 2)):
        cache = make_cache(g, [500], 16, 2, 64, dtype)
        Q = torch.randn((4, n, 64), generator=g).to(dtype).to(DEV)
        idx = torch.tensor([0, 3], dtype=torch.int32, device=DEV).expand(4, n, 2).contiguous()
        cache.lens[0] = 470       # the last 30 tokens are behind the sequence's end
        args = (cache, i32([0]), i32([0, n]), Q, idx, 60)
        want = B.sl_paged_span_attention(*args)
        for k, t in enumerate([470, 480, 499, 61, 100, 179, 250]):
            cache.K[0, int(cache.tables[0, t // 16]), :, t % 16] = [math.nan, math.inf, -math.inf][k % 3]
        got = B.sl_paged_span_attention(*args)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_lists_in_the_layout_of_the_batched_search():
    """idx and scores [B][Hq][topk] of one new token per sequence, as views [Hq, B, topk]."""
    g = torch.Generator().manual_seed(22)
    for dtype in (BF16, F32):
        cache = make_cache(g, [300, 500, 90], 32, 2, 128, dtype)
        Q = torch.randn((8, 3, 128), generator=g).to(dtype).to(DEV)
        idx = choose(g, 8, 3, 4, 8).transpose(0, 1).contiguous().transpose(0, 1)
        scores = torch.randn((3, 8, 4), generator=g).to(DEV).transpose(0, 1)
        assert idx.stride() == (4, 32, 1) and scores.stride() == (4, 32, 1)
        O, LSE = B.sl_paged_span_attention(cache, i32([0, 1, 2]), i32([0, 1, 2, 3]), Q, idx, 40)
        check(cache, [0, 1, 2], [0, 1, 2, 3], Q, idx, None, 40, O, LSE)
        O = B.sl_paged_span_attention_combined(cache, i32([0, 1, 2]), i32([0, 1, 2, 3]), Q, idx, scores, 40)
        check(cache, [0, 1, 2], [0, 1, 2, 3], Q, idx, scores, 40, O)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_results_do_not_change_from_run_to_run(dtype):
    """Places in a bucket are handed out by atomics: no result may depend on them."""
    g = torch.Generator().manual_seed(23)
    cache = make_cache(g, [3000], 64, 2, 128, dtype)
    Q = torch.randn((8, 900, 128), generator=g).to(dtype).to(DEV)
    idx = choose(g, 8, 900, 4, 40)
    want = None
    for _ in range(6):
        got = B.sl_paged_span_attention(cache, i32([0]), i32([0, 900]), Q, idx, 64)
        want = want or got
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_two_captured_graphs_and_eager_calls_between():
    """Scratch of a captured call is the graph's own: replays in any order, with eager calls of other sizes between them."""
    g = torch.Generator().manual_seed(24)
    cache = make_cache(g, [2000, 700], 64, 2, 128, BF16)
    jobs = []
    for seq, n, topk in ((0, 200, 4), (1, 1, 3)):
        Q = torch.randn((8, n, 128), generator=g).to(BF16).to(DEV)
        idx, cu, seqs = choose(g, 8, n, topk, 20), i32([0, n]), i32([seq])
        jobs.append((lambda q=Q, i=idx, c=cu, s=seqs: B.sl_paged_span_attention(cache, s, c, q, i, 64)))
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
        graphs[k].replay()
        jobs[1 - k]()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[k], want[k]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("topk", [0, 8])
@pytest.mark.parametrize("cu,rows", [([0, 512] * 50 + [512], 512), ([0, 4] * 6 + [4], 4), ([300, 20, 512, -40, 512, 1 << 30, 7], 512),
                                     ([0, -5, 1 << 30, 3, 512], 512)])
def test_rows_out_of_order_stay_inside_the_arrays(cu, rows, topk, dtype):
    """cu_rows that decrease name rows twice, or rows that are none: results may be anything, what lies around them stays."""
    g = torch.Generator().manual_seed(25)
    cache = make_cache(g, [6400, 300], 64, 1, 64, dtype)
    B_ = len(cu) - 1
    seqs, cu = i32([0] * (B_ - 1) + [1]), i32(cu)
    Q = torch.randn((16, rows, 64), generator=g).to(dtype).to(DEV)
    idx = choose(g, 16, rows, topk, 18) if topk else None
    S = 320 if topk else 10000
    tables, lens, refs = cache.tables.clone(), cache.lens.clone(), cache.refs.clone()
    a = B.SlPagedAttention(16, S, topk, 0.0, 0, 0, 0, 0)
    b = cache.batch(seqs, cu, rows, 6400)
    need = B.load().sl_paged_attention_workspace_bytes(cache.record, b, a)
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device=DEV)   # (every float in it is NaN)
    O = torch.full((Q.numel() + 2048,), 7.0, dtype=dtype, device=DEV)
    LSE = torch.full((16 * rows + 2048,), 7.0, device=DEV)
    for n in range(2):
        st = B.load().sl_paged_span_attention(cache.record, b, a, Q.data_ptr(), None if idx is None else idx.data_ptr(), O.data_ptr() + 2048,
                                              LSE.data_ptr() + 4096, ws.data_ptr(), need, cache.stream())
        assert st == 0
        torch.cuda.synchronize()
        edge = 2048 // O.element_size()
        assert bool((ws[need:] == 0xFF).all()) and bool((O[:edge] == 7).all()) and bool((O[edge + Q.numel():] == 7).all())
        assert bool((LSE[:1024] == 7).all()) and bool((LSE[1024 + 16 * rows:] == 7).all())
    before = cache.K.clone()
    new = torch.randn((1, rows, 64), generator=g).to(dtype).to(DEV)
    B.sl_paged_append(cache, seqs, cu, new, new)
    cache.K.copy_(before)
    B.sl_paged_span_keys(cache, seqs, cu, torch.empty((2, 1, 20, 64), dtype=dtype, device=DEV), 320)
    torch.cuda.synchronize()
    assert torch.equal(cache.tables, tables) and torch.equal(cache.lens, lens) and torch.equal(cache.refs, refs)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fill", [0, 1, 0x7F, 0x80])
@pytest.mark.parametrize("cu", [[0, 0, 300, 10, 400], [0, 400, 0, 400, 400], [20, 390, 7, 1 << 30, 400]])
def test_rows_out_of_order_whatever_the_workspace_held(cu, fill, dtype):
    """Rows that no entry counted have places in the item list that nobody wrote, and spans that nobody checked."""
    g = torch.Generator().manual_seed(31)
    rows, topk, S = 400, 8, 320
    cache = make_cache(g, [6400, 300], 64, 1, 64, dtype)
    n = len(cu) - 1
    seqs, cu = i32([0] * (n - 1) + [1]), i32(cu)
    Q = torch.randn((16, rows, 64), generator=g).to(dtype).to(DEV)
    idx = choose(g, 16, rows, topk, 18).cpu()
    wild = torch.tensor([1 << 30, (1 << 31) - 1, -(1 << 31), -77, 20, 21], dtype=torch.int32)
    idx = torch.where(torch.rand(idx.shape, generator=g) < 0.3, wild[torch.randint(0, len(wild), idx.shape, generator=g)], idx).to(DEV)
    assert 16 * rows * topk >= 6 * n * 20 and 16 * rows * topk * S >= 1 << 19      # (buckets)
    a, b = B.SlPagedAttention(16, S, topk, 0.0, 0, 0, 0, 0), cache.batch(seqs, cu, rows, 6400)
    need = B.load().sl_paged_attention_workspace_bytes(cache.record, b, a)
    ws = torch.full((need + 8192,), fill, dtype=torch.uint8, device=DEV)
    O = torch.full((Q.numel() + 2048,), 7.0, dtype=dtype, device=DEV)
    LSE = torch.full((16 * rows + 2048,), 7.0, device=DEV)
    edge = 2048 // O.element_size()
    for _ in range(2):
        ws.fill_(fill)
        st = B.load().sl_paged_span_attention(cache.record, b, a, Q.data_ptr(), idx.data_ptr(), O.data_ptr() + 2048, LSE.data_ptr() + 4096,
                                              ws.data_ptr() + 4096, need, cache.stream())
        assert st == 0
        torch.cuda.synchronize()
        assert bool((ws[:4096] == fill).all()) and bool((ws[4096 + need:] == fill).all())
        assert bool((O[:edge] == 7).all()) and bool((O[edge + Q.numel():] == 7).all())
        assert bool((LSE[:1024] == 7).all()) and bool((LSE[1024 + 16 * rows:] == 7).all())


@pytest.mark.parametrize("dtype,n", [(BF16, 2), (BF16, 150), (F32, 2), (F32, 60), (F32, 150)])
def test_a_row_that_lists_a_span_twice_spoils_no_other(dtype, n):
    g = torch.Generator().manual_seed(26)
    cache = make_cache(g, [700], 32, 2, 64, dtype)
    Q = torch.randn((8, n, 64), generator=g).to(dtype).to(DEV)
    idx = choose(g, 8, n, 4, 14)
    idx[:, 0] = 3
    want, other = B.sl_paged_span_attention(cache, i32([0]), i32([0, n]), Q, idx, 40), idx.clone()
    other[:, 0] = i32([3, -1, -1, -1])
    got = B.sl_paged_span_attention(cache, i32([0]), i32([0, n]), Q, other, 40)
    check(cache, [0], [0, n], Q, other, None, 40, *got)
    tol = 1e-4 if dtype == F32 else 2.0 ** -7 * 5      # (places in a tile differ: two roundings each of outputs below 5)
    assert float((want[0] - got[0])[:, 1:].float().abs().max()) <= tol and float((want[1] - got[1])[:, 1:].abs().max()) <= 1e-4


def test_more_workgroups_than_a_grid_dimension_takes():
    """1200 rows of 64 heads with 16 spans of 4 tokens each, all but alone in their spans: 1.2 million pieces, against calls of 300 rows."""
    g = torch.Generator(device=DEV).manual_seed(27)
    L, ps, n, topk = 1 << 20, 64, 1200, 16
    K, V = (torch.randn((1, L // ps, 2, ps, 64), generator=g, device=DEV).to(BF16) for _ in range(2))
    tables = torch.randperm(L // ps, generator=g, device=DEV).to(torch.int32).view(1, -1)
    cache = B.PageCache(K, V, tables, i32([L]), torch.ones(L // ps, dtype=torch.int32, device=DEV))
    Q = torch.randn((64, n, 64), generator=g, device=DEV).to(BF16)
    idx = torch.randint(0, L // 4 // topk, (64, n, topk), generator=g, device=DEV, dtype=torch.int32) * topk + torch.arange(topk, dtype=torch.int32, device=DEV)
    O, LSE = B.sl_paged_span_attention(cache, i32([0]), i32([0, n]), Q, idx, 4)
    for r in range(0, n, 300):
        cache.lens.fill_(L - n + r + 300)
        o, lse = B.sl_paged_span_attention(cache, i32([0]), i32([0, 300]), Q[:, r:r + 300].contiguous(), idx[:, r:r + 300].contiguous(), 4)
        assert float((LSE[:, r:r + 300] - lse).abs().max()) <= 1e-4
        assert float((O[:, r:r + 300].float() - o.float()).abs().max()) <= 2.0 ** -7 * 5     # (two roundings each of outputs below 5)


def test_more_tiles_of_buckets_than_a_grid_dimension_takes():
    """3200 rows of 64 heads, each with sixteen of 262144 spans of 4 tokens, in buckets: a launch goes on in y beyond 2^20 workgroups, and
    what it is rounded up by has nothing to do.  Against calls of 400 rows, which take the spans one by one."""
    g = torch.Generator(device=DEV).manual_seed(29)
    L, S, ps, n, topk, Hq, Hkv = 1 << 20, 4, 64, 3200, 16, 64, 4
    items, buckets = Hq * n * topk, Hkv * (L // S)
    tiles = items // 256 + min(items, buckets)       # of the buckets
    assert items >= 3 * buckets and tiles > 1 << 20 and tiles + (n * Hq // Hkv // 256 + 1) * Hkv < 2 << 20   # (or this tests something else)
    K, V = (torch.randn((1, L // ps, Hkv, ps, 64), generator=g, device=DEV).to(BF16) for _ in range(2))
    tables = torch.randperm(L // ps, generator=g, device=DEV).to(torch.int32).view(1, -1)
    cache = B.PageCache(K, V, tables, i32([L]), torch.ones(L // ps, dtype=torch.int32, device=DEV))
    Q = torch.randn((Hq, n, 64), generator=g, device=DEV).to(BF16)
    idx = torch.randint(0, (L - n) // S // topk, (Hq, n, topk), generator=g, device=DEV, dtype=torch.int32) * topk
    idx += torch.arange(topk, dtype=torch.int32, device=DEV)
    O, LSE = B.sl_paged_span_attention(cache, i32([0]), i32([0, n]), Q, idx, S)
    for r in range(0, n, 400):
        assert Hq * 400 * topk < 3 * buckets
        cache.lens.fill_(L - n + r + 400)
        o, lse = B.sl_paged_span_attention(cache, i32([0]), i32([0, 400]), Q[:, r:r + 400].contiguous(), idx[:, r:r + 400].contiguous(), S)
        assert float((LSE[:, r:r + 400] - lse).abs().max()) <= 1e-4
        assert float((O[:, r:r + 400].float() - o.float()).abs().max()) <= 2.0 ** -7 * 5     # (two roundings each of outputs below 5)


@pytest.mark.parametrize("dtype,B_,Hkv,n", [(BF16, 32768, 32, 1), (BF16, 29200, 32, 33), (F32, 26300, 32, 33)])
def test_more_tiles_of_windows_than_a_grid_dimension_takes(dtype, B_, Hkv, n):
    """Dense calls of many short sequences (they share a page: attention does not look at refs) without any spans, narrow and wide tiles,
    against calls of an eighth of the sequences."""
    g = torch.Generator(device=DEV).manual_seed(30)
    narrow = n * B_ <= 32 * B_
    cols = 32 if narrow else 128 if dtype == F32 else 256
    assert 1 << 20 < (B_ * n // cols + B_) * Hkv < 2 << 20 and B_ * n * Hkv < 1 << 26
    K, V = (torch.randn((1, 1, Hkv, 40, 64), generator=g, device=DEV).to(dtype) for _ in range(2))
    lens = torch.randint(n, 41, (B_,), generator=g, device=DEV, dtype=torch.int32)
    cache = B.PageCache(K, V, torch.zeros((B_, 1), dtype=torch.int32, device=DEV), lens, i32([B_]))
    seqs, cu = torch.arange(B_, dtype=torch.int32, device=DEV), torch.arange(B_ + 1, dtype=torch.int32, device=DEV) * n
    Q = torch.randn((Hkv, B_ * n, 64), generator=g, device=DEV, dtype=dtype)
    O, LSE = B.sl_paged_span_attention(cache, seqs, cu, Q, None, 1000)
    tol = 1e-4 if dtype == F32 else 2.0 ** -7 * 5     # (two roundings each of outputs below 5)
    m = -(-B_ // 8)
    for b in range(0, B_, m):
        part = seqs[b:b + m]
        rows = slice(b * n, (b + part.numel()) * n)
        o, lse = B.sl_paged_span_attention(cache, part, cu[:part.numel() + 1], Q[:, rows], None, 1000)
        assert float((LSE[:, rows] - lse).abs().max()) <= 1e-4
        assert float((O[:, rows].float() - o.float()).abs().max()) <= tol
    # a few rows by hand
    for e in (0, B_ // 2, B_ - 1):
        for r in (0, n - 1):
            pos = int(lens[e]) - n + r
            z = torch.einsum("hd,htd->ht", Q[:, e * n + r].double().cpu(), K[0, 0, :, :pos + 1].double().cpu()) / 8
            want = torch.einsum("ht,htd->hd", torch.softmax(z, 1), V[0, 0, :, :pos + 1].double().cpu())
            assert float((LSE[:, e * n + r].double().cpu() - torch.logsumexp(z, 1)).abs().max()) <= 1e-4
            assert float((O[:, e * n + r].double().cpu() - want).abs().max()) <= tol


@pytest.mark.parametrize("dtype,n,D,ps", [(BF16, 3400, 128, 64), (BF16, 6700, 64, 40), (F32, 1800, 128, 16)])
def test_records_beyond_the_caches(dtype, n, D, ps):
    """Calls with more than 200 MB of records, joint and gated, against calls of 400 rows."""
    g = torch.Generator(device=DEV).manual_seed(28)
    L, S, topk, Hq = 20000, 128, 8, 32
    pages = -(-L // ps)
    K, V = (torch.randn((1, pages, 4, ps, D), generator=g, device=DEV).to(dtype) for _ in range(2))
    tables = torch.randperm(pages, generator=g, device=DEV).to(torch.int32).view(1, -1)
    cache = B.PageCache(K, V, tables, i32([L]), torch.ones(pages, dtype=torch.int32, device=DEV))
    Q = torch.randn((Hq, n, D), generator=g, device=DEV).to(dtype)
    idx = torch.randint(0, (L - n) // S // topk, (Hq, n, topk), generator=g, device=DEV, dtype=torch.int32) * topk
    idx += torch.arange(topk, dtype=torch.int32, device=DEV)
    scores = torch.randn(idx.shape, generator=g, device=DEV)
    O, LSE = B.sl_paged_span_attention(cache, i32([0]), i32([0, n]), Q, idx, S)
    C = B.sl_paged_span_attention_combined(cache, i32([0]), i32([0, n]), Q, idx, scores, S)
    tol = 1e-4 if dtype == F32 else 2.0 ** -7 * 5     # (two roundings each of outputs below 5)
    for r in range(0, n, 400):
        rows = slice(r, min(r + 400, n))
        m = rows.stop - r
        cache.lens.fill_(L - n + rows.stop)
        q, i, sc = (x[:, rows].contiguous() for x in (Q, idx, scores))
        o, lse = B.sl_paged_span_attention(cache, i32([0]), i32([0, m]), q, i, S)
        c = B.sl_paged_span_attention_combined(cache, i32([0]), i32([0, m]), q, i, sc, S)
        assert float((LSE[:, rows] - lse).abs().max()) <= 1e-4
        assert float((O[:, rows].float() - o.float()).abs().max()) <= tol and float((C[:, rows].float() - c.float()).abs().max()) <= tol


def test_append_and_span_keys():
    for dtype, Hkv, D, ps, S, ns, have, token_major in [
            (BF16, 2, 128, 64, 32, [1, 1, 1], [31, 0, 100], False), (F32, 3, 64, 10, 7, [50, 0, 13], [3, 5, 69], True),
            (BF16, 1, 64, 16, 200, [1000], [0], False), (F32, 1, 128, 33, 1, [5, 64], [10, 31], False)]:
        g = torch.Generator().manual_seed(ps)
        Ls = [n + h for n, h in zip(ns, have)]
        cache = make_cache(g, Ls, ps, Hkv, D, dtype, token_major, layers=2)
        cu = [2 + sum(ns[:b]) for b in range(len(ns) + 1)]
        T = cu[-1] + 3
        K, V = (torch.randn((T, Hkv, D), generator=g).to(dtype).to(DEV).transpose(0, 1) for _ in range(2))
        want_K, want_V = cache.K.clone(), cache.V.clone()
        Ks = torch.full((len(Ls), Hkv, max(Ls) // S + 2, D), 9.0, dtype=dtype, device=DEV)
        want_s = Ks.clone()
        cache.tables[0, 0] = -1 if have[0] == 31 else cache.tables[0, 0]
        for b, (n, L) in enumerate(zip(ns, Ls)):
            for t in range(L - n, L):
                page = int(cache.tables[b, t // ps])
                if page < 0:
                    continue
                r = cu[b] + t - (L - n)
                want_K[1, page, :, t % ps], want_V[1, page, :, t % ps] = K[:, r], V[:, r]
                if (t + 1) % S == 0:
                    want_s[b, :, t // S] = K[:, r]
        seqs = i32(list(range(len(Ls))))
        B.sl_paged_append(cache, seqs, i32(cu), K, V, layer=1)
        B.sl_paged_span_keys(cache, seqs, i32(cu), Ks, S, layer=1)
        torch.cuda.synchronize()
        assert torch.equal(cache.K.nan_to_num(3.0), want_K.nan_to_num(3.0)) and torch.equal(cache.V.nan_to_num(3.0), want_V.nan_to_num(3.0))
        assert torch.equal(Ks, want_s)
        few = torch.full((len(Ls), Hkv, 1, D), 9.0, dtype=dtype, device=DEV)     # room for one span only
        B.sl_paged_span_keys(cache, seqs, i32([0] + [sum(Ls[:b + 1]) for b in range(len(Ls))]), few, S, layer=1)   # all keys anew
        for b, L in enumerate(Ls):
            page = int(cache.tables[b, (S - 1) // ps])
            if L >= S and page >= 0:
                assert torch.equal(few[b, :, 0], cache.K[1, page, :, (S - 1) % ps])
            else:
                assert bool((few[b] == 9).all())


def test_appending_past_the_sequence_writes_nothing():
    g = torch.Generator().manual_seed(3)
    cache = make_cache(g, [20, 40], 16, 1, 64, BF16)
    before = cache.K.clone()
    K = torch.ones((1, 40, 64), dtype=BF16, device=DEV)
    B.sl_paged_append(cache, i32([77, -1]), i32([0, 5, 9]), K, K)
    torch.cuda.synchronize()
    assert torch.equal(cache.K.nan_to_num(3.0), before.nan_to_num(3.0))
    B.sl_paged_append(cache, i32([0]), i32([0, 35]), K, K)       # 35 rows, 20 tokens: the last 20 of them
    torch.cuda.synchronize()
    for t in range(20):
        assert bool((cache.K[0, int(cache.tables[0, t // 16]), 0, t % 16] == 1).all())
    assert int((cache.K == 1).all(-1).sum()) == 20


@pytest.mark.parametrize("dtype,ps", [(BF16, 16), (F32, 7)])
def test_rows_that_no_page_was_found_for_leave_other_sequences_tokens(dtype, ps):
    """A fork of a sequence that ends on a page's end shares its last page.  Without a free page it is not extended, and rows appended to it
    all the same would lie at its last tokens, which are the source's too."""
    g = torch.Generator().manual_seed(32)
    cache = B.PageCache.empty(3, ps, 2, 64, 4, 4, layers=2, dtype=dtype)
    seqs, cu = i32([0]), i32([0, 3 * ps])
    K, V = (torch.randn((2, 3 * ps, 64), generator=g).to(dtype).to(DEV) for _ in range(2))
    assert B.sl_pages_extend(cache, seqs, cu).tolist() == [1]
    for layer in range(2):
        B.sl_paged_append(cache, seqs, cu, K, V, layer)
    assert B.sl_pages_fork(cache, i32([0, 0]), i32([2, 3])).tolist() == [1, 1]
    before = cache.K.clone(), cache.V.clone()
    new = torch.ones((2, 2 * ps, 64), dtype=dtype, device=DEV)
    assert B.sl_pages_extend(cache, i32([2, 3]), i32([0, ps, 2 * ps])).tolist() == [0, 0]
    B.sl_paged_append(cache, i32([2, 3]), i32([0, ps, 2 * ps]), new, new, 1)
    torch.cuda.synchronize()
    assert torch.equal(cache.K, before[0]) and torch.equal(cache.V, before[1])
    # a source that goes on writes into a page of its own, and into its last one again once the forks are gone
    B.sl_pages_free(cache, i32([2, 3]))
    B.sl_paged_append(cache, seqs, i32([0, ps]), new[:, :ps], new[:, :ps], 1)
    torch.cuda.synchronize()
    last = int(cache.tables[0, 2])
    assert bool((cache.K[1, last] == 1).all()) and int((cache.K == 1).all(-1).sum()) == 2 * ps and torch.equal(cache.K[0], before[0][0])


@pytest.mark.parametrize("seed,n_pages,ps,n_seqs,dtype,layers", [(1, 40, 4, 12, BF16, 1), (2, 300, 3, 30, F32, 2), (3, 70, 1, 9, BF16, 1),
                                                                 (4, 17000, 2, 40, BF16, 1), (5, 1, 8, 3, BF16, 1)])
def test_page_turns(seed, n_pages, ps, n_seqs, dtype, layers):
    """Random turns of a scheduler, bad entries among them, against the bookkeeping done one step after the other."""
    rng = random.Random(seed)
    g = torch.Generator().manual_seed(seed)
    max_pages = max(2, n_pages // 3)
    cache = B.PageCache.empty(n_pages, ps, 2, 64, n_seqs, max_pages, layers, dtype)
    cache.K.copy_(torch.randn(cache.K.shape, generator=g))
    cache.V.copy_(torch.randn(cache.V.shape, generator=g))
    model = ref.Pages(cache)
    most = max_pages * ps
    for turn in range(14):
        seqs = [rng.randint(-1, n_seqs) for _ in range(rng.randint(1, n_seqs))]
        cu = [rng.randint(0, 5)]
        for _ in seqs:
            cu.append(cu[-1] + rng.choice([0, 1, rng.randint(0, most // 2 + 1), rng.randint(0, 3 * ps)]))
        ok = B.sl_pages_extend(cache, i32(seqs), i32(cu))
        assert ok.tolist() == model.extend(seqs, cu), turn
        model.agrees(cache)
        src = [rng.randint(-1, n_seqs) for _ in range(rng.randint(1, 2 * n_seqs))]
        dst = [rng.randint(-1, n_seqs) for _ in src]
        ok = B.sl_pages_fork(cache, i32(src), i32(dst))
        assert ok.tolist() == model.fork(src, dst), turn
        model.agrees(cache)
        gone = [rng.randint(-2, n_seqs + 1) for _ in range(rng.randint(0, n_seqs // 2 + 1))]
        gone += gone[:1]
        B.sl_pages_free(cache, i32(gone))
        model.free(sorted(set(gone)))
        model.agrees(cache)
        if turn % 2:
            where = B.sl_pages_compact(cache)
            assert where.tolist() == model.compact()
            model.agrees(cache)
    B.sl_pages_free(cache, i32(list(range(n_seqs))))
    assert int(cache.refs.abs().sum()) == 0 and int((cache.tables != -1).sum()) == 0


@pytest.mark.parametrize("seed,n_pages,ps,n_seqs", [(6, 70000, 1, 12), (7, 140000, 2, 7)])
def test_page_turns_in_large_pools(seed, n_pages, ps, n_seqs):
    """Pools whose counts are looked at sixteen at a time, in several passes."""
    test_page_turns(seed, n_pages, ps, n_seqs, BF16, 1)


@pytest.mark.parametrize("n_pages", [3000, 70000])
def test_tables_whose_pages_together_pass_32_bits(n_pages):
    """4096 entries of tables of 2^20 pages each: needs are summed in 64 bits.  Chunks of less than nothing are not served."""
    cache = B.PageCache.empty(n_pages, 1, 1, 64, 8, 1 << 20)
    model = ref.Pages(cache)
    rng = random.Random(n_pages)
    for _ in range(3):
        seqs = [rng.choice([-1, 8, 1 << 30, rng.randint(0, 7)]) for _ in range(4096)]
        cu = [0]
        for _ in seqs:
            cu.append(max(0, cu[-1] + rng.choice([0, 1, 3, n_pages // 5, -2, -n_pages // 5])))
        ok = B.sl_pages_extend(cache, i32(seqs), i32(cu))
        assert ok.tolist() == model.extend(seqs, cu) and 1 in ok.tolist()
        assert cache.lens.tolist() == model.lens and cache.refs.tolist() == model.refs
        assert cache.tables[:, :n_pages].tolist() == [t[:n_pages] for t in model.tables] and bool((cache.tables[:, n_pages:] == -1).all())


def test_lists_as_long_as_they_may_be():
    """4096 entries of one token each, with 4000 pages: the entry at which they run out, and that every later one is refused."""
    cache = B.PageCache.empty(4000, 16, 1, 64, 5000, 2)
    seqs, cu = i32(list(range(4096))), i32(list(range(4097)))
    ok = B.sl_pages_extend(cache, seqs, cu)
    assert ok.tolist() == [1] * 4000 + [0] * 96
    assert cache.tables[:4000, 0].tolist() == list(range(4000)) and int(cache.lens.sum()) == 4000
    again = B.sl_pages_extend(cache, seqs, cu)        # the pages have room: only the unserved ones need more
    assert again.tolist() == [1] * 4000 + [0] * 96
    B.sl_pages_free(cache, i32(list(range(0, 4096, 2))))
    ok = B.sl_pages_fork(cache, i32([1] * 4096), i32(list(range(904, 5000))))
    free_slots = [i for i, d in enumerate(range(904, 5000)) if d % 2 == 0 or d >= 4000]
    want = [0] * 4096
    for i in free_slots[:2000]:
        want[i] = 1
    assert ok.tolist() == want
    with pytest.raises(B.SlError) as e:
        B.sl_pages_extend(cache, i32([0] * 4097), i32([0] * 4098))
    assert e.value.status == 2


def test_a_serving_run_equals_the_contiguous_entry_points():
    """Prompts in chunks, span-search on the gathered keys, paged attention; forks that go on by single tokens; compaction in
    between.  Outputs against the contiguous entry points on each sequence's own tokens."""
    g = torch.Generator().manual_seed(11)
    Hq, Hkv, D, S, topk, ps = 8, 2, 128, 64, 4, 32
    cache = B.PageCache.empty(90, ps, Hkv, D, 6, 40)
    n_spans = 40 * ps // S
    Ks = torch.zeros((6, Hkv, n_spans, D), dtype=BF16, device=DEV)
    tokens = {s: (torch.empty((Hkv, 0, D), dtype=BF16, device=DEV),) * 2 for s in range(6)}

    def step(seqs, ns):
        T, cu = sum(ns), [sum(ns[:b]) for b in range(len(ns) + 1)]
        K, V = (torch.randn((Hkv, T, D), generator=g).to(BF16).to(DEV) for _ in range(2))
        Q = torch.randn((Hq, T, D), generator=g).to(BF16).to(DEV)
        ds, dcu = i32(seqs), i32(cu)
        assert B.sl_pages_extend(cache, ds, dcu).tolist() == [1] * len(seqs)
        B.sl_paged_append(cache, ds, dcu, K, V)
        B.sl_paged_span_keys(cache, ds, dcu, Ks, S)
        idx, scores = torch.empty((Hq, T, topk), dtype=torch.int32, device=DEV), torch.empty((Hq, T, topk), device=DEV)
        want = []
        for b, s in enumerate(seqs):
            rows = slice(cu[b], cu[b + 1])
            tokens[s] = tuple(torch.cat([old, new[:, rows]], 1) for old, new in zip(tokens[s], (K, V)))
            k, v = tokens[s]
            L, q = k.shape[1], Q[:, rows].contiguous()
            # (search reads Ks alone: a tensor of n_spans * S tokens stands for the cache)
            stand = torch.empty((Hkv, n_spans * S, D), dtype=BF16, device=DEV)
            i, sc = B.sl_span_search_prefill(q, stand, Ks[s], S, topk, q_pos0=L - ns[b], want_scores=True)
            wi = B.sl_span_search_prefill(q, k, None, S, topk, q_pos0=L - ns[b])
            assert torch.equal(i, wi)
            idx[:, rows], scores[:, rows] = i, sc
            want.append((B.sl_span_attention_prefill(q, k, v, i, S, q_pos0=L - ns[b]),
                         B.sl_span_attention_combined_prefill(q, k, v, i, sc, S, q_pos0=L - ns[b])))
        O, LSE = B.sl_paged_span_attention(cache, ds, dcu, Q, idx, S)
        C = B.sl_paged_span_attention_combined(cache, ds, dcu, Q, idx, scores, S)
        check(cache, seqs, cu, Q, idx, None, S, O, LSE)
        for b in range(len(seqs)):
            rows = slice(cu[b], cu[b + 1])
            (wO, wL), wC = want[b]
            assert float((O[:, rows].float() - wO.float()).abs().max()) <= 2e-2
            assert float((C[:, rows].float() - wC.float()).abs().max()) <= 2e-2
            assert float((LSE[:, rows] - wL).abs().max()) <= 2e-2

    step([0, 1], [200, 333])
    step([0, 1, 2], [150, 1, 70])
    assert B.sl_pages_fork(cache, i32([1, 1, 0]), i32([3, 4, 5])).tolist() == [1, 1, 1]
    for d, s in ((3, 1), (4, 1), (5, 0)):
        tokens[d] = tokens[s]
        Ks[d] = Ks[s]
    step([3, 4, 5, 1], [1, 1, 1, 1])
    step([4, 3, 2], [40, 1, 9])
    B.sl_pages_free(cache, i32([1, 2]))
    tokens[1] = tokens[2] = (torch.empty((Hkv, 0, D), dtype=BF16, device=DEV),) * 2
    where = B.sl_pages_compact(cache)
    used = int((cache.refs > 0).sum())
    assert bool((cache.refs[:used] > 0).all()) and int((where >= 0).sum()) == used
    step([0, 3, 4, 5, 1], [1, 1, 1, 1, 100])


@pytest.mark.parametrize("dtype,D,S,n", [(BF16, 128, 64, 1), (BF16, 128, 64, 300), (BF16, 64, 40, 70), (F32, 128, 32, 130), (F32, 64, 17, 1)])
def test_search_over_the_keys_of_a_paged_sequence(dtype, D, S, n):
    """Ks[s] without any K, against the contiguous search over the sequence's own tokens; after a fork, the keys made anew."""
    g = torch.Generator().manual_seed(35)
    Hq, Hkv, ps, L, spans = 8, 2, 16, 1000, 70
    cache = B.PageCache.empty(80, ps, Hkv, D, 5, 64, dtype=dtype)
    Ks = torch.full((5, Hkv, spans, D), math.nan, dtype=dtype, device=DEV)
    K = torch.randn((Hkv, 2 * L, D), generator=g).to(dtype).to(DEV)
    seqs, cu = i32([3, 1]), i32([0, L, 2 * L - 250])
    assert B.sl_pages_extend(cache, seqs, cu).tolist() == [1, 0]        # (80 pages)
    seqs = B.sl_pages_served(cache, seqs, i32([1, 0]))
    B.sl_paged_append(cache, seqs, cu, K, K)
    B.sl_paged_span_keys(cache, seqs, cu, Ks, S)
    Q = torch.randn((Hq, n, D), generator=g).to(dtype).to(DEV)
    want = B.sl_span_search_prefill(Q, K[:, :L].contiguous(), None, S, 4, q_pos0=L - n, want_scores=True)

    def same(got):      # (a sum of 128 products below 30, in another order)
        assert torch.equal(got[0], want[0]) and float((got[1] - want[1]).abs().nan_to_num(0).max()) <= 1e-3

    same(B.sl_span_search_prefill(Q, None, Ks[3], S, 4, q_pos0=L - n, want_scores=True))
    src, dst = i32([3, 3, 3]), i32([0, 4, 3])        # (the last is not made)
    assert B.sl_pages_fork(cache, src, dst).tolist() == [1, 1, 0]
    B.sl_paged_span_keys(cache, dst, torch.nn.functional.pad(cache.lens[dst].cumsum(0), (1, 0)).int(), Ks, S)
    for s in (0, 4, 3):
        assert torch.equal(Ks[s].nan_to_num(5.0), Ks[3].nan_to_num(5.0))
        same(B.sl_span_search_prefill(Q, None, Ks[s], S, 4, q_pos0=L - n, want_scores=True))
    assert bool(Ks[[1, 2]].isnan().all())
    with pytest.raises(B.SlError):      # rows at positions that the table has no spans for
        B.sl_span_search_prefill(Q, None, Ks[3], S, 4, q_pos0=spans * S - n + 1)


def test_a_captured_step_is_replayed():
    """extend, append, keys and attention in one graph: each replay is the next step, eager calls in between."""
    g = torch.Generator().manual_seed(12)
    Hq, Hkv, D, S, ps, n = 8, 2, 64, 32, 16, 3
    cache = B.PageCache.empty(64, ps, Hkv, D, 4, 30)
    Ks = torch.zeros((4, Hkv, 20, D), dtype=BF16, device=DEV)
    seqs, cu = i32([2, 0]), i32([0, n, n + 1])
    K, V = (torch.randn((Hkv, n + 1, D), generator=g).to(BF16).to(DEV) for _ in range(2))
    Q = torch.randn((Hq, n + 1, D), generator=g).to(BF16).to(DEV)
    idx = choose(g, Hq, n + 1, 3, 4)
    O, LSE = torch.empty_like(Q), torch.empty((Hq, n + 1), device=DEV)
    ok = torch.empty(2, dtype=torch.int32, device=DEV)
    ws = B.Workspace()
    ws.get(1 << 22)

    def step():
        B.sl_pages_extend(cache, seqs, cu, ok)
        B.sl_paged_append(cache, seqs, cu, K, V)
        B.sl_paged_span_keys(cache, seqs, cu, Ks, S)
        B.sl_paged_span_attention(cache, seqs, cu, Q, idx, S, ws=ws, out=(O, LSE))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(2, 40):
        for x in (K, V, Q):
            x.copy_(torch.randn(x.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        assert cache.lens.tolist() == [i, 0, i * n, 0] and ok.tolist() == [1, 1]
        if i % 5 == 0:
            got = O.clone()
            check(cache, [2, 0], [0, n, n + 1], Q, idx, None, S, O, LSE)
            O2, _ = B.sl_paged_span_attention(cache, seqs, cu, Q, idx, S)
            assert torch.equal(got, O2)


def test_the_packed_strides_of_pages_whose_tokens_come_first():
    """[n_pages][page_size][Hkv][D]: a page stride of 0 stands for page_size * kv_stride_t there."""
    g = torch.Generator().manual_seed(33)
    ps, Hkv, D = 16, 3, 64
    K, V = (torch.zeros((2, 4, ps, Hkv, D), dtype=BF16, device=DEV) for _ in range(2))
    whole = B.PageCache(K.transpose(2, 3), V.transpose(2, 3), i32([[2, 0, 3]]), i32([40]), i32([1, 0, 1, 1]))
    assert (whole.record.page_stride, whole.record.layer_stride) == (ps * Hkv * D, 4 * ps * Hkv * D)
    whole.record.page_stride = whole.record.layer_stride = 0
    new = torch.randn((Hkv, 40, D), generator=g).to(BF16).to(DEV)
    B.sl_paged_append(whole, i32([0]), i32([0, 40]), new, new, layer=1)
    for t in range(40):
        assert torch.equal(K[1, [2, 0, 3][t // ps], t % ps], new[:, t])
    assert int((K != 0).any(-1).sum()) == 40 * Hkv and torch.equal(K, V)
    Q = torch.randn((6, 40, D), generator=g).to(BF16).to(DEV)
    O, LSE = B.sl_paged_span_attention(whole, i32([0]), i32([0, 40]), Q, None, 100, layer=1)
    check(whole, [0], [0, 40], Q, None, None, 100, O, LSE, layer=1)


def test_a_captured_step_goes_on_where_pages_run_out():
    """extend, the served list, append, keys and attention in one graph, over a pool that runs out: sequences that no page is found for keep
    their tokens and keys, and their rows are rows without a token; once others are freed they go on."""
    g = torch.Generator().manual_seed(34)
    Hq, Hkv, D, S, ps, n, layers = 4, 2, 64, 8, 4, 3, 2
    cache = B.PageCache.empty(9, ps, Hkv, D, 4, 12, layers)
    model = ref.Pages(cache)
    Ks = torch.zeros((4, Hkv, 12 * ps // S, D), dtype=BF16, device=DEV)
    want_Ks = Ks.clone()
    seqs, cu = i32([2, 0, 3]), i32([0, n, 2 * n, 3 * n])
    K, V, Q = (torch.randn((h, 3 * n, D), generator=g).to(BF16).to(DEV) for h in (Hkv, Hkv, Hq))
    O, LSE = torch.empty_like(Q), torch.empty((Hq, 3 * n), device=DEV)
    ok, served = torch.empty(3, dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)
    ws = B.Workspace()
    ws.get(1 << 22)

    def step():
        B.sl_pages_extend(cache, seqs, cu, ok)
        B.sl_pages_served(cache, seqs, ok, served)
        for layer in range(layers):
            B.sl_paged_append(cache, served, cu, K, V, layer)
        B.sl_paged_span_keys(cache, served, cu, Ks, S, layer=1)
        B.sl_paged_span_attention(cache, served, cu, Q, None, 1000, layer=1, ws=ws, out=(O, LSE))

    def follow():
        torch.cuda.synchronize()
        got = model.extend([2, 0, 3], [0, n, 2 * n, 3 * n])
        assert ok.tolist() == got and served.tolist() == [s if k else -1 for s, k in zip([2, 0, 3], got)]
        for b, (s, k) in enumerate(zip([2, 0, 3], got)):
            for r in range(n if k else 0):
                t = model.lens[s] - n + r
                page = model.tables[s][t // ps]
                for mine, new in ((model.K, K), (model.V, V)):
                    mine[:, page, :, t % ps] = new[:, b * n + r].double().cpu()
                if (t + 1) % S == 0:
                    want_Ks[s, :, t // S] = K[:, b * n + r]
        model.agrees(cache)
        assert torch.equal(Ks, want_Ks)
        check(cache, served.tolist(), [0, n, 2 * n, 3 * n], Q, None, None, 1000, O, LSE, layer=1)
        for b, k in enumerate(got):
            rows = slice(b * n, b * n + n)
            assert bool((LSE[:, rows] == -math.inf).all()) == (not k) and bool((O[:, rows] == 0).all()) == (not k)
        return got

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    follow()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    seen = []
    for turn in range(14):
        for x in (K, V, Q):
            x.copy_(torch.randn(x.shape, generator=g))
        graph.replay()
        seen.append(follow())
        if turn == 6:
            B.sl_pages_free(cache, i32([2]))
            model.free([2])
        if turn == 9:      # a fork shares its source's pages, and goes on where there are some
            B.sl_pages_free(cache, i32([3]))
            model.free([3])
            assert B.sl_pages_fork(cache, i32([0]), i32([3])).tolist() == model.fork([0], [3])
        if turn == 11:
            B.sl_pages_free(cache, i32([0]))
            model.free([0])
    assert any(0 in k for k in seen[:7]) and any(all(k) for k in seen[:3]) and any(0 in k and 1 in k for k in seen)
    seqs_too = seqs.clone()
    assert B.sl_pages_served(cache, seqs_too, i32([0, 5, -1]), seqs_too) is seqs_too and seqs_too.tolist() == [-1, 0, 3]


def test_two_streams_at_once():
    """Calls without a workspace of the caller's do not share scratch."""
    g = torch.Generator().manual_seed(13)
    cache = make_cache(g, [3000, 2500], 64, 2, 128, BF16)
    Q = torch.randn((2, 8, 300, 128), generator=g).to(BF16).to(DEV)
    cu = i32([0, 300])
    idx = choose(g, 8, 300, 4, 40)
    alone = [B.sl_paged_span_attention(cache, i32([b]), cu, Q[b], idx, 64)[0] for b in range(2)]
    seqs = [i32([b]) for b in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(5):
        for b in range(2):
            with torch.cuda.stream(streams[b]):
                got[b] = B.sl_paged_span_attention(cache, seqs[b], cu, Q[b], idx, 64)[0]
        torch.cuda.synchronize()
        assert torch.equal(got[0], alone[0]) and torch.equal(got[1], alone[1])


def test_a_cache_beyond_32_bit_offsets():
    """Pages behind 2^32 bytes and 2^31 elements of the pool."""
    ps, Hkv, D = 64, 4, 128
    n_pages = (9 << 30) // 2 // (ps * Hkv * D)      # 9 GB of K: 4.8e9 elements
    K, V = (torch.zeros((1, n_pages, Hkv, ps, D), dtype=BF16, device=DEV) for _ in range(2))
    g = torch.Generator().manual_seed(14)
    pages = [n_pages - 1, 3, n_pages // 2 + 1, n_pages - 2]
    for p in pages:
        K[0, p], V[0, p] = (torch.randn((Hkv, ps, D), generator=g).to(BF16).to(DEV) for _ in range(2))
    tables = torch.full((2, 6), -1, dtype=torch.int32, device=DEV)
    tables[0, :4] = i32(pages)
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[torch.tensor(pages, device=DEV)] = 1
    cache = B.PageCache(K, V, tables, i32([250, 0]), refs)
    for n in (1, 200):
        Q = torch.randn((8, n, D), generator=g).to(BF16).to(DEV)
        idx = choose(g, 8, n, 2, 4)
        O, LSE = B.sl_paged_span_attention(cache, i32([0]), i32([0, n]), Q, idx, 50)
        torch.cuda.synchronize()
        small = B.PageCache(K[:, pages].contiguous(), V[:, pages].contiguous(), i32([[0, 1, 2, 3, -1, -1]] * 2), i32([250, 0]), i32([2] * 4))
        wO, wL = B.sl_paged_span_attention(small, i32([0]), i32([0, n]), Q, idx, 50)
        assert torch.equal(O, wO) and torch.equal(LSE, wL)
        check(small, [0], [0, n], Q, idx, None, 50, O, LSE)
    new = torch.ones((Hkv, 3, D), dtype=BF16, device=DEV)
    B.sl_paged_append(cache, i32([0]), i32([0, 3]), new, new)
    assert bool((K[0, n_pages - 2, :, 55:58] == 1).all()) and not bool((K[0, n_pages - 2, :, 54] == 1).any())
    assert B.sl_pages_fork(cache, i32([0]), i32([1])).tolist() == [1]
    assert torch.equal(K[0, 0, :, :58], K[0, n_pages - 2, :, :58]) and not bool(K[0, 0, :, 58:].any())
    B.sl_pages_compact(cache)
    assert sorted(cache.tables[0, :4].tolist()) == [0, 1, 2, 3] or int((cache.refs > 0).sum()) == 5
    last = int(cache.tables[0, 3])
    assert bool((K[0, last, :, 55:58] == 1).all())


def test_compaction_beyond_32_bit_offsets_moves_every_page():
    """Two sequences, forked, in pages at the far end of a pool of 9 GB: tables, counts, the map and all that the pages held."""
    ps, Hkv, D = 64, 4, 128
    n_pages = (9 << 30) // 2 // (ps * Hkv * D)
    K, V = (torch.zeros((1, n_pages, Hkv, ps, D), dtype=BF16, device=DEV) for _ in range(2))
    g = torch.Generator().manual_seed(36)
    first, second = [n_pages - 1, 3, n_pages // 2 + 1, n_pages - 2], [n_pages - 7, 1]
    for p in first + second:
        K[0, p], V[0, p] = (torch.randn((Hkv, ps, D), generator=g).to(BF16).to(DEV) for _ in range(2))
    tables = torch.full((4, 6), -1, dtype=torch.int32, device=DEV)
    tables[0, :4], tables[2, :2] = i32(first), i32(second)
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[torch.tensor(first + second, device=DEV)] = 1
    cache = B.PageCache(K, V, tables, i32([250, 0, 128, 0]), refs)
    assert B.sl_pages_fork(cache, i32([0, 2]), i32([1, 3])).tolist() == [1, 1]      # (page 0 for the last, partly filled one)
    held = {(s, k): (K[0, int(tables[s, k])].clone(), V[0, int(tables[s, k])].clone()) for s in range(4) for k in range(6) if tables[s, k] >= 0}
    used = {0: 1, 1: 2, 3: 2, n_pages // 2 + 1: 2, n_pages - 7: 2, n_pages - 2: 1, n_pages - 1: 2}
    assert {int(p): int(refs[p]) for p in (refs != 0).nonzero()} == used
    where = B.sl_pages_compact(cache)
    to = {0: 0, 1: 1, 3: 3, n_pages // 2 + 1: 2, n_pages - 7: 4, n_pages - 2: 5, n_pages - 1: 6}
    assert {int(p): int(where[p]) for p in (where != -1).nonzero()} == to
    assert tables.tolist() == [[to[p] for p in first] + [-1] * 2, [to[p] for p in first[:3]] + [0] + [-1] * 2,
                               [to[p] for p in second] + [-1] * 4, [to[p] for p in second] + [-1] * 4]
    assert refs[:7].tolist() == [n for _, n in sorted((to[p], n) for p, n in used.items())] and int((refs != 0).sum()) == 7
    for (s, k), (kept_K, kept_V) in held.items():
        assert torch.equal(K[0, int(tables[s, k])], kept_K) and torch.equal(V[0, int(tables[s, k])], kept_V)


def test_pages_of_more_pieces_than_32_bits_count():
    """A page of 2^26 tokens has 2^31 pieces of 16 bytes a head: compaction moves all of them, and a fork copies all that are filled.  (34 GB a
    page; K and V are one tensor here.)"""
    torch.cuda.empty_cache()
    ps, D = 1 << 26, 128
    K = torch.empty((1, 2, 1, ps, D), device=DEV)
    for x in K[0, 0, 0], K[0, 1, 0]:
        x.fill_(-1.0)
    mark = torch.arange(ps, dtype=torch.float32, device=DEV)      # (a row's number, rounded, and its last bits)
    K[0, 1, 0, :, 0], K[0, 1, 0, :, D - 1] = mark, mark.remainder(1021)
    cache = B.PageCache(K, K, i32([[1], [-1]]), i32([ps, 0]), i32([0, 1]))
    assert B.sl_pages_compact(cache).tolist() == [-1, 0] and cache.tables.tolist() == [[0], [-1]]
    assert torch.equal(K[0, 0, 0, :, 0], mark) and torch.equal(K[0, 0, 0, :, D - 1], mark.remainder(1021))
    K[0, 1].fill_(-1.0)
    filled = ps - 3
    cache.lens[0] = filled
    assert B.sl_pages_fork(cache, i32([0]), i32([1])).tolist() == [1] and cache.tables.tolist() == [[0], [1]]
    assert torch.equal(K[0, 1, 0, :filled, 0], mark[:filled]) and torch.equal(K[0, 1, 0, :filled, D - 1], mark[:filled].remainder(1021))
    assert bool((K[0, 1, 0, filled:] == -1).all()) and bool((K[0, 1, 0, :filled:4099, 1:D - 1] == -1).all())
    del cache, K
    torch.cuda.empty_cache()
