"""Span-attention over a cache in 4 bits, form by form: tiles of 128 and of 256 columns with results and with records, records past the caches,
few columns in every variant of their kernel, launches beyond 2^20 workgroups.

Tolerances are those of tests/test_paged_fp4_gpu.py.  Held values are at most 3 here: fp32, below 1e-4; bf16, the output's rounding (2^-8 |O|),
weights rounded once (2^-8 of A = sum p |v|), partial outputs to 11 bits of their largest element (2^-11 * 3), beside the fp32 part."""
import pytest
import torch

from paper_2601_18401_amd import binding as B
from tests import paged_whole_reference as whole

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def make_cache(g, Ls, ps, Hkv, D, dtype):
    """Sequences of Ls tokens in pages of random order; every code, scales of 1/4 and 1/2: values of a variance about 1, at most 3.  Places that
    no sequence holds are NaN."""
    need = [-(-L // ps) for L in Ls]
    n_pages, size, at = sum(need) + 3, B.PageCache.page_bytes(ps, D), ps * (D // 2)
    K, V = (torch.randint(0, 256, (1, n_pages, Hkv, size), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2))
    tables = torch.full((len(Ls), max(need) + 1), -1, dtype=torch.int32, device=DEV)
    order, first = torch.randperm(n_pages, generator=g, device=DEV), 0
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    for x in (K, V):
        x[..., at:] = 125 + x[..., at:] % 2
    for s, (L, n) in enumerate(zip(Ls, need)):
        mine = order[first:first + n]
        first += n
        tables[s, :n] = mine.int()
        refs[mine] = 1
        left = L - (n - 1) * ps
        for x in (K, V):
            x[:, mine[-1], :, at + left * (D // 32):] = 255
    for x in (K, V):
        x[:, order[first:], :, at:] = 255
    return B.PageCache(K, V, tables, i32(Ls), refs, page_size=ps, D=D, dtype=dtype)


def spoil(cache, name, s, t):
    """The second block of token t of sequence s becomes NaN, in all heads."""
    ps, D = cache.page_size, cache.D
    getattr(cache, name)[0, int(cache.tables[s, t // ps]), :, ps * (D // 2) + t % ps * (D // 32) + 1] = 255


def distinct_spans(g, Hq, n, topk, spans):
    """Random spans below `spans` (a multiple of topk is used), distinct in a row, and some empty slots."""
    idx = torch.randint(0, spans // topk, (Hq, n, topk), generator=g, device=DEV, dtype=torch.int32) * topk
    idx += torch.arange(topk, dtype=torch.int32, device=DEV)
    idx[torch.rand(idx.shape, generator=g, device=DEV) < 0.02] = -1
    return idx


def check(cache, want, O, LSE=None):
    wO, A, wL = want
    got, spoilt = O.double(), torch.isnan(wO)
    assert torch.equal(torch.isnan(got), spoilt)
    tol = 1e-4 + (0 if cache.dtype == F32 else 2.0 ** -8 * (wO.abs() + A) + 2.0 ** -11 * 3)
    off = torch.where(spoilt, -1.0, (got - wO).abs() - tol)
    assert float(off.max()) <= 0, float(off.max())
    if LSE is not None:
        got = LSE.double()
        assert torch.equal(torch.isnan(got), torch.isnan(wL)) and torch.equal(torch.isinf(got), torch.isinf(wL))
        fin = torch.isfinite(wL)
        assert bool(((got - wL)[fin].abs() <= 1e-4).all())


def both(cache, cu, Q, idx, S, g, L=0):
    """The joint and the gated form."""
    seqs = list(range(len(cu) - 1))
    O, LSE = B.sl_paged_span_attention(cache, i32(seqs), i32(cu), Q, idx, S, L=L)
    check(cache, whole.attention(cache, seqs, cu, Q, idx, None, S), O, LSE)
    scores = torch.randn(idx.shape, generator=g, device=DEV)
    O = B.sl_paged_span_attention_combined(cache, i32(seqs), i32(cu), Q, idx, scores, S, L=L)
    check(cache, whole.attention(cache, seqs, cu, Q, idx, scores, S), O)


# ---- wide tiles
@pytest.mark.parametrize("D,ps", [(128, 64), (64, 48), (128, 40), (64, 7)])
def test_prompts_in_tiles_of_256_columns(D, ps):
    """One piece a row, which the tiles write themselves; a page that is missing, blocks held as NaN that some rows attend."""
    g = torch.Generator(device=DEV).manual_seed(D + ps)
    Hq, Hkv, ns, Ls = 64, 4, [2600, 1, 1499], [3000, 5, 1600]
    cu = [0, 2600, 2601, 4100]
    assert cu[-1] * Hq >= 1 << 18
    cache = make_cache(g, Ls, ps, Hkv, D, BF16)
    cache.tables[0, 700 // ps] = -1
    spoil(cache, "V", 0, 2990)
    spoil(cache, "K", 2, 1590)
    Q = torch.randn((cu[-1], Hq, D), generator=g, device=DEV).to(BF16).transpose(0, 1)
    O, LSE = B.sl_paged_span_attention(cache, i32([0, 1, 2]), i32(cu), Q, None, 1 << 20, L=max(Ls))
    check(cache, whole.attention(cache, [0, 1, 2], cu, Q, None, None, 1 << 20), O, LSE)


def width_of_tiles(items, columns, buckets):
    """Columns of the tiles that bf16 rows in buckets are taken by: fewer where those of 256 would stand a third emptier."""
    assert items >= 3 * buckets
    n = items // buckets
    emptier = -(-n // 256) * 256 * 3 >= -(-n // 128) * 128 * 4
    return 256 if columns + items >= 1 << 18 and not emptier else 128


@pytest.mark.parametrize("D,ps,spans,width", [(64, 64, 300, 256), (128, 64, 300, 256), (64, 20, 300, 256), (128, 33, 300, 256),
                                              (64, 64, 200, 128), (128, 64, 200, 128), (64, 20, 200, 128), (128, 33, 200, 128)])
def test_buckets_of_both_widths(D, ps, spans, width):
    """1000 rows of 32 heads with eight spans of 64 tokens each, from two sequences."""
    g = torch.Generator(device=DEV).manual_seed(spans + D + ps)
    Hq, Hkv, S, topk, cu, Ls = 32, 4, 64, 8, [0, 640, 1000], [spans * 32, spans * 32]
    assert width_of_tiles(Hq * 1000 * topk, 1000 * Hq, 2 * Hkv * (spans // 2)) == width
    cache = make_cache(g, Ls, ps, Hkv, D, BF16)
    cache.tables[1, 900 // ps] = 1 << 20
    spoil(cache, "V", 0, 5 * S + 3)
    spoil(cache, "K", 1, 9 * S + 60)
    Q = torch.randn((Hq, 1000, D), generator=g, device=DEV).to(BF16)
    both(cache, cu, Q, distinct_spans(g, Hq, 1000, topk, spans // 2), S, g, L=max(Ls))


@pytest.mark.parametrize("dtype,n,D,ps,S,L,width", [
    (BF16, 3400, 128, 64, 128, 20000, 256), (BF16, 6700, 64, 40, 128, 20000, 256), (BF16, 3400, 128, 25, 128, 20000, 256),
    (BF16, 6700, 64, 16, 128, 20000, 256), (BF16, 3400, 128, 64, 32, 21760, 128), (BF16, 3400, 128, 40, 32, 21760, 128),
    (BF16, 6700, 64, 64, 16, 21440, 128), (BF16, 6700, 64, 9, 16, 21440, 128),
    (F32, 1800, 128, 16, 128, 20000, 128), (F32, 1800, 128, 9, 128, 20000, 128), (F32, 3700, 64, 32, 128, 20000, 128), (F32, 3700, 64, 50, 128, 20000, 128)])
def test_records_beyond_the_caches(dtype, n, D, ps, S, L, width):
    """Calls with 230 MiB of records and more, which are written past the caches."""
    g = torch.Generator(device=DEV).manual_seed(n + ps)
    Hq, Hkv, topk, spans = 32, 4, 8, -(-L // S)
    assert Hq * n * (topk + 1) * D * (2 if dtype == BF16 else 4) >= 230 << 20
    assert dtype == F32 or width_of_tiles(Hq * n * topk, n * Hq, Hkv * spans) == width
    cache = make_cache(g, [L], ps, Hkv, D, dtype)
    cache.tables[0, 3000 // ps] = -1
    spoil(cache, "V", 0, 77 * S + 3)
    Q = torch.randn((Hq, n, D), generator=g, device=DEV).to(dtype)
    both(cache, [0, n], Q, distinct_spans(g, Hq, n, topk, (L - n) // S), S, g, L=L)


# ---- few columns
@pytest.mark.parametrize("D,ps", [(64, 64), (128, 32), (64, 8), (128, 40), (64, 20), (128, 7)])
@pytest.mark.parametrize("Hq,Hkv,ns", [
    (8, 2, [1, 1, 1]), (3, 1, [1, 5, 4]), (15, 3, [2, 3, 0]), (16, 1, [1, 1, 1]),      # up to 16 columns
    (24, 1, [1, 1, 1]), (9, 3, [10, 7, 9]), (64, 2, [1, 1, 0]), (20, 4, [6, 5, 6]),    # up to 32
    (64, 1, [3, 1, 2])])                                                              # more, in spans alone
def test_few_columns(Hq, Hkv, ns, D, ps):
    """Pages of a multiple of 32 tokens, of 8, and others; groups that are no power of two; dense calls, and spans of 70, 24 and 6 tokens, of
    which a workgroup takes a piece, one, and several."""
    g = torch.Generator(device=DEV).manual_seed(Hq * D + ps)
    Ls = [1600, 77, 903]
    cu = [sum(ns[:b]) for b in range(len(ns) + 1)]
    cache = make_cache(g, Ls, ps, Hkv, D, BF16)
    cache.tables[0, 300 // ps] = -1
    spoil(cache, "V", 2, 500)
    Q = torch.randn((Hq, cu[-1], D), generator=g, device=DEV).to(BF16)
    if cu[-1] * (Hq // Hkv) <= 32 * len(ns):
        O, LSE = B.sl_paged_span_attention(cache, i32([0, 1, 2]), i32(cu), Q, None, 5000)
        check(cache, whole.attention(cache, [0, 1, 2], cu, Q, None, None, 5000), O, LSE)
    spoil(cache, "K", 0, 1000)
    for S, topk in ((70, 4), (24, 7), (6, 32)):
        assert Hq * cu[-1] * topk < 3 * 3 * Hkv * (16000 // S)       # (as many spans as L has are no buckets)
        idx = distinct_spans(g, Hq, cu[-1], topk, max(max(Ls) // S, topk))
        idx[:, ::2] = idx[:1, ::2]       # heads that share their spans
        idx[idx == 500 // S] = -1        # (the spoilt blocks spoil few rows)
        idx[: Hq // 2][idx[: Hq // 2] == 1000 // S] = -1
        wide = torch.full((3, -(-16000 // ps)), -1, dtype=torch.int32, device=DEV)
        wide[:, :cache.tables.shape[1]] = cache.tables
        both(B.PageCache(cache.K, cache.V, wide, cache.lens, cache.refs, page_size=ps, D=D), cu, Q, idx, S, g)


@pytest.mark.parametrize("dtype,n", [(BF16, 2), (BF16, 150), (F32, 2), (F32, 60), (F32, 150)])
@pytest.mark.parametrize("S", [40, 5])
def test_a_row_that_lists_a_span_twice_spoils_no_other(dtype, n, S):
    """(Spans of five tokens: a workgroup takes several slots of a row.)"""
    g = torch.Generator(device=DEV).manual_seed(26)
    cache = make_cache(g, [700], 32, 2, 64, dtype)
    Q = torch.randn((8, n, 64), generator=g, device=DEV).to(dtype)
    once = distinct_spans(g, 8, n, 4, 540 // S)
    once[:, 0] = i32([6, 2, -1, -1])
    once[:, 1:, 2] = 2      # others list what the first row lists
    twice = once.clone()
    twice[:, 0] = i32([6, 2, 2, 6])
    want = [x[:, 1:] for x in whole.attention(cache, [0], [0, n], Q, once, None, S)]
    for lists in (once, twice):
        O, LSE = B.sl_paged_span_attention(cache, i32([0]), i32([0, n]), Q, lists, S)
        check(cache, want, O[:, 1:], LSE[:, 1:])


def test_more_units_of_few_columns_than_a_grid_dimension_takes():
    """17000 rows of 64 heads, each with one of 262144 spans of 4 tokens: more than 2^20 lists, against calls of 2000 rows."""
    g = torch.Generator(device=DEV).manual_seed(27)
    L, ps, n, S, Hq, Hkv = 1 << 20, 64, 17000, 4, 64, 2
    assert 1 << 20 < n * Hq < 3 * Hkv * (L // S)
    cache = make_cache(g, [L - 64], ps, Hkv, 64, BF16)
    assert cache.tables.shape[1] * ps == L
    Q = torch.randn((Hq, n, 64), generator=g, device=DEV).to(BF16)
    idx = torch.randint(0, (L - 64 - n) // S, (Hq, n, 1), generator=g, device=DEV, dtype=torch.int32)
    O, LSE = B.sl_paged_span_attention(cache, i32([0]), i32([0, n]), Q, idx, S)
    for r in range(0, n, 2000):
        rows = slice(r, min(r + 2000, n))
        m = rows.stop - r
        cache.lens.fill_(L - 64 - n + rows.stop)
        o, lse = B.sl_paged_span_attention(cache, i32([0]), i32([0, m]), Q[:, rows].contiguous(), idx[:, rows].contiguous(), S)
        assert float((LSE[:, rows] - lse).abs().max()) <= 1e-4
        assert float((O[:, rows].float() - o.float()).abs().max()) <= 2.0 ** -7 * 3     # (two roundings each of outputs below 3)


@pytest.mark.parametrize("dtype,B_,Hkv,n", [(BF16, 32768, 32, 1), (BF16, 32700, 32, 20), (BF16, 29200, 32, 33), (F32, 26300, 32, 33)])
def test_more_tiles_of_windows_than_a_grid_dimension_takes(dtype, B_, Hkv, n):
    """Dense calls of many short sequences (they share a page: attention does not look at refs), tiles of 16, 32, 256 and 128 columns, against calls
    of an eighth of the sequences."""
    g = torch.Generator(device=DEV).manual_seed(30)
    cols = 16 if n <= 16 else 32 if n <= 32 else 128 if dtype == F32 else 256
    assert 1 << 20 < (B_ * n // cols + B_) * Hkv < 2 << 20 and B_ * n * Hkv < 1 << 26
    cache = make_cache(g, [40], 40, Hkv, 64, dtype)
    page = int(cache.tables[0, 0])
    lens = torch.randint(n, 41, (B_,), generator=g, device=DEV, dtype=torch.int32)
    many = B.PageCache(cache.K, cache.V, torch.full((B_, 1), page, dtype=torch.int32, device=DEV), lens, cache.refs, page_size=40, D=64, dtype=dtype)
    seqs, cu = torch.arange(B_, dtype=torch.int32, device=DEV), torch.arange(B_ + 1, dtype=torch.int32, device=DEV) * n
    Q = torch.randn((Hkv, B_ * n, 64), generator=g, device=DEV, dtype=dtype)
    O, LSE = B.sl_paged_span_attention(many, seqs, cu, Q, None, 1000)
    m = -(-B_ // 8)
    for b in range(0, B_, m):
        part = seqs[b:b + m]
        rows = slice(b * n, (b + part.numel()) * n)
        o, lse = B.sl_paged_span_attention(many, part, cu[:part.numel() + 1], Q[:, rows], None, 1000)
        assert float((LSE[:, rows] - lse).abs().max()) <= 1e-4
        # (two roundings each of outputs below 3)
        assert float((O[:, rows].float() - o.float()).abs().max()) <= (1e-4 if dtype == F32 else 2.0 ** -7 * 3)
    few = [0, 1, B_ // 2, B_ - 1]      # by hand
    some = B.PageCache(cache.K, cache.V, many.tables[few], lens[few], cache.refs, page_size=40, D=64, dtype=dtype)
    rows = torch.cat([torch.arange(e * n, (e + 1) * n, device=DEV) for e in few])
    want = whole.attention(some, [0, 1, 2, 3], [k * n for k in range(5)], Q[:, rows], None, None, 1000)
    check(some, want, O[:, rows], LSE[:, rows])


@pytest.mark.parametrize("dtype,n,ps,Hq", [(BF16, 3, 32, 4), (BF16, 3, 27, 40), (BF16, 130, 32, 4), (BF16, 130, 27, 4), (F32, 3, 32, 4), (F32, 300, 27, 4),
                                           (F32, 200, 16, 32)])
@pytest.mark.parametrize("tensor", ["K", "V"])
def test_infinite_blocks_where_some_rows_attend(tensor, dtype, n, ps, Hq):
    """Scales 253 and 254, which no append writes: rows that attend such a token are not finite (in its 32 channels, or, of a key, all), and no
    other is."""
    g = torch.Generator(device=DEV).manual_seed(n)
    L, S = 400, 50
    cache, marked = (make_cache(torch.Generator(device=DEV).manual_seed(n), [L], ps, 2, 128, dtype) for _ in range(2))
    for t, scale in ((L - 2, 253), (120, 254)):
        page, at = int(cache.tables[0, t // ps]), ps * 64 + t % ps * 4 + 1
        x = getattr(cache, tensor)[0, page]
        x[:, t % ps * 64 + 16:t % ps * 64 + 32] = 0x77      # sixes
        x[:, at] = scale
        spoil(marked, tensor, 0, t)
    Q = torch.randn((Hq, n, 128), generator=g, device=DEV).to(dtype)
    idx = torch.tensor([[[0, 2], [0, 1]][(h + r) % 2] for h in range(Hq) for r in range(n)], dtype=torch.int32, device=DEV).view(Hq, n, 2)
    scores = torch.randn(idx.shape, generator=g, device=DEV)
    seqs, cu = i32([0]), i32([0, n])
    for got, want in ((B.sl_paged_span_attention(cache, seqs, cu, Q, idx, S)[0], whole.attention(marked, [0], [0, n], Q, idx, None, S)),
                      (B.sl_paged_span_attention_combined(cache, seqs, cu, Q, idx, scores, S), whole.attention(marked, [0], [0, n], Q, idx, scores, S)),
                      (B.sl_paged_span_attention(cache, seqs, cu, Q, None, 4000)[0], whole.attention(marked, [0], [0, n], Q, None, None, 4000))):
        check(cache, want, torch.where(torch.isfinite(got), got, torch.nan))
