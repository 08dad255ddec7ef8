"""Rows of any paged cache read back: what pages hold, bit by bit."""
import pytest
import torch

from paper_2601_18401_amd import binding as B
from tests import paged_whole_reference as whole
from tests.test_paged_fp4_forms_gpu import make_cache as codes_cache
from tests.test_paged_gpu import i32, make_cache as rows_cache

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def same(got, want):
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.double().nan_to_num(0.0), want.nan_to_num(0.0))


@pytest.mark.parametrize("dtype,Hkv,D,ps,layers,token_major", [
    (BF16, 4, 128, 64, 1, False), (BF16, 3, 128, 7, 2, True), (BF16, 1, 64, 48, 3, False), (BF16, 8, 64, 1, 1, True),
    (F32, 2, 128, 16, 2, True), (F32, 1, 128, 100, 1, False), (F32, 5, 64, 9, 1, False)])
def test_rows_of_unquantised_pages(dtype, Hkv, D, ps, layers, token_major):
    """Ragged ends of sequences and whole ones; results packed, tokens first, and K and V in turn in one tensor."""
    g = torch.Generator().manual_seed(D + ps)
    Ls = [300, 1, 129, 70]
    cache = rows_cache(g, Ls, ps, Hkv, D, dtype, token_major, layers=layers)
    cache.tables[2, 0] = -1
    for ns in ([257, 1, 129, 0], [1, 0, 40, 70], Ls):
        cu = [3 + sum(ns[:b]) for b in range(5)]
        T, layer = cu[-1] + 2, layers - 1
        want = [torch.full((Hkv, T, D), 7.0, dtype=torch.float64, device=DEV) for _ in range(2)]
        for x, name in zip(want, "KV"):
            v = whole.values(cache, name, layer)
            for s, n in enumerate(ns):
                t = torch.arange(Ls[s] - n, Ls[s], device=DEV)
                page = cache.tables[s].long()[t // ps]
                x[:, cu[s]:cu[s + 1]] = torch.where((page >= 0)[:, None, None], v[page, :, t % ps], 0.0).transpose(0, 1)
        packed = torch.full((2, Hkv, T, D), 7.0, dtype=dtype, device=DEV)
        tokens = torch.full((2, T, Hkv, D), 7.0, dtype=dtype, device=DEV).transpose(1, 2)
        turns = torch.full((Hkv, T, 2 * D), 7.0, dtype=dtype, device=DEV)
        heads = torch.full((T, Hkv, 2, D), 7.0, dtype=dtype, device=DEV).permute(2, 1, 0, 3)
        for out in (tuple(packed), tuple(tokens), (turns[..., :D], turns[..., D:]), tuple(heads)):
            B.sl_paged_read(cache, i32([0, 1, 2, 3]), i32(cu), T, layer=layer, out=out)
            assert all(same(x, w) for x, w in zip(out, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_k_and_v_in_turn_from_4_bits(dtype):
    """K's and V's rows in one tensor, and results that meet are refused: the caller's tensors stay."""
    g = torch.Generator(device=DEV).manual_seed(3)
    cache = codes_cache(g, [100], 24, 2, 64, dtype)
    t = torch.arange(100, device=DEV)
    want = [whole.values(cache, name)[cache.tables[0].long()[t // 24], :, t % 24].transpose(0, 1) for name in "KV"]
    turns = torch.zeros((2, 100, 128), dtype=dtype, device=DEV)
    B.sl_paged_read(cache, i32([0]), i32([0, 100]), 100, out=(turns[..., :64], turns[..., 64:]))
    assert same(turns[..., :64], want[0]) and same(turns[..., 64:], want[1])
    before = turns.clone()
    for out in ((turns[..., :64], turns[..., :64]), (turns[..., :64], turns[..., 32:96]), (turns[:1, :, :64].expand(2, 100, 64),) * 2):
        with pytest.raises((B.SlError, ValueError)):
            B.sl_paged_read(cache, i32([0]), i32([0, 100]), 100, out=out)
    torch.cuda.synchronize()
    assert torch.equal(turns, before)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_every_code_under_every_scale(dtype, D):
    """A code's value times 2^(scale - 127) in rows of either type, below the normal range too; 2^128 and more, of scales that no append writes,
    is infinite; scale 255: NaN."""
    ps = 256
    cache = B.PageCache.empty(1, ps, 1, D, n_seqs=1, max_pages=1, dtype=dtype, fp4=True)
    cache.tables.zero_(), cache.refs.fill_(1), cache.lens.fill_(ps)
    codes = torch.arange(D, device=DEV) % 16
    for x in (cache.K, cache.V):
        x[0, 0, 0, :ps * D // 2] = (codes[0::2] | codes[1::2] << 4).to(torch.uint8).repeat(ps)
        x[0, 0, 0, ps * D // 2:] = torch.arange(ps, device=DEV).repeat_interleave(D // 32).to(torch.uint8)
    want = whole.values(cache, "K")[0]
    want = torch.where(want.abs() >= 2.0 ** 128, want.sign() * torch.inf, want)
    for x in B.sl_paged_read(cache, i32([0]), i32([0, ps]), ps):
        assert same(x, want)
    Ks = torch.zeros((1, 1, ps, D), dtype=dtype, device=DEV)
    B.sl_paged_span_keys(cache, i32([0]), i32([0, ps]), Ks, 1)
    assert same(Ks[0], want)
