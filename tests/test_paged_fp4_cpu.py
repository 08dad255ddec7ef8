"""What a paged cache in 4 bits refuses, without a GPU; and the plain format that its other tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2601_18401_amd import binding as B
from tests import fp4_reference as fp4
from tests.test_paged_cpu import BAD_ATTENTION, BAD_BATCH, P, records

PART = B.PageCache.page_bytes(64, 128)
GOOD = dict(dtype=B.SL_MXFP4 + B.SL_BF16)


def cache_calls(lib, c, b):
    return [lib.sl_pages_extend(c, b, P, None), lib.sl_pages_fork(c, P, P, 1, P, None), lib.sl_pages_free(c, P, 1, None),
            lib.sl_pages_compact(c, P, P, 1 << 40, None), lib.sl_paged_append(c, b, P, P, 0, 0, None), lib.sl_paged_read(c, b, P, P, 0, 0, None),
            lib.sl_paged_span_keys(c, b, 64, 10, P, None)]


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=15), 1), (dict(dtype=18), 1), (dict(dtype=2), 1), (dict(dtype=-1), 1), (dict(K=None), 1), (dict(V=P + 8), 1), (dict(D=96), 2),
    (dict(kv_stride_t=32), 1), (dict(kv_stride_t=128), 1), (dict(kv_stride_h=PART - 16), 1), (dict(kv_stride_h=PART + 8), 1),
    (dict(page_stride=PART - 16), 1), (dict(page_stride=4 * PART + 8), 1), (dict(layer_stride=64), 1), (dict(kv_stride_h=-16), 1),
    (dict(page_stride=1 << 50), 2), (dict(n_pages=1 << 20, page_stride=1 << 40), 2), (dict(layers=512, layer_stride=1 << 48), 2),
    (dict(max_pages=1 << 25, page_size=64), 2), (dict(page_size=0), 1), (dict(Hkv=2048), 2)])
def test_caches_are_refused(kw, status):
    lib = B.load()
    c, b, a = records(**{**GOOD, **kw})
    args = [ctypes.byref(x) for x in (c, b, a)]
    assert cache_calls(lib, *args[:2]) == [status] * 7
    assert lib.sl_pages_compact_workspace_bytes(args[0]) == B.WORKSPACE_INVALID
    assert lib.sl_paged_attention_workspace_bytes(*args) == B.WORKSPACE_INVALID
    assert lib.sl_paged_span_attention(*args, P, P, P, P, P, 1 << 40, None) == status
    assert lib.sl_paged_span_attention_combined(*args, P, P, P, P, P, 1 << 40, None) == status


@pytest.mark.parametrize("kw", [dict(), dict(kv_stride_t=64), dict(kv_stride_h=PART, page_stride=4 * PART, layer_stride=400 * PART),
                                dict(kv_stride_h=PART + 16), dict(dtype=B.SL_MXFP4), dict(D=64), dict(page_size=7, max_pages=1 << 20),
                                dict(page_size=1 << 30, max_pages=1, n_pages=1 << 12)])
def test_caches_are_taken(kw):
    c, b, a = (ctypes.byref(x) for x in records(**{**GOOD, **kw}))
    assert B.load().sl_paged_attention_workspace_bytes(c, b, a) not in (0, B.WORKSPACE_INVALID)
    assert B.load().sl_pages_compact_workspace_bytes(c) != B.WORKSPACE_INVALID


@pytest.mark.parametrize("dtype", [B.SL_F32, B.SL_BF16, B.SL_MXFP4 + B.SL_F32, B.SL_MXFP4 + B.SL_BF16])
def test_reads_are_refused(dtype):
    lib = B.load()
    for kw, status in BAD_BATCH:
        c, b, _ = (ctypes.byref(x) for x in records(dtype=dtype, **kw))
        assert lib.sl_paged_read(c, b, P, P, 0, 0, None) == status
    c, b, _ = (ctypes.byref(x) for x in records(dtype=dtype))
    for args, status in (((None, P, 0, 0), 1), ((P, None, 0, 0), 1), ((P + 8, P, 0, 0), 1), ((P, P + 4, 0, 0), 1), ((P, P, -8, 0), 1),
                         ((P, P, 0, -8), 1), ((P, P, 0, 120), 1), ((P, P, 0, 130), 1), ((P, P, 4 * 128 + 2, 128), 1), ((P, P, 64, 512), 1), ((P, P, 128, 128), 1),
                         ((P, P, 39 * 128, 128), 1), ((P, P, 128, 3 * 128), 1),
                         ((P, P, 1 << 50, 0), 2), ((P, P, 0, 1 << 40), 2)):
        assert lib.sl_paged_read(c, b, *args, None) == status
    for kw in (dict(B=0, seqs=None, cu_rows=None), dict(rows=0)):
        c, b, _ = (ctypes.byref(x) for x in records(dtype=dtype, **kw))
        assert lib.sl_paged_read(c, b, None, None, 0, 0, None) == 0


def test_attention_and_appends_are_refused_as_of_other_caches():
    lib = B.load()
    for kw, status in BAD_BATCH + BAD_ATTENTION:
        args = [ctypes.byref(x) for x in records(**{**GOOD, **kw})]
        assert lib.sl_paged_span_attention(*args, P, P, P, P, P, 1 << 40, None) == status
    c, b, a = (ctypes.byref(x) for x in records(**GOOD))
    size = lib.sl_paged_attention_workspace_bytes(c, b, a)
    assert lib.sl_paged_span_attention(c, b, a, P, P, P, P, P, size - 1, None) == 3
    assert lib.sl_paged_span_attention(c, b, a, P + 8, P, P, P, P, size, None) == 1
    assert lib.sl_paged_append(c, b, P, None, 0, 0, None) == 1 and lib.sl_paged_append(c, b, P, P, 0, 100, None) == 1


def test_contiguous_calls_take_no_cache_in_4_bits():
    lib = B.load()
    for dtype in (16, 17):
        p = B.SlParams(4096, 4096, 0, 8, 2, 128, 64, 4, dtype, 0.0, 0, 0, 0, 0, 0)
        assert lib.sl_workspace_bytes(ctypes.byref(p), B.OP_ATTENTION_PREFILL) == B.WORKSPACE_INVALID
        assert lib.sl_span_keys(ctypes.byref(p), P, P, None) == 1


def test_the_binding_refuses_tensors_that_do_not_fit():
    cache = B.PageCache.empty(6, 16, 2, 64, 3, 4, device="cpu", fp4=True)
    size = 16 * 34
    assert cache.K.shape == (1, 6, 2, size) and cache.K.dtype == torch.uint8 and cache.dtype == torch.bfloat16
    assert cache.record.dtype == 17 and cache.record.kv_stride_h == size and cache.record.kv_stride_t == 0
    assert B.PageCache.empty(6, 16, 2, 64, 3, 4, dtype=torch.float32, device="cpu", fp4=True).record.dtype == 16
    assert B.PageCache.page_bytes(7, 64) == 240 and B.PageCache.page_bytes(16, 128) == 16 * 68
    K, rest = cache.K, (cache.tables, cache.lens, cache.refs)
    B.PageCache(K[0], K[0].clone(), *rest, page_size=16, D=64)
    ok = dict(page_size=16, D=64)
    for kv, kw in (((K, K), {}), ((K, K), dict(page_size=16)), ((K, K), dict(page_size=15, D=64)), ((K, K), dict(page_size=16, D=128)),
                   ((K, K), dict(page_size=8, D=96)), ((K[..., :-16], K[..., :-16]), ok), ((K, K[:, :5]), ok), ((K, K.bfloat16()), ok),
                   ((K[..., ::2], K[..., ::2]), ok), ((K[:, :1].expand(1, 6, 2, size), K[:, :1].expand(1, 6, 2, size)), ok)):
        with pytest.raises(ValueError):
            B.PageCache(*kv, *rest, **kw)
    odd = torch.zeros((1, 6, 2, size + 1), dtype=torch.uint8)
    with pytest.raises(ValueError):
        B.PageCache(odd[..., 1:], odd[..., 1:], *rest, **ok)
    with pytest.raises(TypeError):
        B.PageCache(K, K.clone(), *rest, **ok, dtype=torch.float16)
    rows = torch.zeros((1, 6, 2, 16, 64), dtype=torch.bfloat16)
    B.PageCache(rows, rows.clone(), *rest, page_size=16, D=64, dtype=torch.bfloat16)
    for kw in (dict(page_size=8), dict(D=128), dict(dtype=torch.float32)):
        with pytest.raises(ValueError):
            B.PageCache(rows, rows.clone(), *rest, **kw)
    one, two = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    new = torch.zeros((2, 3, 64), dtype=torch.bfloat16)
    for out in ((new, new.float()), (new.float(), new.float()), (new[:1], new[:1]), (new, new.transpose(0, 1).contiguous().transpose(0, 1)),
                (new[:, :1].expand(2, 3, 64), new[:, :1].expand(2, 3, 64))):
        with pytest.raises(ValueError):
            B.sl_paged_read(cache, one, two, 3, out=out)
    with pytest.raises(ValueError):
        B.sl_paged_read(cache, one, two, 2, out=(new, new.clone()))
    with pytest.raises(ValueError):
        B.sl_paged_append(cache, one, two, new.float(), new.float())
    with pytest.raises(ValueError):
        B._paged_attention(cache, one, two, torch.zeros((4, 3, 64)), None, None, 16, 0, 0, 0.0, None)
    with pytest.raises(ValueError):      # a cache in host memory
        B.sl_paged_read(cache, one, two, 3)


def test_the_plain_format():
    """Half way to the even code; the power of two that leaves the largest value below 7; ends of the range; blocks that are not finite."""
    row = np.zeros(32)
    row[:11] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6.99, -6.99, 0.2501, -0.0]
    assert fp4.hold(row[None])[0, :11].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, -6, 0.5, 0]
    for top, scale in ((6.99, 127), (7.0, 128), (13.99, 128), (3.49, 126), (3.5, 127), (0.0, 2), (2.0 ** -140, 2), (3.3e38, 252)):
        row[:] = 0
        row[3] = -top
        assert fp4.block_scale(row) == scale
        held = fp4.hold(row[None])[0, 3]
        # half a step of e2m1 (1 in [4, 6]), what is cut off above 6, or, at the ends of the scales' range, half of the smallest step
        assert abs(held + top) <= max(top / 6, 2.0 ** -127) or scale == 252
    row[3] = np.nan
    assert fp4.block_scale(row) == 255 and np.isnan(fp4.hold(row[None])).all()
    codes = np.arange(64, dtype=np.uint8).reshape(2, 32) % 16
    assert np.array_equal(fp4.unpack(fp4.pack(codes)), codes)


@pytest.mark.parametrize("dtype", [B.SL_F32, B.SL_BF16, B.SL_MXFP4 + B.SL_F32, B.SL_MXFP4 + B.SL_BF16])
def test_reads_into_rows_of_k_that_are_rows_of_v_are_refused(dtype):
    """40 rows of 4 heads, 128 channels; V begins so many elements behind K, or before it."""
    lib = B.load()
    es = 2 if dtype % 16 == B.SL_BF16 else 4
    c, b, _ = (ctypes.byref(x) for x in records(dtype=dtype))
    for behind, sh, st in ((0, 0, 0), (120, 0, 0), (128, 0, 0), (4 * 40 * 128 - 8, 0, 0), (128, 40 * 256, 256 - 16), (8, 128, 4 * 128),
                           (3 * 40 * 256 + 39 * 256, 0, 256), (40 * 128 + 8, 2 * 40 * 128, 128)):
        meets = any(abs(behind - h * (sh or 40 * (st or 128)) - t * (st or 128)) < 128 for h in range(-3, 4) for t in range(-39, 40))
        assert meets
        for k, v in ((P, P + behind * es), (P + behind * es, P)):
            assert lib.sl_paged_read(c, b, k, v, sh, st, None) == 1


def test_limits_under_address_and_undefined_sanitizers(tmp_path):
    """Validation, size arithmetic, and whether rows meet, of records at and beyond every limit, in a build of the host side with ASan + UBSan."""
    import glob
    import os
    import shutil
    import subprocess
    from paper_2601_18401_amd import build as _build
    clang = "/opt/rocm/lib/llvm/bin/clang"
    if not os.path.exists(clang) or not shutil.which("hipcc"):
        pytest.skip("no ROCm clang")
    sources = _build.sources() + glob.glob(os.path.join(_build.CSRC, "*.h")) + [os.path.join(_build.ROOT, "include", "sl.h")]
    built = os.path.exists(_build.SAN_LIB) and os.path.getmtime(_build.SAN_LIB) > max(os.path.getmtime(s) for s in sources)
    lib = _build.SAN_LIB if built else _build.build(sanitize=True)
    exe = str(tmp_path / "fp4_limits_from_c")
    subprocess.run([clang, "-std=c99", "-Wall", "-Wextra", "-Werror", "-g", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=undefined", "-shared-libsan", "-I", os.path.join(_build.ROOT, "include"),
                    os.path.join(_build.ROOT, "tests", "cabi", "fp4_limits_from_c.c"), "-o", exe, "-ldl"], check=True)
    rt = os.path.dirname(glob.glob("/opt/rocm*/lib/llvm/lib/clang/*/lib/*/libclang_rt.asan*.so")[0])
    env = dict(os.environ, LD_LIBRARY_PATH=rt, ASAN_OPTIONS="detect_leaks=0")
    run = subprocess.run([exe, lib], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0 and "wrong=0" in run.stdout, (run.stdout, run.stderr[-3000:])
    assert "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr, run.stderr[-3000:]


def test_reads_into_heads_beyond_what_64_bits_address_are_refused():
    c, b, _ = (ctypes.byref(x) for x in records(**GOOD, rows=1 << 25))
    assert B.load().sl_paged_read(c, b, P, P, 0, 1 << 32, None) == 2
    c, b, _ = (ctypes.byref(x) for x in records(**GOOD, rows=1 << 25, Hkv=1024))
    assert B.load().sl_paged_read(c, b, P, P, 0, 1 << 25, None) == 2
