"""The paged cache's refusals, without a GPU: every status comes back before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_2601_18401_amd import binding as B

P = 1 << 20  # a pointer that nothing dereferences


def records(**kw):
    c = B.SlPageCache(P, P, P, P, P, 0, 0, 0, 0, 2, 100, 8, 50, 64, 4, 128, B.SL_BF16)
    b = B.SlPagedBatch(P, P, 40, 0, 3, 1)
    a = B.SlPagedAttention(32, 256, 8, 0.0, 0, 0, 0, 0)
    for k, v in kw.items():
        for r in (c, b, a):
            if k in [f[0] for f in r._fields_]:
                setattr(r, k, v)
                break
        else:
            raise KeyError(k)
    return c, b, a


def need(**kw):
    c, b, a = records(**kw)
    return B.load().sl_paged_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(b), ctypes.byref(a))


def test_record_sizes():
    assert ctypes.sizeof(B.SlPageCache) == 5 * 8 + 4 * 8 + 8 * 4
    assert ctypes.sizeof(B.SlPagedBatch) == 2 * 8 + 2 * 8 + 8
    assert ctypes.sizeof(B.SlPagedAttention) == 16 + 4 * 8


BAD_CACHE = [(dict(K=None), 1), (dict(V=P + 8), 1), (dict(tables=None), 1), (dict(tables=P + 2), 1), (dict(lens=None), 1), (dict(refs=None), 1),
             (dict(refs=P + 4), 1), (dict(layers=0), 1), (dict(n_pages=0), 1), (dict(n_seqs=0), 1), (dict(max_pages=0), 1),
             (dict(page_size=0), 1), (dict(Hkv=0), 1), (dict(dtype=2), 1), (dict(D=96), 2), (dict(max_pages=1 << 25, page_size=64), 2),
             (dict(kv_stride_t=-8), 1), (dict(kv_stride_t=1 << 21, kv_stride_h=8, page_stride=1 << 22), 2), (dict(kv_stride_t=120), 1), (dict(kv_stride_t=132), 1), (dict(kv_stride_h=4), 1),
             (dict(page_stride=12), 1), (dict(layer_stride=-8), 1), (dict(page_stride=8), 1), (dict(page_stride=1 << 50), 2), (dict(Hkv=2048), 2),
             (dict(n_pages=(1 << 30) + 1), 2), (dict(n_pages=1 << 20, page_stride=1 << 40), 2), (dict(layers=512, layer_stride=1 << 48), 2)]
BAD_BATCH = [(dict(B=-1), 1), (dict(B=65536), 2), (dict(rows=-1), 1), (dict(rows=(1 << 25) + 1), 2), (dict(L=-1), 1), (dict(layer=2), 1),
             (dict(layer=-1), 1), (dict(seqs=None), 1), (dict(cu_rows=None), 1), (dict(cu_rows=P + 2), 1)]
BAD_ATTENTION = [(dict(Hq=0), 1), (dict(Hq=30), 1), (dict(Hq=512), 2), (dict(S=0), 1), (dict(topk=-1), 1), (dict(topk=33), 2), (dict(scale=-1.0), 1),
                 (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(q_stride_t=64), 1), (dict(q_stride_h=4), 1),
                 (dict(q_stride_t=-128), 1), (dict(idx_stride_h=-1), 1), (dict(q_stride_h=1 << 50), 2)]


@pytest.mark.parametrize("kw,status", BAD_CACHE + BAD_BATCH + BAD_ATTENTION)
def test_attention_refuses(kw, status):
    lib = B.load()
    assert need(**kw) == B.WORKSPACE_INVALID
    c, b, a = records(**kw)
    args = [ctypes.byref(x) for x in (c, b, a)]
    assert lib.sl_paged_span_attention(*args, P, P, P, P, P, 1 << 40, None) == status
    assert lib.sl_paged_span_attention_combined(*args, P, P, P, P, P, 1 << 40, None) == status


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_page_calls_refuse_bad_caches(kw, status):
    lib = B.load()
    c, b, _ = records(**kw)
    c, b = ctypes.byref(c), ctypes.byref(b)
    assert lib.sl_pages_extend(c, b, P, None) == status
    assert lib.sl_pages_fork(c, P, P, 1, P, None) == status
    assert lib.sl_pages_free(c, P, 1, None) == status
    assert lib.sl_pages_compact_workspace_bytes(c) == B.WORKSPACE_INVALID
    assert lib.sl_pages_compact(c, P, P, 1 << 40, None) == status
    assert lib.sl_paged_append(c, b, P, P, 0, 0, None) == status
    assert lib.sl_paged_span_keys(c, b, 64, 10, P, None) == status


@pytest.mark.parametrize("kw,status", BAD_BATCH)
def test_page_calls_refuse_bad_batches(kw, status):
    lib = B.load()
    c, b, _ = records(**kw)
    c, b = ctypes.byref(c), ctypes.byref(b)
    assert lib.sl_pages_extend(c, b, P, None) == status
    assert lib.sl_paged_append(c, b, P, P, 0, 0, None) == status
    assert lib.sl_paged_span_keys(c, b, 64, 10, P, None) == status


def test_missing_pointers_workspaces_and_long_lists():
    lib = B.load()
    c, b, a = records()
    c, b, a = (ctypes.byref(x) for x in (c, b, a))
    size = need()
    assert 0 < size < 1 << 30
    ok = (c, b, a, P, P, P, P, P)
    assert lib.sl_paged_span_attention(*ok, size - 1, None) == 3
    assert lib.sl_paged_span_attention(*ok[:-1], None, size, None) == 3
    assert lib.sl_paged_span_attention(*ok[:-1], P + 16, size, None) == 3
    for missing in (3, 4, 5, 6):
        args = list(ok)
        args[missing] = None
        assert lib.sl_paged_span_attention(*args, size, None) == 1
        assert lib.sl_paged_span_attention_combined(*args, size, None) == 1
    assert lib.sl_paged_span_attention(c, b, a, P + 8, P, P, P, P, size, None) == 1
    assert lib.sl_pages_extend(c, b, None, None) == 1
    assert lib.sl_pages_fork(c, None, P, 1, P, None) == 1 and lib.sl_pages_fork(c, P, P, -1, P, None) == 1
    assert lib.sl_pages_fork(c, P, P, 4097, P, None) == 2
    assert lib.sl_pages_free(c, None, 1, None) == 1 and lib.sl_pages_free(c, P, -1, None) == 1 and lib.sl_pages_free(c, P, 65536, None) == 2
    assert lib.sl_pages_compact(c, None, P, 1 << 20, None) == 1 and lib.sl_pages_compact(c, P, P, 16, None) == 3
    assert lib.sl_paged_append(c, b, None, P, 0, 0, None) == 1 and lib.sl_paged_append(c, b, P, P, 0, 100, None) == 1
    assert lib.sl_paged_append(c, b, P, P, -8, 0, None) == 1 and lib.sl_paged_append(c, b, P, P, 1 << 50, 0, None) == 2
    assert lib.sl_paged_span_keys(c, b, 0, 10, P, None) == 1 and lib.sl_paged_span_keys(c, b, 64, 0, P, None) == 1
    assert lib.sl_paged_span_keys(c, b, 64, 10, None, None) == 1 and lib.sl_paged_span_keys(c, b, 64, 1 << 23, P, None) == 2


def test_nothing_to_do_enqueues_nothing():
    lib = B.load()
    for kw in (dict(B=0, seqs=None, cu_rows=None), dict(rows=0)):
        c, b, a = records(**kw)
        c, b, a = (ctypes.byref(x) for x in (c, b, a))
        assert lib.sl_paged_attention_workspace_bytes(c, b, a) == 0
        assert lib.sl_paged_span_attention(c, b, a, None, None, None, None, None, 0, None) == 0
        assert lib.sl_paged_append(c, b, None, None, 0, 0, None) == 0
    c, b, _ = (ctypes.byref(x) for x in records(B=0, seqs=None, cu_rows=None))
    assert lib.sl_pages_extend(c, b, None, None) == 0
    assert lib.sl_pages_fork(c, None, None, 0, None, None) == 0 and lib.sl_pages_free(c, None, 0, None) == 0


def test_the_largest_problems_ask_for_sizes_that_fit():
    """Sizes are computed in 64 bits: 2^26 rows and heads, 32 spans of the longest length."""
    for kw in (dict(), dict(dtype=B.SL_F32)):
        size = need(rows=(1 << 25) - 1, Hq=2, Hkv=2, topk=32, S=1 << 24, max_pages=1 << 24, page_size=64, **kw)
        assert size != B.WORKSPACE_INVALID
        size = need(rows=1 << 20, Hq=32, Hkv=4, topk=32, S=512, max_pages=1 << 15, page_size=32, B=4, **kw)
        assert size != B.WORKSPACE_INVALID and (1 << 25) * 33 * 128 * 2 <= size < 1 << 46
    assert need(rows=1 << 25, Hq=2, Hkv=2) == B.WORKSPACE_INVALID     # a row, its head and a slot count in 31 bits
    assert need(rows=1 << 21, Hq=32) == B.WORKSPACE_INVALID


def test_the_binding_refuses_tensors_that_do_not_fit():
    K = torch.zeros((1, 6, 2, 16, 64), dtype=torch.bfloat16)
    tables, lens, refs = (torch.zeros(s, dtype=torch.int32) for s in ((3, 4), (3,), (6,)))
    cache = B.PageCache(K, K.clone(), tables, lens, refs)
    assert cache.record.page_stride == 2 * 16 * 64 and cache.record.layers == 1
    B.PageCache(K[0], K[0].clone(), tables, lens, refs)
    for bad in ((K, K.float(), tables, lens, refs), (K, K[:, :5], tables, lens, refs), (K, K, tables.long(), lens, refs),
                (K, K, tables, lens[:2], refs), (K, K, tables, lens, refs[:5]), (K, K, tables[0], lens, refs),
                (K[..., ::2], K[..., ::2], tables, lens, refs), (K, K.transpose(2, 3).contiguous().transpose(2, 3), tables, lens, refs)):
        with pytest.raises(ValueError):
            B.PageCache(*bad)
    with pytest.raises(TypeError):
        B.PageCache(K.half(), K.half(), tables, lens, refs)
    one, two = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for seqs, cu in ((one.long(), two), (one, one), (one, two.float()), (two[::2][:1].expand(1), two[:1])):
        with pytest.raises(ValueError):
            cache.batch(seqs, cu)
    assert cache.batch(one, two).B == 1
    with pytest.raises(ValueError):      # a cache in host memory
        cache.stream()
    with pytest.raises(ValueError):
        B.sl_pages_fork(cache, one, two)
    with pytest.raises(ValueError):
        B.sl_pages_free(cache, one.long())
    with pytest.raises(ValueError):
        B.sl_paged_append(cache, one, two, K[0, 0], K[0, 0, :1])
    with pytest.raises(ValueError):
        B.sl_paged_span_keys(cache, one, two, K[0], 16)
    Q = torch.zeros((4, 1, 64), dtype=torch.bfloat16)
    idx = torch.zeros((4, 1, 2), dtype=torch.int32)
    wide = torch.zeros((4, 3, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):      # rows that are one row repeated: no stride says that
        B._paged_attention(cache, one, two, wide[:, :1].expand(4, 3, 64), None, None, 16, 0, 0, 0.0, None)
    with pytest.raises(ValueError):
        B._paged_attention(cache, one, two, wide, idx.expand(4, 3, 2), None, 16, 0, 0, 0.0, None)
    with pytest.raises(ValueError):
        B.PageCache(K[:, :1].expand(1, 6, 2, 16, 64), K[:, :1].expand(1, 6, 2, 16, 64), tables, lens, refs)
    with pytest.raises(ValueError):
        B.sl_paged_append(cache, one, two, wide[:2, :1].expand(2, 3, 64), wide[:2, :1].expand(2, 3, 64))
    for out in (Q.float(), Q[:2], wide[:, :1]):
        with pytest.raises(ValueError):
            B._result(out, Q.shape, Q.dtype, -1)
    for q, i, s in ((Q.float(), idx, None), (Q[0], idx, None), (Q, idx.long(), None), (Q, idx[:2], None), (Q, idx, idx),
                    (Q, idx, torch.zeros((4, 1, 1)))):
        with pytest.raises(ValueError):
            B._paged_attention(cache, one, two, q, i, s, 16, 0, 0, 0.0, None)


def test_a_span_longer_than_any_sequence_is_not_cut_off():
    """S is 32 bits wide in the record; ctypes would drop the bits above without a word."""
    K = torch.zeros((6, 2, 16, 64), dtype=torch.bfloat16)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    cache = B.PageCache(K, K.clone(), i32(3, 4), i32(3), i32(6))

    class Room:
        def get(self, n):
            return 0, n

    for S, want in ((1 << 40, 0x7fffffff), ((1 << 32) + 5, 0x7fffffff), (100, 100)):
        a, *_ = B._paged_attention(cache, i32(1), i32(2), torch.zeros((4, 1, 64), dtype=torch.bfloat16), None, None, S, 0, 0, 0.0, Room())
        assert a.S == want


def test_integers_beyond_32_bits_are_not_cut_off(monkeypatch):
    """What the records hold in 32 bits: ctypes would drop the bits above, and a span of 2^32 + 4 would be one of 4."""
    K = torch.zeros((6, 2, 16, 64), dtype=torch.bfloat16)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    cache = B.PageCache(K, K.clone(), i32(3, 4), i32(3), i32(6))
    seen = []

    class Lib:
        def sl_paged_span_keys(self, c, b, S, n_spans, Ks, stream):
            seen.append(ctypes.c_int32(S).value)        # what the library gets
            return 0

    monkeypatch.setattr(B, "load", lambda: Lib())
    monkeypatch.setattr(B.PageCache, "stream", lambda self: None)
    Ks = torch.zeros((3, 2, 5, 64), dtype=torch.bfloat16)
    for S in (1 << 40, (1 << 32) + 4, 0x7fffffff, 100, 0, -4, -(1 << 32) + 4):
        B.sl_paged_span_keys(cache, i32(1), i32(2), Ks, S)
    assert seen[:4] == [0x7fffffff] * 3 + [100] and all(S <= 0 for S in seen[4:])
    for layer, want in ((0, 0), (1 << 32, 0x7fffffff), ((1 << 33) + 1, 0x7fffffff), (7, 7)):
        assert cache.batch(i32(1), i32(2), layer=layer).layer == want
    for layer in (-1, -(1 << 32), -(1 << 32) + 1):
        assert cache.batch(i32(1), i32(2), layer=layer).layer < 0

    class Room:
        def get(self, n):
            return 0, n

    monkeypatch.undo()
    for S in (0, -1, -(1 << 32) + 5):
        a, *_ = B._paged_attention(cache, i32(1), i32(2), torch.zeros((4, 1, 64), dtype=torch.bfloat16), None, None, S, 0, 0, 0.0, Room())
        assert a.S <= 0


def test_search_without_a_key_tensor_refuses_tables_that_do_not_fit():
    Q, Ks = torch.zeros((4, 1, 64)), torch.zeros((2, 6, 64))
    for bad in (None, Ks[0], Ks[:, ::2], Ks.bfloat16(), Ks.transpose(0, 1)):
        with pytest.raises(ValueError):
            B.sl_span_search_prefill(Q, None, bad, 16, 2)


def test_the_served_list_refuses():
    lib = B.load()
    assert lib.sl_pages_served(P, P, 0, P, None) == 0 and lib.sl_pages_served(None, None, 0, None, None) == 0
    for args, status in (((P, P, -1, P), 1), ((None, P, 3, P), 1), ((P, None, 3, P), 1), ((P, P, 3, None), 1), ((P + 2, P, 3, P), 1),
                         ((P, P + 1, 3, P), 1), ((P, P, 3, P + 3), 1), ((P, P, 65536, P), 2)):
        assert lib.sl_pages_served(*args, None) == status
    cache = B.PageCache.empty(6, 16, 2, 64, 3, 4, device="cpu")
    three, two = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for args in ((three, two), (three, three.long()), (three.float(), three), (three, three, two)):
        with pytest.raises(ValueError):
            B.sl_pages_served(cache, *args)


def test_sizes_at_the_limits_under_address_and_undefined_sanitizers(tmp_path):
    """Validation and size arithmetic of records at and beyond every limit, in a build of the host side with ASan + UBSan."""
    import glob
    import os
    import shutil
    import subprocess
    from paper_2601_18401_amd import build as _build
    clang = "/opt/rocm/lib/llvm/bin/clang"
    if not os.path.exists(clang) or not shutil.which("hipcc"):
        pytest.skip("no ROCm clang")
    lib = _build.build(sanitize=True)
    exe = str(tmp_path / "size_paged_from_c")
    subprocess.run([clang, "-std=c99", "-Wall", "-Wextra", "-Werror", "-g", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=undefined", "-shared-libsan", "-I", os.path.join(_build.ROOT, "include"),
                    os.path.join(_build.ROOT, "tests", "cabi", "size_paged_from_c.c"), "-o", exe, "-ldl"], check=True)
    rt = os.path.dirname(glob.glob("/opt/rocm*/lib/llvm/lib/clang/*/lib/*/libclang_rt.asan*.so")[0])
    env = dict(os.environ, LD_LIBRARY_PATH=rt, ASAN_OPTIONS="detect_leaks=0")
    run = subprocess.run([exe, lib], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0 and "wrong=0" in run.stdout, (run.stdout, run.stderr[-3000:])
    assert "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr, run.stderr[-3000:]
