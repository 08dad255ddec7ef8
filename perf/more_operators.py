"""A paged KV cache held in 4 bits, to be timed and compared: span-attention that reads it, rows that are quantised as they are written,
rows that are read back.

A row of D channels of K or V is D / 32 blocks: 32 codes of 4 bits (e2m1: a sign, and 0, 0.5, 1, 1.5, 2, 3, 4 or 6) and a scale of 8 bits, a
power of two.  A page holds, for each head, the codes of its tokens (D / 2 bytes each, the even channel in the low half of a byte) and then
their scales (D / 32 bytes each), 16-byte aligned.  Three kinds of work: span-attention of a ragged batch of new tokens over such pages, joint,
gated or dense (`attention`); new tokens written, with the search keys of the spans that they complete, and handed back as the cache
holds them, which is what the rest of the step goes on with (`append`); the last tokens of sequences, or all of them, as rows again (`read`).
Random inputs of unit variance; pages lie in random order, as they do in a cache that has been in use.
"""
import math
import random

import torch

own = False
DEV = "cuda"

_LISTED = [
    # attention: a few short sequences, one new token each, everything attended: the smallest step, where latency counts
    {"name": "step_short", "kind": "attention", "form": "joint", "dtype": "bf16", "B": 6, "n_lo": 1, "n_hi": 1, "L_lo": 300,
     "L_hi": 2500, "Hq": 16, "Hkv": 4, "D": 64, "S": 0, "topk": 0, "ps": 32, "ragged": 101},
    # one sequence, one new token behind a million, sixteen spans of 1024
    {"name": "step_1m", "kind": "attention", "form": "joint", "dtype": "bf16", "B": 1, "n_lo": 1, "n_hi": 1, "L_lo": 1048576,
     "L_hi": 1048576, "Hq": 32, "Hkv": 4, "D": 128, "S": 1024, "topk": 16, "ps": 256, "ragged": 102},
    # a serving batch's step: 40 sequences of very different lengths, gated
    {"name": "step_batch_gated", "kind": "attention", "form": "gated", "dtype": "bf16", "B": 40, "n_lo": 1, "n_hi": 1, "L_lo": 2000,
     "L_hi": 200000, "Hq": 32, "Hkv": 4, "D": 128, "S": 512, "topk": 8, "ps": 64, "ragged": 103},
    # drafts of a few tokens checked at once, everything attended, odd pages
    {"name": "draft_dense", "kind": "attention", "form": "joint", "dtype": "bf16", "B": 12, "n_lo": 1, "n_hi": 9, "L_lo": 3000,
     "L_hi": 40000, "Hq": 24, "Hkv": 8, "D": 128, "S": 0, "topk": 0, "ps": 40, "ragged": 104},
    # chunked prefill of a long prompt: 1500 new rows, eight spans of 256
    {"name": "chunk_80k", "kind": "attention", "form": "joint", "dtype": "bf16", "B": 1, "n_lo": 1500, "n_hi": 1500, "L_lo": 81920,
     "L_hi": 81920, "Hq": 32, "Hkv": 4, "D": 128, "S": 256, "topk": 8, "ps": 64, "ragged": 105},
    # whole prompts of a batch, dense: the most arithmetic
    {"name": "prompts_dense", "kind": "attention", "form": "joint", "dtype": "bf16", "B": 3, "n_lo": 2000, "n_hi": 5500, "L_lo": 1,
     "L_hi": 1, "Hq": 32, "Hkv": 8, "D": 128, "S": 0, "topk": 0, "ps": 128, "ragged": 106},
    # rows in full precision: drafts of a small model
    {"name": "draft_f32", "kind": "attention", "form": "gated", "dtype": "f32", "B": 7, "n_lo": 1, "n_hi": 30, "L_lo": 500,
     "L_hi": 9000, "Hq": 8, "Hkv": 2, "D": 64, "S": 128, "topk": 4, "ps": 16, "ragged": 107},
    # append: one token of each of 48 sequences: the smallest call
    {"name": "append_step", "kind": "append", "dtype": "bf16", "B": 48, "n_lo": 1, "n_hi": 1, "L_lo": 100, "L_hi": 30000, "Hkv": 4,
     "D": 128, "S": 128, "ps": 64, "ragged": 108},
    # the prompts of a large batch
    {"name": "append_prompts", "kind": "append", "dtype": "bf16", "B": 20, "n_lo": 1000, "n_hi": 14000, "L_lo": 1, "L_hi": 1,
     "Hkv": 8, "D": 128, "S": 256, "ps": 64, "ragged": 109},
    # chunks of a small model in full precision, odd pages
    {"name": "append_chunks_f32", "kind": "append", "dtype": "f32", "B": 9, "n_lo": 10, "n_hi": 2000, "L_lo": 1, "L_hi": 9000,
     "Hkv": 2, "D": 64, "S": 50, "ps": 23, "ragged": 110},
    # read: the last tokens of a few sequences, as a window that goes on in the contiguous entry points
    {"name": "read_windows", "kind": "read", "dtype": "bf16", "B": 10, "n_lo": 64, "n_hi": 700, "L_lo": 700, "L_hi": 50000, "Hkv": 4,
     "D": 128, "ps": 64, "ragged": 111},
    # whole sequences
    {"name": "read_sequences", "kind": "read", "dtype": "bf16", "B": 5, "n_lo": 8000, "n_hi": 60000, "L_lo": 1, "L_hi": 1, "Hkv": 8,
     "D": 128, "ps": 128, "ragged": 112},
]


def listed():
    return [dict(c) for c in _LISTED]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "step", "step", "draft", "draft", "chunk", "prompts", "f32", "append", "append", "read", "read"])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 3, 4, 8]) if Hkv < 8 else rng.choice([1, 4])
    D = rng.choice([64, 128, 128])
    ps = rng.choice([16, 32, 64, 64, 128, 256, rng.randint(9, 200)])
    ragged = rng.randrange(1 << 30)
    base = {"kind": "attention", "form": rng.choice(["joint", "joint", "gated"]), "dtype": "bf16", "ragged": ragged}
    heads = {"Hq": G * Hkv, "Hkv": Hkv, "D": D}
    if kind == "step":  # one new token each
        B = _log_int(rng, 1, 64)
        top = min(1000000, int(4e6 / B))
        L_hi = _log_int(rng, 1000, top)
        dense = rng.random() < 0.25 and L_hi * B < 1000000
        S = rng.choice([64, 128, 256, 512, 1024, rng.randint(20, 700)])
        return {**base, "form": "joint" if dense else base["form"], "B": B, "n_lo": 1, "n_hi": 1, "L_lo": max(1, L_hi // rng.choice([1, 4, 50])),
                "L_hi": L_hi, **heads, "S": 0 if dense else S, "topk": 0 if dense else rng.choice([1, 4, 8, 16]), "ps": ps}
    if kind == "draft":
        B = _log_int(rng, 1, 40)
        routed = rng.random() < 0.5
        return {**base, "form": base["form"] if routed else "joint", "B": B, "n_lo": 1, "n_hi": rng.randint(2, 16), "L_lo": 20,
                "L_hi": _log_int(rng, 1000, 16000), **heads, "S": rng.randint(30, 600) if routed else 0,
                "topk": rng.choice([2, 8]) if routed else 0, "ps": ps}
    if kind == "chunk":
        n = _log_int(rng, 100, 1800)
        L = _log_int(rng, 4000, min(200000, int(1.2e8 / n)))
        return {**base, "B": 1, "n_lo": n, "n_hi": n, "L_lo": max(L, n), "L_hi": max(L, n), **heads,
                "S": rng.choice([64, 128, 256, 512, rng.randint(40, 600)]), "topk": rng.choice([2, 4, 8, 16]), "ps": ps}
    if kind == "prompts":
        return {**base, "form": "joint", "B": rng.randint(1, 3), "n_lo": 20, "n_hi": _log_int(rng, 200, 4500), "L_lo": 1, "L_hi": 1, **heads,
                "S": 0, "topk": 0, "ps": ps}
    if kind == "f32":
        return {**base, "dtype": "f32", "B": rng.randint(1, 8), "n_lo": 1, "n_hi": _log_int(rng, 1, 300), "L_lo": 50,
                "L_hi": _log_int(rng, 500, 12000), "Hq": G * min(Hkv, 4), "Hkv": min(Hkv, 4), "D": D, "S": rng.randint(16, 200),
                "topk": rng.choice([1, 4, 8]), "ps": ps}
    rows = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"]), "Hkv": Hkv, "D": D, "ps": ps, "ragged": ragged}
    B = _log_int(rng, 1, 80)
    if kind == "append":
        n_hi = _log_int(rng, 1, 120000 // B)
        return {**rows, "B": B, "n_lo": max(1, n_hi // 20), "n_hi": n_hi, "L_lo": 1, "L_hi": _log_int(rng, 2, 10000), "S": rng.randint(20, 600)}
    n_hi = _log_int(rng, 1, 150000 // B)
    return {**rows, "B": B, "n_lo": max(1, n_hi // 10), "n_hi": n_hi, "L_lo": 1, "L_hi": _log_int(rng, 2, 20000)}


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _sizes(case):
    """New tokens and lengths (new tokens included) of the batch's sequences."""
    rng = random.Random(case["ragged"])
    ns = [_log_int(rng, case["n_lo"], case["n_hi"]) for _ in range(case["B"])]
    return ns, [max(n, _log_int(rng, case["L_lo"], case["L_hi"])) for n in ns]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _page_bytes(ps, D):
    return -(-ps * (D // 2 + D // 32) // 16) * 16


# ---- the format, in elementary operations: every step is exact, so that 32 bits are enough
def _encode(x):
    """Codes [..., D / 2] and scales [..., D / 32] (uint8) of rows [..., D]."""
    blocks = x.float().unflatten(-1, (-1, 32))
    top = blocks.abs().amax(-1)
    mantissa, exponent = torch.frexp(top)          # top = mantissa * 2^exponent, mantissa in [0.5, 1): the largest goes to [1.75, 7/2) * 2
    scale = (exponent - 3 + (mantissa >= 0.875) + 127).clamp(2, 252).to(torch.int32)
    a = blocks * ((254 - scale) << 23).view(torch.float32)[..., None]
    negative, a = torch.signbit(a), a.abs().clamp(max=6)
    q = torch.where(a < 2, torch.round(2 * a) / 2, torch.where(a < 4, torch.round(a), torch.round(a / 2) * 2))
    code = torch.where(q < 2, 2 * q, torch.where(q < 4, q + 2, q / 2 + 4)).to(torch.uint8) + 8 * negative.to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], scale.to(torch.uint8)


def _decode(codes, scales):
    """Rows [..., D] in 32 bits."""
    size = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    values = torch.cat([size, -size])
    x = torch.stack([values[(codes & 15).int()], values[(codes >> 4).int()]], -1).flatten(-2)
    return (x.unflatten(-1, (-1, 32)) * (scales.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _parts(pages, ps, D):
    """Views [..., ps, D / 2] of the codes and [..., ps, D / 32] of the scales of pages [..., bytes]."""
    at = ps * (D // 2)
    return pages[..., :at].unflatten(-1, (ps, -1)), pages[..., at:at + ps * (D // 32)].unflatten(-1, (ps, -1))


def _fill(pages, ps, D, g):
    """Pages of random rows, a few at a time."""
    codes, scales = _parts(pages, ps, D)
    step = max(1, (1 << 26) // (pages.shape[1] * ps * D))
    for k in range(0, pages.shape[0], step):
        n = min(step, pages.shape[0] - k)
        x = torch.randn((n, pages.shape[1], ps, D), generator=g, device=DEV)
        codes[k:k + n], scales[k:k + n] = _encode(x)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    kind, dt, ps, B, D = case["kind"], _dtype(case), case["ps"], case["B"], case["D"]
    ns, Ls = _sizes(case)
    max_pages = -(-max(Ls) // ps) + 1
    need = sum(-(-L // ps) for L in Ls)
    n_pages = need + need // 8 + 2
    K, V = (torch.zeros((1, n_pages, case["Hkv"], _page_bytes(ps, D)), dtype=torch.uint8, device=DEV) for _ in range(2))
    for x in (K, V):
        _fill(x[0], ps, D, g)
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    tables = torch.full((B, max_pages), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, L in enumerate(Ls):
        k = -(-L // ps)
        tables[s, :k] = order[at:at + k]
        at += k
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[order[:at].long()] = 1
    T = sum(ns)
    st = {"case": case, "ns": ns, "Ls": Ls, "T": T, "K": K, "V": V, "tables": tables, "lens": _i32(Ls), "refs": refs,
          "seqs": torch.arange(B, dtype=torch.int32, device=DEV), "cu": _i32([sum(ns[:b]) for b in range(B + 1)])}
    if kind == "read":
        return st
    S = case["S"] or max_pages * ps
    st["S"], spans = S, max_pages * ps // S + 1
    if kind == "append":
        st["Kn"], st["Vn"] = (torch.randn((case["Hkv"], T, D), generator=g, device=DEV).to(dt) for _ in range(2))
        st["Ks"] = torch.zeros((B, case["Hkv"], spans, D), device=DEV, dtype=dt)
        return st
    st["Q"] = torch.randn((case["Hq"], T, D), generator=g, device=DEV).to(dt)
    st["idx"] = None
    if case["topk"]:
        pos = torch.cat([torch.arange(L - n, L, device=DEV) for n, L in zip(ns, Ls)])
        like = torch.rand((case["Hq"], T, max(spans, case["topk"])), generator=g, device=DEV)
        like.masked_fill_(torch.arange(like.shape[2], device=DEV) >= (pos // S)[None, :, None], -1.0)
        best = like.topk(case["topk"], dim=2)
        idx = torch.where(best.values >= 0, best.indices, 1 << 30).sort(dim=2).values
        st["idx"] = torch.where(idx < 1 << 30, idx, -1).to(torch.int32).contiguous()
        st["scores"] = torch.randn(idx.shape, generator=g, device=DEV) * 2
    return st


# ---- plain forms
def _dense(pages, tables, ps, D):
    """[B, Hkv, max_pages * page_size, D] in 32 bits."""
    x = _decode(*_parts(pages[tables.clamp(min=0).long()], ps, D))
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _rows(st):
    """Entry, place in the chunk, position and page of each row."""
    seqs, cu, ps = st["seqs"].long(), st["cu"].long(), st["case"]["ps"]
    row = torch.arange(st["T"], device=DEV)
    b = torch.searchsorted(cu[1:], row, right=True)
    pos = st["lens"][seqs].long()[b] - cu[b + 1] + row
    return b, row - cu[b], pos, st["tables"][seqs[b], pos // ps].long()


def _plain_attention(st):
    c, S, gated = st["case"], st["S"], st["case"]["form"] == "gated"
    Hq, Hkv, D, topk, ps = c["Hq"], c["Hkv"], c["D"], c["topk"], c["ps"]
    Q, seqs, B, most = st["Q"], st["seqs"].long(), c["B"], max(st["ns"])
    K, V = _dense(st["K"][0], st["tables"][seqs], ps, D), _dense(st["V"][0], st["tables"][seqs], ps, D)
    Lc = -(-K.shape[2] // S) * S
    K, V = (torch.nn.functional.pad(x, (0, 0, 0, Lc - x.shape[2])) for x in (K, V))
    b, i, at_pos, _ = _rows(st)
    pos = torch.zeros((B, most), device=DEV, dtype=torch.long)
    pos[b, i] = at_pos
    Qp = torch.zeros((B, most, Hq, D), device=DEV)
    Qp[b, i] = Q.float().transpose(0, 1)
    Qp = Qp.permute(0, 2, 1, 3).reshape(B, Hkv, -1, D)
    s = torch.matmul(Qp, K.transpose(2, 3).contiguous()).mul_(1 / math.sqrt(D)).view(B, Hq, most, Lc // S, S)
    first = pos // S
    span, token = torch.arange(Lc // S, device=DEV), torch.arange(Lc, device=DEV).view(-1, S)
    window = (token >= (first * S)[..., None, None]) & (token <= pos[..., None, None])
    if topk:
        chosen = torch.full((B, most, Hq, topk), -1, device=DEV, dtype=torch.long)
        chosen[b, i] = st["idx"].long().transpose(0, 1)
        chosen = chosen.transpose(1, 2)
        empty = (chosen < 0) | (chosen >= first[:, None, :, None])
        at = torch.where(empty, Lc // S, chosen)
        took = torch.zeros((B, Hq, most, Lc // S + 1), device=DEV, dtype=torch.bool).scatter_(3, at, True)[..., :-1]
        s.masked_fill_(~(took[..., None] | window[:, None]), -math.inf)
    else:
        s.masked_fill_(~window[:, None], -math.inf)
    m = s.amax(dim=(3, 4), keepdim=True)
    p = s.sub_(m).exp_()
    total = None
    if gated and topk:
        sums = p.sum(4)
        own_span = (span == first[..., None])[:, None]
        in_window = (sums * own_span).sum(3, keepdim=True)
        gate = torch.full((B, most, Hq, topk), -math.inf, device=DEV)
        gate[b, i] = st["scores"].transpose(0, 1)
        gate = torch.softmax(gate.transpose(1, 2).masked_fill(empty, -math.inf), 3).nan_to_num(0.0)
        alpha = torch.zeros((B, Hq, most, Lc // S + 1), device=DEV).scatter_(3, at, gate)[..., :-1]
        factor = alpha / (sums + in_window)
        alone = empty.all(3, keepdim=True)
        factor = torch.where(own_span, torch.where(alone, 1 / in_window, factor.masked_fill(own_span, 0).sum(3, keepdim=True)), factor)
        p.mul_(factor[..., None])
    else:
        total = p.sum(dim=(3, 4))
    o = torch.matmul(p.view(B, Hkv, -1, Lc), V).view(B, Hq, most, D)
    if total is None:
        return {"O": o[b, :, i].transpose(0, 1).to(Q.dtype)}
    o = o / total[..., None]
    return {"O": o[b, :, i].transpose(0, 1).to(Q.dtype), "LSE": (m.view(B, Hq, most) + total.log())[b, :, i].transpose(0, 1)}


def _plain_read(st):
    D, ps, dt = st["case"]["D"], st["case"]["ps"], _dtype(st["case"])
    _, _, pos, page = _rows(st)
    out = {}
    for name in ("K", "V"):
        codes, scales = _parts(st[name][0], ps, D)
        out[name] = _decode(codes[page, :, pos % ps], scales[page, :, pos % ps]).to(dt).transpose(0, 1).contiguous()
    return out


def _plain_append(st):
    D, ps, S = st["case"]["D"], st["case"]["ps"], st["S"]
    b, _, pos, page = _rows(st)
    for pages, new in ((st["K"], st["Kn"]), (st["V"], st["Vn"])):
        codes, scales = _parts(pages[0], ps, D)
        codes[page, :, pos % ps], scales[page, :, pos % ps] = _encode(new.transpose(0, 1))
    out = _plain_read(st)
    Ks = torch.cat([st["Ks"], st["Ks"][:, :, :1]], 2)  # rows that complete no span go to a row of their own
    Ks[st["seqs"].long()[b], :, torch.where(pos % S == S - 1, pos // S, Ks.shape[2] - 1)] = out["K"].transpose(0, 1)
    st["Ks"].copy_(Ks[:, :, :-1])
    return {**out, "Ks": st["Ks"]}


# ---- the framework's calls
def _own(st):
    from paper_2601_18401_amd import binding as sl
    c = st["case"]
    if "cache" not in st:
        st["cache"] = sl.PageCache(st["K"], st["V"], st["tables"], st["lens"], st["refs"], page_size=c["ps"], D=c["D"], dtype=_dtype(c))
    cache, seqs, cu = st["cache"], st["seqs"], st["cu"]
    if c["kind"] == "attention":
        if c["form"] == "gated":
            return {"O": sl.sl_paged_span_attention_combined(cache, seqs, cu, st["Q"], st["idx"], st["scores"], st["S"], L=max(st["Ls"]))}
        O, LSE = sl.sl_paged_span_attention(cache, seqs, cu, st["Q"], st["idx"], st["S"], L=max(st["Ls"]))
        return {"O": O, "LSE": LSE}
    if c["kind"] == "append":
        sl.sl_paged_append(cache, seqs, cu, st["Kn"], st["Vn"])
        sl.sl_paged_span_keys(cache, seqs, cu, st["Ks"], st["S"])
    K, V = sl.sl_paged_read(cache, seqs, cu, st["T"])
    return {"K": K, "V": V, "Ks": st["Ks"]} if c["kind"] == "append" else {"K": K, "V": V}


def run(state):
    if own:
        return _own(state)
    return {"attention": _plain_attention, "append": _plain_append, "read": _plain_read}[state["case"]["kind"]](state)


def work(case):
    es, kind, D = (4 if case["dtype"] == "f32" else 2), case["kind"], case["D"]
    held, row = case["Hkv"] * (D // 2 + D // 32), case["Hkv"] * D * es
    ns, Ls = _sizes(case)
    T = sum(ns)
    if kind == "attention":
        S = case["S"] or (1 << 40)
        G, read, keys = case["Hq"] // case["Hkv"], 0.0, 0.0
        for n, L in zip(ns, Ls):
            c = (L - n // 2) // S
            k = min(case["topk"], c)
            window = sum((L - n + i) % S + 1 for i in range(n))
            keys += n * k * S + window
            # distinct spans that the group's heads and the rows ask for, and the rows' windows
            read += c * S * (1 - (1 - k / c) ** (G * n) if k else 0) + min(L, (L - n) % S + n)
        io = 2 * case["Hq"] * T * D * es + case["Hq"] * T * 4 * (1 + case["topk"] * (2 if case["form"] == "gated" else 1))
        return {"bytes": 2 * read * held + io, "flops": 4.0 * keys * case["Hq"] * D}
    if kind == "append":  # rows read and written in 4 bits; handed back in the rows' type; keys of the completed spans
        spans = sum(L // case["S"] - (L - n) // case["S"] for n, L in zip(ns, Ls))
        return {"bytes": 2 * T * (2 * row + held) + spans * row, "flops": 0}
    return {"bytes": 2 * T * (held + row), "flops": 0}


# ---- the definition in 64 bits
def _tokens(pages, page, at, head, ps, D):
    """Rows [n, D] in 64 bits: tokens `at` of pages `page`, one head."""
    raw = pages[0, page, head]
    first = at[:, None] * (D // 2) + torch.arange(D // 2, device=DEV)
    byte = raw.gather(1, first).long()
    code = torch.stack([byte % 16, byte // 16], 2).reshape(len(page), D)
    power = raw.gather(1, ps * (D // 2) + at[:, None] * (D // 32) + torch.arange(D, device=DEV) // 32).double() - 127
    size, odd = code % 8, code % 2
    exponent = torch.clamp(size // 2 - 1, min=0).double()
    magnitude = torch.where(size < 2, 0.5 * odd.double(), (1 + 0.5 * odd.double()) * 2.0 ** exponent)
    return torch.where(code >= 8, -magnitude, magnitude) * 2.0 ** power


def _held(x):
    """What rows [n, D] in 64 bits become when they are held in 4 bits."""
    blocks = x.reshape(x.shape[0], -1, 32)
    top = blocks.abs().amax(2, keepdim=True)
    # the smallest power of two at which the largest value, rounded, is no more than 6: below 7 at that power
    power = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 8)) - 1
    for _ in range(3):
        power = torch.where(top >= 7 * 2.0 ** power, power + 1, power)
    power = power.clamp(-125, 125)
    a = blocks.abs() / 2.0 ** power
    step = torch.zeros_like(a, dtype=torch.long)
    for k, middle in enumerate([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]):
        step += (a > middle) | ((a == middle) & (k % 2 == 1))  # half way: to the even code
    size = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV, dtype=torch.float64)[step]
    return (torch.sign(blocks) * size * 2.0 ** power).reshape(x.shape)


def _exact_attention(case, seed):
    st = prepare(case, seed)
    ns, Ls, S, ps, D, G = st["ns"], st["Ls"], st["S"], case["ps"], case["D"], case["Hq"] // case["Hkv"]
    T = sum(ns)
    O = torch.zeros((case["Hq"], T, D), dtype=torch.float64, device=DEV)
    LSE = torch.zeros((case["Hq"], T), dtype=torch.float64, device=DEV)
    at = 0
    for b, (n, L) in enumerate(zip(ns, Ls)):
        t = torch.arange(L, device=DEV)
        page = st["tables"][b].long()[t // ps]
        block = max(1, min(n, int(3e8 // (L * G))))
        for kv in range(case["Hkv"]):
            K, V = (_tokens(x, page, t % ps, kv, ps, D) for x in (st["K"], st["V"]))
            heads = slice(kv * G, kv * G + G)
            for r0 in range(0, n, block):
                rows = torch.arange(r0, min(n, r0 + block), device=DEV)
                pos = (L - n + rows)[None, :, None]
                z = (st["Q"][heads, at + rows].double() @ K.T) / math.sqrt(D)
                near = (t >= pos // S * S) & (t <= pos)
                slots = [st["idx"][heads, at + rows, k, None].long() for k in range(case["topk"])]
                live = [(j >= 0) & (j < pos // S) for j in slots]
                if case["form"] == "gated" and case["topk"]:
                    gate = torch.stack([torch.where(e[..., 0], st["scores"][heads, at + rows, k].double(), -math.inf) for k, e in enumerate(live)])
                    none = ~torch.stack([e[..., 0] for e in live]).any(0)
                    alpha = torch.softmax(gate.masked_fill(none, 0.0), 0)
                    o = 0
                    for k, (j, e) in enumerate(zip(slots, live)):
                        a = torch.softmax(z.masked_fill(~(near | (e & (t // S == j))), -math.inf), -1) @ V
                        o = o + alpha[k][..., None] * a
                    O[heads, at + rows] = o
                else:
                    seen = near.expand_as(z).clone()
                    for j, e in zip(slots, live):
                        seen |= e & (t // S == j)
                    z.masked_fill_(~seen, -math.inf)
                    LSE[heads, at + rows] = torch.logsumexp(z, -1)
                    O[heads, at + rows] = torch.softmax(z, -1) @ V
        at += n
    return {"O": O} if case["form"] == "gated" else {"O": O, "LSE": LSE}


def _exact_rows(case, seed):
    st = prepare(case, seed)
    ps, D, T, append = case["ps"], case["D"], st["T"], case["kind"] == "append"
    K, V = (torch.zeros((case["Hkv"], T, D), dtype=torch.float64, device=DEV) for _ in range(2))
    Ks = st["Ks"].double() if append else None
    at = 0
    for b, (n, L) in enumerate(zip(st["ns"], st["Ls"])):
        t = torch.arange(L - n, L, device=DEV)
        page = st["tables"][b].long()[t // ps]
        for h in range(case["Hkv"]):
            for x, pages, new in ((K, "K", "Kn"), (V, "V", "Vn")):
                x[h, at:at + n] = _held(st[new][h, at:at + n].double()) if append else _tokens(st[pages], page, t % ps, h, ps, D)
            if append:
                last = t[(t + 1) % case["S"] == 0]
                Ks[b, h, last // case["S"]] = K[h, at + last - (L - n)]
        at += n
    return {"K": K, "V": V, "Ks": Ks} if append else {"K": K, "V": V}


def exact(case, seed):
    return (_exact_attention if case["kind"] == "attention" else _exact_rows)(case, seed)
