"""A paged KV cache and span-attention over it: what a serving program does with one, to be timed and compared.

Four kinds of work: span-attention of a ragged batch of new tokens over the pages, joint or gated (`attention`); new tokens
written into pages, with the search keys of the spans that they complete (`append`); a scheduler's turn, which frees the
sequences that ended, forks others and gives them pages for the tokens to come (`turn`); compaction of a fragmented cache
(`compact`).  Random inputs of unit variance; pages lie in random order, as they do in a cache that has been in use.
"""
import math
import random

import torch

own = False
DEV = "cuda"

_LISTED = [
    # attention: one sequence, one new token behind a million, sixteen spans of 1024: the longest cache, latency of one step
    {"name": "step_1m", "kind": "attention", "form": "joint", "dtype": "bf16", "B": 1, "n_lo": 1, "n_hi": 1, "L_lo": 1048576,
     "L_hi": 1048576, "Hq": 32, "Hkv": 4, "D": 128, "S": 1024, "topk": 16, "ps": 256, "ragged": 1},
    # a serving batch's step: 24 sequences of very different lengths, gated
    {"name": "step_batch_gated", "kind": "attention", "form": "gated", "dtype": "bf16", "B": 24, "n_lo": 1, "n_hi": 1, "L_lo": 1500,
     "L_hi": 120000, "Hq": 32, "Hkv": 4, "D": 128, "S": 256, "topk": 8, "ps": 64, "ragged": 2},
    # drafts of a few tokens checked at once, short sequences that attend everything (the dense fallback), D = 64, odd pages
    {"name": "draft_dense", "kind": "attention", "form": "joint", "dtype": "bf16", "B": 16, "n_lo": 1, "n_hi": 8, "L_lo": 500,
     "L_hi": 9000, "Hq": 16, "Hkv": 2, "D": 64, "S": 0, "topk": 0, "ps": 48, "ragged": 3},
    # chunked prefill of a long prompt: 2000 new rows, eight spans of 512
    {"name": "chunk_64k", "kind": "attention", "form": "joint", "dtype": "bf16", "B": 1, "n_lo": 2000, "n_hi": 2000, "L_lo": 65536,
     "L_hi": 65536, "Hq": 32, "Hkv": 4, "D": 128, "S": 512, "topk": 8, "ps": 64, "ragged": 4},
    # whole prompts of a batch, dense: the most arithmetic
    {"name": "prompts_dense", "kind": "attention", "form": "joint", "dtype": "bf16", "B": 4, "n_lo": 2500, "n_hi": 6000, "L_lo": 1,
     "L_hi": 1, "Hq": 32, "Hkv": 8, "D": 128, "S": 0, "topk": 0, "ps": 128, "ragged": 5},
    # a small model in full precision: ragged chunks, spans of 64
    {"name": "chunks_f32", "kind": "attention", "form": "joint", "dtype": "f32", "B": 5, "n_lo": 1, "n_hi": 400, "L_lo": 300,
     "L_hi": 4096, "Hq": 4, "Hkv": 4, "D": 64, "S": 64, "topk": 4, "ps": 16, "ragged": 6},
    # append: one token of each of 64 sequences: the smallest call
    {"name": "append_step", "kind": "append", "dtype": "bf16", "B": 64, "n_lo": 1, "n_hi": 1, "L_lo": 100, "L_hi": 20000, "Hkv": 4,
     "D": 128, "S": 128, "ps": 64, "ragged": 7},
    # the prompts of a large batch
    {"name": "append_prompts", "kind": "append", "dtype": "bf16", "B": 24, "n_lo": 1000, "n_hi": 16000, "L_lo": 1, "L_hi": 1,
     "Hkv": 8, "D": 128, "S": 256, "ps": 64, "ragged": 8},
    # turn: a few forks in a small cache, as a search over continuations makes them at every step
    {"name": "turn_small", "kind": "turn", "dtype": "bf16", "pages": 3000, "base": 8, "forks": 8, "L_lo": 200, "L_hi": 9000,
     "n_lo": 1, "n_hi": 64, "layers": 2, "Hkv": 4, "D": 128, "ps": 64, "ragged": 9},
    # many forks of long prompts in a large cache
    {"name": "turn_large", "kind": "turn", "dtype": "bf16", "pages": 60000, "base": 16, "forks": 200, "L_lo": 8000, "L_hi": 90000,
     "n_lo": 1, "n_hi": 3000, "layers": 2, "Hkv": 2, "D": 64, "ps": 32, "ragged": 10},
    # compact: a small cache, a third of it free
    {"name": "compact_small", "kind": "compact", "dtype": "bf16", "pages": 400, "seqs": 12, "used": 0.6, "layers": 1, "Hkv": 4,
     "D": 64, "ps": 16, "ragged": 11},
    # a large one, half empty
    {"name": "compact_large", "kind": "compact", "dtype": "bf16", "pages": 12000, "seqs": 40, "used": 0.5, "layers": 4, "Hkv": 4,
     "D": 128, "ps": 64, "ragged": 12},
]


def listed():
    return [dict(c) for c in _LISTED]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "step", "draft", "chunk", "prompts", "f32", "append", "append", "turn", "turn", "compact", "compact"])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 3, 4, 8]) if Hkv < 8 else rng.choice([1, 4])
    D = rng.choice([64, 128, 128])
    ps = rng.choice([16, 32, 64, 64, 128, 256, rng.randint(9, 200)])
    ragged = rng.randrange(1 << 30)
    base = {"kind": "attention", "form": rng.choice(["joint", "joint", "gated"]), "dtype": "bf16", "ragged": ragged}
    heads = {"Hq": G * Hkv, "Hkv": Hkv, "D": D}
    if kind == "step":  # one new token each
        B = _log_int(rng, 1, 48)
        top = min(1000000, int(4e6 / B))
        L_hi = _log_int(rng, 2000, top)
        S = rng.choice([64, 128, 256, 512, 1024, rng.randint(20, 700)])
        return {**base, "B": B, "n_lo": 1, "n_hi": 1, "L_lo": max(1, L_hi // rng.choice([1, 4, 50])), "L_hi": L_hi, **heads, "S": S,
                "topk": rng.choice([1, 4, 8, 16]), "ps": ps}
    if kind == "draft":
        B = _log_int(rng, 1, 40)
        routed = rng.random() < 0.5
        return {**base, "form": base["form"] if routed else "joint", "B": B, "n_lo": 1, "n_hi": rng.randint(2, 16), "L_lo": 20,
                "L_hi": _log_int(rng, 1000, 16000), **heads, "S": rng.randint(30, 600) if routed else 0,
                "topk": rng.choice([2, 8]) if routed else 0, "ps": ps}
    if kind == "chunk":
        n = _log_int(rng, 100, 2000)
        L = _log_int(rng, 4000, min(200000, int(1.3e8 / n)))
        return {**base, "B": 1, "n_lo": n, "n_hi": n, "L_lo": max(L, n), "L_hi": max(L, n), **heads,
                "S": rng.choice([64, 128, 256, 512, rng.randint(40, 600)]), "topk": rng.choice([2, 4, 8, 16]), "ps": ps}
    if kind == "prompts":
        B = rng.randint(1, 5)
        return {**base, "form": "joint", "B": B, "n_lo": 20, "n_hi": _log_int(rng, 200, 4000), "L_lo": 1, "L_hi": 1, **heads,
                "S": 0, "topk": 0, "ps": ps}
    if kind == "f32":
        return {**base, "dtype": "f32", "B": rng.randint(1, 6), "n_lo": 1, "n_hi": _log_int(rng, 2, 500), "L_lo": 50,
                "L_hi": _log_int(rng, 500, 6000), "Hq": G * min(Hkv, 4), "Hkv": min(Hkv, 4), "D": D, "S": rng.randint(16, 200),
                "topk": rng.choice([1, 4, 8]), "ps": ps}
    if kind == "append":
        B = _log_int(rng, 1, 100)
        n_hi = _log_int(rng, 1, 200000 // B)
        return {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"]), "B": B, "n_lo": max(1, n_hi // 20), "n_hi": n_hi, "L_lo": 1,
                "L_hi": _log_int(rng, 2, 10000), "Hkv": Hkv, "D": D, "S": rng.randint(20, 600), "ps": ps, "ragged": ragged}
    if kind == "turn":
        return {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"]), "pages": _log_int(rng, 1500, 50000), "base": rng.randint(1, 20),
                "forks": _log_int(rng, 1, 200), "L_lo": 50, "L_hi": _log_int(rng, 300, 50000), "n_lo": 1, "n_hi": _log_int(rng, 1, 2000),
                "layers": rng.randint(1, 3), "Hkv": min(Hkv, 2), "D": 64, "ps": rng.choice([16, 32, rng.randint(9, 40)]), "ragged": ragged}
    return {"kind": "compact", "dtype": rng.choice(["bf16", "bf16", "f32"]), "pages": _log_int(rng, 100, 8000), "seqs": rng.randint(1, 60),
            "used": round(rng.uniform(0.05, 0.95), 3), "layers": rng.randint(1, 3), "Hkv": min(Hkv, 4), "D": D, "ps": rng.choice([16, 32, 64]),
            "ragged": ragged}


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _sizes(case):
    """New tokens and lengths (new tokens included) of the batch's sequences."""
    rng = random.Random(case["ragged"])
    ns = [_log_int(rng, case["n_lo"], case["n_hi"]) for _ in range(case["B"])]
    return ns, [max(n, _log_int(rng, case["L_lo"], case["L_hi"])) for n in ns]


def _turn_sizes(case):
    """Lengths of the sequences that stay (as many as fit three quarters of the cache), what is forked, and the tokens each fork is to get."""
    rng, room, Ls = random.Random(case["ragged"]), case["pages"] * 3 // 4, []
    for _ in range(case["base"]):
        L = min(_log_int(rng, case["L_lo"], case["L_hi"]), room * case["ps"])
        room -= -(-L // case["ps"])
        Ls.append(L)
    return Ls, [rng.randrange(case["base"]) for _ in range(case["forks"])], [_log_int(rng, case["n_lo"], case["n_hi"]) for _ in range(case["forks"])]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _paged(case, Ls, n_seqs, n_pages, max_pages, g, layers=1):
    """A cache whose first len(Ls) sequences hold Ls tokens, in pages of random order."""
    ps, shape = case["ps"], (layers, n_pages, case["Hkv"], case["ps"], case["D"])
    K, V = (torch.randn(shape, generator=g, device=DEV, dtype=_dtype(case)) for _ in range(2))
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    tables = torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, L in enumerate(Ls):
        k = -(-L // ps)
        tables[s, :k] = order[at:at + k]
        at += k
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[order[:at].long()] = 1
    lens = torch.zeros(n_seqs, dtype=torch.int32, device=DEV)
    lens[:len(Ls)] = _i32(Ls)
    return {"K": K, "V": V, "tables": tables, "lens": lens, "refs": refs}


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    kind, dt = case["kind"], _dtype(case)
    if kind in ("attention", "append"):
        ns, Ls = _sizes(case)
        ps, B, D = case["ps"], case["B"], case["D"]
        max_pages = -(-max(Ls) // ps) + 1
        need = sum(-(-L // ps) for L in Ls)
        st = {"case": case, "ns": ns, "Ls": Ls, **_paged(case, Ls, B, need + need // 8 + 2, max_pages, g)}
        st["seqs"] = torch.arange(B, dtype=torch.int32, device=DEV)
        st["cu"] = _i32([sum(ns[:b]) for b in range(B + 1)])
        T, S = sum(ns), case["S"] or max_pages * ps
        st["S"], spans = S, max_pages * ps // S + 1
        if kind == "append":
            st["Kn"], st["Vn"] = (torch.randn((case["Hkv"], T, D), generator=g, device=DEV, dtype=dt) for _ in range(2))
            st["Ks"] = torch.zeros((B, case["Hkv"], spans, D), device=DEV, dtype=dt)
            return st
        st["Q"] = torch.randn((case["Hq"], T, D), generator=g, device=DEV, dtype=dt)
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
    if kind == "turn":
        Ls, src, ns = _turn_sizes(case)
        most = -(-max(max(Ls) + max(ns), 1) // case["ps"]) + 1
        st = {"case": case, **_paged(case, Ls, case["base"] + case["forks"], case["pages"], most, g, case["layers"])}
        st["src"], st["dst"] = _i32(src), torch.arange(case["base"], case["base"] + case["forks"], dtype=torch.int32, device=DEV)
        st["cu"], st["most_new"] = _i32([sum(ns[:b]) for b in range(len(ns) + 1)]), sum(n // case["ps"] + 1 for n in ns)
        return st
    used = max(1, int(case["pages"] * case["used"]))
    per = [used // case["seqs"] + (s < used % case["seqs"]) for s in range(case["seqs"])]
    st = {"case": case, **_paged(case, [p * case["ps"] for p in per], case["seqs"], case["pages"], max(per) + 1, g, case["layers"])}
    st["fragmented"] = st["tables"].clone(), st["refs"].clone()
    return st


# ---- plain forms
def _dense(pages, tables):
    """[B, Hkv, max_pages * page_size, D] in 32 bits."""
    x = pages[tables.clamp(min=0).long()].float()
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _plain_attention(st):
    c, S, gated = st["case"], st["S"], st["case"]["form"] == "gated"
    Hq, Hkv, D, topk = c["Hq"], c["Hkv"], c["D"], c["topk"]
    Q, seqs, cu = st["Q"], st["seqs"].long(), st["cu"].long()
    T, B, most = Q.shape[1], c["B"], max(st["ns"])
    K, V = _dense(st["K"][0], st["tables"][seqs]), _dense(st["V"][0], st["tables"][seqs])
    Lc = -(-K.shape[2] // S) * S
    K, V = (torch.nn.functional.pad(x, (0, 0, 0, Lc - x.shape[2])) for x in (K, V))
    row = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu[1:], row, right=True)
    i = row - cu[b]
    n = cu[1:] - cu[:-1]
    pos = torch.full((B, most), 0, device=DEV, dtype=torch.long)
    pos[b, i] = st["lens"][seqs].long()[b] - n[b] + i
    Qp = torch.zeros((B, most, Hq, D), device=DEV)
    Qp[b, i] = Q.float().transpose(0, 1)
    Qp = Qp.permute(0, 2, 1, 3).reshape(B, Hkv, -1, D)
    s = torch.matmul(Qp, K.transpose(2, 3).contiguous()).mul_(1 / math.sqrt(D)).view(B, Hq, most, Lc // S, S)
    first = pos // S
    span, token = torch.arange(Lc // S, device=DEV), torch.arange(Lc, device=DEV).view(-1, S)
    window = (token >= (first * S)[..., None, None]) & (token <= pos[..., None, None])
    factor = None
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
        total = None
    else:
        total = p.sum(dim=(3, 4))
    o = torch.matmul(p.view(B, Hkv, -1, Lc), V).view(B, Hq, most, D)
    if total is None:
        return {"O": o[b, :, i].transpose(0, 1).to(Q.dtype)}
    o = o / total[..., None]
    return {"O": o[b, :, i].transpose(0, 1).to(Q.dtype), "LSE": (m.view(B, Hq, most) + total.log())[b, :, i].transpose(0, 1)}


def _plain_append(st):
    seqs, cu, S, ps = st["seqs"].long(), st["cu"].long(), st["S"], st["case"]["ps"]
    row = torch.arange(st["Kn"].shape[1], device=DEV)
    b = torch.searchsorted(cu[1:], row, right=True)
    pos = st["lens"][seqs].long()[b] - cu[b + 1] + row
    page = st["tables"][seqs[b], pos // ps].long()
    st["K"][0][page, :, pos % ps] = st["Kn"].transpose(0, 1)
    st["V"][0][page, :, pos % ps] = st["Vn"].transpose(0, 1)
    Ks = torch.cat([st["Ks"], st["Ks"][:, :, :1]], 2)  # rows that complete no span go to a row of their own
    Ks[seqs[b], :, torch.where(pos % S == S - 1, pos // S, Ks.shape[2] - 1)] = st["Kn"].transpose(0, 1)
    st["Ks"].copy_(Ks[:, :, :-1])
    return {"K": st["K"], "V": st["V"], "Ks": st["Ks"]}


def _free_pages(refs):
    """The pages in the order in which they are given out, and how many are free."""
    return torch.argsort((refs > 0).to(torch.int8), stable=True), (refs <= 0).sum()


def _put(tables, at, valid, pages):
    flat = torch.cat([tables.view(-1), tables.new_empty(1)])
    flat[torch.where(valid, at, tables.numel())] = pages.to(torch.int32)
    tables.copy_(flat[:-1].view_as(tables))


def _plain_turn(st):
    tables, lens, refs, ps = st["tables"], st["lens"], st["refs"], st["case"]["ps"]
    src, dst, cu = st["src"].long(), st["dst"].long(), st["cu"].long()
    most = tables.shape[1]
    # free
    gone = tables[dst]
    refs.index_add_(0, gone.clamp(min=0).view(-1).long(), -(gone >= 0).view(-1).to(torch.int32))
    tables[dst] = -1
    lens[dst] = 0
    # fork
    order, free = _free_pages(refs)
    L = lens[src].long()
    part = L % ps
    need = (part > 0).long()
    end = need.cumsum(0)
    ok_fork = (need == 0) | (end <= free)
    fresh, last = order[(end - need).clamp(max=order.numel() - 1)], (L // ps).clamp(max=most - 1)
    old = tables[src, last].clamp(min=0).long()
    rows = tables[src]
    rows[torch.arange(len(src), device=DEV), last] = torch.where(need > 0, fresh.to(torch.int32), rows[torch.arange(len(src), device=DEV), last])
    rows = torch.where(ok_fork[:, None], rows, -1)
    tables[dst] = rows
    lens[dst] = torch.where(ok_fork, L, 0).to(torch.int32)
    refs.index_add_(0, rows.clamp(min=0).view(-1).long(), (rows >= 0).view(-1).to(torch.int32))
    copied = ok_fork & (need > 0)
    to = torch.where(copied, fresh, old)
    held = (torch.arange(ps, device=DEV)[None, :] < part[:, None])[None, :, None, :, None]
    for pages in (st["K"], st["V"]):
        pages[:, to] = torch.where(held, pages[:, old], pages[:, to])
    # extend
    order, free = _free_pages(refs)
    have, n = lens[dst].long(), cu[1:] - cu[:-1]
    got = (have + ps - 1) // ps
    need = (have + n + ps - 1) // ps - got
    end = need.cumsum(0)
    ok = (need == 0) | (end <= free)
    k = torch.arange(min(st["most_new"], refs.numel()), device=DEV)
    b = torch.searchsorted(end, k, right=True).clamp(max=len(dst) - 1)
    valid = (k < end[-1]) & ok[b]
    at = dst[b] * most + got[b] + k - (end - need)[b]
    _put(tables, at, valid, order[: k.numel()])
    refs.index_add_(0, order[: k.numel()], valid.to(torch.int32))
    lens[dst] = (have + torch.where(ok, n, 0)).to(torch.int32)
    return {"ok_fork": ok_fork.to(torch.int32), "ok": ok.to(torch.int32), "tables": tables, "lens": lens, "refs": refs, "K": st["K"], "V": st["V"]}


def _plain_compact(st):
    st["tables"].copy_(st["fragmented"][0])
    st["refs"].copy_(st["fragmented"][1])
    refs = st["refs"]
    page, used = torch.arange(refs.numel(), device=DEV), refs > 0
    n = used.sum()
    hole, moves = (page < n) & ~used, (page >= n) & used
    to, frm = torch.argsort((~hole).to(torch.int8), stable=True), torch.argsort((~moves).to(torch.int8), stable=True)
    source = torch.cat([page, page[:1]])
    source[torch.where(page < moves.sum(), to, refs.numel())] = frm
    source = source[:-1]
    where = torch.full((refs.numel(),), -1, dtype=torch.int32, device=DEV)
    new = torch.where(page < n, source, refs.numel())
    where = torch.cat([where, where[:1]]).index_put_((new,), page.to(torch.int32))[:-1]
    st["K"].copy_(st["K"][:, source])
    st["V"].copy_(st["V"][:, source])
    refs.copy_(torch.where(page < n, refs[source], 0))
    t = st["tables"]
    t.copy_(torch.where(t >= 0, where[t.clamp(min=0).long()], -1))
    return {"map": where, "tables": t, "refs": refs, "K": st["K"], "V": st["V"]}


# ---- the framework's calls
def _cache(st, sl):
    if "cache" not in st:
        st["cache"] = sl.PageCache(st["K"], st["V"], st["tables"], st["lens"], st["refs"])
    return st["cache"]


def _own(st):
    from paper_2601_18401_amd import binding as sl
    kind, cache = st["case"]["kind"], _cache(st, sl)
    if kind == "attention":
        if st["case"]["form"] == "gated":
            return {"O": sl.sl_paged_span_attention_combined(cache, st["seqs"], st["cu"], st["Q"], st["idx"], st["scores"], st["S"], L=max(st["Ls"]))}
        O, LSE = sl.sl_paged_span_attention(cache, st["seqs"], st["cu"], st["Q"], st["idx"], st["S"], L=max(st["Ls"]))
        return {"O": O, "LSE": LSE}
    if kind == "append":
        sl.sl_paged_append(cache, st["seqs"], st["cu"], st["Kn"], st["Vn"])
        sl.sl_paged_span_keys(cache, st["seqs"], st["cu"], st["Ks"], st["S"])
        return {"K": st["K"], "V": st["V"], "Ks": st["Ks"]}
    if kind == "turn":
        sl.sl_pages_free(cache, st["dst"])
        ok_fork = sl.sl_pages_fork(cache, st["src"], st["dst"])
        ok = sl.sl_pages_extend(cache, st["dst"], st["cu"])
        return {"ok_fork": ok_fork, "ok": ok, "tables": st["tables"], "lens": st["lens"], "refs": st["refs"], "K": st["K"], "V": st["V"]}
    st["tables"].copy_(st["fragmented"][0])
    st["refs"].copy_(st["fragmented"][1])
    where = sl.sl_pages_compact(cache)
    return {"map": where, "tables": st["tables"], "refs": st["refs"], "K": st["K"], "V": st["V"]}


def run(state):
    if own:
        return _own(state)
    return {"attention": _plain_attention, "append": _plain_append, "turn": _plain_turn, "compact": _plain_compact}[state["case"]["kind"]](state)


def work(case):
    es, kind = (4 if case["dtype"] == "f32" else 2), case["kind"]
    row = case["Hkv"] * case["D"] * es
    if kind == "attention":
        ns, Ls = _sizes(case)
        S = case["S"] or (1 << 40)
        G, read, keys = case["Hq"] // case["Hkv"], 0.0, 0.0
        for n, L in zip(ns, Ls):
            c = (L - n // 2) // S
            k = min(case["topk"], c)
            window = sum((L - n + i) % S + 1 for i in range(n))
            keys += n * k * S + window
            # distinct spans that the group's heads and the rows ask for, and the rows' windows
            read += c * S * (1 - (1 - k / c) ** (G * n) if k else 0) + min(L, (L - n) % S + n)
        T = sum(ns)
        io = 2 * case["Hq"] * T * case["D"] * es + case["Hq"] * T * 4 * (1 + case["topk"] * (2 if case["form"] == "gated" else 1))
        return {"bytes": 2 * read * row + io, "flops": 4.0 * keys * case["Hq"] * case["D"]}
    if kind == "append":
        ns, Ls = _sizes(case)
        spans = sum(L // case["S"] - (L - n) // case["S"] for n, L in zip(ns, Ls))
        return {"bytes": 4 * sum(ns) * row + 2 * spans * row, "flops": 0}
    if kind == "turn":
        Ls, src, ns = _turn_sizes(case)
        parts = sum(Ls[s] % case["ps"] for s in src)
        entries = sum(Ls[s] // case["ps"] + 1 for s in src)
        # forks freed (table rows and counts read and written), forked (read, written, counts), extended; pages of all layers copied
        return {"bytes": 4 * case["layers"] * parts * row + 4 * (8 * entries + 4 * sum(ns) // case["ps"] + case["pages"]), "flops": 0}
    used = max(1, int(case["pages"] * case["used"]))
    moved = used * (1 - used / case["pages"])
    return {"bytes": 4 * case["layers"] * moved * case["ps"] * row + 4 * (3 * case["pages"] + 4 * used), "flops": 0}


# ---- the definition in 64 bits
def _exact_attention(case, seed):
    st = prepare(case, seed)
    ns, Ls, S, ps, G = st["ns"], st["Ls"], st["S"], case["ps"], case["Hq"] // case["Hkv"]
    T = sum(ns)
    O = torch.zeros((case["Hq"], T, case["D"]), dtype=torch.float64, device=DEV)
    LSE = torch.zeros((case["Hq"], T), dtype=torch.float64, device=DEV)
    at = 0
    for b, (n, L) in enumerate(zip(ns, Ls)):
        pages = st["tables"][b, : -(-L // ps)].long()
        t = torch.arange(L, device=DEV)
        block = max(1, min(n, int(3e8 // (L * G))))
        for kv in range(case["Hkv"]):
            K, V = (x[0][pages, kv].reshape(-1, case["D"])[:L].double() for x in (st["K"], st["V"]))
            for r0 in range(0, n, block):
                rows = torch.arange(r0, min(n, r0 + block), device=DEV)
                pos = (L - n + rows)[None, :, None]
                heads = slice(kv * G, kv * G + G)
                z = (st["Q"][heads, at + rows].double() @ K.T) / math.sqrt(case["D"])
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


def _exact_append(case, seed):
    st = prepare(case, seed)
    K, V, Ks = st["K"].double(), st["V"].double(), st["Ks"].double()
    at = 0
    for b, (n, L) in enumerate(zip(st["ns"], st["Ls"])):
        t = torch.arange(L - n, L, device=DEV)
        page = st["tables"][b].long()[t // case["ps"]]
        for h in range(case["Hkv"]):
            new = st["Kn"][h, at:at + n].double()
            K[0, page, h, t % case["ps"]] = new
            V[0, page, h, t % case["ps"]] = st["Vn"][h, at:at + n].double()
            last = t[(t + 1) % case["S"] == 0]
            Ks[b, h, last // case["S"]] = new[last - (L - n)]
        at += n
    return {"K": K, "V": V, "Ks": Ks}


def _exact_turn(case, seed):
    st = prepare(case, seed)
    K, V, ps = st["K"].double(), st["V"].double(), case["ps"]
    refs, tables, lens = st["refs"].tolist(), st["tables"].tolist(), st["lens"].tolist()
    free = sorted(p for p, r in enumerate(refs) if r <= 0)
    for s in st["src"].tolist():
        if lens[s] % ps:
            if not free:
                break
            page = free.pop(0)
            for x in (K, V):
                x[:, page, :, : lens[s] % ps] = x[:, tables[s][lens[s] // ps], :, : lens[s] % ps]
    return {"ok_fork": None, "ok": None, "tables": None, "lens": None, "refs": None, "K": K, "V": V}


def _exact_compact(case, seed):
    st = prepare(case, seed)
    K, V = st["K"].double(), st["V"].double()
    used = [r > 0 for r in st["refs"].tolist()]
    n = sum(used)
    holes, moved = [p for p in range(n) if not used[p]], [p for p in range(n, len(used)) if used[p]]
    for x in (K, V):
        x[:, holes] = x[:, moved]
    return {"map": None, "tables": None, "refs": None, "K": K, "V": V}


def exact(case, seed):
    return {"attention": _exact_attention, "append": _exact_append, "turn": _exact_turn, "compact": _exact_compact}[case["kind"]](case, seed)
