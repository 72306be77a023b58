"""Timing cases of the paged 8-bit cache: its page tables, its writers and the attention that reads it.

What follows an eviction in a serving program, one call a pass, on this repository's attention shapes (head_dim
128; 32 query heads over 8 KV heads unless a case says otherwise). `op` names the call:

  pages    block tables, page releases and slot maps of every (layer, sequence) from their lengths
  gather   the kept and the window rows of an eviction, written into the cache in 8 bits
  store    new tokens' keys and values of one layer, written by slot: one a request, or whole prompts
  attend   attention of one layer's new tokens over the cache

A cache value is an e4m3 code times the power of two that its (page, head) holds as a scale. Codes are
returned as 8-bit floats beside the scales.
"""

from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128
DEV = "cuda"
F8 = torch.float8_e4m3fn


def _case(name, op, **kw):
    c = dict(op=op, hq=32, hkv=8, layers=1, page=64)
    c.update(kw)
    return dict(c, name=name) if name else c


def _spread(seed, n, lo, hi):
    """n lengths, log-uniform in [lo, hi], as the text of a case."""
    r = random.Random(seed)
    return ",".join(str(_log_int(r, lo, hi)) for _ in range(n))


def listed():
    return [
        # a decode step of 16 conversations on a 32-layer model: most grow by a token, some end (the call does not
        # depend on the heads: one keeps the cache small)
        _case("pages-decode-32layer-16", "pages", hq=4, hkv=1, layers=32, page=32, lens=_spread(1, 16, 96, 700), grow=1,
              fresh=False),
        # a wave of 48 prompts admitted at once, with the slots of every token
        _case("pages-prompts-32layer-48", "pages", hq=4, hkv=1, layers=32, page=16, lens=_spread(2, 48, 500, 32768), grow=0,
              fresh=True),
        # the compact cache of one long prompt (budget 64, window 32), all layers
        _case("gather-32layer-B64", "gather", layers=32, page=32, lens="8192", budget=64, window=32),
        # a batch of prompts with a larger budget, an odd number of rows and a short window
        _case("gather-8layer-16req-B509", "gather", layers=8, page=64, lens=_spread(3, 16, 300, 4096), budget=509, window=8),
        # one new token of each of 16 conversations
        _case("store-decode-16", "store", page=64, lens=_spread(4, 16, 1, 700), new=1, fused=True),
        # one new token of each of 256 conversations, some slots of the batch empty
        _case("store-decode-256", "store", page=16, lens=_spread(5, 256, 1, 4096), new=1, fused=True),
        # five prompts of 24k tokens in all, kept whole
        _case("store-prompts-24k", "store", page=64, lens="0,0,0,0,0", new=0, tokens="9473,1,4099,2050,8192", fused=False),
        # one conversation over a cache evicted to a budget of 64 with its window of 32: latency
        _case("attend-1x96", "attend", page=32, lens="96", q_tokens=1, fused=True),
        # 16 conversations over evicted caches that have grown by their answers, layer 1 of 2
        _case("attend-16-evicted", "attend", layers=2, page=32, lens=_spread(6, 16, 96, 700), q_tokens=1, fused=True),
        # 64 conversations of ragged length, some slots of the batch empty: ordinary serving
        _case("attend-64-ragged", "attend", page=64, lens=_spread(7, 60, 512, 16384) + ",0,0,1,1", q_tokens=1, fused=True),
        # one very long document that was not evicted
        _case("attend-1x131072", "attend", page=128, lens="131072", q_tokens=1, fused=False),
        # four drafted tokens of 24 conversations checked at once
        _case("attend-24x4-drafts", "attend", page=16, lens=_spread(8, 24, 500, 8192), q_tokens=4, fused=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["pages", "gather", "store", "attend", "attend", "attend"])
    page = rng.choice([16, 32, 64, 128])
    seed = rng.randrange(1 << 30)
    hq, hkv = rng.choice([(32, 8), (32, 8), (32, 4), (32, 2), (16, 16), (40, 8), (24, 2), (8, 1)])
    if op == "pages":
        if rng.random() < 0.5:
            return _case(None, op, hq=4, hkv=1, layers=rng.choice([1, _log_int(rng, 2, 32), 32]), page=page,
                         lens=_spread(seed, _log_int(rng, 1, 256), 1, 4096), grow=rng.choice([1, 1, 4, 7]), fresh=False)
        return _case(None, op, hq=4, hkv=1, layers=_log_int(rng, 1, 32), page=page,
                     lens=_spread(seed, _log_int(rng, 1, 40), 1, 32768), grow=0, fresh=True)
    if op == "gather":
        budget, n = _log_int(rng, 16, 512), _log_int(rng, 1, 12)
        window = min(rng.choice([1, 8, 8, 16]), 128 // (hq // hkv))
        layers = _log_int(rng, 1, max(1, min(32, 480000 // (n * hkv * budget))))
        return _case(None, op, hq=hq, hkv=hkv, layers=layers, page=page, lens=_spread(seed, n, window + 1, 4096), budget=budget,
                     window=window)
    if op == "store":
        if rng.random() < 0.5:
            return _case(None, op, hq=hq, hkv=hkv, page=page, lens=_spread(seed, _log_int(rng, 1, 512), 1, 2048),
                         new=rng.choice([1, 1, 3, 8]), fused=rng.random() < 0.5)
        n = _log_int(rng, 1, 12)
        return _case(None, op, page=page, lens=",".join(str(rng.choice([0, rng.randrange(1, 100)])) for _ in range(n)), new=0,
                     tokens=_spread(seed, n, 1, 1900), fused=rng.random() < 0.5)
    n = _log_int(rng, 1, 96)
    t = min(rng.choice([1, 1, 1, 2, 4, 5, 8]), 128 // (hq // hkv))
    hi = max(2, min(131072, (1 << 20) // (hkv * n), 8000000 // (hq * t * n)))
    return _case(None, op, hq=hq, hkv=hkv, layers=rng.choice([1, 1, 2]), page=page,
                 lens=_spread(seed, n, rng.choice([1, max(1, hi // 16)]), hi), q_tokens=t, fused=rng.random() < 0.5)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _up(a, b):
    return -(-a // b)


# ------------------------------------------------------------------------------------------------ inputs

def _random_rows(g, shape, spread=1.0):
    """bf16 rows as attention makes them: normal, with channels that are larger than others."""
    gain = torch.exp(0.5 * spread * torch.randn((D,), generator=g, device=DEV))
    return (torch.randn(shape, generator=g, device=DEV) * gain).to(torch.bfloat16)


def _quantise(x, amax):
    """(codes, scale) of rows whose largest magnitude is amax, broadcast over the rows; amax in fp32."""
    s = _need(amax)
    return (x.float() / s).to(F8), s


def _need(amax):
    """The smallest power of two s >= 2^-126 with amax <= 448 s (amax finite, fp32)."""
    m, e = torch.frexp(amax.double())   # amax = m 2^e, m in [0.5, 1): 448 = 0.875 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(min=-126)
    return torch.pow(2.0, e.double()).float()


def _pool(g, case, pages):
    """A cache whose every page is written: codes [pages][H][P][d] as bytes, scales [pages][H]."""
    h, p = case["hkv"], case["page"]
    out = []
    for _ in range(2):
        code = torch.empty((pages, h, p, D), dtype=torch.uint8, device=DEV)
        scale = torch.empty((pages, h), dtype=torch.float32, device=DEV)
        step = max(1, (1 << 26) // (h * p * D))
        for a in range(0, pages, step):
            b = min(pages, a + step)
            x = _random_rows(g, (b - a, h, p, D)).float()
            x *= torch.exp(0.3 * torch.randn((b - a, h, 1, 1), generator=g, device=DEV))
            x = x.to(torch.bfloat16)
            c, s = _quantise(x, x.abs().amax(dim=(2, 3), keepdim=True).float())
            code[a:b] = c.view(torch.uint8)
            scale[a:b] = s[:, :, 0, 0]
        out += [code, scale]
    return out


def _table(g, have, max_pages, pages):
    """A table whose sequences hold have[i] pages each, taken in a shuffled order; -1 behind them."""
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    have = torch.tensor(have, device=DEV, dtype=torch.int64)
    first = torch.cumsum(have, 0) - have
    j = torch.arange(max_pages, device=DEV)
    ids = order[(first[:, None] + j[None]).clamp(max=pages - 1)]
    return torch.where(j[None] < have[:, None], ids, torch.full_like(ids, -1)), order


def _spec(case):
    return dict(num_layers=case["layers"], num_q_heads=case["hq"], num_kv_heads=case["hkv"], head_dim=D,
                window=case.get("window", 1), budget=case.get("budget", 1), pool_kernel=7, candidate_factor=1,
                norm_eps=1e-12)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case=case, op=case["op"])
    make = {"pages": _prepare_pages, "gather": _prepare_gather, "store": _prepare_store, "attend": _prepare_attend}
    make[case["op"]](case, g, s, random.Random(seed))
    if own:
        from paper_2609_30738_gb300 import kv_evict
        s["cache"] = kv_evict.Cache8(_spec(case), max_seqs=s["n_seq"], num_pages=s["n_pages"], max_pages=s["max_pages"],
                                     page_tokens=case["page"], k=s.get("k8"), v=s.get("v8"), k_scale=s.get("ks"),
                                     v_scale=s.get("vs"))
        if case["op"] == "gather":
            s["plan"] = kv_evict.Plan(_spec(case), _ints(case["lens"]))
    return s


def _prepare_pages(case, g, s, rng):
    p, layers = case["page"], case["layers"]
    lens = _ints(case["lens"])
    n = len(lens)
    rows_from, rows_to = [], []
    for _ in range(layers):
        if case["fresh"]:   # empty sequences get their prompts, which an eviction has cut differently by layer
            rows_from.append([0] * n)
            rows_to.append([max(1, x - rng.randrange(0, min(x, 64))) for x in lens])
        else:               # every sequence grows, but for those that have ended
            rows_from.append([max(1, x - rng.randrange(0, min(x, 64))) for x in lens])
            rows_to.append(list(rows_from[-1]))
    if not case["fresh"]:
        for i in range(n):
            ended = rng.random() < 0.1
            for l in range(layers):
                rows_to[l][i] = 0 if ended else rows_to[l][i] + case["grow"]
    have = [_up(x, p) for row in rows_from for x in row]
    s["n_seq"] = n
    grow = 0 if case["fresh"] else case["grow"]
    s["max_pages"] = _up(max(lens) + grow, p)
    s["n_pages"] = layers * sum(_up(x + grow, p) for x in lens) + 37   # room for all, whatever the seed
    table, order = _table(g, have, s["max_pages"], s["n_pages"])
    used = sum(have)
    head = rng.randrange(s["n_pages"])
    ring = torch.roll(torch.cat([order[used:], order[:used]]), head)
    s["table"] = table.view(layers, n, s["max_pages"]).contiguous()
    s["free"] = ring.contiguous()
    s["ring_in"] = torch.tensor([head, s["n_pages"] - used], dtype=torch.int32, device=DEV)
    s["ring_out"] = torch.zeros_like(s["ring_in"])
    s["from"] = torch.tensor(rows_from, dtype=torch.int32, device=DEV)
    s["to"] = torch.tensor(rows_to, dtype=torch.int32, device=DEV)
    s["lens"] = torch.zeros_like(s["to"])
    s["slots"] = torch.zeros((layers, n * grow or sum(lens)), dtype=torch.int32, device=DEV)


def _prepare_gather(case, g, s, rng):
    p, layers, h = case["page"], case["layers"], case["hkv"]
    lens, b, w = _ints(case["lens"]), case["budget"], case["window"]
    n, total = len(lens), sum(lens)
    s["k"] = _random_rows(g, (layers, h, total, D))
    s["v"] = _random_rows(g, (layers, h, total, D))
    kept = [min(b, x - w) for x in lens]
    idx = torch.full((n, layers, h, b), -1, dtype=torch.int32, device=DEV)
    for r, x in enumerate(lens):
        pick = torch.rand((layers, h, x - w), generator=g, device=DEV).topk(kept[r], dim=-1).indices
        idx[r, :, :, :kept[r]] = pick.sort(dim=-1).values.to(torch.int32)
    s["indices"] = idx.view(-1, b)
    s["n_seq"], s["max_pages"] = n, _up(b + w, p)
    have = [_up(m + w, p) for m in kept for _ in range(layers)]
    s["n_pages"] = sum(have) + 5
    table, order = _table(g, have, s["max_pages"], s["n_pages"])
    s["table"], s["spare"] = table.view(n, layers, -1).transpose(0, 1).contiguous(), order[-1].long()
    s["k8"], s["ks"], s["v8"], s["vs"] = _pool(g, case, s["n_pages"])
    s["kept"] = torch.tensor(kept, device=DEV)
    s["lens"] = torch.tensor(lens, device=DEV)


def _prepare_store(case, g, s, rng):
    p, h = case["page"], case["hkv"]
    lens = _ints(case["lens"])
    new = _ints(case["tokens"]) if case["new"] == 0 else [case["new"]] * len(lens)
    if case["new"] and len(lens) > 100:   # empty slots of a padded batch
        new = [0 if rng.random() < 0.05 else x for x in new]
    have = [_up(a + b, p) for a, b in zip(lens, new)]
    most = [_up(a + max(b, case["new"]), p) for a, b in zip(lens, new)]
    s["n_seq"], s["max_pages"], s["n_pages"] = len(lens), max(most), sum(most) + 3
    table = _table(g, have, s["max_pages"], s["n_pages"])[0].cpu().numpy()
    slots = []
    for i, (a, b) in enumerate(zip(lens, new)):
        pos = np.arange(a, a + b)
        slots.append(table[i, pos // p].astype(np.int64) * p + pos % p if b else np.full(max(1, case["new"]), -1))
    slots = np.concatenate(slots)
    s["slots"] = torch.from_numpy(slots.astype(np.int32)).to(DEV)
    n = len(slots)
    heads = case["hq"] + 2 * h
    if case["fused"]:      # slices of the projection's output
        x = _random_rows(g, (n, heads, D))
        s["k_new"], s["v_new"] = x[:, case["hq"]:case["hq"] + h], x[:, case["hq"] + h:]
    else:
        s["k_new"], s["v_new"] = _random_rows(g, (n, h, D)), _random_rows(g, (n, h, D))
    s["k8"], s["ks"], s["v8"], s["vs"] = _pool(g, case, s["n_pages"])


def _prepare_attend(case, g, s, rng):
    p, h, layers, t = case["page"], case["hkv"], case["layers"], case["q_tokens"]
    lens = _ints(case["lens"])
    n = len(lens)
    have = [_up(x, p) for x in lens] * layers
    s["n_seq"], s["max_pages"], s["n_pages"] = n, max(1, max(have)), sum(have) + 3
    s["table"] = _table(g, have, s["max_pages"], s["n_pages"])[0].view(layers, n, -1).contiguous()
    s["lens"] = torch.tensor([lens] * layers, dtype=torch.int32, device=DEV)
    s["k8"], s["ks"], s["v8"], s["vs"] = _pool(g, case, s["n_pages"])
    s["layer"] = layers - 1
    heads = case["hq"] + (2 * h if case["fused"] else 0)
    # logits of standard deviation 1.5 or so: some rows peaked, most spread
    s["q"] = (_random_rows(g, (n, t, heads, D), 0.5) * 0.8).to(torch.bfloat16)[:, :, :case["hq"]]
    s["out"] = torch.empty((n, t, case["hq"], D), dtype=torch.bfloat16, device=DEV)
    s["lse"] = torch.empty((n, t, case["hq"]), dtype=torch.float32, device=DEV)


# ------------------------------------------------------------------------------------------------ passes

def run(s):
    if own:
        c = s["cache"]
        if s["op"] == "pages":
            c.pages(s["from"], s["to"], s["table"], s["free"], s["ring_in"], s["ring_out"], s["lens"], s["slots"])
        elif s["op"] == "gather":
            c.gather(s["plan"], s["k"], s["v"], s["indices"], s["table"])
        elif s["op"] == "store":
            c.store(s["k_new"], s["v_new"], s["slots"])
        else:
            c.attend(s["q"], s["table"], s["lens"], s["layer"], s["out"], s["lse"])
    else:
        {"pages": _plain_pages, "gather": _plain_gather, "store": _plain_store, "attend": _plain_attend}[s["op"]](s)
    if s["op"] == "pages":
        return dict(table=s["table"], free=s["free"], ring=s["ring_out"], lens=s["lens"], slots=s["slots"])
    if s["op"] == "attend":
        return dict(out=s["out"], lse=s["lse"])
    return dict(k=s["k8"].view(F8), v=s["v8"].view(F8), k_scale=s["ks"], v_scale=s["vs"])


def _plain_pages(s):
    p, n_pages = s["case"]["page"], s["n_pages"]
    a, b = s["from"].long(), s["to"].long()
    layers, n = a.shape
    have, need = (a + p - 1) // p, (b + p - 1) // p
    grow = (need - have).clamp(min=0).view(-1)
    gone = (have - need).clamp(min=0).view(-1)
    grow_at, gone_at = torch.cumsum(grow, 0) - grow, torch.cumsum(gone, 0) - gone
    head, count = s["ring_in"][0].long(), s["ring_in"][1].long()
    ok = grow.sum() <= count   # the cases have room: all or nothing otherwise
    j = torch.arange(s["max_pages"], device=DEV)[None]
    table = s["table"].view(layers * n, -1)
    have, need = have.view(-1, 1), need.view(-1, 1)
    page = s["free"][(head + grow_at[:, None] + (j - have).clamp(min=0)) % n_pages]
    back = (head + count + gone_at[:, None] + (j - need).clamp(min=0)) % n_pages
    free = torch.cat([s["free"], s["free"][:1]])
    free[torch.where((j >= need) & (j < have) & ok, back, torch.full_like(back, n_pages))] = table
    s["free"].copy_(free[:n_pages])
    table.copy_(torch.where((j >= have) & (j < need) & ok, page, table))
    s["ring_out"][0] = torch.where(ok, (head + grow.sum()) % n_pages, head)
    s["ring_out"][1] = torch.where(ok, count - grow.sum() + gone.sum(), count)
    s["lens"].copy_(torch.where(ok, b, a))
    new = (b - a).clamp(min=0)
    end = torch.cumsum(new, 1)
    at = torch.arange(s["slots"].shape[1], device=DEV).expand(layers, -1).contiguous()
    seq = torch.searchsorted(end, at, right=True)
    inside = (seq < n) & ok
    seq = seq.clamp(max=n - 1)
    pos = a.gather(1, seq) + at - (end - new).gather(1, seq)
    row = torch.arange(layers, device=DEV)[:, None] * n + seq
    slot = table[row, (pos // p).clamp(max=s["max_pages"] - 1)].long() * p + pos % p
    s["slots"].copy_(torch.where(inside, slot, torch.full_like(slot, -1)))


def _plain_gather(s):
    case = s["case"]
    p, w, b = case["page"], case["window"], case["budget"]
    layers, n, h = case["layers"], s["n_seq"], case["hkv"]
    rows = s["max_pages"] * p
    j = torch.arange(rows, device=DEV)
    m = s["kept"][:, None, None, None]                                   # [n][1][1][1]
    idx = s["indices"].view(n, layers, h, b)
    pick = idx[..., j.clamp(max=b - 1)].long()
    win = (s["lens"] - w)[:, None, None, None] + j - m
    src = torch.where(j < m, pick, win)
    good = (j < m + w).expand(n, layers, h, rows)
    src = torch.where(good, src, torch.zeros_like(src)) + (torch.cumsum(s["lens"], 0) - s["lens"])[:, None, None, None]
    l = torch.arange(layers, device=DEV)[None, :, None, None]
    hh = torch.arange(h, device=DEV)[None, None, :, None]
    table = s["table"].permute(1, 0, 2).long()                           # [n][layers][pages]
    valid = good.view(n, layers, h, -1, p)
    held = (table >= 0) & valid.any(-1)[:, :, 0]
    at = torch.where(held, table, s["spare"])
    put = held[:, :, None].expand(n, layers, h, -1)
    _write_pages(s["k"][l, hh, src].view(n, layers, h, -1, p, D), valid, at, put, s["k8"], s["ks"])
    _write_pages(s["v"][l, hh, src].view(n, layers, h, -1, p, D), valid, at, put, s["v8"], s["vs"])


def _write_pages(x, valid, at, put, code, scale):
    """Rows x of whole pages into the pages `at` (where put): codes of the valid rows, and the scales."""
    x = torch.where(valid[..., None], x.float(), torch.zeros((), device=DEV))
    q, s = _quantise(x, x.abs().amax(dim=(-1, -2), keepdim=True))
    page = at[:, :, None].expand(put.shape)
    head = torch.arange(put.shape[2], device=DEV)[None, None, :, None].expand(put.shape)
    old, old_s = code[page, head], scale[page, head]
    code[page, head] = torch.where((valid & put[..., None])[..., None], q.view(torch.uint8), old)
    scale[page, head] = torch.where(put, s[..., 0, 0], old_s)


def _plain_store(s):
    p, n_pages = s["case"]["page"], s["n_pages"]
    slot = s["slots"].long()
    # what the empty slots of the batch would write goes to a page behind the last
    page = torch.where(slot >= 0, slot // p, torch.full_like(slot, n_pages))
    off = torch.where(slot >= 0, slot % p, torch.zeros_like(slot))
    first = torch.full((n_pages + 1,), p, device=DEV).scatter_reduce(0, page, off, "amin")[:n_pages]
    for x, code, scale in ((s["k_new"], s["k8"], s["ks"]), (s["v_new"], s["v8"], s["vs"])):
        x = x.float()
        amax = torch.zeros((n_pages + 1, x.shape[1]), device=DEV).scatter_reduce(
            0, page[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")[:n_pages]
        written = (first < p)[:, None]
        held = torch.where((first > 0)[:, None], scale, torch.zeros_like(scale))
        to = torch.where(written, torch.maximum(held, _need(amax)), scale)
        older = written[:, :, None] & (torch.arange(p, device=DEV)[None, None] < first[:, None, None])
        moved = (code.view(F8).float() * (held / to)[..., None, None]).to(F8).view(torch.uint8)
        new = torch.where(older[..., None], moved, code)
        new = torch.cat([new, new[:1]])
        q = (x / torch.cat([to, to[:1]])[page][..., None]).to(F8).view(torch.uint8)
        new[page, :, off] = q
        code.copy_(new[:n_pages])
        scale.copy_(to)


def _plain_attend(s):
    case = s["case"]
    h, t, n = case["hkv"], case["q_tokens"], s["n_seq"]
    g = case["hq"] // h
    lens = s["lens"][s["layer"]].long()
    ids = s["table"][s["layer"]].long().clamp(min=0)

    def rows(code, scale):   # [n][h][tokens][d]
        x = code[ids].view(F8).float() * scale[ids][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(n, h, -1, D)

    q = s["q"].float().reshape(n, t, h, g, D).permute(0, 2, 1, 3, 4).reshape(n, h, t * g, D)
    pos = torch.arange(ids.shape[1] * case["page"], device=DEV)
    x = torch.matmul(q, rows(s["k8"], s["ks"]).transpose(-1, -2)) * (1.0 / math.sqrt(D))
    seen = (lens[:, None] - t + 1 + torch.arange(t, device=DEV)).repeat_interleave(g, 1)[:, None, :, None]
    mask = pos < seen
    x = x.masked_fill(~mask, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    v = rows(s["v8"], s["vs"]).masked_fill((pos >= lens[:, None])[:, None, :, None], 0.0)
    o = torch.matmul(e, v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = torch.log(total) + top
    s["out"].copy_(o.view(n, h, t, g, D).permute(0, 2, 1, 3, 4).reshape(n, t, h * g, D))
    s["lse"].copy_(lse.view(n, h, t, g).permute(0, 2, 1, 3).reshape(n, t, h * g))


# ------------------------------------------------------------------------------------------------ exact

_E4M3 = np.array([(-1.0 if c & 128 else 1.0) * ((c & 7) / 8 * 2.0 ** -6 if (c >> 3) & 15 == 0
                                              else (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7))
                  if c & 127 != 127 else math.nan for c in range(256)])


def _values(code):
    return torch.from_numpy(_E4M3).to(DEV)[code.long()]


_POWERS = np.array([2.0 ** e for e in range(-6, 10)])


def _round8(x):
    """x (64 bits, |x| <= 448) to the nearest e4m3 value, ties to the even one."""
    powers = torch.from_numpy(_POWERS).to(DEV)
    binade = (torch.searchsorted(powers, x.abs().contiguous(), right=True) - 1).clamp(min=0)
    ulp = powers[binade] / 8
    return torch.round(x / ulp) * ulp


def _power(amax):
    """The scale of one block's largest magnitude, by search over the exponents."""
    e = -126
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def exact(case, seed):
    if case["op"] == "pages" or work(case)["bytes"] > 1.5e9:
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"gather": _exact_gather, "store": _exact_store, "attend": _exact_attend}[case["op"]](s)


def _exact_scales(amax):
    return torch.tensor([_power(float(x)) for x in amax.view(-1).cpu()], dtype=torch.float64, device=DEV).view(amax.shape)


def _exact_gather(s):
    case = s["case"]
    p, w, layers, h = case["page"], case["window"], case["layers"], case["hkv"]
    lens = _ints(case["lens"])
    idx = s["indices"].view(len(lens), layers, h, -1).long()
    out = {}
    for name, src, code, scale in (("k", s["k"], s["k8"], s["ks"]), ("v", s["v"], s["v8"], s["vs"])):
        val, sc = _values(code), scale.double()
        at = 0
        for r, x in enumerate(lens):
            m = min(case["budget"], x - w)
            rows = torch.cat([idx[r, :, :, :m], torch.arange(x - w, x, device=DEV).expand(layers, h, w)], -1) + at
            full = src.gather(2, rows[..., None].expand(-1, -1, -1, D)).double()
            for j in range(_up(m + w, p)):
                part = full[:, :, j * p:(j + 1) * p]
                f = _exact_scales(part.abs().amax(dim=(2, 3)))
                ids = s["table"][:, r, j].long()
                val[ids, :, :part.shape[2]] = _round8(part / f[..., None, None])
                sc[ids] = f
            at += x
        out[name], out[name + "_scale"] = val, sc
    return out


def _exact_store(s):
    p = s["case"]["page"]
    slots = s["slots"].cpu().tolist()
    out = {}
    for name, src, code, scale in (("k", s["k_new"], s["k8"], s["ks"]), ("v", s["v_new"], s["v8"], s["vs"])):
        val, sc, t = _values(code), scale.double(), 0
        while t < len(slots):
            e = t + 1
            while slots[t] >= 0 and e < len(slots) and slots[e] == slots[e - 1] + 1 and slots[e] % p:
                e += 1
            if slots[t] >= 0:
                page, off = divmod(slots[t], p)
                x = src[t:e].double().transpose(0, 1)                     # [h][rows][d]
                f = _exact_scales(x.abs().amax(dim=(1, 2)))
                if off:
                    f = torch.maximum(f, sc[page])
                    val[page, :, :off] = _round8(val[page, :, :off] * (sc[page] / f)[:, None, None])
                val[page, :, off:off + e - t] = _round8(x / f[:, None, None])
                sc[page] = f
            t = e
        out[name], out[name + "_scale"] = val, sc
    return out


def _exact_attend(s):
    case = s["case"]
    p, h, t = case["page"], case["hkv"], case["q_tokens"]
    g = case["hq"] // h
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    for r, x in enumerate(_ints(case["lens"])):
        ids = s["table"][s["layer"], r, :_up(x, p)].long()
        k, v = ((_values(c[ids]) * f[ids].double()[..., None, None]).transpose(1, 2).reshape(-1, h, D)[:x]
                for c, f in ((s["k8"], s["ks"]), (s["v8"], s["vs"])))
        for i in range(t):
            seen = x - t + i + 1
            if seen > 0:
                a = torch.einsum("hgd,nhd->hgn", s["q"][r, i].double().reshape(h, g, D), k[:seen]) / math.sqrt(D)
                lse[r, i] = torch.logsumexp(a, -1).reshape(-1)
                out[r, i] = torch.einsum("hgn,nhd->hgd", torch.softmax(a, -1), v[:seen]).reshape(-1, D)
    return dict(out=out, lse=lse)


# ------------------------------------------------------------------------------------------------ work

def work(case):
    """Bytes: each input read once, each output written once. Flops: the two products of the attention."""
    lens, p, layers, h = _ints(case["lens"]), case["page"], case["layers"], case["hkv"]
    n = len(lens)
    if case["op"] == "pages":
        grown = sum(lens) * layers if case["fresh"] else n * layers * case["grow"]
        new = sum(_up(x, p) for x in lens) * layers if case["fresh"] else _up(grown, p)
        return {"bytes": 12 * n * layers + 8 * new + 4 * grown, "flops": 0}
    if case["op"] == "gather":
        rows = sum(min(case["budget"], x - case["window"]) + case["window"] for x in lens)
        pages = sum(_up(min(case["budget"], x - case["window"]) + case["window"], p) for x in lens)
        return {"bytes": layers * h * (rows * D * 6 + rows * 4 + pages * 8) + layers * pages * 4, "flops": 0}
    if case["op"] == "store":
        toks = sum(_ints(case["tokens"])) if case["new"] == 0 else n * case["new"]
        pages = max(n, toks // p)
        return {"bytes": toks * (h * D * 6 + 4) + pages * h * 16, "flops": 0}
    t, tok = case["q_tokens"], sum(lens)
    pages = sum(_up(x, p) for x in lens)
    return {"bytes": tok * h * D * 2 + pages * (4 + 8 * h) + n * t * case["hq"] * (D * 4 + 4),
            "flops": 4 * D * tok * case["hq"] * t}
