"""Timing cases of rotary positions and of the paged 4-bit cache.

A decode step as a serving program makes it behind an eviction: queries and keys are rotated by their positions, the
rotated keys and the values go into the paged cache in the same call, and the cache is attended over; in 4 bits it
holds twice the tokens. On this repository's attention shapes (head_dim 128; 32 query heads over 8 KV heads unless a
case says otherwise). `op` names the call:

  rotate   rotary positions of rows [tokens][heads][d]: both pairings, part of the head, the transpose for gradients
  append   new tokens' queries and keys rotated, keys and values written into the paged 8-bit cache by slot
  gather4  the kept and the window rows of an eviction, written into the 4-bit cache
  store4   new tokens' keys and values of one layer into the 4-bit cache by slot
  attend4  attention of one layer's new tokens over the 4-bit cache

A 4-bit row has 128 codes c in 0 .. 15, two in a byte (the even element in the low half), and two bf16 numbers,
s and z: an element stands for s c + z. Packed codes are whole numbers, equal or not; s and z are returned beside them.
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
    if op in ("rotate", "append"):
        c.update(rotary=128, interleaved=False, scaling="none", base=10000.0, factor=1.0, original=8192, start=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _spread(seed, n, lo, hi):
    """n lengths, log-uniform in [lo, hi], as the text of a case."""
    r = random.Random(seed)
    return ",".join(str(_log_int(r, lo, hi)) for _ in range(n))


def listed():
    return [
        # the window queries of one prompt of 32768 tokens, all layers at once, before they score its keys: rows by head
        _case("rotate-window-32layer", "rotate", tokens=32, heads=1024, head_major=True, start=32736),
        # the gradient of a training batch's queries and keys, slices of the projection's: half of the head, pairs side
        # by side, a context stretched eightfold
        _case("rotate-gradient-16k", "rotate", tokens=16411, heads=40, head_major=False, rotary=64, interleaved=True,
              scaling="yarn", factor=8.0, original=4096, transpose=True),
        # one new token of each of 16 conversations, far beyond what their caches kept
        _case("append-decode-16", "append", lens=_spread(4, 16, 1, 700), new=1, start=30000),
        # five prompts of 24k tokens in all, kept whole
        _case("append-prompts-24k", "append", lens="0,0,0,0,0", new=0, tokens="9473,1,4099,2050,8192", scaling="parts",
              base=500000.0, factor=8.0),
        # the compact cache of one long prompt (budget 64, window 32), all layers
        _case("gather4-32layer-B64", "gather4", layers=32, page=32, lens="8192", budget=64, window=32),
        # a batch of prompts with a larger budget, an odd number of rows and a short window
        _case("gather4-8layer-16req-B509", "gather4", layers=8, page=64, lens=_spread(3, 16, 300, 4096), budget=509, window=8),
        # one new token of each of 256 conversations, some slots of the batch empty
        _case("store4-decode-256", "store4", page=16, lens=_spread(5, 256, 1, 4096), new=1, fused=True),
        # the same five prompts into the 4-bit cache
        _case("store4-prompts-24k", "store4", page=64, lens="0,0,0,0,0", new=0, tokens="9473,1,4099,2050,8192", fused=False),
        # 16 conversations over evicted caches that have grown by their answers, layer 1 of 2: latency
        _case("attend4-16-evicted", "attend4", layers=2, page=32, lens=_spread(6, 16, 96, 700), q_tokens=1, fused=True),
        # 64 conversations of ragged length, some slots of the batch empty: ordinary serving
        _case("attend4-64-ragged", "attend4", page=64, lens=_spread(7, 60, 512, 16384) + ",0,0,1,1", q_tokens=1, fused=True),
        # one very long document that was not evicted
        _case("attend4-1x131072", "attend4", page=128, lens="131072", q_tokens=1, fused=False),
        # four drafted tokens of 24 conversations checked at once
        _case("attend4-24x4-drafts", "attend4", page=16, lens=_spread(8, 24, 500, 8192), q_tokens=4, fused=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rotary(rng):
    scaling = rng.choice(["none", "none", "linear", "ntk", "parts", "yarn"])
    return dict(rotary=rng.choice([128, 128, 96, 64, 32]), interleaved=rng.random() < 0.5, scaling=scaling,
                base=rng.choice([10000.0, 500000.0, 1000000.0]), factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]),
                original=rng.choice([2048, 4096, 8192, 32768]), start=rng.choice([0, 0, _log_int(rng, 1, 4000000)]))


def draw(rng):
    op = rng.choice(["rotate", "append", "gather4", "store4", "attend4", "attend4"])
    page = rng.choice([16, 32, 64, 128])
    seed = rng.randrange(1 << 30)
    hq, hkv = rng.choice([(32, 8), (32, 8), (32, 4), (32, 2), (16, 16), (40, 8), (24, 2), (8, 1)])
    if op == "rotate":
        heads = rng.choice([1, 2, 8, 32, 40, _log_int(rng, 1, 1024)])
        return _case(None, op, tokens=_log_int(rng, 1, max(1, 640000 // heads)), heads=heads, head_major=rng.random() < 0.3,
                     transpose=rng.random() < 0.3, **_draw_rotary(rng))
    if op == "append":
        rotary = _draw_rotary(rng)
        if rng.random() < 0.5:
            return _case(None, op, hq=hq, hkv=hkv, page=page, lens=_spread(seed, _log_int(rng, 1, 512), 1, 2048),
                         new=rng.choice([1, 1, 3, 8]), **rotary)
        n = _log_int(rng, 1, 12)
        return _case(None, op, page=page, lens=",".join(str(rng.choice([0, rng.randrange(1, 100)])) for _ in range(n)), new=0,
                     tokens=_spread(seed, n, 1, 1900), **rotary)
    if op == "gather4":
        budget, n = _log_int(rng, 16, 512), _log_int(rng, 1, 12)
        window = min(rng.choice([1, 8, 8, 16]), 128 // (hq // hkv))
        layers = _log_int(rng, 1, max(1, min(32, 480000 // (n * hkv * budget))))
        return _case(None, op, hq=hq, hkv=hkv, layers=layers, page=page, lens=_spread(seed, n, window + 1, 4096), budget=budget,
                     window=window)
    if op == "store4":
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


def _need(amax):
    """The smallest power of two s >= 2^-126 with amax <= 448 s (amax finite, fp32)."""
    m, e = torch.frexp(amax.double())   # amax = m 2^e, m in [0.5, 1): 448 = 0.875 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(min=-126)
    return torch.pow(2.0, e.double()).float()


def _quantise4(x):
    """(packed codes [..., 64], s and z [..., 2]) of finite bf16 rows [..., 128], in fp32: s = (hi - lo) / 15 rounded to
    bf16 (a spread below 15 * 2^-120 counts as none), z = lo, c = (x - lo) / s to the nearest, ties to the even one. Counted
    in units of 2^4, so that no difference overflows."""
    x = x.float() * 0.0625
    lo, hi = x.amin(-1, keepdim=True) + 0.0, x.amax(-1, keepdim=True)
    s = ((hi - lo) * (16.0 / 15.0)).to(torch.bfloat16)
    s = torch.where(s.float() >= 2.0 ** -120, s, torch.zeros_like(s))
    unit = s.float() * 0.0625
    c = torch.round((x - lo) / torch.where(unit > 0, unit, torch.ones_like(unit))).clamp(max=15.0)
    c = torch.where(unit > 0, c, torch.zeros_like(c)).to(torch.uint8)
    return c[..., 0::2] | c[..., 1::2] << 4, torch.cat([s, (lo * 16.0).to(torch.bfloat16)], -1)


def _pool8(g, case, pages):
    """An 8-bit cache whose every page is written: codes [pages][H][P][d] as bytes, scales [pages][H]."""
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
            s = _need(x.abs().amax(dim=(2, 3), keepdim=True))
            code[a:b] = (x / s).to(F8).view(torch.uint8)
            scale[a:b] = s[:, :, 0, 0]
        out += [code, scale]
    return out


def _pool4(g, case, pages):
    """A 4-bit cache whose every page is written: codes [pages][H][P][64] as bytes, s and z [pages][H][P][2]."""
    h, p = case["hkv"], case["page"]
    out = []
    for _ in range(2):
        code = torch.empty((pages, h, p, D // 2), dtype=torch.uint8, device=DEV)
        param = torch.empty((pages, h, p, 2), dtype=torch.bfloat16, device=DEV)
        step = max(1, (1 << 25) // (h * p * D))
        for a in range(0, pages, step):
            b = min(pages, a + step)
            x = _random_rows(g, (b - a, h, p, D)).float()
            x *= torch.exp(0.3 * torch.randn((b - a, h, p, 1), generator=g, device=DEV))
            code[a:b], param[a:b] = _quantise4(x.to(torch.bfloat16))
        out += [code, param]
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
    make = {"rotate": _prepare_rotate, "append": _prepare_store, "gather4": _prepare_gather, "store4": _prepare_store,
            "attend4": _prepare_attend}
    make[case["op"]](case, g, s, random.Random(seed))
    if own:
        from paper_2609_30738_gb300 import kv_evict
        if case["op"] in ("rotate", "append"):
            s["rotary"] = kv_evict.Rotary(D, case["rotary"], base=case["base"], interleaved=case["interleaved"],
                                          scaling=case["scaling"], factor=case["factor"], original_length=case["original"])
        if case["op"] != "rotate":
            sizes = dict(max_seqs=s["n_seq"], num_pages=s["n_pages"], max_pages=s["max_pages"], page_tokens=case["page"])
            if case["op"] == "append":
                s["cache"] = kv_evict.Cache8(_spec(case), k=s["k8"], v=s["v8"], k_scale=s["ks"], v_scale=s["vs"], **sizes)
            else:
                s["cache"] = kv_evict.Cache4(_spec(case), k=s["k4"], v=s["v4"], k_param=s["kp"], v_param=s["vp"], **sizes)
        if case["op"] == "gather4":
            s["plan"] = kv_evict.Plan(_spec(case), _ints(case["lens"]))
    else:
        if case["op"] in ("rotate", "append"):
            s["freq"], s["amplitude"] = _frequencies(case)
    return s


def _prepare_rotate(case, g, s, rng):
    n, h = case["tokens"], case["heads"]
    if case["head_major"]:
        s["x"] = _random_rows(g, (h, n, D)).transpose(0, 1)
        s["out"] = torch.empty((h, n, D), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    else:   # a slice of the projection's output, whose last heads are the values
        s["x"] = _random_rows(g, (n, h + max(1, h // 4), D))[:, :h]
        s["out"] = torch.empty((n, h, D), dtype=torch.bfloat16, device=DEV)
    s["positions"] = (torch.arange(n, device=DEV) + case["start"] + rng.randrange(64)).to(torch.int32)


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
    table, _ = _table(g, have, s["max_pages"], s["n_pages"])
    s["table"] = table.view(n, layers, -1).transpose(0, 1).contiguous()
    s["k4"], s["kp"], s["v4"], s["vp"] = _pool4(g, case, s["n_pages"])
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
    slots, positions = [], []
    for i, (a, b) in enumerate(zip(lens, new)):
        pos = np.arange(a, a + b)
        # what an eviction dropped still counts in a token's position
        positions.append(pos + case.get("start", 0) + rng.randrange(1000) if b else np.zeros(max(1, case["new"]), np.int64))
        slots.append(table[i, pos // p].astype(np.int64) * p + pos % p if b else np.full(max(1, case["new"]), -1))
    slots, positions = np.concatenate(slots), np.concatenate(positions)
    s["slots"] = torch.from_numpy(slots.astype(np.int32)).to(DEV)
    n, hq = len(slots), case["hq"]
    if case["op"] == "append":
        s["positions"] = torch.from_numpy(positions.astype(np.int32)).to(DEV)
        s["q_out"] = torch.empty((n, hq, D), dtype=torch.bfloat16, device=DEV)
    if case.get("fused", True):      # slices of the projection's output
        x = _random_rows(g, (n, hq + 2 * h, D))
        s["q"], s["k_new"], s["v_new"] = x[:, :hq], x[:, hq:hq + h], x[:, hq + h:]
    else:
        s["k_new"], s["v_new"] = _random_rows(g, (n, h, D)), _random_rows(g, (n, h, D))
    if case["op"] == "append":
        s["k8"], s["ks"], s["v8"], s["vs"] = _pool8(g, case, s["n_pages"])
    else:
        s["k4"], s["kp"], s["v4"], s["vp"] = _pool4(g, case, s["n_pages"])


def _prepare_attend(case, g, s, rng):
    p, h, layers, t = case["page"], case["hkv"], case["layers"], case["q_tokens"]
    lens = _ints(case["lens"])
    n = len(lens)
    have = [_up(x, p) for x in lens] * layers
    s["n_seq"], s["max_pages"], s["n_pages"] = n, max(1, max(have)), sum(have) + 3
    s["table"] = _table(g, have, s["max_pages"], s["n_pages"])[0].view(layers, n, -1).contiguous()
    s["lens"] = torch.tensor([lens] * layers, dtype=torch.int32, device=DEV)
    s["k4"], s["kp"], s["v4"], s["vp"] = _pool4(g, case, s["n_pages"])
    s["layer"] = layers - 1
    heads = case["hq"] + (2 * h if case["fused"] else 0)
    # logits of standard deviation 1.5 or so: some rows peaked, most spread
    s["q"] = (_random_rows(g, (n, t, heads, D), 0.5) * 0.8).to(torch.bfloat16)[:, :, :case["hq"]]
    s["out"] = torch.empty((n, t, case["hq"], D), dtype=torch.bfloat16, device=DEV)
    s["lse"] = torch.empty((n, t, case["hq"]), dtype=torch.float32, device=DEV)


def _frequencies(case):
    """(radians a position of each pair, in 64 bits, and what cos and sin are multiplied by)."""
    n, base, factor = case["rotary"], case["base"], case["factor"]
    j = torch.arange(n // 2, dtype=torch.float64, device=DEV)
    if case["scaling"] == "ntk":   # the base is stretched, so that the slowest pair turns `factor` times slower
        base = base * factor ** (n / (n - 2.0))
    f = torch.exp(j * (-2.0 * math.log(base) / n))
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "parts":   # pairs that turn once or less within the original length slow down, those that turn 4 times do not
        keep = ((f * (case["original"] / (2.0 * math.pi)) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 1.0
    if case["scaling"] == "yarn":    # the same between 32 turns and 1, linear in the pair's number
        at = [n * math.log(case["original"] / (2.0 * math.pi * r)) / (2.0 * math.log(base)) for r in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), n - 1)
        keep = 1.0 - ((j - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0
    return f, 1.0


# ------------------------------------------------------------------------------------------------ passes

def run(s):
    op = s["op"]
    if own:
        if op == "rotate":
            s["rotary"].rotate(s["x"], s["positions"], out=s["out"], transpose=s["case"].get("transpose", False))
        elif op == "append":
            s["cache"].append(s["rotary"], s["positions"], s["k_new"], s["v_new"], s["slots"], q=s["q"], q_out=s["q_out"])
        elif op == "gather4":
            s["cache"].gather(s["plan"], s["k"], s["v"], s["indices"], s["table"])
        elif op == "store4":
            s["cache"].store(s["k_new"], s["v_new"], s["slots"])
        else:
            s["cache"].attend(s["q"], s["table"], s["lens"], s["layer"], s["out"], s["lse"])
    else:
        {"rotate": _plain_rotate, "append": _plain_append, "gather4": _plain_gather, "store4": _plain_store,
         "attend4": _plain_attend}[op](s)
    if op == "rotate":
        return s["out"]
    if op == "append":
        return dict(q=s["q_out"], k=s["k8"].view(F8), v=s["v8"].view(F8), k_scale=s["ks"], v_scale=s["vs"])
    if op == "attend4":
        return dict(out=s["out"], lse=s["lse"])
    return dict(k=s["k4"], v=s["v4"], k_param=s["kp"], v_param=s["vp"])


def _rotated(x, s, transpose=False):
    """fp32 rows [tokens][heads][d] turned by their positions; the angles in 64 bits."""
    case, n = s["case"], s["case"]["rotary"]
    angle = s["positions"].double()[:, None, None] * s["freq"]
    cos, sin = (torch.cos(angle) * s["amplitude"]).float(), (torch.sin(angle) * s["amplitude"]).float()
    if transpose:
        sin = -sin
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if case["interleaved"] else (x[..., :n // 2], x[..., n // 2:n])
    a, b = a.float(), b.float()
    u, v = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([u, v], -1).flatten(-2) if case["interleaved"] else torch.cat([u, v], -1)
    return torch.cat([y, x[..., n:].float()], -1)


def _plain_rotate(s):
    s["out"].copy_(_rotated(s["x"], s, s["case"].get("transpose", False)))


def _plain_append(s):
    s["q_out"].copy_(_rotated(s["q"], s))
    _store8(s, _rotated(s["k_new"], s).to(torch.bfloat16), s["v_new"])


def _store8(s, k_new, v_new):
    p, n_pages = s["case"]["page"], s["n_pages"]
    slot = s["slots"].long()
    # what the empty slots of the batch would write goes to a page behind the last
    page = torch.where(slot >= 0, slot // p, torch.full_like(slot, n_pages))
    off = torch.where(slot >= 0, slot % p, torch.zeros_like(slot))
    first = torch.full((n_pages + 1,), p, device=DEV).scatter_reduce(0, page, off, "amin")[:n_pages]
    for x, code, scale in ((k_new, s["k8"], s["ks"]), (v_new, s["v8"], s["vs"])):
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
        new[page, :, off] = (x / torch.cat([to, to[:1]])[page][..., None]).to(F8).view(torch.uint8)
        code.copy_(new[:n_pages])
        scale.copy_(to)


def _plain_gather(s):
    case = s["case"]
    p, w, b = case["page"], case["window"], case["budget"]
    layers, n, h = case["layers"], s["n_seq"], case["hkv"]
    j = torch.arange(b + w, device=DEV)
    m = s["kept"][:, None, None, None]                                   # [n][1][1][1]
    idx = s["indices"].view(n, layers, h, b)
    good = (j < m + w).expand(n, layers, h, b + w)
    src = torch.where(j < m, idx[..., j.clamp(max=b - 1)].long(), (s["lens"] - w)[:, None, None, None] + j - m)
    src = torch.where(good, src, torch.zeros_like(src)) + (torch.cumsum(s["lens"], 0) - s["lens"])[:, None, None, None]
    l = torch.arange(layers, device=DEV)[None, :, None, None]
    hh = torch.arange(h, device=DEV)[None, None, :, None]
    at = s["table"].permute(1, 0, 2)[:, :, j // p].long() * p + j % p    # [n][layers][rows]
    at = (at[:, :, None] // p * h + hh) * p + at[:, :, None] % p         # rows of the pool, [n][layers][h][rows]
    _write_rows(at[good], s["k"][l, hh, src][good], s["k4"], s["kp"])
    _write_rows(at[good], s["v"][l, hh, src][good], s["v4"], s["vp"])


def _write_rows(at, x, code, param):
    code.view(-1, D // 2)[at], param.view(-1, 2)[at] = _quantise4(x)


def _plain_store(s):
    p, h = s["case"]["page"], s["case"]["hkv"]
    slot = s["slots"].long()
    use = slot >= 0
    at = (slot[use][:, None] // p * h + torch.arange(h, device=DEV)) * p + slot[use][:, None] % p
    _write_rows(at, s["k_new"][use], s["k4"], s["kp"])
    _write_rows(at, s["v_new"][use], s["v4"], s["vp"])


def _plain_attend(s):
    case = s["case"]
    h, t, n = case["hkv"], case["q_tokens"], s["n_seq"]
    g = case["hq"] // h
    lens = s["lens"][s["layer"]].long()
    ids = s["table"][s["layer"]].long().clamp(min=0)

    def rows(code, param):   # [n][h][tokens][d]
        x, f = code[ids], param[ids].float()
        x = torch.stack([x & 15, x >> 4], -1).flatten(-2).float() * f[..., :1] + f[..., 1:]
        return x.permute(0, 2, 1, 3, 4).reshape(n, h, -1, D)

    q = s["q"].float().reshape(n, t, h, g, D).permute(0, 2, 1, 3, 4).reshape(n, h, t * g, D)
    pos = torch.arange(ids.shape[1] * case["page"], device=DEV)
    x = torch.matmul(q, rows(s["k4"], s["kp"]).transpose(-1, -2)) * (1.0 / math.sqrt(D))
    seen = (lens[:, None] - t + 1 + torch.arange(t, device=DEV)).repeat_interleave(g, 1)[:, None, :, None]
    x = x.masked_fill(~(pos < seen), -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    v = rows(s["v4"], s["vp"]).masked_fill((pos >= lens[:, None])[:, None, :, None], 0.0)
    o = torch.matmul(e, v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = torch.log(total) + top
    s["out"].copy_(o.view(n, h, t, g, D).permute(0, 2, 1, 3, 4).reshape(n, t, h * g, D))
    s["lse"].copy_(lse.view(n, h, t, g).permute(0, 2, 1, 3).reshape(n, t, h * g))


# ------------------------------------------------------------------------------------------------ exact

_E4M3 = np.array([(-1.0 if c & 128 else 1.0) * ((c & 7) / 8 * 2.0 ** -6 if (c >> 3) & 15 == 0
                                              else (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7))
                  if c & 127 != 127 else math.nan for c in range(256)])
_POWERS = np.array([2.0 ** e for e in range(-6, 10)])


def _values(code):
    return torch.from_numpy(_E4M3).to(DEV)[code.long()]


def _round8(x):
    """x (64 bits, |x| <= 448) to the nearest e4m3 value, ties to the even one."""
    powers = torch.from_numpy(_POWERS).to(DEV)
    binade = (torch.searchsorted(powers, x.abs().contiguous(), right=True) - 1).clamp(min=0)
    ulp = powers[binade] / 8
    return torch.round(x / ulp) * ulp


def _exact_scales(amax):
    out = []
    for a in amax.view(-1).cpu().tolist():
        e = -126
        while a > 448.0 * 2.0 ** e:
            e += 1
        out.append(2.0 ** e)
    return torch.tensor(out, dtype=torch.float64, device=DEV).view(amax.shape)


def exact(case, seed):
    if work(case)["bytes"] > 1.5e9:
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"rotate": _exact_rotate, "append": _exact_append, "gather4": _exact_gather, "store4": _exact_store,
            "attend4": _exact_attend}[case["op"]](s)


def _exact_frequencies(case):
    """The same from the definitions, one pair at a time, as numbers of Python."""
    n, theta, factor, out = case["rotary"], case["base"], case["factor"], []
    for j in range(n // 2):
        f = (theta * factor ** (n / (n - 2)) if case["scaling"] == "ntk" else theta) ** (-2 * j / n)
        if case["scaling"] == "linear":
            f /= factor
        elif case["scaling"] in ("parts", "yarn"):
            if case["scaling"] == "parts":
                turns = case["original"] * f / (2 * math.pi)
                slow = 1.0 - min(max((turns - 1) / 3, 0.0), 1.0)
            else:
                ends = [n * math.log(case["original"] / (2 * math.pi * r), theta) / 2 for r in (32, 1)]
                ends = max(math.floor(ends[0]), 0), min(math.ceil(ends[1]), n - 1)
                slow = min(max((j - ends[0]) / max(ends[1] - ends[0], 0.001), 0.0), 1.0)
            f = slow * f / factor + (1 - slow) * f
        out.append(f)
    return out, 1 + 0.1 * math.log(factor) if case["scaling"] == "yarn" else 1.0


def _exact_turn(x, s, back=False):
    """Pairs as complex numbers times amplitude * exp(+-i * angle)."""
    case, n = s["case"], s["case"]["rotary"]
    f, amplitude = _exact_frequencies(case)
    angle = torch.outer(s["positions"].double(), torch.tensor(f, dtype=torch.float64, device=DEV))
    turn = torch.polar(torch.full_like(angle, amplitude), -angle if back else angle)[:, None]
    y = x.double()
    head = y[..., :n].unflatten(-1, (n // 2, 2) if case["interleaved"] else (2, n // 2))
    if not case["interleaved"]:
        head = head.transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
    y[..., :n] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
    return y


def _exact_rotate(s):
    n = s["x"].shape[0]
    step = max(1, (1 << 23) // (s["x"].shape[1] * D))
    part = lambda a: dict(s, positions=s["positions"][a:a + step])  # noqa: E731
    return torch.cat([_exact_turn(s["x"][a:a + step], part(a), s["case"].get("transpose", False)) for a in range(0, n, step)])


def _exact_append(s):
    p = s["case"]["page"]
    slots = s["slots"].cpu().tolist()
    q = _exact_rotate(dict(s, x=s["q"]))
    keys = _exact_rotate(dict(s, x=s["k_new"])).to(torch.bfloat16)   # a key is rounded before it is coded
    out = dict(q=q)
    for name, src, code, scale in (("k", keys, s["k8"], s["ks"]), ("v", s["v_new"], s["v8"], s["vs"])):
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


def _exact_param(rows):
    lo, hi = rows.double().amin(-1), rows.double().amax(-1)
    return torch.stack([(hi - lo) / 15, lo], -1)


def _exact_gather(s):
    case = s["case"]
    p, w, layers, h = case["page"], case["window"], case["layers"], case["hkv"]
    lens = _ints(case["lens"])
    idx = s["indices"].view(len(lens), layers, h, -1).long()
    out = dict(k=None, v=None)
    for name, src, param in (("k_param", s["k"], s["kp"]), ("v_param", s["v"], s["vp"])):
        f, at = param.double(), 0
        for r, x in enumerate(lens):
            m = min(case["budget"], x - w)
            rows = torch.cat([idx[r, :, :, :m], torch.arange(x - w, x, device=DEV).expand(layers, h, w)], -1) + at
            full = _exact_param(src.gather(2, rows[..., None].expand(-1, -1, -1, D)))   # [layers][h][rows][2]
            for j in range(_up(m + w, p)):
                part = full[:, :, j * p:(j + 1) * p]
                f[s["table"][:, r, j].long(), :, :part.shape[2]] = part
            at += x
        out[name] = f
    return out


def _exact_store(s):
    p = s["case"]["page"]
    out = dict(k=None, v=None)
    slots = [(t, x // p, x % p) for t, x in enumerate(s["slots"].cpu().tolist()) if x >= 0]
    t, page, off = (torch.tensor(x, device=DEV) for x in zip(*slots))
    for name, src, param in (("k_param", s["k_new"], s["kp"]), ("v_param", s["v_new"], s["vp"])):
        f = param.double()
        f[page, :, off] = _exact_param(src[t])
        out[name] = f
    return out


def _exact_attend(s):
    case = s["case"]
    p, h, t = case["page"], case["hkv"], case["q_tokens"]
    g = case["hq"] // h
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)

    def rows(code, param, ids, x):
        c = torch.empty((*code[ids].shape[:3], D), dtype=torch.float64, device=DEV)
        c[..., 0::2], c[..., 1::2] = code[ids] % 16, code[ids] // 16
        f = param[ids].double()
        return (f[..., :1] * c + f[..., 1:]).transpose(1, 2).reshape(-1, h, D)[:x]

    for r, x in enumerate(_ints(case["lens"])):
        ids = s["table"][s["layer"], r, :_up(x, p)].long()
        k, v = rows(s["k4"], s["kp"], ids, x), rows(s["v4"], s["vp"], ids, x)
        for i in range(t):
            seen = x - t + i + 1
            if seen > 0:
                a = torch.einsum("hgd,nhd->hgn", s["q"][r, i].double().reshape(h, g, D), k[:seen]) / math.sqrt(D)
                lse[r, i] = torch.logsumexp(a, -1).reshape(-1)
                out[r, i] = torch.einsum("hgn,nhd->hgd", torch.softmax(a, -1), v[:seen]).reshape(-1, D)
    return dict(out=out, lse=lse)


# ------------------------------------------------------------------------------------------------ work

def work(case):
    """Bytes: each input read once, each output written once. Flops: the two products of the attention, and a rotation's
    products and sums."""
    op = case["op"]
    if op == "rotate":
        rows = case["tokens"] * case["heads"]
        return {"bytes": rows * D * 4 + case["tokens"] * 4, "flops": rows * case["rotary"] * 3}
    lens, p, layers, h = _ints(case["lens"]), case["page"], case["layers"], case["hkv"]
    n, row4 = len(lens), D // 2 + 4
    if op == "gather4":
        rows = sum(min(case["budget"], x - case["window"]) + case["window"] for x in lens)
        pages = sum(_up(min(case["budget"], x - case["window"]) + case["window"], p) for x in lens)
        return {"bytes": layers * h * (rows * 2 * (D * 2 + row4) + rows * 4) + layers * pages * 4, "flops": 0}
    if op in ("append", "store4"):
        toks = sum(_ints(case["tokens"])) if case["new"] == 0 else n * case["new"]
        if op == "store4":
            return {"bytes": toks * (h * 2 * (D * 2 + row4) + 4), "flops": 0}
        pages = max(n, toks // p)
        return {"bytes": toks * (h * D * 6 + case["hq"] * D * 4 + 8) + pages * h * 16,
                "flops": toks * (case["hq"] + h) * case["rotary"] * 3}
    t, tok = case["q_tokens"], sum(lens)
    pages = sum(_up(x, p) for x in lens)
    return {"bytes": tok * h * 2 * row4 + pages * 4 + n * t * case["hq"] * (D * 4 + 4),
            "flops": 4 * D * tok * case["hq"] * t}
