"""Measured cases of the operators around appending and block caches: appending new rows to a cache with the rotation on the way,
the same into a cache held in 8 bits with a scale for each block of tokens and head, attention of single tokens over such a cache,
and the same over blocks that a cheap score selects for each query.

Each case runs either in a plain form (elementary torch operations in 32 bits) or, with `own` set, through the public
binding of the library.  `exact` states the definitions once more in 64 bits.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_BYTES = {"f32": 4, "bf16": 2, "e4m3": 1, "e5m2": 1}
_TOP = {"e4m3": 448.0, "e5m2": 57344.0}
_TINY = 2.0 ** -100     # a block with nothing as large as this is stored as zeros


# ------------------------------------------------------------------------------------------------------------ cases

def _append(name, **kw):
    c = dict(op="append", layers=1, batch=1, hq=32, hkv=8, d=128, dtype="bf16", page=16, cached_lo=0, cached_hi=0, new_lo=1, new_hi=1,
             spare=64, rot_dim=128, style="halves", axes=1)
    c.update(kw)
    return dict(c, name=name) if name else c


def _fill(name, **kw):
    c = dict(op="fill", layers=1, batch=1, hq=32, hkv=8, d=128, block=32, paged=True, cached_lo=0, cached_hi=0, new_lo=1, new_hi=1,
             spare=64, rot_dim=128, style="halves", axes=1)
    c.update(kw)
    return dict(c, name=name) if name else c


def _attend(name, **kw):
    c = dict(op="attend", layers=1, batch=1, hq=32, hkv=8, d=128, block=32, paged=True, cached_lo=1, cached_hi=1, spare=64, select=0, sink=0,
             recent=0, scale=1.0)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the new token of a decode step, all layers of the Llama-8B shape, retained lengths after pruning
        _append("append_token_llama8b", layers=32, batch=8, cached_lo=900, cached_hi=1300),
        # a whole prompt into an empty contiguous cache, one layer
        _append("append_prompt_8192", page=0, new_lo=8192, new_hi=8192),
        # a serving batch that mixes single tokens with chunks of prompts, quantised paged cache, part of the row rotated in
        # neighbouring pairs, positions in time, height and width
        _append("append_mixed_e4m3", layers=2, batch=16, hq=28, hkv=4, dtype="e4m3", cached_lo=100, cached_hi=4000, new_lo=1, new_hi=513,
                rot_dim=64, style="pairs", axes=3),
        # the same three over block caches: a decode step's token, a prompt, a ragged mixed batch
        _fill("block_append_token_llama8b", layers=32, batch=8, cached_lo=900, cached_hi=1300),
        _fill("block_append_prompt_8205", new_lo=8205, new_hi=8205),
        _fill("block_append_mixed_64", layers=2, batch=16, hq=28, hkv=4, block=64, paged=False, cached_lo=100, cached_hi=4000, new_lo=1, new_hi=701, axes=3),
        # a decode step of all layers of the Llama-8B shape over a block cache
        _attend("block_attend_llama8b", layers=32, batch=8, cached_lo=900, cached_hi=1300),
        # one layer of it, as a model's layer loop issues it: latency
        _attend("block_attend_one_layer", batch=8, cached_lo=900, cached_hi=1300),
        # one sequence with a very long context
        _attend("block_attend_131072", block=64, paged=False, cached_lo=131072, cached_hi=131072),
        # a ragged serving batch of long contexts, Qwen-7B shape, small blocks
        _attend("block_attend_ragged_qwen7b", layers=2, batch=16, hq=28, hkv=4, block=16, cached_lo=1024, cached_hi=32768),
        # long contexts of which each query reads a sixteenth
        _attend("block_select_32768", batch=8, cached_lo=32768, cached_hi=32768, select=64, sink=1, recent=2),
        # ragged odd lengths, narrow heads, four layers at once
        _attend("block_select_ragged_64", layers=4, batch=5, hq=14, hkv=2, d=64, block=16, cached_lo=999, cached_hi=20011, select=100, sink=1, recent=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "fill", "attend", "attend", "select"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.randint(1, 8)
    layers = rng.choice([1, 1, 2, 4, 16])
    if kind in ("append", "fill"):
        batch, new, cached = _log_int(rng, 1, 32), _log_int(rng, 1, 6000), _log_int(rng, 1, 4096) if rng.random() < 0.8 else 0
        while layers > 1 and layers * batch * hq * d * new > 8192 * 40 * 128:
            layers //= 2
        while batch > 1 and layers * batch * hq * d * new > 8192 * 40 * 128:
            batch //= 2
        kw = dict(layers=layers, batch=batch, hq=hq, hkv=hkv, d=d, cached_lo=cached if rng.random() < 0.3 else cached // rng.randint(2, 20),
                  cached_hi=cached, new_lo=new if rng.random() < 0.5 else max(1, new // rng.randint(2, 50)), new_hi=new, spare=rng.randint(0, 300),
                  rot_dim=rng.choice([d, d, 2 * rng.randint(4, d // 2)]), style=rng.choice(["halves", "pairs"]), axes=rng.randint(1, 4))
        if kind == "append":
            return _append(None, dtype=rng.choice(["bf16", "bf16", "f32", "e4m3", "e5m2"]), page=rng.choice([0, 16]), **kw)
        return _fill(None, block=rng.choice([16, 32, 64, 128]), paged=rng.random() < 0.6, **kw)
    batch, cached = _log_int(rng, 1, 48), _log_int(rng, 1 if kind == "attend" else 500, 131072)
    while layers > 1 and layers * batch * hkv * cached > 2.0e6:
        layers //= 2
    while batch > 1 and batch * hkv * cached > 2.0e6:
        batch //= 2
    c = _attend(None, layers=layers, batch=batch, hq=hq, hkv=hkv, d=d, block=rng.choice([16, 32, 64, 128]), paged=rng.random() < 0.6,
                cached_lo=cached if rng.random() < 0.4 else max(1, cached // rng.randint(2, 20)), cached_hi=cached, spare=rng.randint(0, 300),
                scale=rng.choice([1.0, 1.0, 2.0, 3.0]))
    if kind == "select":
        c["select"] = max(4, int(cached / c["block"] * rng.choice([0.03, 0.06, 0.12, 0.25])))
        c["sink"], c["recent"] = rng.randint(0, 2), rng.randint(0, 2)
    return c


# ---------------------------------------------------------------------------------------------- lengths and sizes

def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly spread in their logarithm."""
    if lo <= 0:
        return [int(round(lo + (hi - lo) * (i + 1) / n)) for i in range(n)]
    return [int(round(lo * (hi / lo) ** (i / max(1, n - 1)))) if n > 1 else hi for i in range(n)]


def _lengths(c, order=None):
    """(cached, new) tokens of every sequence; `order` permutes the cached lengths."""
    cached = _spread(c["cached_lo"], c["cached_hi"], c["batch"])
    new = _spread(c["new_lo"], c["new_hi"], c["batch"]) if "new_lo" in c else [0] * c["batch"]
    return ([cached[i] for i in order] if order is not None else cached), new


def work(case):
    c = case
    cached, new = _lengths(c)
    L, H, d, hq = c["layers"], c["hkv"], c["d"], c["hq"]
    tokens = sum(new)
    if c["op"] == "append":
        act, kv = (4 if c["dtype"] == "f32" else 2), _BYTES[c["dtype"]]
        rows = L * tokens * H
        return {"bytes": rows * (2 * d * (act + kv) + 8) + 2 * L * tokens * hq * d * act + 4 * c["axes"] * tokens,
                "flops": 3 * L * tokens * (H + hq) * d}
    if c["op"] == "fill":
        # new rows read; closed blocks (with the open rows that they take in) and the open rows written; the rows read back
        total = 0
        for n0, t in zip(cached, new):
            n1 = n0 + t
            closed = n1 // c["block"] - n0 // c["block"]
            taken = n0 % c["block"] if closed else 0
            left = n1 % c["block"] if closed else t
            total += 2 * d * (2 * t + 2 * taken + closed * c["block"] + 2 * left) + closed * (8 + 2 * d)     # the append
            back = t + taken
            total += 2 * d * (2 * back + (back - left if closed else 0) + 2 * left)                          # reading back
        return {"bytes": L * H * total + 4 * L * tokens * hq * d + 4 * c["axes"] * tokens, "flops": 3 * L * tokens * (H + hq) * d}
    T, total, seen = c["block"], 0, 0
    for n in cached:
        full, left = n // T, n % T
        if c["select"]:
            total += full * (2 * d + 4)
            full = min(full, c["select"])
            total += 4 * full
        total += full * (T * 2 * d + 8) + left * 4 * d
        seen += full * T + left
    rows = L * c["batch"] * hq
    return {"bytes": L * H * total + rows * (4 * d + 4), "flops": 4 * L * seen * hq * d}


# ------------------------------------------------------------------------------------------------------------- inputs

_context = []


def _ctx():
    """The library context of this process."""
    if not _context:
        from paper_2511_06029_b200 import binding
        _context.append(binding.Context(0))
    return _context[0]


def _codes(x):
    """Blocks [..., T, D] as codes of 8 bits and their scales."""
    top = x.abs().amax((-1, -2))
    some = top >= _TINY
    scale = torch.where(some, top / 127.0, 0.0)
    inv = torch.where(some, 127.0 / top, 0.0)
    return torch.round(x * inv[..., None, None]).clamp(-127, 127).to(torch.int8), scale


def prepare(case, seed):
    c, dev = case, torch.device("cuda", 0)
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 11 + 5)
    L, B, H, d, hq = c["layers"], c["batch"], c["hkv"], c["d"], c["hq"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    order = np.random.RandomState(int(seed) % (1 << 31)).permutation(B)
    cached, new = _lengths(c, order)
    slots = max(_lengths(c)[0]) + max(new) + c["spare"]
    s = {"c": c, "cached": cached, "new": new}
    ln = torch.tensor(cached, dtype=torch.int32, device=dev).view(1, B, 1).expand(L, B, H).contiguous()
    s["len"], s["len0"] = ln.clone(), ln
    if c["op"] != "attend":
        act = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
        N = sum(new)
        s["q"], s["k_new"], s["v_new"] = normal(L, N, hq, d).to(act), normal(L, N, H, d).to(act), normal(L, N, H, d).to(act)
        s["q_out"] = torch.empty_like(s["q"])
        s["chunk_start"] = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=dev)
        s["max_chunk"] = max(new)
        t = torch.tensor(np.concatenate([cached[b] + np.arange(new[b]) for b in range(B)]), dtype=torch.int32, device=dev)
        s["token_pos"] = t
        # text runs on in every axis; images step through height and width
        s["axis_pos"] = torch.stack([t, t // 16, t % 16, torch.randint(0, 50, (N,), generator=g, device=dev)][:c["axes"]]).to(torch.int32).contiguous()
        half = c["rot_dim"] // 2
        s["pair_axis"] = [p * c["axes"] // half for p in range(half)]
        s["pair_freq"] = [10000.0 ** (-p / half) for p in range(half)]
        s["pair_axis_dev"] = torch.tensor(s["pair_axis"], device=dev)
        s["pair_freq_dev"] = torch.tensor(s["pair_freq"], device=dev, dtype=torch.float64)
        if own:
            from paper_2511_06029_b200 import binding
            s["rotary"] = binding.Rotary(s["pair_axis"], s["pair_freq"], s["axis_pos"],
                                         style=binding.ROT_HALVES if c["style"] == "halves" else binding.ROT_PAIRS)
    if c["op"] == "append":
        kv, page = _DT[c["dtype"]], c["page"]
        if page:
            slots = -(-slots // page) * page
        s["slots"] = slots
        s["k_scale"] = [0.02 + 0.005 * i for i in range(L)] if c["dtype"] in _TOP else None
        s["v_scale"] = [0.015 + 0.005 * i for i in range(L)] if c["dtype"] in _TOP else None
        k, v = normal(L * B * H * slots, d).to(kv), normal(L * B * H * slots, d).to(kv)
        s["page_table"] = None
        if page:
            n_pages = L * B * H * slots // page
            s["page_table"] = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32).view(L, B, H, -1).contiguous()
            s["k"], s["v"] = k.view(n_pages, page, d), v.view(n_pages, page, d)
        else:
            s["k"], s["v"] = k.view(L, B, H, slots, d), v.view(L, B, H, slots, d)
        s["rel"] = torch.rand((L, B, H, slots), generator=g, device=dev)
        s["pos"] = torch.arange(slots, device=dev, dtype=torch.int32).expand(L, B, H, slots).contiguous()
        if own:
            s["ctx"] = _ctx()
            s["cache"] = binding.Cache(hq, s["k"], s["v"], s["rel"], s["pos"], s["len"], s["page_table"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return s

    T = c["block"]
    blocks = max(1, -(-slots // T))
    s["blocks"] = blocks
    n_pages = L * B * H * blocks
    k, v = torch.empty((n_pages, T, d), dtype=torch.int8, device=dev), torch.empty((n_pages, T, d), dtype=torch.int8, device=dev)
    ks, vs = torch.empty(n_pages, device=dev), torch.empty(n_pages, device=dev)
    kr = torch.empty((n_pages, 2, d), dtype=torch.int8, device=dev)
    for p in range(0, n_pages, 65536):      # in pieces: the 32-bit values of a large pool are not held all at once
        m = min(65536, n_pages - p)
        x = normal(m, T, d)
        # the keys of a block have something in common, one key in a hundred is three times as long (anchors)
        x = (0.8 * x + 0.6 * normal(m, 1, d)) * torch.where(torch.rand((m, T, 1), generator=g, device=dev) < 0.01, 3.0, 1.0)
        k[p:p + m], ks[p:p + m] = _codes(x)
        kr[p:p + m, 0], kr[p:p + m, 1] = k[p:p + m].amin(1), k[p:p + m].amax(1)
        v[p:p + m], vs[p:p + m] = _codes(normal(m, T, d) * torch.exp(0.5 * normal(m, 1, 1)))
    lead = (L, B, H, blocks)
    s["page_table"] = None
    if c["paged"]:
        s["page_table"] = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32).view(lead).contiguous()
    else:
        k, v, ks, vs, kr = k.view(*lead, T, d), v.view(*lead, T, d), ks.view(lead), vs.view(lead), kr.view(*lead, 2, d)
    s["k"], s["v"], s["k_scale"], s["v_scale"], s["k_range"] = k, v, ks, vs, kr
    s["k_open"], s["v_open"] = normal(L, B, H, T, d).to(torch.bfloat16), normal(L, B, H, T, d).to(torch.bfloat16)
    if c["op"] == "fill":
        # what is read back: the new rows and the open ones that went into a block with them
        T0 = [n % T for n in cached]
        s["slot_begin"] = torch.tensor([n - o for n, o in zip(cached, T0)], dtype=torch.int32, device=dev)
        s["n_read"] = max(new) + T - 1
        s["k_read"] = torch.empty((L, B, H, s["n_read"], d), dtype=torch.bfloat16, device=dev)
        s["v_read"] = torch.empty_like(s["k_read"])
    else:
        s["q"] = normal(L, B, hq, d).to(torch.bfloat16)
        s["scale"] = [c["scale"] / math.sqrt(d) / (1 + 0.25 * (i % 4)) for i in range(L)]
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((L, B, hq), dtype=torch.float32, device=dev)
        s["selected"] = torch.empty((L, B, H, c["select"]), dtype=torch.int32, device=dev) if c["select"] else None
    if own:
        from paper_2511_06029_b200 import binding
        s["ctx"] = _ctx()
        s["cache"] = binding.BlockCache(hq, k, v, ks, vs, kr, s["k_open"], s["v_open"], s["len"], s["page_table"])
    return s


# --------------------------------------------------------------------------------------------------------- one pass

def run(state):
    s = state
    c = s["c"]
    L = c["layers"]
    if c["op"] == "append":
        s["len"].copy_(s["len0"])
        if own:
            s["ctx"].append(s["cache"], 0, L, s["chunk_start"], s["max_chunk"], s["k_new"], s["v_new"], s["token_pos"], rotary=s["rotary"], q=s["q"], q_out=s["q_out"])
        else:
            _plain_append(s)
        return {"q": s["q_out"], "k": s["k"], "v": s["v"], "rel": s["rel"], "pos": s["pos"], "len": s["len"]}
    if c["op"] == "fill":
        s["len"].copy_(s["len0"])
        if own:
            s["ctx"].block_append(s["cache"], 0, L, s["chunk_start"], s["max_chunk"], s["k_new"], s["v_new"], rotary=s["rotary"], q=s["q"], q_out=s["q_out"])
            s["ctx"].block_read(s["cache"], 0, L, s["slot_begin"], s["k_read"], s["v_read"])
        else:
            _plain_fill(s)
            _plain_read(s)
        return {"q": s["q_out"], "k": s["k_read"], "v": s["v_read"], "k_open": s["k_open"], "v_open": s["v_open"], "len": s["len"]}
    if own:
        if c["select"]:
            s["ctx"].block_select(s["cache"], 0, L, s["q"], c["sink"], c["recent"], s["selected"])
        s["ctx"].block_attend(s["cache"], 0, L, s["q"], s["scale"], s["out"], lse=s["lse"], selected=s["selected"])
        return {"out": s["out"], "lse": s["lse"], "selected": s["selected"]}
    sel = _plain_select(s) if c["select"] else None
    out, lse = _plain_attend(s, sel)
    return {"out": out, "lse": lse, "selected": sel}


def _rotated(s, x):
    c = s["c"]
    half = c["rot_dim"] // 2
    angle = s["axis_pos"][s["pair_axis_dev"]].double().t() * s["pair_freq_dev"]            # [tokens][pairs], in 64 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    y = x.float()
    z = y.clone()
    a, b = (y[..., :half], y[..., half:2 * half]) if c["style"] == "halves" else (y[..., 0:2 * half:2], y[..., 1:2 * half:2])
    u, w = a * cos - b * sin, a * sin + b * cos
    if c["style"] == "halves":
        z[..., :half], z[..., half:2 * half] = u, w
    else:
        z[..., 0:2 * half:2], z[..., 1:2 * half:2] = u, w
    return z.to(x.dtype)


def _of_tokens(s):
    """The sequence of each packed token, and its place among the sequence's new ones."""
    start, dev = s["chunk_start"].long(), s["k_new"].device
    n = torch.arange(s["k_new"].shape[1], device=dev)
    seq = torch.searchsorted(start, n, right=True) - 1
    return seq, n - start[seq]


def _plain_append(s):
    c = s["c"]
    L, B, H, d, dev = c["layers"], c["batch"], c["hkv"], c["d"], s["k_new"].device
    s["q_out"].copy_(_rotated(s, s["q"]))
    kn, vn = _rotated(s, s["k_new"]), s["v_new"]
    seq, at = _of_tokens(s)
    slot = s["len"].long()[:, seq, :] + at[None, :, None]                                  # [L][N][H]
    item = (torch.arange(L, device=dev)[:, None, None] * B + seq[None, :, None]) * H + torch.arange(H, device=dev)
    row = item * s["slots"] + slot
    where = row
    if s["page_table"] is not None:
        page = c["page"]
        where = s["page_table"].view(-1, s["slots"] // page)[item, slot // page].long() * page + slot % page
    kf, vf = s["k"].view(-1, d), s["v"].view(-1, d)
    if s["k_scale"] is not None:
        top = _TOP[c["dtype"]]
        kn = (kn.float() / torch.tensor(s["k_scale"], device=dev).view(L, 1, 1, 1)).clamp(-top, top).to(kf.dtype)
        vn = (vn.float() / torch.tensor(s["v_scale"], device=dev).view(L, 1, 1, 1)).clamp(-top, top).to(vf.dtype)
    raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[kf.element_size()]
    kf.view(raw)[where] = kn.view(raw)
    vf.view(raw)[where] = vn.view(raw)
    s["pos"].view(-1)[row] = s["token_pos"][None, :, None].expand_as(row).contiguous()
    s["rel"].view(-1)[row] = torch.zeros(1, device=dev)
    s["len"] += (s["chunk_start"][1:] - s["chunk_start"][:-1]).view(1, B, 1)


def _plain_fill(s):
    c = s["c"]
    L, B, H, d, T, dev = c["layers"], c["batch"], c["hkv"], c["d"], c["block"], s["k_new"].device
    s["q_out"].copy_(_rotated(s, s["q"]))
    start = s["chunk_start"].long()
    n0 = s["len"][0, :, 0].long()                                                          # every layer and head has the same
    n1 = n0 + start[1:] - start[:-1]
    closed = n1 // T - n0 // T
    count = sum((a + t) // T - a // T for a, t in zip(s["cached"], s["new"]))
    k, v = s["k"].view(-1, T, d), s["v"].view(-1, T, d)
    layer, head = torch.arange(L, device=dev)[:, None, None], torch.arange(H, device=dev)
    new = (("k", _rotated(s, s["k_new"])), ("v", s["v_new"]))
    if count:
        seq = torch.repeat_interleave(torch.arange(B, device=dev), closed, output_size=count)
        blk = n0[seq] // T + torch.arange(count, device=dev) - (torch.cumsum(closed, 0) - closed)[seq]
        slot = blk[:, None] * T + torch.arange(T, device=dev)                              # [blocks][T]
        tok = (start[seq, None] + slot - n0[seq, None]).clamp(min=0)
        held = (slot < n0[seq, None])[None, :, :, None, None]
        item = (layer * B + seq[None, :, None]) * H + head                                 # [L][blocks][H]
        page = item * s["blocks"] + blk[None, :, None]
        if s["page_table"] is not None:
            page = s["page_table"].view(-1)[page].long()
        for name, x in new:
            rows = torch.where(held, s[name + "_open"][:, seq].permute(0, 1, 3, 2, 4).float(), x[:, tok].float())
            codes, scale = _codes(rows.permute(0, 1, 3, 2, 4))
            s[name].view(-1, T, d)[page], s[name + "_scale"].view(-1)[page] = codes, scale
            if name == "k":
                s["k_range"].view(-1, 2, d)[page] = torch.stack([codes.amin(-2), codes.amax(-2)], -2)
    # what is left goes to the open blocks
    left = sum((a + t) % T if (a + t) // T > a // T else t for a, t in zip(s["cached"], s["new"]))
    if left:
        keep = torch.where(closed > 0, n1 % T, n1 - n0)
        seq = torch.repeat_interleave(torch.arange(B, device=dev), keep, output_size=left)
        slot = n1[seq] - keep[seq] + torch.arange(left, device=dev) - (torch.cumsum(keep, 0) - keep)[seq]
        for name, x in new:
            s[name + "_open"][:, seq, :, slot % T] = x[:, start[seq] + slot - n0[seq]].permute(1, 0, 2, 3)
    s["len"] += (start[1:] - start[:-1]).to(torch.int32).view(1, B, 1)


def _plain_read(s):
    c = s["c"]
    L, B, H, d, T, dev = c["layers"], c["batch"], c["hkv"], c["d"], c["block"], s["k"].device
    slot = (s["slot_begin"].long()[:, None] + torch.arange(s["n_read"], device=dev))[None, :, None].expand(L, B, H, -1)
    n = s["len"].long()[..., None]
    blk = (slot // T).clamp(max=s["blocks"] - 1)
    page = torch.arange(L * B * H, device=dev).view(L, B, H, 1) * s["blocks"] + blk
    if s["page_table"] is not None:
        page = s["page_table"].view(-1)[page].long()
    full, real = (slot < n // T * T)[..., None], (slot < n)[..., None]
    for name in ("k", "v"):
        stored = s[name].view(-1, T, d)[page, slot % T].float() * s[name + "_scale"].view(-1)[page][..., None]
        still = torch.gather(s[name + "_open"], 3, (slot % T)[..., None].expand(*slot.shape, d)).float()
        s[name + "_read"].copy_(torch.where(real, torch.where(full, stored, still), 0.0))


def _pages(s):
    """The page of every block of every item."""
    c = s["c"]
    if s["page_table"] is not None:
        return s["page_table"].long()
    return torch.arange(s["k_scale"].numel(), device=s["k"].device).view(c["layers"], c["batch"], c["hkv"], s["blocks"])


def _plain_select(s):
    c = s["c"]
    L, B, H, d, T, G, dev = c["layers"], c["batch"], c["hkv"], c["d"], c["block"], c["hq"] // c["hkv"], s["q"].device
    q = s["q"].float().view(L, B, H, G, d)
    top = q.abs().amax((-1, -2), keepdim=True)
    code = torch.round(q * torch.where(top >= _TINY, 127.0 / top, 0.0)).clamp(-127, 127)
    up, down = code.clamp(min=0).sum(-2), code.clamp(max=0).sum(-2)                         # whole numbers
    page = _pages(s)
    r = s["k_range"].view(-1, 2, d)[page].float()                                          # [L][B][H][blocks][2][d]
    # whole numbers below 2^24: exact in 32 bits in any order
    bound = torch.matmul(r[..., 1, :], up[..., None])[..., 0] + torch.matmul(r[..., 0, :], down[..., None])[..., 0]
    score = s["k_scale"].view(-1)[page] * bound + 0.0
    full = (s["len"].long() // T)[..., None]
    blk = torch.arange(s["blocks"], device=dev)
    score = torch.where((blk < c["sink"]) | (blk >= full - c["recent"]), math.inf, score)
    score = torch.where(blk < full, score, -math.inf)
    n = min(c["select"], s["blocks"])
    pick = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :n]
    pick = torch.where(pick < full, pick, s["blocks"]).sort(-1)[0]
    pick = torch.where(pick < full, pick, -1)
    return torch.nn.functional.pad(pick, (0, c["select"] - n), value=-1).to(torch.int32)


def _plain_attend(s, sel):
    c = s["c"]
    L, B, H, d, T, G, dev = c["layers"], c["batch"], c["hkv"], c["d"], c["block"], c["hq"] // c["hkv"], s["q"].device
    n = s["len"].long()
    page = _pages(s)
    if sel is not None:
        live = sel >= 0
        page = torch.gather(page, 3, sel.long().clamp(min=0))
    else:
        live = torch.arange(s["blocks"], device=dev) < (n // T)[..., None]
    M = page.shape[3] * T

    def rows(name):
        full = s[name].view(-1, T, d)[page].float() * s[name + "_scale"].view(-1)[page][..., None, None]
        return torch.cat([torch.where(live[..., None, None], full, 0.0).view(L, B, H, M, d), s[name + "_open"].float()], 3)

    see = torch.cat([live[..., None].expand(L, B, H, -1, T).reshape(L, B, H, M), torch.arange(T, device=dev) < (n % T)[..., None]], 3)
    q = s["q"].float().view(L, B, H, G, d)
    x = torch.matmul(q, rows("k").transpose(-1, -2)) * torch.tensor(s["scale"], device=dev).view(L, 1, 1, 1, 1)
    x = torch.where(see[..., None, :], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    V = torch.where(see[..., None], rows("v"), 0.0)
    out = torch.matmul(p / torch.where(total > 0, total, 1.0), V)
    return out.view(L, B, H * G, d).to(s["q"].dtype), (top + torch.log(total)).view(L, B, H * G)


# --------------------------------------------------------------------------------------------- definitions in 64 bits

def _turned(s, x):
    """Rows in 64 bits, rotated."""
    c = s["c"]
    half = c["rot_dim"] // 2
    z = x.double().clone()
    for p in range(half):
        i0, i1 = (p, p + half) if c["style"] == "halves" else (2 * p, 2 * p + 1)
        turn = s["axis_pos"][s["pair_axis"][p]].double() * s["pair_freq"][p]
        a, b, cs, sn = z[..., i0].clone(), z[..., i1].clone(), torch.cos(turn)[None, :, None], torch.sin(turn)[None, :, None]
        z[..., i0], z[..., i1] = a * cs - b * sn, b * cs + a * sn
    return z


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    dev = s["k"].device
    L, B, H, d, G = c["layers"], c["batch"], c["hkv"], c["d"], c["hq"] // c["hkv"]
    if c["op"] in ("append", "fill"):
        first = s["chunk_start"].tolist()
        k_new, v_new = _turned(s, s["k_new"]), s["v_new"].double()
        res = {"q": _turned(s, s["q"])}
    if c["op"] == "append":
        page, unit = c["page"], {1: torch.uint8, 2: torch.int16, 4: torch.int32}[s["k"].element_size()]
        # values of a byte cache stand for scale * value; they come back as they are stored, without the scale
        for name, x in (("k", k_new), ("v", v_new)):
            y = s[name].double()
            for l in range(L):
                z = x[l] if s[name + "_scale"] is None else (x[l] / float(np.float32(s[name + "_scale"][l]))).clamp(-_TOP[c["dtype"]], _TOP[c["dtype"]])
                for b in range(B):
                    t0, t1, n = first[b], first[b + 1], s["cached"][b]
                    for h in range(H):
                        if page:
                            at = torch.arange(n, n + t1 - t0, device=dev)
                            y[s["page_table"][l, b, h].long()[at // page], at % page] = z[t0:t1, h]
                        else:
                            y[l, b, h, n:n + t1 - t0] = z[t0:t1, h]
            res[name] = y
        rel = s["rel"].double()
        for b in range(B):
            rel[:, b, :, s["cached"][b]:s["cached"][b] + s["new"][b]] = 0
        return dict(res, rel=rel, pos=None, len=None)
    T = c["block"]
    if c["op"] == "fill":
        for name, x in (("k", k_new), ("v", v_new)):
            still = s[name + "_open"].double()
            back = torch.zeros(s[name + "_read"].shape, dtype=torch.float64, device=dev)
            for b in range(B):
                t0, t1, n = first[b], first[b + 1], s["cached"][b]
                o = n % T
                # the open rows and the new ones (rounded as they are held), cut into blocks from slot n - o on
                rows = torch.cat([still[:, b, :, :o], x[:, t0:t1].to(torch.bfloat16).double().transpose(1, 2)], 2)       # [L][H][o + new][d]
                m = rows.shape[2] // T
                if m:
                    cut = rows[:, :, :m * T].reshape(L, H, m, T * d)
                    step = cut.abs().amax(-1, keepdim=True) / 127
                    back[:, b, :, :m * T] = (torch.round(cut / step) * step).view(L, H, m * T, d)
                back[:, b, :, m * T:rows.shape[2]] = rows[:, :, m * T:]
                r = rows.shape[2] - m * T
                still[:, b, :, :r] = rows[:, :, m * T:]
            res[name], res[name + "_open"] = back, still
        return dict(res, len=None)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=dev)
    page, pool = _pages(s), {x: s[x].view(-1, T, d) for x in ("k", "v")}
    for l in range(L):
        for b in range(B):
            n = s["cached"][b]
            m = n // T
            for h in range(H):
                q = s["q"][l, b, h * G:(h + 1) * G]
                pg = page[l, b, h, :m]
                if c["select"] and m > c["select"]:
                    big = float(q.float().abs().max())
                    qi = torch.round(q.float() * float(np.float32(127.0) / np.float32(big))).clamp(-127, 127).long()
                    lo, hi = s["k_range"].view(-1, 2, d)[pg].long().unbind(1)
                    most = sum(torch.maximum(qi[g] * lo, qi[g] * hi).sum(1) for g in range(G))
                    score = (s["k_scale"].view(-1)[pg] * most.float()).cpu().numpy() + np.float32(0)
                    must = np.zeros(m, bool)
                    must[:c["sink"]] = True
                    must[m - c["recent"]:] = True
                    best = np.lexsort((np.arange(m), -score, ~must))[:c["select"]]
                    pg = pg[torch.from_numpy(np.sort(best)).to(dev)]
                K, V = (torch.cat([(pool[x][pg].double() * s[x + "_scale"].view(-1)[pg].double()[:, None, None]).reshape(-1, d),
                                   s[x + "_open"][l, b, h, :n - m * T].double()]) for x in ("k", "v"))
                e = q.double() @ K.T * float(np.float32(s["scale"][l]))
                z = torch.logsumexp(e, 1)
                out[l, b, h * G:(h + 1) * G] = torch.exp(e - z[:, None]) @ V
                lse[l, b, h * G:(h + 1) * G] = z
    return {"out": out, "lse": lse, "selected": None}
