"""Measured cases of the operators that work on a chunk of new tokens: attention of the chunk over the (pruned, paged)
cache with the relevance update, the same with modified scores, and rotary positions with several axes.

Each case runs either in a plain form (elementary torch operations in 32 bits) or, with `own` set, through the public
binding of the library.  `exact` states the definitions once more in 64 bits.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_BYTES = {"f32": 4, "bf16": 2, "e4m3": 1, "e5m2": 1}
_GAMMA = 0.99
_STRETCH = 1.5          # original positions of a pruned cache: about every third token has been evicted


# ------------------------------------------------------------------------------------------------------------ cases

def _attend(name, **kw):
    c = dict(op="attend", layers=1, batch=1, hq=32, hkv=8, d=128, dtype="bf16", page=16, cached_lo=0, cached_hi=0,
             new_lo=1, new_hi=1, spare=64, scale=1.0, softcap=0.0, slopes=False, window=0, doc=0, prefix=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _rotate(name, **kw):
    c = dict(op="rotate", layers=1, tokens=1, hq=32, hkv=8, d=128, rot_dim=128, dtype="bf16", axes=3, style="halves",
             inverse=False, far=0, grid=16)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # verification of four drafted tokens per sequence on the Llama-8B shape after pruning to about 1100 tokens
        _attend("verify_4_llama8b", batch=8, cached_lo=900, cached_hi=1300, new_lo=4, new_hi=4),
        # one chunk of a chunked prompt behind 1024 retained tokens, Llama-8B shape, contiguous cache
        _attend("chunk_512_llama8b", batch=8, page=0, cached_lo=1024, cached_hi=1024, new_lo=512, new_hi=512),
        # a whole long prompt into an empty cache
        _attend("prompt_8192_llama8b", batch=1, page=0, new_lo=8192, new_hi=8192),
        # a serving batch that mixes decode steps with chunks of prompts, Qwen-7B shape, ragged paged cache
        _attend("mixed_ragged_qwen7b", batch=16, hq=28, hkv=4, cached_lo=1024, cached_hi=8192, new_lo=1, new_hi=256),
        # the fp32 shape of the small configuration, an odd chunk
        _attend("tiny_f32_33", batch=1, hq=8, hkv=2, d=64, dtype="f32", page=0, cached_lo=512, cached_hi=512,
                new_lo=33, new_hi=33),
        # chunks over a quantised cache
        _attend("chunk_e4m3_llama8b", batch=4, dtype="e4m3", page=0, cached_lo=1500, cached_hi=2500, new_lo=200, new_hi=300),
        # single tokens of a model with capped scores and a sliding window
        _attend("token_softcap_window", batch=32, cached_lo=1500, cached_hi=2600, new_lo=1, new_hi=1, scale=3.0,
                softcap=30.0, window=1024),
        # a chunk with capped scores and a bias that falls with distance
        _attend("chunk_softcap_slopes", batch=4, hq=28, hkv=4, cached_lo=900, cached_hi=1100, new_lo=450, new_hi=512,
                scale=3.0, softcap=30.0, slopes=True),
        # packed documents of a prompt, each seeing itself only
        _attend("documents_4096", batch=2, page=0, cached_lo=0, cached_hi=200, new_lo=4000, new_hi=4096, doc=700),
        # a decode step's queries and keys, positions in time, height and width
        _rotate("rotate_step_8", tokens=8),
        # the queries and keys of a long prompt with images
        _rotate("rotate_prompt_8192", tokens=8192),
        # the way back (gradients), neighbouring pairs, part of the row, two axes, far positions
        _rotate("rotate_back_f32", tokens=1003, hq=8, hkv=2, d=64, rot_dim=48, dtype="f32", axes=2, style="pairs",
                inverse=True, far=1000000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.25:
        d = rng.choice([64, 128])
        hkv = rng.choice([1, 2, 4, 8])
        return _rotate(None, layers=rng.choice([1, 1, 2]), tokens=_log_int(rng, 1, 6000), hq=hkv * rng.randint(1, 8), hkv=hkv, d=d,
                       rot_dim=rng.choice([d, d, 2 * rng.randint(4, d // 2)]), dtype=rng.choice(["bf16", "f32"]),
                       axes=rng.randint(1, 4), style=rng.choice(["halves", "pairs"]), inverse=rng.random() < 0.4,
                       far=rng.choice([0, 0, _log_int(rng, 1000, 10000000)]), grid=rng.randint(4, 40))
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8])
    dtype = rng.choice(["bf16", "bf16", "bf16", "e4m3", "e5m2", "f32"])
    batch = _log_int(rng, 1, 32)
    new = _log_int(rng, 1, 4096 if dtype != "f32" else 512)
    cached = _log_int(rng, 1, 16384 if dtype != "f32" else 4096) if rng.random() < 0.85 else 0
    # no dearer than the longest listed prompt: products of rows and keys, and the padded form's size, are bounded
    while batch > 1 and batch * hq * new * (cached + new) > 1.0e9:
        batch //= 2
    while hq * new * (cached + new) > 1.0e9:
        new, cached = (new + 1) // 2, cached // 2
    new_lo = new if rng.random() < 0.5 else max(1, new // rng.randint(2, 50))
    cached_lo = cached if rng.random() < 0.4 else cached // rng.randint(2, 20)
    c = _attend(None, layers=rng.choice([1, 1, 1, 2]) if batch * hq * new * (cached + new) < 4e8 else 1, batch=batch, hq=hq,
                hkv=hkv, d=d, dtype=dtype, page=rng.choice([0, 16]), cached_lo=cached_lo, cached_hi=cached, new_lo=new_lo,
                new_hi=new, spare=rng.randint(0, 300))
    if rng.random() < 0.45:
        c["scale"] = rng.choice([1.0, 2.0, 3.0])
        if rng.random() < 0.6:
            c["softcap"] = rng.choice([15.0, 30.0, 50.0])
        if rng.random() < 0.4:
            c["slopes"] = True
        kind = rng.randint(0, 3)
        if kind == 1:
            c["window"] = _log_int(rng, 16, 4096)
        elif kind == 2:
            c["doc"] = _log_int(rng, 20, 2000)
        elif kind == 3:
            c["prefix"] = int((cached + new) * _STRETCH * rng.random()) + 1
    return c


# ---------------------------------------------------------------------------------------------- lengths and positions

def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly spread in their logarithm."""
    if lo <= 0:
        return [int(round(lo + (hi - lo) * (i + 1) / n)) for i in range(n)]
    return [int(round(lo * (hi / lo) ** (i / max(1, n - 1)))) if n > 1 else hi for i in range(n)]


def _lengths(c, order=None):
    """(cached, new) tokens of every sequence; `order` permutes the cached lengths."""
    cached, new = _spread(c["cached_lo"], c["cached_hi"], c["batch"]), _spread(c["new_lo"], c["new_hi"], c["batch"])
    return ([cached[i] for i in order] if order is not None else cached), new


def _modified(c):
    return bool(c["softcap"] or c["slopes"] or c["window"] or c["doc"] or c["prefix"])


def _visible(c, cached, new):
    """Pairs of (new token, slot) that the masks leave in one sequence, and the slots that some token sees."""
    if not (c["window"] or c["doc"] or c["prefix"]):
        return new * cached + new * (new + 1) // 2, cached + new
    slot = np.arange(cached + new)
    pos = np.where(slot < cached, np.floor(slot * _STRETCH), int(cached * _STRETCH) + slot - cached).astype(np.int64)
    pairs, seen = 0, np.zeros(cached + new, bool)
    for i in range(0, new, 256):
        rows = np.arange(i, min(new, i + 256))
        pq = (int(cached * _STRETCH) + rows)[:, None]
        m = slot[None] <= cached + rows[:, None]
        if c["prefix"]:
            m |= pos[None] < c["prefix"]
        if c["window"]:
            m &= pq - pos[None] < c["window"]
        if c["doc"]:
            m &= pos[None] >= pq // c["doc"] * c["doc"]
        pairs += int(m.sum())
        seen |= m.any(0)
    return pairs, int(seen.sum())


def work(case):
    c = case
    if c["op"] == "rotate":
        e = _BYTES[c["dtype"]]
        values = c["layers"] * c["tokens"] * (c["hq"] + c["hkv"]) * c["d"]
        return {"bytes": 2 * values * e + 4 * c["axes"] * c["tokens"], "flops": 3 * values}
    cached, new = _lengths(c)
    pairs, rows, slots = 0, 0, 0
    for a, b in zip(cached, new):
        p, s = _visible(c, a, b)
        pairs, rows, slots = pairs + p, rows + s, slots + a + b
    act, kv = (4 if c["dtype"] == "f32" else 2), _BYTES[c["dtype"]]
    tokens = sum(new)
    per_layer = (rows * 2 * c["hkv"] * c["d"] * kv                                  # keys and values that some token sees
                 + slots * c["hkv"] * 8                                             # the relevance, read and written
                 + tokens * 2 * c["hkv"] * c["d"] * (act + kv)                      # the new rows, read and appended
                 + tokens * c["hq"] * (2 * c["d"] * act + 4))                       # queries, outputs and log-sum-exps
    return {"bytes": c["layers"] * per_layer, "flops": 4 * c["layers"] * pairs * c["hq"] * c["d"]}


# ------------------------------------------------------------------------------------------------------------- inputs

_context = []


def _ctx():
    """The library context of this process."""
    if not _context:
        from paper_2511_06029_b200 import binding
        _context.append(binding.Context(0))
    return _context[0]


def prepare(case, seed):
    c, dev = case, torch.device("cuda", 0)
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7 + 3)
    L, d = c["layers"], c["d"]
    act = torch.float32 if c["dtype"] == "f32" else torch.bfloat16

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    if c["op"] == "rotate":
        n, half = c["tokens"], c["rot_dim"] // 2
        s = {"c": c, "q": normal(L, n, c["hq"], d).to(act), "k": normal(L, n, c["hkv"], d).to(act)}
        t = torch.arange(n, device=dev) + c["far"] + int(seed) % 5
        grid = c["grid"]      # text runs on in every axis; images step through height and width
        axes = [t, t // grid, t % grid, torch.randint(0, 50, (n,), generator=g, device=dev)][:c["axes"]]
        s["axis_pos"] = torch.stack(axes).to(torch.int32).contiguous()
        s["pair_axis"] = [p * c["axes"] // half for p in range(half)]
        s["pair_freq"] = [10000.0 ** (-p / half) for p in range(half)]
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        s["pair_axis_dev"] = torch.tensor(s["pair_axis"], device=dev)
        s["pair_freq_dev"] = torch.tensor(s["pair_freq"], device=dev, dtype=torch.float64)
        if own:
            from paper_2511_06029_b200 import binding
            s["ctx"] = _ctx()
            s["rotary"] = binding.Rotary(s["pair_axis"], s["pair_freq"], s["axis_pos"],
                                         style=binding.ROT_HALVES if c["style"] == "halves" else binding.ROT_PAIRS)
        return s

    B, H = c["batch"], c["hkv"]
    order = np.random.RandomState(int(seed) % (1 << 31)).permutation(B)
    cached, new = _lengths(c, order)
    N = sum(new)
    slots = max(_lengths(c)[0]) + max(new) + c["spare"]
    if c["page"]:
        slots = -(-slots // c["page"]) * c["page"]
    kv = _DT[c["dtype"]]
    # keys: Gaussian, one row in a hundred three times as long (anchors)
    k = normal(L * B * H * slots, d)
    k *= torch.where(torch.rand(k.shape[0], generator=g, device=dev) < 0.01, 3.0, 1.0)[:, None]
    v = normal(L * B * H * slots, d)
    s = {"c": c, "slots": slots, "cached": cached, "new": new, "k_scale": None, "v_scale": None}
    if kv.itemsize == 1:
        s["k_scale"], s["v_scale"] = [0.02 + 0.005 * i for i in range(L)], [0.015 + 0.005 * i for i in range(L)]
        top = 448.0 if c["dtype"] == "e4m3" else 57344.0
        per = lambda x, sc: (x.view(L, -1) / torch.tensor(sc, device=dev)[:, None]).clamp(-top, top).view(x.shape)  # noqa: E731
        k, v = per(k, s["k_scale"]), per(v, s["v_scale"])
    k, v = k.to(kv), v.to(kv)
    ln = torch.tensor(cached, dtype=torch.int32, device=dev).view(1, B, 1).expand(L, B, H).contiguous()
    if c["page"]:
        n_pages = L * B * H * slots // c["page"]
        s["page_table"] = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32).view(L, B, H, -1).contiguous()
        s["k"], s["v"] = k.view(n_pages, c["page"], d), v.view(n_pages, c["page"], d)
    else:
        s["page_table"] = None
        s["k"], s["v"] = k.view(L, B, H, slots, d), v.view(L, B, H, slots, d)
    # relevance and lengths in one buffer, so that one copy takes a speculative step back
    items = L * B * H
    s["book"] = torch.empty(items * slots + items, dtype=torch.int32, device=dev)
    s["rel"], s["len"] = s["book"][:items * slots].view(torch.float32).view(L, B, H, slots), s["book"][items * slots:].view(L, B, H)
    s["rel"].copy_(torch.rand((L, B, H, slots), generator=g, device=dev) * (torch.arange(slots, device=dev) < ln[..., None]))
    s["len"].copy_(ln)
    s["book0"] = s["book"].clone()
    s["pos"] = torch.floor(torch.arange(slots, device=dev, dtype=torch.float64) * _STRETCH).to(torch.int32).expand(L, B, H, slots).contiguous()
    s["q"] = normal(L, N, c["hq"], d).to(act)
    s["k_new"], s["v_new"] = normal(L, N, H, d).to(act), normal(L, N, H, d).to(act)
    start = np.concatenate([[0], np.cumsum(new)])
    s["chunk_start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    s["max_chunk"] = max(new)
    first = [int(x * _STRETCH) for x in cached]
    tp = np.concatenate([first[b] + np.arange(new[b]) for b in range(B)])
    s["token_pos"] = torch.tensor(tp, dtype=torch.int32, device=dev)
    s["scale"] = [c["scale"] / math.sqrt(d) / (1 + 0.25 * i) for i in range(L)]
    s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / c["hq"]) for h in range(c["hq"])], dtype=torch.float32, device=dev) if c["slopes"] else None
    s["doc_start"] = (s["token_pos"] // c["doc"] * c["doc"]).to(torch.int32) if c["doc"] else None
    s["prefix_len"] = torch.full((B,), c["prefix"], dtype=torch.int32, device=dev) if c["prefix"] else None
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((L, N, c["hq"]), dtype=torch.float32, device=dev)
    if own:
        from paper_2511_06029_b200 import binding
        s["ctx"] = _ctx()
        s["cache"] = binding.Cache(c["hq"], s["k"], s["v"], s["rel"], s["pos"], s["len"], s["page_table"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        s["mod"] = binding.ScoreMod(softcap=c["softcap"], window=c["window"], slopes=s["slopes"], doc_start=s["doc_start"],
                                    prefix_len=s["prefix_len"]) if _modified(c) else None
    return s


# --------------------------------------------------------------------------------------------------------- one pass

def run(state):
    s = state
    c = s["c"]
    if c["op"] == "rotate":
        if own:
            s["ctx"].rotate(s["rotary"], s["q"], s["k"], s["q_out"], s["k_out"], inverse=c["inverse"])
            return {"q": s["q_out"], "k": s["k_out"]}
        return {"q": _plain_rotate(s, s["q"]), "k": _plain_rotate(s, s["k"])}
    s["book"].copy_(s["book0"])
    if own:
        s["ctx"].chunk_attend(s["cache"], 0, c["layers"], s["chunk_start"], s["max_chunk"], s["q"], s["k_new"], s["v_new"],
                              s["token_pos"], s["scale"], _GAMMA, s["out"], lse=s["lse"], mod=s["mod"])
        out, lse = s["out"], s["lse"]
    else:
        out, lse = _plain_attend(s)
    return {"out": out, "lse": lse, "rel": s["rel"], "len": s["len"], "pos": s["pos"], "k": s["k"], "v": s["v"]}


def _plain_rotate(s, x):
    c = s["c"]
    half = c["rot_dim"] // 2
    angle = s["axis_pos"][s["pair_axis_dev"]].double().t() * s["pair_freq_dev"]            # [tokens][pairs], in 64 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if c["inverse"]:
        sin = -sin
    y = x.float()
    z = y.clone()
    a, b = (y[..., :half], y[..., half:2 * half]) if c["style"] == "halves" else (y[..., 0:2 * half:2], y[..., 1:2 * half:2])
    u, w = a * cos - b * sin, a * sin + b * cos
    if c["style"] == "halves":
        z[..., :half], z[..., half:2 * half] = u, w
    else:
        z[..., 0:2 * half:2], z[..., 1:2 * half:2] = u, w
    return z.to(x.dtype)


def _plain_attend(s):
    c = s["c"]
    L, B, H, d, G = c["layers"], c["batch"], c["hkv"], c["d"], c["hq"] // c["hkv"]
    dev, T = s["q"].device, s["max_chunk"]
    start = s["chunk_start"].long()
    new = start[1:] - start[:-1]
    n0 = s["len"].long()                                                                  # [L][B][H]
    # rows of the packed tokens in a padded [B][T] grid
    i = torch.arange(T, device=dev)
    real = i[None] < new[:, None]
    tok = (start[:-1, None] + i[None]).clamp(max=s["q"].shape[1] - 1)
    # append: row of every (layer, token, head) in the flattened cache
    seq = torch.searchsorted(start, torch.arange(s["q"].shape[1], device=dev), right=True) - 1
    at = torch.arange(s["q"].shape[1], device=dev) - start[seq]
    slot = n0[:, seq, :] + at[None, :, None]                                              # [L][N][H]
    item = (torch.arange(L, device=dev)[:, None, None] * B + seq[None, :, None]) * H + torch.arange(H, device=dev)
    kf, vf = s["k"].view(-1, d), s["v"].view(-1, d)

    def row_of(item, slot):
        if s["page_table"] is None:
            return item * s["slots"] + slot
        pt = c["page"]
        return s["page_table"].view(-1, s["slots"] // pt)[item, slot // pt].long() * pt + slot % pt

    where = row_of(item, slot)
    kn, vn = s["k_new"], s["v_new"]
    ks = vs = torch.ones(L, device=dev)
    if s["k_scale"] is not None:
        ks, vs = torch.tensor(s["k_scale"], device=dev), torch.tensor(s["v_scale"], device=dev)
        top = 448.0 if c["dtype"] == "e4m3" else 57344.0
        kn = (kn.float() / ks.view(L, 1, 1, 1)).clamp(-top, top).to(kf.dtype)
        vn = (vn.float() / vs.view(L, 1, 1, 1)).clamp(-top, top).to(vf.dtype)
    raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[kf.element_size()]
    kf.view(raw)[where] = kn.view(raw)
    vf.view(raw)[where] = vn.view(raw)
    s["pos"].view(-1)[item * s["slots"] + slot] = s["token_pos"][None, :, None].expand_as(slot).contiguous()
    s["len"] += new.view(1, B, 1).to(torch.int32)
    # padded keys and values, in 32 bits
    M = max(s["cached"]) + T
    M = min(M, s["slots"])
    j = torch.arange(M, device=dev)
    items = torch.arange(L * B * H, device=dev).view(L, B, H, 1)
    rows = row_of(items, j.view(1, 1, 1, M).expand(L, B, H, M))
    used = j < s["len"].long()[..., None]                                                 # [L][B][H][M]
    K = torch.where(used[..., None], kf.view(raw)[rows].view(kf.dtype).float(), 0.0) * ks.view(L, 1, 1, 1, 1)
    V = torch.where(used[..., None], vf.view(raw)[rows].view(vf.dtype).float(), 0.0) * vs.view(L, 1, 1, 1, 1)
    q = s["q"][:, tok].float().view(L, B, T, H, G, d).permute(0, 1, 3, 4, 2, 5)            # [L][B][H][G][T][d]
    x = torch.matmul(q.reshape(L, B, H, G * T, d), K.transpose(-1, -2)).view(L, B, H, G, T, M)
    x = x * torch.tensor(s["scale"], device=dev).view(L, 1, 1, 1, 1, 1)
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    pq = s["token_pos"][tok].view(1, B, 1, T, 1)
    pk = s["pos"][..., :M].view(L, B, H, 1, M)
    if c["slopes"]:
        x = x - s["slopes"].view(1, 1, H, G, 1, 1) * (pq - pk).abs().float()[:, :, :, None]
    see = j.view(1, 1, 1, 1, M) <= n0[..., None, None] + i.view(1, 1, 1, T, 1)
    if c["prefix"]:
        see = see | ((pk < s["prefix_len"].view(1, B, 1, 1, 1)) & used[..., None, :])
    if c["window"]:
        see = see & (pq - pk < c["window"])
    if c["doc"]:
        see = see & (pk >= s["doc_start"][tok].view(1, B, 1, T, 1))
    see = (see & real.view(1, B, 1, T, 1))[:, :, :, None]
    x = torch.where(see, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total))[..., 0]                                                # [L][B][H][G][T]
    o = torch.matmul(p.view(L, B, H, G * T, M), V).view(L, B, H, G, T, d)
    # relevance: decayed once per new token, what later tokens gave counts more
    weight = torch.where(real, torch.tensor(_GAMMA, device=dev, dtype=torch.float64) ** (new[:, None] - 1 - i[None]).clamp(min=0), 0.0).float()
    got = (p * weight.view(1, B, 1, 1, T, 1)).sum((3, 4))                                  # [L][B][H][M]
    decay = (torch.tensor(_GAMMA, device=dev, dtype=torch.float64) ** new).float().view(1, B, 1, 1)
    old = torch.where(j < n0[..., None], s["rel"][..., :M], 0.0)
    s["rel"][..., :M] = torch.where(used, decay * old + got, s["rel"][..., :M])
    pick = (seq, at)
    out = o.permute(0, 1, 4, 2, 3, 5).reshape(L, B, T, H * G, d)[:, pick[0], pick[1]].to(s["q"].dtype)
    lse = lse.permute(0, 1, 4, 2, 3).reshape(L, B, T, H * G)[:, pick[0], pick[1]]
    return out, lse


# --------------------------------------------------------------------------------------------- definitions in 64 bits

def exact(case, seed):
    c = case
    s = prepare(case, seed)
    dev = s["q"].device
    if c["op"] == "rotate":
        half = c["rot_dim"] // 2
        res = {}
        for name in ("q", "k"):
            z = s[name].double().clone()
            for p in range(half):
                i0, i1 = (p, p + half) if c["style"] == "halves" else (2 * p, 2 * p + 1)
                turn = s["axis_pos"][s["pair_axis"][p]].double() * s["pair_freq"][p] * (-1 if c["inverse"] else 1)
                a, b = z[..., i0].clone(), z[..., i1].clone()
                cs, sn = torch.cos(turn)[None, :, None], torch.sin(turn)[None, :, None]
                z[..., i0], z[..., i1] = a * cs - b * sn, b * cs + a * sn
            res[name] = z
        return res
    L, B, H, d, G = c["layers"], c["batch"], c["hkv"], c["d"], c["hq"] // c["hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=dev)
    rel = s["rel"].double()
    first = s["chunk_start"].tolist()
    unit = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[s["k"].element_size()]

    def stored(x, scale):
        """What the cache holds of new rows, and what that stands for."""
        if scale is None:
            return x.double()
        top = 448.0 if c["dtype"] == "e4m3" else 57344.0
        return (x.float() / scale).clamp(-top, top).to(_DT[c["dtype"]]).double() * float(np.float32(scale))

    for l in range(L):
        for b in range(B):
            t0, t1, n = first[b], first[b + 1], s["cached"][b]
            m = t1 - t0
            pq = s["token_pos"][t0:t1].long()
            for h in range(H):
                if s["page_table"] is None:
                    K, V = s["k"][l, b, h, :n].double(), s["v"][l, b, h, :n].double()
                else:
                    pages = s["page_table"][l, b, h].long()
                    K = s["k"].view(unit)[pages].view(s["k"].dtype).reshape(-1, d)[:n].double()
                    V = s["v"].view(unit)[pages].view(s["v"].dtype).reshape(-1, d)[:n].double()
                ksc, vsc = (None, None) if s["k_scale"] is None else (s["k_scale"][l], s["v_scale"][l])
                if ksc is not None:
                    K, V = K * float(np.float32(ksc)), V * float(np.float32(vsc))
                K = torch.cat([K, stored(s["k_new"][l, t0:t1, h], ksc)])
                V = torch.cat([V, stored(s["v_new"][l, t0:t1, h], vsc)])
                pk = torch.cat([s["pos"][l, b, h, :n].long(), pq])
                j = torch.arange(n + m, device=dev)
                ok = j[None, :] <= n + torch.arange(m, device=dev)[:, None]
                if c["prefix"]:
                    ok = ok | (pk[None, :] < c["prefix"])
                if c["window"]:
                    ok = ok & (pq[:, None] - pk[None, :] < c["window"])
                if c["doc"]:
                    ok = ok & (pk[None, :] >= (pq // c["doc"] * c["doc"])[:, None])
                w = _GAMMA ** torch.arange(m - 1, -1, -1, dtype=torch.float64, device=dev)
                mass = torch.zeros(n + m, dtype=torch.float64, device=dev)
                for g in range(G):
                    e = s["q"][l, t0:t1, h * G + g].double() @ K.T * float(np.float32(s["scale"][l]))
                    if c["softcap"]:
                        e = torch.tanh(e / c["softcap"]) * c["softcap"]
                    if c["slopes"]:
                        e = e - float(s["slopes"][h * G + g]) * (pq[:, None] - pk[None, :]).abs()
                    e = e.masked_fill(~ok, -math.inf)
                    z = torch.logsumexp(e, 1)
                    p = torch.exp(e - torch.where(torch.isinf(z), 0.0, z)[:, None])
                    out[l, t0:t1, h * G + g] = p @ V
                    lse[l, t0:t1, h * G + g] = z
                    mass += w @ p
                old = torch.cat([rel[l, b, h, :n], torch.zeros(m, dtype=torch.float64, device=dev)])
                rel[l, b, h, :n + m] = _GAMMA ** m * old + mass
    return {"out": out, "lse": lse, "rel": rel, "len": None, "pos": None, "k": None, "v": None}
