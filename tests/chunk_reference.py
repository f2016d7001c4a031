"""Plain 64-bit statement of lethe_chunk_attend and lethe_rotate for the tests, with the error bounds that the arithmetic of the
kernels allows (so that tolerances follow from the inputs)."""
import math

import numpy as np
import torch

FP8_MAX = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}


def stored(x, dtype, scale):
    """New rows as the cache holds them."""
    if dtype not in FP8_MAX:
        return x.to(dtype)
    top = FP8_MAX[dtype]
    return (x.float() / torch.tensor(scale, dtype=torch.float32)).clamp(-top, top).to(dtype)


class State:
    """CPU cache: k, v [L][B][H][cap][D] in storage type, rel, pos, len; layout and page table for the device copy."""

    def __init__(self, L, B, Hq, Hkv, D, cap, lens, dtype, page=0, seed=0, k_scale=None, v_scale=None, junk=float("nan"), spare_pages=3,
                 gaps=True, key_gain=1.0):
        g = torch.Generator().manual_seed(seed)
        self.L, self.B, self.Hq, self.Hkv, self.D, self.cap, self.dtype, self.page = L, B, Hq, Hkv, D, cap, dtype, page
        self.len = torch.as_tensor(lens, dtype=torch.int32).expand(L, B, Hkv).clone() if not (isinstance(lens, torch.Tensor) and lens.dim() == 3) else lens.to(torch.int32).clone()
        self.k_scale = k_scale if dtype in FP8_MAX else None
        self.v_scale = v_scale if dtype in FP8_MAX else None
        if dtype in FP8_MAX:
            self.k_scale, self.v_scale = self.k_scale or [0.02] * L, self.v_scale or [0.015] * L
        k, v = torch.randn((L, B, Hkv, cap, D), generator=g) * key_gain, torch.randn((L, B, Hkv, cap, D), generator=g)
        one = [1.0] * L
        self.k = torch.stack([stored(k[l], dtype, (self.k_scale or one)[l]).view(self.raw) for l in range(L)]).view(dtype)
        self.v = torch.stack([stored(v[l], dtype, (self.v_scale or one)[l]).view(self.raw) for l in range(L)]).view(dtype)
        self.rel = torch.rand((L, B, Hkv, cap), generator=g)
        step = torch.randint(1, 4 if gaps else 2, (L, B, Hkv, cap), generator=g)
        self.pos = (step.cumsum(-1) - step[..., :1]).to(torch.int32)
        beyond = torch.arange(cap) >= self.len[..., None]
        if junk is not None:   # slots beyond len may hold anything
            bad = torch.full((), junk).to(dtype).view(self.raw)
            self.k.view(self.raw)[beyond] = bad
            self.v.view(self.raw)[beyond] = bad
            self.rel[beyond] = junk
        self.n_pages = L * B * Hkv * (cap // page) + spare_pages if page else 0
        if page:
            assert cap % page == 0
            self.table = torch.randperm(self.n_pages, generator=g)[:L * B * Hkv * (cap // page)].to(torch.int32).view(L, B, Hkv, -1).contiguous()

    @property
    def raw(self):
        return {1: torch.uint8, 2: torch.int16, 4: torch.int32}[self.dtype.itemsize]

    def device_cache(self, dev="cuda"):
        from paper_2511_06029_b200 import binding
        table = None
        k, v = self.k, self.v
        if self.page:
            def pool(x):
                p = torch.zeros((self.n_pages, self.page, self.D), dtype=self.raw)
                p[self.table.long().view(-1)] = x.view(self.raw).reshape(-1, self.page, self.D)
                return p.view(self.dtype)
            k, v, table = pool(k), pool(v), self.table.to(dev)
        return binding.Cache(self.Hq, k.to(dev), v.to(dev), self.rel.to(dev), self.pos.to(dev), self.len.to(dev), table,
                             k_scale=self.k_scale, v_scale=self.v_scale)

    def rows_of(self, gc):
        """The device cache's K and V back in the contiguous layout (raw integers)."""
        k, v = gc.k.view(self.raw).cpu(), gc.v.view(self.raw).cpu()
        if self.page:
            at = self.table.long()
            k, v = (x[at].reshape(self.L, self.B, self.Hkv, self.cap, self.D) for x in (k, v))
        return k, v


def make_chunk(st, new, l0=0, l1=None, seed=1, lead=0, trail=0, first_pos=None):
    """Packed tokens for sequences with new[b] tokens each; lead / trail padding rows around them."""
    l1 = st.L if l1 is None else l1
    g = torch.Generator().manual_seed(seed)
    act = torch.float32 if st.dtype == torch.float32 else torch.bfloat16
    N = lead + sum(new) + trail
    start = torch.tensor([lead + sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32)
    tp = torch.zeros(N, dtype=torch.int32)
    for b in range(st.B):
        p0 = int(st.pos[:, b].max()) + 1 if first_pos is None else first_pos[b]
        tp[int(start[b]):int(start[b + 1])] = p0 + torch.arange(new[b], dtype=torch.int32)
    rn = lambda h: torch.randn((l1 - l0, N, h, st.D), generator=g).to(act)  # noqa: E731
    return {"q": rn(st.Hq), "k_new": rn(st.Hkv), "v_new": rn(st.Hkv), "token_pos": tp, "chunk_start": start, "N": N,
            "max_chunk": max(1, max(new)), "l0": l0, "l1": l1}


def chunk_attend(st, ch, scale, gamma, softcap=0.0, window=0, slopes=None, doc_start=None, prefix_len=None, append=True):
    """Updates st in place (k, v, rel, pos, len) and returns out, lse (double), and elementwise error bounds of out, lse, rel."""
    L, B, H, D, G = st.L, st.B, st.Hkv, st.D, st.Hq // st.Hkv
    start = ch["chunk_start"].tolist()
    q = ch["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64)
    tol_out, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    tol_rel = torch.zeros(st.rel.shape, dtype=torch.float64)
    rel64 = st.rel.double()
    tensor_cores = st.dtype != torch.float32
    u = 2.0 ** -23          # fp32 accumulation, a whole step per add (the tensor cores truncate)
    refused = []
    one = [1.0] * L
    for l in range(ch["l0"], ch["l1"]):
        li = l - ch["l0"]
        s32 = float(torch.tensor(scale[l], dtype=torch.float32))
        ks = float(torch.tensor((st.k_scale or one)[l], dtype=torch.float32))
        vs = float(torch.tensor((st.v_scale or one)[l], dtype=torch.float32))
        for b in range(B):
            t0, t1 = start[b], start[b + 1]
            T = t1 - t0
            if T == 0:
                continue
            pq = ch["token_pos"][t0:t1].long()
            for h in range(H):
                n = int(st.len[l, b, h])
                if append:
                    if n + T > st.cap:
                        refused.append((l * B + b) * H + h)
                        continue
                    st.k.view(st.raw)[l, b, h, n:n + T] = stored(ch["k_new"][li, t0:t1, h], st.dtype, ks).view(st.raw)
                    st.v.view(st.raw)[l, b, h, n:n + T] = stored(ch["v_new"][li, t0:t1, h], st.dtype, vs).view(st.raw)
                    st.pos[l, b, h, n:n + T] = pq.to(torch.int32)
                    rel64[l, b, h, n:n + T] = 0
                    st.len[l, b, h] = n + T
                m = int(st.len[l, b, h])
                K, V = st.k[l, b, h, :m].double() * ks, st.v[l, b, h, :m].double() * vs
                pk = st.pos[l, b, h, :m].long()
                j, i = torch.arange(m), torch.arange(T)
                see = (j[None] <= n + i[:, None]) if append else torch.ones((T, m), dtype=torch.bool)
                if prefix_len is not None:
                    see = see | (pk[None] < int(prefix_len[b]))
                if window:
                    see = see & (pq[:, None] - pk[None] < window)
                if doc_start is not None:
                    see = see & (pk[None] >= doc_start[t0:t1].long()[:, None])
                wt = gamma ** (T - 1 - i).double()
                mass = torch.zeros(m, dtype=torch.float64)
                mass_err = torch.zeros(m, dtype=torch.float64)
                for gi in range(G):
                    hq = h * G + gi
                    qq = q[li, t0:t1, hq]
                    x = qq @ K.T * s32
                    err = (qq.abs() @ K.abs().T * abs(s32)) * (D + 4) * u      # the product, accumulated in fp32
                    if softcap:
                        x = softcap * torch.tanh(x / softcap)
                        err = err + softcap * 2.0 ** -21 + x.abs() * 2.0 ** -21
                    err = err + x.abs() * 4 * u
                    if slopes is not None:
                        bias = float(slopes[hq]) * (pq[:, None] - pk[None]).abs().double()
                        x = x - bias
                        err = err + (bias + x.abs()) * 4 * u
                    x = torch.where(see, x, -math.inf)
                    z = torch.logsumexp(x, 1) if m else torch.full((T,), -math.inf, dtype=torch.float64)
                    p = torch.exp(x - torch.where(z == -math.inf, 0.0, z)[:, None])
                    p = torch.where(see, p, 0.0)
                    e_row = torch.where(see, err, 0.0).amax(1) if m else torch.zeros(T, dtype=torch.float64)
                    # a probability: exponent, statistics, 2^x (2 steps), the running rescales and the sums
                    e_p = 2 * e_row + (z.abs().where(z != -math.inf, torch.zeros(())) + 8) * 4 * u + (m / 16 + 16) * u
                    o = p @ V
                    out[li, t0:t1, hq], lse[li, t0:t1, hq] = o, z
                    half = 2.0 ** -8 if tensor_cores else 2.0 ** -24          # half a step of the probabilities' / outputs' type
                    tol_out[li, t0:t1, hq] = (p @ V.abs()) * ((2 * e_p + (half if tensor_cores else 0) + (m / 16 + 16) * u)[:, None]) + o.abs() * half + 1e-30
                    tol_lse[li, t0:t1, hq] = e_row + (z.abs().where(z != -math.inf, torch.zeros(())) + 8) * 4 * u + (m / 16 + 16) * u
                    mass += wt @ p
                    mass_err += (wt * (2 * e_p + 4 * u * (T - 1 - i) * abs(math.log2(gamma)) + (T * G / 16 + 16) * u)) @ p
                rel64[l, b, h, :m] = gamma ** T * rel64[l, b, h, :m] + mass
                tol_rel[l, b, h, :m] = mass_err + rel64[l, b, h, :m].abs() * (8 + 4 * T * abs(math.log2(gamma))) * u + 1e-30
    st.rel = rel64
    return out, lse, tol_out, tol_lse, tol_rel, refused


def rotate(x, pair_axis, pair_freq, axis_pos, pairs=False, inverse=False):
    """lethe_rotate in 64 bits; x [nl][N][H][D]."""
    half = len(pair_axis)
    z = x.double().clone()
    # angles in 80 bits, reduced there: a position of 2^31 times 2 pi has half a step of 2^-20 radians in 64
    two_pi = np.longdouble("6.283185307179586476925286766559")
    turns = axis_pos.numpy().astype(np.longdouble)[np.array(pair_axis)] * (np.array(pair_freq).astype(np.longdouble) / two_pi)[:, None]
    turn = torch.from_numpy(((turns - np.rint(turns)) * two_pi).astype(np.float64))                              # [pairs][N]
    c, s = turn.cos().t()[None, :, None], turn.sin().t()[None, :, None] * (-1 if inverse else 1)
    i0 = torch.arange(0, 2 * half, 2) if pairs else torch.arange(half)
    i1 = i0 + 1 if pairs else i0 + half
    a, b = x.double()[..., i0], x.double()[..., i1]
    z[..., i0], z[..., i1] = a * c - b * s, a * s + b * c
    size = torch.zeros_like(z)
    size[..., i0] = size[..., i1] = a.abs() + b.abs()
    return z, size
