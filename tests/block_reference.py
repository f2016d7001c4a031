"""Plain statement of block caches (8 bits, one scale for each block of tokens) for the tests: filling in fp32 as the definition says,
everything that follows in 64 bits, with the error bounds that the arithmetic of the kernels allows."""
import numpy as np
import torch

TINY = 2.0 ** -100


def quantise(x):
    """fp32 blocks [..., T, D] (numpy) -> codes int8, scales fp32."""
    finite = np.where(np.isfinite(x), np.abs(x), 0).astype(np.float32)
    top = finite.max((-1, -2))
    some = top >= np.float32(TINY)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        scale = np.where(some, top / np.float32(127), np.float32(0)).astype(np.float32)
        inv = np.where(some, np.float32(127) / top, np.float32(0)).astype(np.float32)
        y = x.astype(np.float32) * inv[..., None, None]
    y = np.clip(np.rint(np.where(np.isnan(y), np.float32(0), y)), -127, 127)
    return y.astype(np.int8), scale


class BlockState:
    """CPU block cache: what each item holds as full blocks and open rows; layout and page table for the device copy."""

    def __init__(self, L, B, Hq, Hkv, D, T, capacity, lens, paged=False, seed=0, junk=True, spare_pages=3):
        g = torch.Generator().manual_seed(seed)
        self.L, self.B, self.Hq, self.Hkv, self.D, self.T, self.capacity, self.paged = L, B, Hq, Hkv, D, T, capacity, paged
        self.G = Hq // Hkv
        self.len = torch.as_tensor(lens, dtype=torch.int32).expand(L, B, Hkv).clone()
        shape = (L, B, Hkv, capacity, T, D)
        draw = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        # blocks of different size, keys with something in common
        k = draw(*shape) + 0.5 * draw(L, B, Hkv, capacity, 1, D)
        v = draw(*shape) * torch.exp(0.7 * draw(L, B, Hkv, capacity, 1, 1))
        kc, ks = quantise(k.numpy())
        vc, vs = quantise(v.numpy())
        self.k, self.v, self.k_scale, self.v_scale = (torch.from_numpy(x) for x in (kc, vc, ks, vs))
        self.k_open, self.v_open = draw(L, B, Hkv, T, D).to(torch.bfloat16), draw(L, B, Hkv, T, D).to(torch.bfloat16)
        self.k_range = torch.stack([self.k.amin(4), self.k.amax(4)], 4)
        if junk:  # what lies behind the full blocks and behind the open rows may be anything
            full = self.len // T
            beyond = torch.arange(capacity) >= full[..., None]
            self.k_scale[beyond] = float("nan")
            self.v_scale[beyond] = float("nan")
            rows = torch.arange(T) >= (self.len % T)[..., None]
            self.k_open[rows] = float("nan")
            self.v_open[rows] = float("nan")
        self.n_pages = L * B * Hkv * capacity + spare_pages if paged else 0
        if paged:
            self.table = torch.randperm(self.n_pages, generator=g)[:L * B * Hkv * capacity].to(torch.int32).view(L, B, Hkv, capacity).contiguous()

    def device_cache(self, dev="cuda", with_range=True):
        from paper_2511_06029_b200 import binding

        def place(x):
            if not self.paged:
                return x.contiguous().to(dev)
            p = torch.zeros((self.n_pages,) + tuple(x.shape[4:]), dtype=x.dtype)
            p[self.table.long().view(-1)] = x.reshape((-1,) + tuple(x.shape[4:]))
            return p.to(dev)

        return binding.BlockCache(self.Hq, place(self.k), place(self.v), place(self.k_scale), place(self.v_scale), place(self.k_range) if with_range else None,
                                  self.k_open.to(dev), self.v_open.to(dev), self.len.to(dev), self.table.to(dev) if self.paged else None)

    def back(self, x):
        """A pool of the device in the order of the items."""
        x = x.cpu()
        return x[self.table.long()] if self.paged else x

    def append(self, layer_begin, chunk_start, k_new, v_new):
        """k_new, v_new [nl][n_tokens][Hkv][D] bf16, keys rotated."""
        T = self.T
        for li in range(k_new.shape[0]):
            for b in range(self.B):
                t0, t1 = int(chunk_start[b]), int(chunk_start[b + 1])
                for h in range(self.Hkv):
                    at = (layer_begin + li, b, h)
                    n = int(self.len[at])
                    if n + t1 - t0 > self.capacity * T or t1 == t0:
                        continue
                    o = n % T
                    for open_, new, codes, scales in ((self.k_open, k_new, self.k, self.k_scale), (self.v_open, v_new, self.v, self.v_scale)):
                        rows = torch.cat([open_[at][:o], new[li, t0:t1, h]])
                        m = len(rows) // T
                        if m:
                            c, s = quantise(rows[:m * T].float().numpy().reshape(m, T, self.D))
                            codes[at][n // T:n // T + m], scales[at][n // T:n // T + m] = torch.from_numpy(c), torch.from_numpy(s)
                            open_[at][:len(rows) - m * T] = rows[m * T:]
                        else:
                            open_[at][o:len(rows)] = rows[o:]
                    m = (n + t1 - t0) // T
                    self.k_range[at][n // T:m] = torch.stack([self.k[at][n // T:m].amin(1), self.k[at][n // T:m].amax(1)], 1)
                    self.len[at] = n + t1 - t0

    def rows(self, at, blocks=None):
        """Keys and values of an item in 64 bits: the given full blocks (all: None), then the open rows."""
        n, T = int(self.len[at]), self.T
        pick = torch.arange(n // T) if blocks is None else torch.as_tensor(blocks, dtype=torch.long)
        out = []
        for codes, scales, open_ in ((self.k, self.k_scale, self.k_open), (self.v, self.v_scale, self.v_open)):
            full = codes[at][pick].double() * scales[at][pick].double()[:, None, None]
            out.append(torch.cat([full.reshape(-1, self.D), open_[at][:n % T].double()]))
        return out

    def attend(self, layer_begin, q, scale, selected=None):
        """(out, lse, bound of out, bound of lse) in 64 bits; selected [nl][B][Hkv][n]."""
        nl = q.shape[0]
        out = torch.zeros(q.shape, dtype=torch.float64)
        lse = torch.full(q.shape[:3], -float("inf"), dtype=torch.float64)
        b_out, b_lse = torch.zeros_like(out), torch.zeros_like(lse)
        for li in range(nl):
            for b in range(self.B):
                for h in range(self.Hkv):
                    at = (layer_begin + li, b, h)
                    blocks = None
                    if selected is not None:
                        full = int(self.len[at]) // self.T
                        blocks = [int(x) for x in selected[li, b, h][:full] if 0 <= int(x) < full]
                    K, V = self.rows(at, blocks)
                    if len(K) == 0:
                        continue
                    hs = slice(h * self.G, (h + 1) * self.G)
                    x = q[li, b, hs].double()
                    sc = float(np.float32(scale[layer_begin + li]))
                    e = x @ K.T * sc
                    size = float((x.abs() @ K.abs().T).max()) * abs(sc)
                    z = torch.logsumexp(e, 1)
                    p = torch.exp(e - z[:, None])
                    out[li, b, hs], lse[li, b, hs] = p @ V, z
                    # A logit: D exact products summed in fp32 (a step each), times factors that round a few times.  A probability:
                    # f16 (half a step, 2^-11), exp2 and log2 of the special-function unit, sums in fp32.
                    err = size * (self.D + 8) * 2.0 ** -23
                    grow = len(K) * 2.0 ** -24 + 2.0 ** -19
                    weight = 2.0 ** -11 + 2 * err + grow
                    b_out[li, b, hs] = (p @ V.abs()) * weight + out[li, b, hs].abs() * 2.0 ** -8 + 1e-30
                    b_lse[li, b, hs] = err + grow + z.abs() * 2.0 ** -22
        return out, lse, b_out, b_lse

    def select(self, layer_begin, q, n_select, sink, recent):
        nl = q.shape[0]
        got = torch.full((nl, self.B, self.Hkv, n_select), -1, dtype=torch.int32)
        for li in range(nl):
            for b in range(self.B):
                for h in range(self.Hkv):
                    at = (layer_begin + li, b, h)
                    full = int(self.len[at]) // self.T
                    if full <= n_select:
                        got[li, b, h, :full] = torch.arange(full)
                        continue
                    code, _ = quantise(q[li, b, h * self.G:(h + 1) * self.G].float().numpy())
                    code = code.astype(np.int64)[:, None]
                    r = self.k_range[at][:full].numpy().astype(np.int64)
                    most = np.maximum(code * r[:, 0], code * r[:, 1]).sum((0, 2))
                    score = self.k_scale[at][:full].numpy() * most.astype(np.float32) + np.float32(0)
                    score = score.astype(np.float64)
                    score[:sink] = np.inf
                    score[full - recent:] = np.inf
                    best = np.argsort(-score, kind="stable")[:n_select]
                    got[li, b, h] = torch.from_numpy(np.sort(best))
        return got


def starts(chunks):
    return torch.tensor(np.concatenate([[0], np.cumsum(chunks)]), dtype=torch.int32)
