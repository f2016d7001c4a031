"""lethe_chunk_attend (a step of several new tokens per sequence, plain and with modified scores) against a plain 64-bit
statement of it; the error bounds follow from the inputs and the number of roundings (chunk_reference.py)."""
import copy
import ctypes
import math

import pytest
import torch

import chunk_reference as ref
from helpers import gpu_context

pytestmark = pytest.mark.gpu

F32, BF16, E4M3, E5M2 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.float8_e5m2


@pytest.fixture(scope="module")
def ctx():
    c = gpu_context()
    yield c
    c.close()


def dev(t):
    return None if t is None else t.cuda()


def run_device(ctx, st, gc, ch, scale, gamma, append=True, mod_kw=None, out=None, lse=None, rotary=None):
    from paper_2511_06029_b200 import binding
    mod = None
    if mod_kw:
        kw = {k: (dev(v) if isinstance(v, torch.Tensor) else v) for k, v in mod_kw.items()}
        mod = binding.ScoreMod(**kw)
    if out is None:
        out = torch.full(ch["q"].shape, 7.0, dtype=ch["q"].dtype, device="cuda")
    if lse is None:
        lse = torch.full(ch["q"].shape[:3], 7.0, dtype=torch.float32, device="cuda")
    ctx.chunk_attend(gc, ch["l0"], ch["l1"], dev(ch["chunk_start"]), ch["max_chunk"], dev(ch["q"]),
                     dev(ch["k_new"]) if append else None, dev(ch["v_new"]) if append else None, dev(ch["token_pos"]), scale, gamma,
                     out, lse, mod=mod, rotary=rotary)
    return out, lse


def compare(st, gc, ch, out, lse, want):
    """st has been updated by the reference; want is what it returned."""
    o, z, tol_o, tol_z, tol_r, _ = want
    out, lse = out.cpu().double(), lse.cpu().double()
    lo, hi = int(ch["chunk_start"][0]), int(ch["chunk_start"][-1])
    assert torch.equal(torch.isnan(out), torch.isnan(o)) and torch.equal(torch.isnan(lse), torch.isnan(z))
    d = torch.where(torch.isnan(o), 0.0, out - o).abs()[:, lo:hi]
    tol_o, tol_z = torch.where(torch.isnan(o), 0.0, tol_o), torch.where(torch.isnan(z), 0.0, tol_z)
    assert bool((d <= tol_o[:, lo:hi]).all()), f"out: worst {float((d / tol_o[:, lo:hi].clamp(min=1e-30)).max()):.3g} of its bound, max abs {float(d.max()):.3g}"
    empty = z[:, lo:hi] == -math.inf
    assert torch.equal(lse[:, lo:hi] == -math.inf, empty)
    d = torch.where(empty | torch.isnan(z[:, lo:hi]), 0.0, lse[:, lo:hi] - torch.where(empty, 0.0, z[:, lo:hi])).abs()
    assert bool((d <= tol_z[:, lo:hi]).all()), f"lse: worst {float((d / tol_z[:, lo:hi].clamp(min=1e-30)).max()):.3g} of its bound"
    for rest in (slice(0, lo), slice(hi, None)):         # padding rows are as they were
        assert bool((out[:, rest] == 7.0).all()) and bool((lse[:, rest] == 7.0).all())
    assert torch.equal(gc.len.cpu(), st.len)
    k, v = st.rows_of(gc)
    assert torch.equal(k, st.k.view(st.raw)) and torch.equal(v, st.v.view(st.raw))
    assert torch.equal(gc.pos.cpu(), st.pos)
    rel = gc.rel.cpu().double()
    live = torch.arange(st.cap) < st.len[..., None]
    assert torch.equal(torch.isnan(rel), torch.isnan(st.rel))
    live = live & ~torch.isnan(st.rel)
    d = (rel - st.rel).abs()[live]
    assert bool((d <= tol_r[live]).all()), f"rel: worst {float((d / tol_r[live].clamp(min=1e-30)).max()):.3g} of its bound"


def check(ctx, st, ch, scale=None, gamma=0.97, append=True, **mod_kw):
    scale = scale or [1.0 / math.sqrt(st.D) / (1 + 0.3 * i) for i in range(st.L)]
    gc = st.device_cache()
    out, lse = run_device(ctx, st, gc, ch, scale, gamma, append, mod_kw)
    want = ref.chunk_attend(st, ch, scale, gamma, append=append, **mod_kw)
    assert ctx.poll_status()[0] == 0
    compare(st, gc, ch, out, lse, want)
    return gc


SHAPES = [  # Hq, Hkv, D
    (8, 2, 64), (32, 8, 128), (28, 4, 128), (5, 1, 64), (6, 2, 128), (8, 1, 128), (3, 3, 64), (12, 2, 128)]
LENGTHS = [  # cached, new
    ([0], [1]), ([1], [1]), ([0], [130]), ([127, 128, 129], [1, 1, 1]), ([300, 0, 5], [4, 9, 0]), ([700, 33, 260], [17, 150, 1]),
    ([1100, 90], [3, 70]), ([64, 500], [257, 300])]


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3, E5M2])
@pytest.mark.parametrize("case", range(len(LENGTHS)))
def test_lengths(ctx, dtype, case):
    cached, new = LENGTHS[case]
    for k in (case % len(SHAPES), (case + 3) % len(SHAPES)):
        Hq, Hkv, D = SHAPES[k]
        B = len(cached)
        cap = max(c + n for c, n in zip(cached, new)) + (case % 3) * 7
        st = ref.State(1, B, Hq, Hkv, D, cap, torch.tensor(cached).view(1, B, 1).expand(1, B, Hkv), dtype, seed=case)
        check(ctx, st, ref.make_chunk(st, new, seed=case + 50))


@pytest.mark.parametrize("Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
def test_shapes_paged_ragged_heads(ctx, Hq, Hkv, D, dtype):
    """Two layers with different scales, ragged lengths per (layer, sequence, head), 16-token pages, padding rows."""
    L, B, cap = 2, 3, 528
    g = torch.Generator().manual_seed(Hq)
    lens = torch.randint(0, cap - 80, (L, B, Hkv), generator=g)
    st = ref.State(L, B, Hq, Hkv, D, cap, lens, dtype, page=16, seed=Hq, k_scale=[0.02, 0.03], v_scale=[0.01, 0.02])
    check(ctx, st, ref.make_chunk(st, [7, 80, 1], seed=4, lead=2, trail=3, first_pos=[2000, 1500, 1800]))


@pytest.mark.parametrize("page", [1, 5, 8, 24, 64, 128, 256])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_page_sizes(ctx, page, dtype):
    cap = page * max(2, -(-420 // page))
    st = ref.State(1, 2, 8, 2, 128, cap, torch.tensor([300, 40]).view(1, 2, 1).expand(1, 2, 2), dtype, page=page, seed=page)
    check(ctx, st, ref.make_chunk(st, [60, 33]))


def test_only_the_named_layers(ctx):
    st = ref.State(3, 2, 8, 2, 64, 200, 100, BF16, seed=3)
    check(ctx, st, ref.make_chunk(st, [20, 5], l0=1, l1=2))


@pytest.mark.parametrize("dtype", [F32, BF16, E5M2])
@pytest.mark.parametrize("kind", ["plain", "prefix", "window"])
def test_without_appending(ctx, dtype, kind):
    st = ref.State(1, 3, 8, 2, 128, 300, torch.tensor([0, 77, 290]).view(1, 3, 1).expand(1, 3, 2), dtype, seed=9)
    kw = {"prefix": {"prefix_len": torch.tensor([5, 40, 100], dtype=torch.int32)}, "window": {"window": 50}}.get(kind, {})
    check(ctx, st, ref.make_chunk(st, [3, 50, 1]), append=False, **kw)


MODS = {
    "softcap": {"softcap": 20.0}, "softcap_small": {"softcap": 1.5}, "slopes": {"slopes": True}, "window": {"window": 100},
    "window_one": {"window": 1}, "docs": {"docs": 90}, "docs_future": {"docs": -1}, "prefix": {"prefix": 250}, "prefix_all": {"prefix": 10 ** 6},
    "all": {"softcap": 30.0, "slopes": True, "window": 400, "docs": 300, "prefix": 120}}


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("kind", sorted(MODS))
@pytest.mark.parametrize("new", [[1, 1], [140, 40]])
def test_modified_scores(ctx, dtype, kind, new):
    m = dict(MODS[kind])
    Hq, Hkv, D, B, cap = 12, 2, 128, 2, 704
    st = ref.State(1, B, Hq, Hkv, D, cap, torch.tensor([500, 120]).view(1, B, 1).expand(1, B, Hkv), dtype, page=16, seed=len(kind))
    ch = ref.make_chunk(st, new, seed=8, first_pos=[1400, 400])
    kw = {k: m[k] for k in ("softcap", "window") if k in m}
    if m.get("slopes"):
        kw["slopes"] = torch.tensor([2.0 ** (-0.5 * (h + 1)) for h in range(Hq)])
    if "docs" in m:
        tp = ch["token_pos"]
        kw["doc_start"] = (tp // m["docs"] * m["docs"]) if m["docs"] > 0 else torch.where(torch.arange(len(tp)) % 3 == 0, tp + 5, tp - 30).to(torch.int32)
        kw["doc_start"] = kw["doc_start"].to(torch.int32)       # docs_future: every third token sees nothing at all
    if "prefix" in m:
        kw["prefix_len"] = torch.tensor([m["prefix"], m["prefix"] // 2], dtype=torch.int32)
    check(ctx, st, ch, scale=[3.0 / math.sqrt(D)], **kw)


@pytest.mark.parametrize("dtype", [F32, BF16, E5M2])
@pytest.mark.parametrize("order", ["grown", "any"])
@pytest.mark.parametrize("kind", ["softcap", "slopes"])
@pytest.mark.parametrize("D", [64, 128])
def test_shaped_scores_with_masks(ctx, dtype, order, kind, D):
    """A cap alone, or slopes alone, together with every mask by position; positions that grow with the slot and others; logits on
    both sides of the cap's bend."""
    Hq, Hkv, B = 10, 2, 2
    st = ref.State(1, B, Hq, Hkv, D, 512, torch.tensor([330, 60]).view(1, B, 1).expand(1, B, Hkv), dtype, page=16 if D == 128 else 0, seed=D + len(kind))
    if order == "any":
        g = torch.Generator().manual_seed(3)
        st.pos[...] = torch.randint(0, 1200, st.pos.shape, generator=g, dtype=torch.int32)
    ch = ref.make_chunk(st, [70, 37], seed=8, first_pos=[1000, 180])
    kw = {"window": 500, "prefix_len": torch.tensor([90, 30], dtype=torch.int32), "doc_start": (ch["token_pos"] // 400 * 400).to(torch.int32)}
    if kind == "softcap":
        kw["softcap"] = 4.0
    else:
        kw["slopes"] = torch.tensor([2.0 ** (-0.8 * (h + 1)) for h in range(Hq)])
    check(ctx, st, ch, scale=[3.0 / math.sqrt(D)], **kw)


def test_positions_in_any_order(ctx):
    """Masks by position do not lean on positions that grow with the slot."""
    st = ref.State(1, 1, 8, 2, 128, 900, 700, BF16, seed=2)
    g = torch.Generator().manual_seed(5)
    st.pos[...] = torch.randint(0, 3000, st.pos.shape, generator=g, dtype=torch.int32)
    ch = ref.make_chunk(st, [150], first_pos=[1200])
    check(ctx, st, ch, window=300, prefix_len=torch.tensor([100], dtype=torch.int32),
          doc_start=torch.full((150,), 50, dtype=torch.int32))


def test_extreme_positions(ctx):
    """Positions at the ends of int32: the window's bound saturates, distances are whole."""
    st = ref.State(1, 1, 4, 1, 64, 300, 200, F32, seed=2)
    st.pos[...] = torch.arange(300, dtype=torch.int32)
    ch = ref.make_chunk(st, [20], first_pos=[2 ** 31 - 30])
    check(ctx, st, ch, window=2 ** 31 - 1)


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_scales(ctx, dtype, scale):
    st = ref.State(1, 1, 8, 2, 128, 400, 300, dtype, seed=4)
    check(ctx, st, ref.make_chunk(st, [40]), scale=[scale])
    st = ref.State(1, 1, 8, 2, 128, 400, 300, dtype, seed=5)
    check(ctx, st, ref.make_chunk(st, [40]), scale=[scale], softcap=10.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_keys_may_be_anything(ctx, dtype):
    """NaN and infinite KEYS of slots that a row does not see leave it alone (hidden by a document mask and by order)."""
    st = ref.State(1, 1, 8, 2, 128, 500, 300, dtype, seed=6)
    clean = ref.State(1, 1, 8, 2, 128, 500, 300, dtype, seed=6)
    st.pos[...] = torch.arange(500, dtype=torch.int32)
    clean.pos.copy_(st.pos)
    st.k[0, 0, :, 10] = float("nan")
    st.k[0, 0, :, 140] = float("inf")
    ch = ref.make_chunk(st, [100], first_pos=[300])
    ds = torch.full((100,), 150, dtype=torch.int32)
    scale = [0.09]
    gc = st.device_cache()
    out, lse = run_device(ctx, st, gc, ch, scale, 0.9, True, {"doc_start": ds})
    want = ref.chunk_attend(clean, ch, scale, 0.9, doc_start=ds)
    assert ctx.poll_status()[0] == 0
    o, z, tol_o, tol_z, tol_r, _ = want
    assert bool(((out.cpu().double() - o).abs() <= tol_o).all()) and bool(((lse.cpu().double() - z).abs() <= tol_z).all())
    live = torch.arange(500) < clean.len[..., None]
    assert bool(((gc.rel.cpu().double() - clean.rel).abs() <= tol_r)[live].all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_equals_single_steps(ctx, dtype):
    """T tokens in one call leave what T calls of lethe_decode_attend leave."""
    T, B, Hq, Hkv, D, cap = 6, 2, 8, 2, 128, 260
    st = ref.State(1, B, Hq, Hkv, D, cap, 200, dtype, seed=12)
    ch = ref.make_chunk(st, [T] * B)
    one, many = st.device_cache(), st.device_cache()
    out, lse = run_device(ctx, st, many, ch, [0.1], 0.95)
    step_out = torch.zeros((1, B, Hq, D), dtype=dtype, device="cuda")
    pick = torch.tensor([0, T])
    got = []
    for i in range(T):
        x = {k: ch[k][:, pick + i].contiguous().cuda() for k in ("q", "k_new", "v_new")}
        ctx.decode_attend(one, 0, 1, x["q"], x["k_new"], x["v_new"], ch["token_pos"][pick + i].cuda(), [0.1], 0.95, step_out)
        got.append(step_out.clone())
    assert ctx.poll_status()[0] == 0
    steps = torch.stack(got, 2)[0].reshape(1, B * T, Hq, D)          # [B][T] tokens, packed
    assert torch.equal(one.len, many.len) and torch.equal(one.pos, many.pos)
    live = torch.arange(cap, device="cuda") < one.len[..., None]
    want = ref.chunk_attend(st, ch, [0.1], 0.95)
    # both are within the bounds of the same value (the single steps decay the relevance T times: T more roundings)
    assert bool(((steps - out).abs().cpu().double() <= 2 * want[2]).all())
    assert torch.allclose(one.rel[live], many.rel[live], rtol=2e-4 if dtype == BF16 else 1e-5, atol=1e-7)


def test_full_item_is_refused_and_the_others_run(ctx):
    from paper_2511_06029_b200 import binding
    for dtype in (F32, BF16, E4M3):
        lens = torch.tensor([[[100, 120], [60, 127]]])
        st = ref.State(1, 2, 8, 2, 64, 130, lens, dtype, seed=1)
        ch = ref.make_chunk(st, [20, 3], first_pos=[500, 500])
        gc = st.device_cache()
        out, lse = run_device(ctx, st, gc, ch, [0.1], 0.9)
        want = ref.chunk_attend(st, ch, [0.1], 0.9)
        assert want[-1] == [1]                                       # 120 + 20 > 130; 127 + 3 just fits
        s, item = ctx.poll_status()
        assert s == binding.ERR_CAPACITY and item == 1
        compare(st, gc, ch, out, lse, want)
        assert bool((out[:, :20, 4:] == 0).all()) and bool((lse[:, :20, 4:] == -math.inf).all())


def test_malformed_chunk_start_does_nothing(ctx):
    from paper_2511_06029_b200 import binding
    for dtype in (F32, BF16):
        st = ref.State(1, 3, 8, 2, 64, 130, 60, dtype, seed=1)
        gc = st.device_cache()
        ch = ref.make_chunk(st, [2, 3, 4])
        for bad, mx in (([0, 5, 3, 9], 9), ([0, 2, 5, 10], 9), ([-1, 2, 5, 9], 9), ([0, 2, 5, 9], 3), ([0, 2, 2 ** 31 - 1, 9], 9)):
            ch["chunk_start"] = torch.tensor(bad, dtype=torch.int32)
            ch["max_chunk"] = mx
            out, lse = run_device(ctx, st, gc, ch, [0.1], 0.9)
            assert ctx.poll_status()[0] == binding.ERR_INVALID_ARG
            assert bool((out == 7.0).all()) and bool((lse == 7.0).all())
            assert torch.equal(gc.len.cpu(), st.len) and torch.equal(gc.pos.cpu(), st.pos)
            assert torch.equal(torch.nan_to_num(gc.rel.cpu(), 3.0), torch.nan_to_num(st.rel, 3.0))
            k, v = st.rows_of(gc)
            assert torch.equal(k, st.k.view(st.raw)) and torch.equal(v, st.v.view(st.raw))


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
def test_bad_page_reads_as_zero_rows(ctx, dtype):
    """An id outside the pool is range-checked: the slots of that page read as zero rows, nothing is written there."""
    from paper_2511_06029_b200 import binding
    st = ref.State(1, 2, 8, 2, 128, 320, torch.tensor([200, 200]).view(1, 2, 1).expand(1, 2, 2), dtype, page=16, seed=1)
    ch = ref.make_chunk(st, [20, 30])
    gc = st.device_cache()
    table = gc.page_table.clone()
    table[0, 0, 1, 3] = gc.c.n_pages + 7                             # cached slots 48..63
    table[0, 1, 0, 13] = -5                                          # new slots 208..223
    bad = binding.Cache(8, gc.k, gc.v, gc.rel, gc.pos, gc.len, table, k_scale=st.k_scale, v_scale=st.v_scale)
    out, lse = run_device(ctx, st, bad, ch, [0.1], 0.9)
    s, item = ctx.poll_status()
    assert s == binding.ERR_PAGE and item in (1, 2)
    st.k.view(st.raw)[0, 0, 1, 48:64] = 0
    st.v.view(st.raw)[0, 0, 1, 48:64] = 0
    zero = {**ch, "k_new": ch["k_new"].clone(), "v_new": ch["v_new"].clone()}
    zero["k_new"][0, 20 + 8:20 + 24, 0] = 0                          # tokens 8..23 of sequence 1 sit on slots 208..223
    zero["v_new"][0, 20 + 8:20 + 24, 0] = 0
    o, z, tol_o, tol_z, tol_r, _ = ref.chunk_attend(st, zero, [0.1], 0.9)
    assert bool(((out.cpu().double() - o).abs() <= tol_o).all()) and bool(((lse.cpu().double() - z).abs() <= tol_z).all())
    live = torch.arange(320) < st.len[..., None]
    assert bool(((gc.rel.cpu().double() - st.rel).abs() <= tol_r)[live].all())
    assert torch.equal(gc.len.cpu(), st.len) and torch.equal(gc.pos.cpu(), st.pos)


def test_other_stream_graph_and_two_calls(ctx):
    """On a stream of its own, captured and replayed, and the same call twice: the same bits."""
    for dtype in (F32, BF16, E4M3):
        st = ref.State(1, 2, 32, 8, 128, 700, torch.tensor([400, 60]).view(1, 2, 1).expand(1, 2, 8), dtype, page=0, seed=3)
        ch = ref.make_chunk(st, [40, 200])
        x = {k: dev(ch[k]) for k in ("q", "k_new", "v_new", "token_pos", "chunk_start")}
        base = st.device_cache()

        def fresh():
            from paper_2511_06029_b200 import binding
            return binding.Cache(32, base.k.clone(), base.v.clone(), base.rel.clone(), base.pos.clone(), base.len.clone(), k_scale=st.k_scale, v_scale=st.v_scale)

        def call(gc, out, lse):
            ctx.chunk_attend(gc, 0, 1, x["chunk_start"], ch["max_chunk"], x["q"], x["k_new"], x["v_new"], x["token_pos"], [0.1], 0.9, out, lse)

        def buffers():
            return torch.zeros_like(x["q"]), torch.zeros(ch["q"].shape[:3], device="cuda")

        a, b, c = fresh(), fresh(), fresh()
        oa, ob, oc = buffers(), buffers(), buffers()
        call(a, *oa)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(b, *ob)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(c, *oc)
        assert torch.equal(c.len, base.len)
        graph.replay()
        assert ctx.poll_status()[0] == 0
        live = torch.arange(700, device="cuda") < a.len[..., None]
        for y, o in ((b, ob), (c, oc)):
            assert torch.equal(oa[0], o[0]) and torch.equal(oa[1], o[1]) and torch.equal(a.len, y.len)
            assert torch.equal(a.rel[live], y.rel[live])
        c.len.copy_(base.len)
        c.rel.copy_(base.rel)
        oc[0].zero_()
        graph.replay()                                               # again, from the same state
        torch.cuda.synchronize()
        assert torch.equal(oa[0], oc[0]) and torch.equal(a.rel[live], c.rel[live])
        del graph


def test_graph_outlives_growth_of_the_scratch():
    """A captured call is replayed after a larger one has made the context's scratch grow."""
    from paper_2511_06029_b200 import binding
    own = binding.Context(0)
    st = ref.State(1, 1, 8, 2, 128, 300, 100, BF16, page=0, seed=3)
    ch = ref.make_chunk(st, [30])
    x = {k: dev(ch[k]) for k in ("q", "k_new", "v_new", "token_pos", "chunk_start")}
    gc = st.device_cache()
    length, rel = gc.len.clone(), gc.rel.clone()
    out = torch.zeros_like(x["q"])

    def call():
        own.chunk_attend(gc, 0, 1, x["chunk_start"], ch["max_chunk"], x["q"], x["k_new"], x["v_new"], x["token_pos"], [0.1], 0.9, out)

    call()
    want, want_rel = out.clone(), gc.rel.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    big = ref.State(2, 4, 32, 8, 128, 4000, 100, BF16, page=0, seed=4)
    many = ref.make_chunk(big, [3000, 1, 2000, 7])
    y = {k: dev(many[k]) for k in ("q", "k_new", "v_new", "token_pos", "chunk_start")}
    own.chunk_attend(big.device_cache(), 0, 2, y["chunk_start"], many["max_chunk"], y["q"], y["k_new"], y["v_new"], y["token_pos"], [0.1, 0.1], 0.9,
                     torch.zeros_like(y["q"]))
    filler = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")  # what a freed buffer could have become
    gc.len.copy_(length)
    gc.rel.copy_(rel)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert own.poll_status()[0] == 0
    assert torch.equal(out, want) and torch.equal(gc.rel[0, 0, :, :130], want_rel[0, 0, :, :130])
    assert bool((filler == 255).all())
    del graph


def test_refusals(ctx):
    from paper_2511_06029_b200 import binding
    st = ref.State(1, 2, 8, 2, 64, 130, 60, BF16, seed=1)
    gc = st.device_cache()
    ch = ref.make_chunk(st, [2, 3])
    x = {k: dev(ch[k]) for k in ("q", "k_new", "v_new", "token_pos", "chunk_start")}
    out = torch.zeros_like(x["q"])

    def call(start=x["chunk_start"], mx=3, q=x["q"], k=x["k_new"], v=x["v_new"], tp=x["token_pos"], gamma=0.9, layers=(0, 1), n=5,
             scale=0.1, mod=None, out=out, rot=None):
        sc = (ctypes.c_float * 1)(scale)
        p = binding._dp
        return ctx.lib.lethe_chunk_attend(ctx.h, ctypes.byref(gc.c), layers[0], layers[1], p(start), n, mx, p(q), p(k), p(v), p(tp), sc, gamma,
                                          None if mod is None else ctypes.byref(mod), None if rot is None else ctypes.byref(rot), p(out), None, binding._stream(0))

    I, U = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    M = binding.lethe_score_mod
    assert call(start=None) == I and call(q=None) == I and call(out=None) == I and call(k=None) == I and call(v=None) == I and call(tp=None) == I
    assert call(mx=0) == I and call(n=-1) == I and call(gamma=0.0) == I and call(gamma=1.5) == I and call(layers=(0, 2)) == I and call(layers=(1, 1)) == I
    assert call(scale=float("nan")) == I and call(mod=M(-1.0, 0, None, None, None)) == I and call(mod=M(float("nan"), 0, None, None, None)) == I
    assert call(mod=M(0.0, -1, None, None, None)) == I and call(mod=M(1e-6, 0, None, None, None)) == I
    assert call(out=x["q"]) == I and call(out=x["q"].view(-1)[64:]) == I
    assert call(k=None, v=None, tp=None, mod=M(0.0, 5, None, None, None)) == I
    q1 = x["q"].view(-1)[1:]
    assert call(q=q1) == I
    f = (ctypes.c_double * 32)(*[0.1] * 32)
    ax = (ctypes.c_int32 * 32)(*[0] * 32)
    R = binding.lethe_rotary
    apos = torch.zeros((1, 5), dtype=torch.int32, device="cuda")
    good = dict(rot_dim=64, style=0, n_axes=1, pair_axis=ax, pair_freq=f, axis_pos=apos.data_ptr())
    for bad in (dict(rot_dim=66), dict(rot_dim=3), dict(rot_dim=0), dict(style=2), dict(n_axes=0), dict(n_axes=5), dict(axis_pos=None),
                dict(pair_axis=(ctypes.c_int32 * 32)(*[1] * 32)), dict(pair_freq=(ctypes.c_double * 32)(*[float("nan")] * 32)),
                dict(pair_freq=(ctypes.c_double * 32)(*[7.0] * 32))):
        assert call(rot=R(**{**good, **bad})) == I, bad
    assert torch.equal(gc.len.cpu(), st.len) and bool((out == 0).all())
    assert call(n=0) == binding.OK and call(n=0, start=None, q=None, out=None) == binding.OK
    assert ctx.poll_status()[0] == 0
    assert call() == binding.OK and call(rot=R(**good)) == binding.OK


def test_a_run_of_steps(ctx):
    """As a server uses it: rotate and append a prompt in two chunks, decode, prune, verify drafted tokens, decode again; the chunk
    calls against the reference from the same state each time."""
    from paper_2511_06029_b200 import binding
    L, B, Hq, Hkv, D, cap = 2, 2, 8, 2, 128, 640
    st = ref.State(L, B, Hq, Hkv, D, cap, 0, BF16, page=16, seed=1)
    gc = st.device_cache()
    scale, gamma = [0.09, 0.06], 0.98
    axes = [p * 3 // 64 for p in range(64)]
    freq = [10000.0 ** (-p / 64) for p in range(64)]
    done = [0, 0]

    def chunk(new, seed, **kw):
        ch = ref.make_chunk(st, new, seed=seed, first_pos=list(done))
        t = ch["token_pos"]
        axis_pos = torch.stack([t, t // 9, t % 9]).to(torch.int32)
        rot = binding.Rotary(axes, freq, axis_pos.cuda())
        out, lse = run_device(ctx, st, gc, ch, scale, gamma, True, kw, rotary=rot)
        # the rotated tensors as lethe_rotate gives them
        q, k = torch.empty_like(ch["q"], device="cuda"), torch.empty_like(ch["k_new"], device="cuda")
        ctx.rotate(rot, ch["q"].cuda(), ch["k_new"].cuda(), q, k)
        ch["q"], ch["k_new"] = q.cpu(), k.cpu()
        st.rel = st.rel.float()
        want = ref.chunk_attend(st, ch, scale, gamma, **kw)
        assert ctx.poll_status()[0] == 0
        compare(st, gc, ch, out, lse, want)
        pull()
        for b in range(B):
            done[b] += new[b]

    def pull():
        """The reference goes on from the device's state."""
        k, v = st.rows_of(gc)
        st.k, st.v = k.view(st.dtype), v.view(st.dtype)
        st.rel, st.pos, st.len = gc.rel.cpu(), gc.pos.cpu(), gc.len.cpu()

    def decode(steps, seed):
        g = torch.Generator().manual_seed(seed)
        for _ in range(steps):
            q = torch.randn((L, B, Hq, D), generator=g).to(BF16).cuda()
            kv = torch.randn((2, L, B, Hkv, D), generator=g).to(BF16).cuda()
            tp = torch.tensor(done, dtype=torch.int32, device="cuda")
            ctx.decode_attend(gc, 0, L, q, kv[0], kv[1], tp, scale, gamma, torch.empty_like(q))
            for b in range(B):
                done[b] += 1
        pull()

    chunk([200, 90], 1)
    chunk([130, 0], 2, prefix_len=torch.tensor([210, 0], dtype=torch.int32))
    decode(5, 3)
    S = torch.zeros((L, B), device="cuda")
    bud = torch.zeros((L, B), dtype=torch.int32, device="cuda")
    ctx.estimate_sparsity(gc, S)
    ctx.alloc_budgets(S, torch.tensor([2 * 150, 2 * 60], dtype=torch.int64, device="cuda"), 20, bud)
    ctx.rasr_prune(gc, bud, 16, 4)
    pull()
    assert int(st.len.max()) < 335
    chunk([4, 4], 5, softcap=30.0, window=150)
    decode(3, 6)
    chunk([1, 1], 7)


@pytest.mark.parametrize("dtype,gain", [(BF16, 3), (E4M3, 1.5), (E4M3, 3)])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("T", [1, 4, 40])
def test_several_tiles_per_cta(ctx, dtype, gain, page, T):
    """Enough items that a CTA walks several key tiles of a unit, with a partly filled last tile: the clearing of what lies behind
    the last slot must not touch a tile that is still on its way.  A few longer keys move the row maxima; three times as long they
    leave e4m3's range and are NaN, which has to come out as NaN."""
    B, Hq, Hkv, D = 12, 32, 8, 128
    lens = torch.tensor([900 + 37 * b for b in range(B)])
    st = ref.State(1, B, Hq, Hkv, D, 1408, lens.view(1, B, 1).expand(1, B, Hkv), dtype, page=page, seed=T)
    g = torch.Generator().manual_seed(T)
    anchors = torch.rand((1, B, Hkv, 1408), generator=g) < 0.01
    k = st.k.float()
    k[anchors] *= gain
    st.k = k.to(dtype)
    ch = ref.make_chunk(st, [T] * B)
    for _ in range(2):
        check(ctx, copy.deepcopy(st), ch)


@pytest.mark.parametrize("dtype,page", [(BF16, 0), (BF16, 16), (E4M3, 0)])
@pytest.mark.parametrize("new", [[1, 1], [300, 20]])
def test_waits_run_out_and_the_context_recovers(ctx, dtype, page, new):
    """With a poll limit of one the tensor-core kernels' first hand-offs give up: the launches return, LETHE_ERR_TIMEOUT is recorded,
    and the next ordinary call on the same context is right."""
    from paper_2511_06029_b200 import binding
    st = ref.State(1, 2, 32, 8, 128, 1600, 1200, dtype, page=page, seed=3)
    ch = ref.make_chunk(st, new)
    broken = st.device_cache()
    try:
        ctx.set_wait_limit(1)
        run_device(ctx, st, broken, ch, [0.09], 0.9)
        assert ctx.poll_status()[0] == binding.ERR_TIMEOUT
        assert ctx.poll_status()[0] == 0
    finally:
        ctx.set_wait_limit(0)
    check(ctx, st, ch, scale=[0.09], gamma=0.9)


def test_two_contexts_on_two_streams(ctx):
    """Calls through two contexts may overlap on the device: each has scratch of its own."""
    from paper_2511_06029_b200 import binding
    other = binding.Context(0)
    st = ref.State(1, 2, 32, 8, 128, 3000, torch.tensor([2500, 900]).view(1, 2, 1).expand(1, 2, 8), BF16, seed=8)
    ch = ref.make_chunk(st, [120, 300])
    caches = [st.device_cache() for _ in range(6)]
    x = {k: dev(ch[k]) for k in ("q", "k_new", "v_new", "token_pos", "chunk_start")}
    outs = [(torch.zeros_like(x["q"]), torch.zeros(ch["q"].shape[:3], device="cuda")) for _ in caches]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i, (gc, (o, z)) in enumerate(zip(caches, outs)):
        with torch.cuda.stream(streams[i % 2]):
            (ctx, other)[i % 2].chunk_attend(gc, 0, 1, x["chunk_start"], ch["max_chunk"], x["q"], x["k_new"], x["v_new"], x["token_pos"], [0.09], 0.9, o, z)
    torch.cuda.synchronize()
    assert ctx.poll_status()[0] == 0 and other.poll_status()[0] == 0
    live = torch.arange(3000, device="cuda") < caches[0].len[..., None]
    for gc, (o, z) in zip(caches[1:], outs[1:]):
        assert torch.equal(o, outs[0][0]) and torch.equal(z, outs[0][1]) and torch.equal(gc.rel[live], caches[0].rel[live])
    other.close()


def test_empty_and_padded_batches(ctx):
    """Sequences without tokens between others, all of them empty with padding rows around, one sequence only."""
    for dtype in (F32, BF16, E4M3):
        st = ref.State(1, 5, 8, 2, 64, 200, torch.tensor([0, 50, 100, 7, 150]).view(1, 5, 1).expand(1, 5, 2), dtype, seed=3)
        check(ctx, copy.deepcopy(st), ref.make_chunk(st, [0, 3, 0, 0, 50], lead=1, trail=2))
        ch = ref.make_chunk(st, [0, 0, 0, 0, 0], lead=3, trail=1)
        check(ctx, copy.deepcopy(st), ch)


def test_long_chunk_of_many_units(ctx):
    """A chunk of several units per item on both sides of every split, odd group size, against the reference."""
    st = ref.State(1, 1, 14, 2, 128, 1500, 333, BF16, page=16 if 1500 % 16 == 0 else 0, seed=5)
    check(ctx, st, ref.make_chunk(st, [1111]))


@pytest.mark.parametrize("D,softcap,dtype", [(64, 0.0, BF16), (64, 20.0, BF16), (128, 0.0, BF16), (128, 0.0, E4M3)])
@pytest.mark.parametrize("short", [(20, 9), (3, 2), (3, 20)])        # one row tile each, or at most 16 rows
def test_single_tile_units_after_pairs(ctx, D, softcap, dtype, short):
    """Units of two row tiles with several key tiles, each followed by two of one row tile and one key tile (in which a CTA's second
    softmax group has nothing to do), so that most CTAs walk pair, short, short.  The second group must not run ahead of the first."""
    L, groups, Hq = 2, 100, 4
    new = [64, *short] * groups
    B = len(new)
    cached = torch.tensor([600, 100, 3] * groups).view(1, B, 1).expand(L, B, 1)
    st = ref.State(L, B, Hq, 1, D, 664, cached, dtype, seed=D)
    ch = ref.make_chunk(st, new, seed=4)
    first = st.device_cache()
    scale = [0.1, 0.07]
    out, lse = run_device(ctx, st, first, ch, scale, 0.97, mod_kw={"softcap": softcap} if softcap else None)
    for _ in range(8):                                               # the same bits however the warps meet
        again = st.device_cache()
        o, z = run_device(ctx, st, again, ch, scale, 0.97, mod_kw={"softcap": softcap} if softcap else None)
        assert torch.equal(o, out) and torch.equal(z, lse) and torch.equal(torch.nan_to_num(again.rel), torch.nan_to_num(first.rel))
    assert ctx.poll_status()[0] == 0
    compare(st, first, ch, out, lse, ref.chunk_attend(st, ch, scale, 0.97, softcap=softcap))


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("T", [3, 40])
@pytest.mark.parametrize("sloped", [False, True])
def test_nan_comes_through_the_cap(ctx, dtype, T, sloped):
    """Capped scores: a NaN query makes its own row NaN and what that row sees NaN in the relevance; a NaN key makes the rows NaN that see
    it.  Everything else is as without it."""
    n, at, head = 300, T // 2, 5                                     # a token in the middle, a head of the second group
    Hq, Hkv, D = 8, 2, 128
    scale, gamma = [0.2], 0.97
    kw = {"softcap": 20.0}
    if sloped:
        kw["slopes"] = torch.tensor([2.0 ** (-0.8 * (h + 1)) for h in range(Hq)])

    def run(where):
        st = ref.State(1, 1, Hq, Hkv, D, n + T, n, dtype, seed=11)
        ch = ref.make_chunk(st, [T], seed=12)
        want = ref.chunk_attend(copy.deepcopy(st), ch, scale, gamma, **kw)
        clean = copy.deepcopy(st)
        ref.chunk_attend(clean, ch, scale, gamma, **kw)
        ch[where] = ch[where].clone()
        ch[where][0, at, head if where == "q" else 1, 3] = float("nan")
        gc = st.device_cache()
        out, lse = run_device(ctx, st, gc, ch, scale, gamma, True, kw)
        assert ctx.poll_status()[0] == 0
        o, z, tol_o, tol_z, tol_r, _ = want
        hit = torch.zeros((1, T, Hq), dtype=torch.bool)
        if where == "q":
            hit[0, at, head] = True
        else:
            hit[0, at:, 4:] = True
        gone = torch.zeros((1, 1, Hkv, n + T), dtype=torch.bool)
        gone[0, 0, 1, :n + at + 1 if where == "q" else n + T] = True
        out, lse, rel = out.cpu().double(), lse.cpu().double(), gc.rel.cpu().double()
        assert torch.equal(torch.isnan(lse), hit) and torch.equal(torch.isnan(rel), gone)
        assert torch.equal(torch.isnan(out), hit[..., None].expand_as(out))
        assert bool(((out - o).abs() <= tol_o)[~hit].all()) and bool(((lse - z).abs() <= tol_z)[~hit].all())
        assert bool(((rel - clean.rel).abs() <= tol_r)[~gone].all())

    run("q")
    run("k_new")


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
def test_slopes_over_the_whole_range_of_positions(ctx, dtype):
    """Distances of up to 2^32 - 1: tiny slopes, half of the keys at the lower end of int32, the others near the tokens at its upper end."""
    st = ref.State(1, 1, 4, 1, 64, 300, 200, dtype, seed=2)
    st.pos[...] = torch.arange(300, dtype=torch.int32) - 2 ** 31
    st.pos[..., 100:] = 2 ** 31 - 1000 + torch.arange(200, dtype=torch.int32)
    ch = ref.make_chunk(st, [20], first_pos=[2 ** 31 - 30])
    check(ctx, st, ch, slopes=torch.tensor([2.0 ** -30, 2.0 ** -31, 2.0 ** -32, 2.0 ** -40]))


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("sloped", [False, True])
def test_capped_scores_do_not_depend_on_what_is_not_seen(ctx, dtype, T, sloped):
    """The same bits whatever lies behind the last slot and in rows that are nobody's tokens."""
    Hq, Hkv, D = 8, 2, 128
    results = []
    for junk in (0.0, float("nan"), 300.0):
        st = ref.State(1, 1, Hq, Hkv, D, 400, 301, dtype, seed=5, junk=junk, k_scale=[0.02], v_scale=[0.015])
        st.rel[..., 301:] = 0
        ch = ref.make_chunk(st, [T], seed=6, trail=30, first_pos=[1000])
        ch["q"][:, T:] = junk
        kw = {"softcap": 30.0}
        if sloped:
            kw["slopes"] = torch.tensor([2.0 ** (-0.8 * (h + 4)) for h in range(Hq)])
        gc = st.device_cache()
        out, lse = run_device(ctx, st, gc, ch, [0.09], 0.97, True, kw)
        assert ctx.poll_status()[0] == 0
        results.append((out[:, :T].clone(), lse[:, :T].clone(), gc.rel[..., :301 + T].clone()))
    for other in results[1:]:
        for x, y in zip(results[0], other):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [2, 40])
@pytest.mark.parametrize("sloped", [False, True])
def test_far_score_leaves_its_neighbours_exact(ctx, dtype, T, sloped):
    """A cap of 1e5 and one key in sixteen whose scores are near minus the cap: it weighs nothing, and the others have to be as exact as
    scores of their own size are, not as the cap's size allows."""
    Hq, Hkv, D, n, cap, s = 8, 2, 128, 320, 1e5, 0.0884
    st = ref.State(1, 1, Hq, Hkv, D, n, n, dtype, seed=5)
    far = torch.arange(n) % 16 == 3
    st.k[..., 0] = 0.0
    st.k[0, 0, :, far, 0] = -56576.0                                 # exact in bf16
    ch = ref.make_chunk(st, [T], seed=6, first_pos=[1000])
    ch["q"][..., 0] = 16.0                                           # scores of -8e4, tanh(-0.8) of the cap
    slopes = torch.tensor([2.0 ** (-h - 4) for h in range(Hq)]) if sloped else torch.zeros(Hq)
    gc = st.device_cache()
    out, lse = run_device(ctx, st, gc, ch, [s], 0.97, False, {"softcap": cap, **({"slopes": slopes} if sloped else {})})
    assert ctx.poll_status()[0] == 0
    u, s32 = 2.0 ** -23, float(torch.tensor(s, dtype=torch.float32))
    rel, rel_err = st.rel.double() * 0.97 ** T, st.rel.double() * 0.97 ** T * (8 + 4 * T * abs(math.log2(0.97))) * u
    for h in range(Hkv):
        K, V = st.k[0, 0, h, ~far].double(), st.v[0, 0, h, ~far].double()
        for g in range(Hq // Hkv):
            hq = h * (Hq // Hkv) + g
            q = ch["q"][0, :, hq].double()
            x = cap * torch.tanh(q @ K.T * s32 / cap)
            # the product, accumulated in fp32; the cap: eight half steps of the argument, the polynomial and its factors, relative to the score
            err = (q.abs() @ K.abs().T * s32) * (D + 4) * u + x.abs() * (2.0 ** -21 + 4 * u)
            bias = float(slopes[hq]) * (ch["token_pos"].long()[:, None] - st.pos[0, 0, h, ~far].long()[None]).abs().double()
            x, err = x - bias, err + (bias + (x - bias).abs()) * 4 * u
            z = torch.logsumexp(x, 1)
            e_z = err.amax(1) + (z.abs() + 8) * 4 * u + (n / 16 + 16) * u   # as in chunk_reference.py
            assert bool(((lse[0, :, hq].cpu().double() - z).abs() <= e_z).all())
            p = torch.exp(x - z[:, None])
            e_p = 2 * (2 * err.amax(1) + (z.abs() + 8) * 4 * u + (n / 16 + 16) * u)
            half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
            o = p @ V
            tol = (p @ V.abs()) * (e_p + (half if dtype == BF16 else 0) + (n / 16 + 16) * u)[:, None] + o.abs() * half
            assert bool(((out[0, :, hq].cpu().double() - o).abs() <= tol).all())
            wt = 0.97 ** (T - 1 - torch.arange(T)).double()
            rel[0, 0, h, ~far] += wt @ p
            rel_err[0, 0, h, ~far] += (wt * (e_p + 4 * u * T * abs(math.log2(0.97)) + (T * Hq / 16 + 16) * u)) @ p
    rel_err += rel.abs() * (8 + 4 * T * abs(math.log2(0.97))) * u
    assert bool(((gc.rel.cpu().double() - rel).abs() <= rel_err + 1e-30).all())


def test_gamma_is_checked_as_a_double(ctx):
    """What fp32 would round into or out of (0, 1]."""
    from paper_2511_06029_b200 import binding
    st = ref.State(1, 1, 8, 2, 64, 130, 60, BF16, seed=1)
    gc = st.device_cache()
    ch = ref.make_chunk(st, [20])
    x = {k: dev(ch[k]) for k in ("q", "k_new", "v_new", "token_pos", "chunk_start")}
    out = torch.zeros_like(x["q"])

    def call(gamma):
        p = binding._dp
        return ctx.lib.lethe_chunk_attend(ctx.h, ctypes.byref(gc.c), 0, 1, p(x["chunk_start"]), 20, 20, p(x["q"]), p(x["k_new"]), p(x["v_new"]),
                                          p(x["token_pos"]), (ctypes.c_float * 1)(0.1), gamma, None, None, p(out), None, binding._stream(0))

    for bad in (1.0 + 1e-9, 0.0, -1e-60, float("nan")):
        assert call(bad) == binding.ERR_INVALID_ARG
    assert torch.equal(gc.len.cpu(), st.len) and bool((out == 0).all())
    assert call(1e-60) == binding.OK and ctx.poll_status()[0] == 0
    ref.chunk_attend(st, ch, [0.1], 1e-60)
    assert torch.equal(gc.len.cpu(), st.len)
    assert torch.allclose(gc.rel.cpu()[..., :80].double(), st.rel[..., :80], rtol=1e-4, atol=1e-30)  # only the last token's weights are left
