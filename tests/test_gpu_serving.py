"""The operators of a decode step on the GPU against their formulas in 64 bits (tests/serving_reference.py has the
bounds and where they come from)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests import serving_reference as R  # noqa: E402
from tests.test_serving import SCALINGS  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bfloat16": torch.bfloat16, "float16": torch.float16, "float32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()


def f64(t):
    return t.detach().double().cpu().numpy()


def rand(g, *shape, dtype):
    return torch.randn(shape, generator=g).to(DT[dtype]).cuda()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def check(got, want, bound, what):
    off = np.abs(f64(got) - want)
    bad = ~(off <= bound)
    assert not bad.any(), (what, int(bad.sum()), float((off / np.maximum(bound, 1e-300)).max()), np.argwhere(bad)[0])


# ---------------------------------------------------------------- rotary positions
ROPE = [(0, 4, 2, 64, 64), (1, 32, 8, 128, 128), (7, 3, 1, 128, 96), (130, 5, 5, 64, 16), (2600, 2, 1, 256, 224),
        (9, 2, 2, 80, 80), (33, 3, 1, 20, 10), (5, 2, 1, 129, 128), (4, 1, 0, 64, 0), (3, 2, 1, 2048, 2048), (12, 0, 3, 64, 64)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shape", ROPE)
def test_rope(shape, layout, dtype):
    T, H, KV, D, rot = shape
    g = gen(T + D)
    scaling = SCALINGS[(T + rot) % len(SCALINGS)]
    rotary = serving.Rotary(D, rot_dim=rot, layout=layout, scaling=scaling)
    theta, factor = R.frequencies(rot, 10000.0, scaling)
    pos = torch.randint(0, 1 << 20, (T,), generator=g).to(torch.int32)
    q, k = rand(g, T, H, D, dtype=dtype), rand(g, T, KV, D, dtype=dtype) if KV else None
    for call, back in ((serving.rope, False), (serving.rope_grad, True)):
        got = call(q, k, pos.cuda(), rotary)
        for x, y in zip((q, k), got):
            if x is None:
                assert y is None
                continue
            want, mag = R.rotate(f64(x), pos.numpy(), theta, factor, layout, back)
            check(y, want, R.rotation_bound(want, mag, rot, dtype), (call.__name__, shape, layout))


@pytest.mark.parametrize("dtype,shift", [("bfloat16", 0), ("bfloat16", 1), ("float32", 3)])
def test_rope_strides_and_in_place(dtype, shift):
    """Views of one projection's rows, one of them off the 16-byte grid, heads before tokens, and results over the inputs."""
    T, H, KV, D = 37, 6, 2, 64
    g = gen(5)
    rotary = serving.Rotary(D)
    theta, factor = R.frequencies(D)
    pos = torch.arange(100, 100 + T, dtype=torch.int32, device="cuda")
    rows = rand(g, T, (H + 2 * KV) * D + 8 + shift, dtype=dtype)[:, shift:]
    q, k = rows[:, :H * D].unflatten(1, (H, D)), rows[:, H * D:(H + KV) * D].unflatten(1, (KV, D))
    by_head = rand(g, H, T, D, dtype=dtype).transpose(0, 1)
    for x, y in ((q, k), (by_head, k), (by_head[::2], k[::2])):
        p = pos[:x.shape[0]].contiguous()
        want = [R.rotate(f64(t), p.cpu().numpy(), theta, factor, "half") for t in (x, y)]
        got = serving.rope(x, y, p, rotary)
        for t, (w, mag) in zip(got, want):
            check(t, w, R.rotation_bound(w, mag, D, dtype), "strided")
        x2, before = x.clone(), rows.clone()
        serving.rope(x2, y, p, rotary, out_q=x2)
        assert torch.equal(x2, got[0]) and torch.equal(rows, before)
    serving.rope(q, k, pos, rotary, out_q=q, out_k=k)
    again = serving.rope(before[:, :H * D].unflatten(1, (H, D)), None, pos, rotary)[0]
    assert torch.equal(q, again) and torch.equal(rows[:, (H + KV) * D:], before[:, (H + KV) * D:])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_gradient_against_differences(layout):
    """The map is linear, so a central difference of <g, rope(x)> is the gradient up to rounding: step 1, sums of 2 x 32
    float32 products of values under 16, so 1e-4 is ample."""
    T, H, KV, D, rot = 5, 2, 1, 32, 24
    g = gen(3)
    rotary = serving.Rotary(D, rot_dim=rot, layout=layout, scaling=SCALINGS[3])
    pos = torch.tensor([0, 1, 77, 4096, 1 << 30], dtype=torch.int32, device="cuda")
    q, k = rand(g, T, H, D, dtype="float32").requires_grad_(), rand(g, T, KV, D, dtype="float32").requires_grad_()
    gq, gk = rand(g, T, H, D, dtype="float32"), rand(g, T, KV, D, dtype="float32")

    def value(x, y):
        with torch.no_grad():
            a, b = serving.rope(x, y, pos, rotary)
        return float((a.double() * gq.double()).sum() + (b.double() * gk.double()).sum())

    a, b = serving.rope(q, k, pos, rotary)
    ((a * gq).sum() + (b * gk).sum()).backward()
    for x, name in ((q, "q"), (k, "k")):
        for _ in range(24):
            at = tuple(int(torch.randint(0, n, (1,), generator=g)) for n in x.shape)
            step = torch.zeros_like(x)
            step[at] = 1.0
            up, down = [value(x + s * step, k) if name == "q" else value(q, x + s * step) for s in (1.0, -1.0)]
            assert abs((up - down) / 2 - float(x.grad[at])) < 1e-4, (name, at)
    theta, factor = R.frequencies(rot, 10000.0, SCALINGS[3])
    want, mag = R.rotate(f64(gq), pos.cpu().numpy(), theta, factor, layout, True)
    check(q.grad, want, R.rotation_bound(want, mag, rot, "float32"), "gradient")


def test_rope_refusals():
    r = serving.Rotary(64)
    q, pos = torch.zeros(3, 2, 64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    bad = [(q.double(), None, pos), (q[0], None, pos), (q, q.bfloat16(), pos), (q, q[:2], pos), (q, None, pos.long()),
           (q, None, pos[:2]), (torch.zeros(3, 2, 128, device="cuda"), None, pos),
           (torch.zeros(3, 64, 2, device="cuda").transpose(1, 2), None, pos), (q, None, pos.cpu())]
    for x, y, p in bad:
        with pytest.raises(gts.GtsError) as e:
            serving.rope(x, y, p, r)
        assert e.value.status == gts.GTS_ERR_INVALID_ARG
    with pytest.raises(gts.GtsError):
        serving.rope(q, None, pos, r, out_q=torch.zeros(2, 2, 64, device="cuda"))


# ---------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("order,page,shape", [("tokens", 16, (1, 32, 8, 128, 128)), ("heads", 48, (300, 4, 2, 128, 96)),
                                              ("tokens", 1, (17, 3, 3, 64, 64)), ("heads", 100, (2500, 2, 1, 256, 256)),
                                              ("tokens", 7, (65, 2, 1, 24, 24)), ("heads", 16, (0, 2, 1, 64, 64))])
def test_append(order, page, shape, dtype):
    T, H, KV, D, rot = shape
    g = gen(T + page)
    layout = "interleaved" if page % 2 == 0 else "half"
    scaling = SCALINGS[page % 4]
    rotary = serving.Rotary(D, rot_dim=rot, layout=layout, scaling=scaling)
    theta, factor = R.frequencies(rot, 10000.0, scaling)
    pages = T // page + 3
    cache = serving.PagedCache.empty(pages, page, KV, D, DT[dtype], order)
    cache.k.fill_(7.0)
    cache.v.fill_(-7.0)
    rows = rand(g, T, H + 2 * KV, D, dtype=dtype)
    q, k, v = rows.split([H, KV, KV], 1)
    pos = torch.randint(0, 1 << 17, (T,), generator=g).to(torch.int32).cuda()
    slots = torch.randperm(pages * page, generator=g)[:T]
    slots[::5] = -1 - slots[::5]
    want_k, want_v = f64(cache.k), f64(cache.v)
    bound_k = np.zeros_like(want_k)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = serving.append_kv(q, k, v, pos, slots.cuda(), rotary, cache, status=status)
    w, mag = R.rotate(f64(q), pos.cpu().numpy(), theta, factor, layout)
    check(got, w, R.rotation_bound(w, mag, rot, dtype), "q")
    w, mag = R.rotate(f64(k), pos.cpu().numpy(), theta, factor, layout)
    b = R.rotation_bound(w, mag, rot, dtype)
    for t, s in enumerate(slots.tolist()):
        if s >= 0:
            want_k[s // page, s % page], bound_k[s // page, s % page] = w[t], b[t]
            want_v[s // page, s % page] = f64(v[t])
    check(cache.k, want_k, bound_k, "k cache")
    check(cache.v, want_v, np.zeros_like(want_v), "v cache")
    assert int(status) == 0


def test_append_reports_slots_beyond_the_cache():
    rotary, cache = serving.Rotary(64), serving.PagedCache.empty(2, 16, 1, 64, torch.float16)
    cache.k.fill_(3.0)
    cache.v.fill_(3.0)
    x = torch.ones(3, 1, 64, dtype=torch.float16, device="cuda")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    slots = torch.tensor([31, 32, 1 << 40], dtype=torch.int64, device="cuda")
    q = serving.append_kv(x, x, x, pos, slots, rotary, cache, status=status)
    assert int(status) == gts.GTS_ERR_INVALID_PARAMS and torch.equal(q, x)
    assert float(cache.k[1, 15].sum()) == 64.0 and float((cache.k == 3.0).sum()) == 31 * 64
    serving.append_kv(x, x, x, pos, slots, rotary, cache)  # the same without a status


def test_append_refusals():
    rotary, cache = serving.Rotary(64), serving.PagedCache.empty(2, 16, 2, 64, torch.float16)
    x = torch.ones(3, 2, 64, dtype=torch.float16, device="cuda")
    pos, slots = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.arange(3, device="cuda")
    for a in [(x.float(), x, x, pos, slots), (x, x[:, :1], x, pos, slots), (x, x, x[:2], pos, slots),
              (x, x, x, pos.long(), slots), (x, x, x, pos, slots.int()), (x, x, x, pos, slots[:2])]:
        with pytest.raises(gts.GtsError) as e:
            serving.append_kv(*a, rotary, cache)
        assert e.value.status == gts.GTS_ERR_INVALID_ARG
    with pytest.raises(gts.GtsError):
        serving.append_kv(x, x, x, pos, slots, serving.Rotary(128), cache)


# ---------------------------------------------------------------- attention
def problem(seed, H, KV, D, page, order, dtype, prefix, lens, new, spread=1.0, rubbish=float("nan")):
    """Inputs on the GPU; whatever no query sees in the cache is rubbish."""
    g = gen(seed)
    B, lens = len(lens), np.array(lens, np.int64)
    per, n_prefix = max(1, -(-max([1, *lens]) // page)), -(-prefix // page)
    held = -(-lens // page)
    ids = torch.randperm(n_prefix + int(held.sum()) + 2, generator=g).numpy().astype(np.int32)
    table, at = np.full((B, per), -5, np.int32), n_prefix
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    cache = serving.PagedCache.empty(len(ids), page, KV, D, DT[dtype], order)
    seen = torch.zeros(len(ids), page, dtype=torch.bool)
    for j in range(prefix):
        seen[ids[j // page], j % page] = True
    for b in range(B):
        for j in range(lens[b]):
            seen[table[b, j // page], j % page] = True
    for c, scale in ((cache.k, spread), (cache.v, 1.0)):
        x = torch.randn(len(ids), page, KV, D, generator=g) * scale
        x[~seen] = rubbish
        c.copy_(x.to(DT[dtype]))
    q = rand(g, B, new, H, D, dtype=dtype)
    return dict(q=q, cache=cache, prefix_pages=torch.from_numpy(ids[:n_prefix].copy()).cuda(), prefix_len=prefix,
                page_table=torch.from_numpy(table).cuda(), lens=torch.from_numpy(lens.astype(np.int32)).cuda())


def reference(p, scale, dtype):
    c = p["cache"]
    return R.attention(f64(p["q"]), f64(c.k), f64(c.v), p["prefix_pages"].cpu().numpy(), p["prefix_len"],
                       p["page_table"].cpu().numpy(), p["lens"].cpu().numpy(), scale, dtype)


def check_attention(p, dtype, scale=None, **kw):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = serving.prefix_attention(**p, scale=scale, status=status, **kw)
    s = p["q"].shape[-1] ** -0.5 if scale is None else scale
    w_out, w_lse, b_out, b_lse = reference(p, s, dtype)
    check(out, w_out, b_out, "out")
    none = np.isneginf(w_lse)
    got = f64(lse)
    assert np.array_equal(np.isneginf(got), none) and np.all(f64(out)[none] == 0)
    off = np.abs(np.where(none, 0, got) - np.where(none, 0, w_lse))
    assert np.all(off <= b_lse), (float((off / b_lse).max()))
    assert int(status) == 0
    return out, lse


LENGTHS = [[0], [1], [0, 1, 2, 15, 16, 17], [127, 128, 129, 0], [300, 1, 64, 65, 1000]]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("prefix", [0, 1, 16, 127, 128, 129, 700])
@pytest.mark.parametrize("lens", LENGTHS)
def test_attention_lengths(lens, prefix, D, dtype):
    n = prefix + len(lens)
    check_attention(problem(n, 8, 2, D, (16, 48, 128, 100)[n % 4], ("tokens", "heads")[n % 2], dtype, prefix, lens, 1), dtype)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("heads", [(1, 1), (4, 4), (14, 2), (32, 8), (16, 1), (40, 1), (130, 1)])
@pytest.mark.parametrize("new,lens", [(2, [0, 1, 2, 40]), (5, [3, 5, 200]), (16, [16, 33]), (33, [0, 20, 150]),
                                      (70, [100, 69])])
def test_attention_new_tokens(new, lens, heads, dtype):
    """Drafts and chunks: causal among the new tokens, rows that see nothing where a sequence holds fewer than them."""
    for prefix in (0, 200):
        check_attention(problem(new + heads[0], *heads, 64, 32, "tokens", dtype, prefix, lens, new), dtype)


@pytest.mark.parametrize("page", [1, 2, 3, 8, 16, 24, 32, 64, 100, 128, 192, 256, 1000])
@pytest.mark.parametrize("order", ["tokens", "heads"])
def test_attention_pages(page, order):
    check_attention(problem(page, 16, 2, 128, page, order, "bfloat16", 515, [130, 3, 77, 256], 1), "bfloat16")


@pytest.mark.parametrize("B,prefix", [(40, 1500), (64, 3000), (129, 640), (256, 1025)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_many_rows(B, prefix, D):
    """Batches whose rows fill several tiles of the prefix."""
    lens = [(7 * b) % 90 for b in range(B)]
    check_attention(problem(B, 8, 2, D, 64, "tokens", "bfloat16", prefix, lens, 1), "bfloat16")
    check_attention(problem(B, 4, 1, D, 16, "heads", "float16", prefix, [x + 3 for x in lens], 3), "float16")


@pytest.mark.parametrize("spread", [0.0, 12.0, 60.0])
@pytest.mark.parametrize("B", [2, 48])
def test_attention_spread_of_scores(spread, B):
    """Equal weights, and scores of which a few take all the weight and the maximum keeps rising."""
    lens = [100 + b for b in range(B)]
    for dtype in ("bfloat16", "float16"):
        check_attention(problem(3, 8, 1, 128, 16, "tokens", dtype, 1000, lens, 1, spread=spread), dtype)


@pytest.mark.parametrize("B", [2, 48])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_attention_scales(scale, B):
    check_attention(problem(4, 8, 1, 64, 16, "tokens", "bfloat16", 600, [50] * B, 1), "bfloat16", scale=scale)


@pytest.mark.parametrize("B", [2, 48])
@pytest.mark.parametrize("rubbish", [float("inf"), -float("inf"), -65504.0])
def test_attention_rubbish_in_the_rest_of_pages(rubbish, B):
    check_attention(problem(4, 8, 1, 128, 48, "tokens", "float16", 601, [50 + b for b in range(B)], 2, rubbish=rubbish),
                    "float16")


@pytest.mark.parametrize("B", [3, 48])
def test_attention_of_a_nan_key_is_nan_for_those_who_see_it(B):
    p = problem(4, 8, 2, 64, 16, "tokens", "bfloat16", 200, [60] * B, 1, rubbish=0.0)
    page = int(p["page_table"][1, 2])
    p["cache"].v[page, 3, 0, 5] = float("nan")
    out, lse = serving.prefix_attention(**p)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[1, 0, :4, 5] = True
    assert torch.equal(torch.isnan(out), bad) and not torch.isnan(lse).any()
    p["cache"].k[page, 3, 0, 5] = float("nan")
    out, lse = serving.prefix_attention(**p)
    bad[1, 0, :4, :] = True
    assert torch.equal(torch.isnan(out), bad) and torch.equal(torch.isnan(lse), bad[..., 0])


@pytest.mark.parametrize("B", [2, 48])
def test_attention_strides_and_outputs(B):
    """Queries and results with heads before tokens and on an 8-byte grid, the caller's own buffers, a larger workspace."""
    p = problem(6, 8, 2, 64, 16, "tokens", "bfloat16", 300, [40 + b % 9 for b in range(B)], 3)
    want = serving.prefix_attention(**p)
    wide = torch.zeros(B, 8, 3, 64 + 4, dtype=torch.bfloat16, device="cuda")
    q = wide[..., 4:].transpose(1, 2)
    q.copy_(p["q"])
    out = torch.full((B, 8, 3, 64 + 1), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(B, 3, 8, device="cuda")
    ws = torch.full((1 << 26,), 255, dtype=torch.uint8, device="cuda")
    got = serving.prefix_attention(**{**p, "q": q}, out=out[..., :64].transpose(1, 2), lse=lse, workspace=ws)
    assert got[1] is lse and torch.equal(got[0], want[0]) and torch.equal(lse, want[1])
    assert torch.all(out[..., 64] == 9.0)
    # a cache whose tokens are not on the 16-byte grid
    c = p["cache"]
    k, v = (torch.zeros(*c.k.shape[:3], 64 + 2, dtype=torch.bfloat16, device="cuda")[..., 1:65] for _ in range(2))
    k.copy_(c.k)
    v.copy_(c.v)
    p["cache"] = serving.PagedCache(k, v)
    check_attention(p, "bfloat16")


def test_attention_repeats_bit_for_bit():
    for B in (3, 64):
        p = problem(8, 8, 2, 128, 16, "tokens", "bfloat16", 3000, [100 + 3 * b for b in range(B)], 1)
        a = serving.prefix_attention(**p)
        for _ in range(5):
            b = serving.prefix_attention(**p)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_attention_on_another_stream():
    p = problem(8, 8, 2, 128, 16, "tokens", "bfloat16", 3000, [100 + 3 * b for b in range(64)], 1)
    want = serving.prefix_attention(**p)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = [serving.prefix_attention(**p, stream=s) for _ in range(4)]
    for _ in range(4):
        serving.prefix_attention(**p)
    torch.cuda.synchronize()
    for o, l in got:
        assert torch.equal(o, want[0]) and torch.equal(l, want[1])


def test_attention_in_a_graph_follows_the_lengths():
    """Lengths and pages are read on the device: a captured call serves the steps after it."""
    p = problem(8, 8, 2, 128, 16, "tokens", "bfloat16", 700, [100 + 3 * b for b in range(20)], 1)
    ws = serving.attention_workspace(p["cache"], p["q"], 700, p["page_table"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serving.prefix_attention(**p, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = serving.prefix_attention(**p, workspace=ws)
    for step in (0, 37):
        p["lens"].sub_(step)
        g.replay()
        torch.cuda.synchronize()
        want = serving.prefix_attention(**p)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_attention_beyond_32_bit_offsets():
    """Pages whose values lie past 2^31 elements and 2^32 bytes, for the append and both kinds of keys."""
    page, KV, D = 64, 4, 128
    n = (1 << 31) // (page * KV * D) + 40
    cache = serving.PagedCache.empty(n, page, KV, D, torch.bfloat16)
    g = gen(2)
    rotary = serving.Rotary(D)
    T, B = 150, 20
    H = 16
    ids = [n - 1, n - 2, n - 3, 5] + [n - 4 - b for b in range(B)]
    slots = torch.tensor([ids[t // page] * page + t % page for t in range(T)] +
                         [ids[4 + b] * page + t for b in range(B) for t in range(20)])
    k, v = rand(g, T + 20 * B, KV, D, dtype="bfloat16"), rand(g, T + 20 * B, KV, D, dtype="bfloat16")
    pos = torch.zeros(T + 20 * B, dtype=torch.int32, device="cuda")
    serving.append_kv(torch.zeros(T + 20 * B, H, D, dtype=torch.bfloat16, device="cuda"), k, v, pos, slots.cuda(), rotary, cache)
    q = rand(g, B, 1, H, D, dtype="bfloat16")
    out, lse = serving.prefix_attention(q, cache, torch.tensor(ids[:3], dtype=torch.int32, device="cuda"), T,
                                        torch.tensor(ids[4:], dtype=torch.int32, device="cuda")[:, None],
                                        torch.full((B,), 20, dtype=torch.int32, device="cuda"))
    small = np.zeros((len(ids), page, KV, D)), np.zeros((len(ids), page, KV, D))
    for c, x in zip(small, (k, v)):
        x = f64(x)
        for t in range(T):
            c[t // page, t % page] = x[t]
        for b in range(B):
            c[4 + b, :20] = x[T + 20 * b:T + 20 * b + 20]
    w_out, w_lse, b_out, b_lse = R.attention(f64(q), *small, np.arange(3), T, 4 + np.arange(B)[:, None], [20] * B, D ** -0.5,
                                             "bfloat16")
    check(out, w_out, b_out, "out")
    check(lse, w_lse, b_lse, "lse")


@pytest.mark.parametrize("B", [2, 48])
def test_attention_reports_pages_and_lengths_out_of_range(B):
    for what in ("prefix", "table_high", "table_low", "lens"):
        p = problem(8, 8, 2, 128, 16, "tokens", "bfloat16", 700, [100] * B, 1, rubbish=0.0)
        if what == "prefix":
            p["prefix_pages"][3] = p["cache"].n_pages
        elif what == "table_high":
            p["page_table"][1, 2] = 1 << 30
        elif what == "table_low":
            p["page_table"][1, 2] = -1
        else:
            p["lens"][1] = 1 << 30
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = serving.prefix_attention(**p, status=status)
        assert int(status) == gts.GTS_ERR_INVALID_PARAMS, what
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        if what != "prefix":  # the other sequences are what they were
            ok = problem(8, 8, 2, 128, 16, "tokens", "bfloat16", 700, [100] * B, 1, rubbish=0.0)
            want = serving.prefix_attention(**ok)
            assert torch.equal(out[0], want[0][0]) and torch.equal(lse[0], want[1][0])
        serving.prefix_attention(**p)  # the same without a status


def test_attention_refusals():
    p = problem(8, 8, 2, 128, 16, "tokens", "bfloat16", 70, [10, 20], 1)
    q, pages = p["q"], p["prefix_pages"]
    for kw in (dict(q=q.half()), dict(q=q[0]), dict(q=q[:, :, :7]), dict(q=q[..., :64]), dict(prefix_len=81), dict(prefix_len=-1),
               dict(prefix_pages=pages.long()), dict(prefix_pages=pages[:4]), dict(page_table=p["page_table"][:1]),
               dict(lens=p["lens"].long()), dict(lens=p["lens"][:1]), dict(lse=torch.zeros(2, 1, 8)),
               dict(status=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(out=q[:1])):
        with pytest.raises(gts.GtsError) as e:
            serving.prefix_attention(**{**p, **kw})
        assert e.value.status == gts.GTS_ERR_INVALID_ARG, kw
    with pytest.raises(gts.GtsError) as e:
        serving.prefix_attention(**p, workspace=torch.zeros(0, dtype=torch.uint8, device="cuda"))
    wide = serving.PagedCache.empty(2, 16, 1, 96, torch.bfloat16)
    with pytest.raises(gts.GtsError) as e:
        serving.prefix_attention(torch.zeros(1, 1, 1, 96, dtype=torch.bfloat16, device="cuda"), wide, pages[:0], 0,
                                 p["page_table"][:1], p["lens"][:1])
    assert e.value.status == gts.GTS_ERR_INVALID_ARG


def test_empty_batches():
    p = problem(8, 8, 2, 128, 16, "tokens", "bfloat16", 70, [10, 20], 1)
    out, lse = serving.prefix_attention(**{**p, "q": p["q"][:, :0]})
    assert out.shape == (2, 0, 8, 128) and lse.shape == (2, 0, 8)
    out, lse = serving.prefix_attention(**{**p, "q": p["q"][:0], "page_table": p["page_table"][:0], "lens": p["lens"][:0]})
    assert out.shape == (0, 1, 8, 128)
