"""The operators of prompts on the GPU against their formulas in 64 bits (tests/prompt_reference.py has the bounds and where they
come from)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests import prompt_reference as R  # noqa: E402
from tests.test_gpu_serving import DT, check, f64, gen, rand  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rows_of(lens, before=0):
    return [before + x for x in np.concatenate([[0], np.cumsum(lens)]).tolist()]


def rubbish(x, value=float("nan")):
    return x.fill_(value)


def problem(seed, lens, H, KV, D, dtype, before=0, after=0, spread=1.0):
    """Packed q, k, v (views of one projection's rows) and starts; rows of no sequence are NaN."""
    g = gen(seed)
    starts = rows_of(lens, before)
    T = starts[-1] + after
    rows = rand(g, T, H + 2 * KV, D, dtype=dtype)
    rows[:, H:H + KV] *= spread
    rubbish(rows[:before]), rubbish(rows[starts[-1]:])
    return (*rows.split([H, KV, KV], 1), starts)


# lengths of the sequences, heads, key heads, head
SHAPES = [([1], 1, 1, 64), ([5], 4, 2, 128), ([0, 1, 0, 2, 3], 8, 2, 64), ([33], 32, 8, 128), ([127, 128, 129], 4, 4, 128),
          ([64, 63, 65, 1, 200], 14, 2, 64), ([500], 8, 1, 128), ([300, 7, 0, 411], 6, 2, 128), ([1000, 2], 3, 1, 64),
          ([257] * 3, 24, 2, 128), ([70, 20], 128, 1, 64), ([45, 3], 200, 2, 128), ([1300], 4, 2, 64), ([17] * 60, 5, 1, 128),
          ([700, 1, 900], 2, 2, 128)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prompt(shape, causal, dtype):
    lens, H, KV, D = SHAPES[shape]
    q, k, v, starts = problem(shape, lens, H, KV, D, dtype, before=shape % 3, after=shape % 5, spread=1.0 + shape % 4)
    status = ints([0])
    out, lse = serving.prompt_attention(q, k, v, ints(starts), causal=causal, status=status)
    (want, w_lse), (bound, b_lse), _, _ = R.packed(f64(q), f64(k), f64(v), starts, D ** -0.5, causal, dtype)
    assert int(status) == 0
    check(out, want, bound, "out")
    lost = np.isinf(w_lse)
    assert np.array_equal(f64(lse)[lost], w_lse[lost])
    check(lse[torch.from_numpy(~lost).cuda()], w_lse[~lost], b_lse[~lost], "lse")
    again = serving.prompt_attention(q, k, v, ints(starts), causal=causal)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prompt_gradient(shape, causal, dtype):
    lens, H, KV, D = SHAPES[shape]
    q, k, v, starts = problem(shape, lens, H, KV, D, dtype, before=shape % 3, after=shape % 5, spread=1.0 + shape % 4)
    g = gen(shape + 100)
    size = [1.0, 2.0 ** -13, 300.0][shape % 3]
    dout = (rand(g, *q.shape, dtype="float32") * size).to(DT[dtype])
    rubbish(dout[:starts[0]]), rubbish(dout[starts[-1]:])
    dlse = rand(g, *q.shape[:2], dtype="float32") * size if shape % 2 else None
    at = ints(starts)
    low = torch.empty_like(q) if shape % 3 else None
    out, lse = serving.prompt_attention(q, k, v, at, causal=causal, low=low)
    status = ints([0])
    got = serving.prompt_attention_grad(dout, q, k, v, out, lse, at, causal=causal, dlse=dlse, low=low, status=status)
    assert int(status) == 0
    _, _, want, bound = R.packed(f64(q), f64(k), f64(v), starts, D ** -0.5, causal, dtype, f64(dout), None if dlse is None else f64(dlse))
    for name, x, w, b in zip(("dq", "dk", "dv"), got, want, bound):
        check(x, w, b, name)
    again = serving.prompt_attention_grad(dout, q, k, v, out, lse, at, causal=causal, dlse=dlse, low=low)
    for x, y in zip(again, got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_what_rounding_took(dtype):
    """out + low has the forward pass's own error alone: that of out without its rounding's half-step, and low's of half a step of it."""
    lens, H, KV, D = [500, 3, 300], 4, 2, 128
    q, k, v, starts = problem(2, lens, H, KV, D, dtype)
    low = torch.full_like(q, 7.0)
    out, _ = serving.prompt_attention(q, k, v, ints(starts), low=low)
    (want, _), (bound, _), _, _ = R.packed(f64(q), f64(k), f64(v), starts, D ** -0.5, True, dtype)
    u = R.HALF_STEP[dtype]
    check(torch.from_numpy(f64(out) + f64(low)), want, bound - u * np.abs(want) + u * u * (np.abs(want) + bound) + (2.0 ** -24 if dtype == "float16" else 0.0), "out + low")
    plain, _ = serving.prompt_attention(q, k, v, ints(starts))
    assert torch.equal(plain, out)


def test_gradient_against_differences():
    """Central differences of <dout, out> + <dlse, lse> in 64 bits: the operator's gradient of the same inputs may differ from that of
    exact arithmetic by the derived bounds, and the difference quotient (step 2^-12) by its third derivative and rounding, 1e-5."""
    lens, H, KV, D = [9, 6], 4, 2, 64
    q, k, v, starts = problem(4, lens, H, KV, D, "bfloat16")
    g = gen(8)
    dout, dlse = rand(g, *q.shape, dtype="bfloat16"), rand(g, *q.shape[:2], dtype="float32")
    leaves = [x.detach().clone().requires_grad_() for x in (q, k, v)]
    out, lse = serving.prompt_attention(*leaves, ints(starts))
    got = torch.autograd.grad([out, lse], leaves, [dout, dlse])
    x = [f64(t) for t in (q, k, v)]
    bound = R.packed(*x, starts, D ** -0.5, True, "bfloat16", f64(dout), f64(dlse))[3]

    def value():
        o, l = R.packed(*x, starts, D ** -0.5, True, "bfloat16")[0]
        return float((o * f64(dout)).sum() + (l * f64(dlse)).sum())
    rng = np.random.default_rng(0)
    for i in range(3):
        for _ in range(16):
            at = tuple(int(rng.integers(0, n)) for n in x[i].shape)
            was, h = x[i][at], 2.0 ** -12
            x[i][at] = was + h
            up = value()
            x[i][at] = was - h
            down = value()
            x[i][at] = was
            assert abs((up - down) / (2 * h) - float(got[i][at])) <= bound[i][at] + 1e-5, (i, at)


def test_autograd():
    """Which inputs want a gradient, which results have one, gradients of any strides (a sum's has none), twice over one graph."""
    lens, H, KV, D = [40, 100], 6, 2, 128
    q, k, v, starts = problem(11, lens, H, KV, D, "bfloat16")
    at = ints(starts)
    low = torch.empty_like(q)
    out, lse = serving.prompt_attention(q, k, v, at, low=low)
    ones = torch.ones_like(out)
    want = serving.prompt_attention_grad(ones, q, k, v, out, lse, at, low=low)
    for which in ([0], [1], [2], [0, 2], [0, 1, 2]):
        x = [t.detach().requires_grad_(i in which) for i, t in enumerate((q, k, v))]
        o, _ = serving.prompt_attention(*x, at)
        assert torch.equal(o, out)
        o.sum().backward(retain_graph=True)
        o.sum().backward()
        for i, t in enumerate(x):
            assert torch.equal(t.grad, want[i] * 2) if i in which else t.grad is None
    x = [t.detach().requires_grad_() for t in (q, k, v)]
    o, l = serving.prompt_attention(*x, at)
    l.sum().backward()
    want = serving.prompt_attention_grad(ones * 0, q, k, v, out, lse, at, dlse=torch.ones_like(lse), low=low)
    assert all(torch.equal(t.grad, w) for t, w in zip(x, want))
    t = ones.transpose(0, 2).contiguous().transpose(0, 2)                       # the head's values are not contiguous
    x = [t.detach().requires_grad_() for t in (q, k, v)]
    got = torch.autograd.grad(serving.prompt_attention(*x, at)[0], x, t)
    want = serving.prompt_attention_grad(ones, q, k, v, out, lse, at, low=low)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(RuntimeError):
        g = torch.autograd.grad(serving.prompt_attention(*x, at)[0], x, ones, create_graph=True)
        g[0].sum().backward()
    for kw in (dict(out=torch.empty_like(out)), dict(lse=torch.empty_like(lse)), dict(low=torch.empty_like(out)), dict(stream=torch.cuda.current_stream()),
               dict(workspace=serving.prompt_workspace(q, k, at))):
        with pytest.raises(gts.GtsError):
            serving.prompt_attention(*x, at, **kw)


@pytest.mark.parametrize("shift", [1, 4, 8])
def test_strides(shift):
    """Views off the 16-byte grid, heads before tokens, every other head or token, results in larger buffers, a gradient that is one
    row for all: the same values."""
    lens, H, KV, D = [150, 1, 290], 4, 2, 128
    q, k, v, starts = (x.contiguous() if torch.is_tensor(x) else x for x in problem(21, lens, H, KV, D, "bfloat16"))
    g, at, T = gen(3), ints(starts), q.shape[0]
    dout = rand(g, 1, 1, D, dtype="bfloat16").expand(T, H, D)
    want = serving.prompt_attention(q, k, v, at)
    grads = serving.prompt_attention_grad(dout.contiguous(), q, k, v, *want, at)

    def off(x):
        y = torch.zeros(x.shape[0], x.shape[1] * D + 16, dtype=x.dtype, device="cuda")[:, shift:shift + x.shape[1] * D].unflatten(1, x.shape[1:])
        return y.copy_(x)

    def by_head(x):
        return x.transpose(0, 1).contiguous().transpose(0, 1)

    def sparse(x):
        y = torch.zeros(2 * x.shape[0], 3 * x.shape[1], D, dtype=x.dtype, device="cuda")[::2, ::3]
        return y.copy_(x)
    for lay in (off, by_head, sparse):
        x = [lay(t) for t in (q, k, v)]
        to = lay(torch.zeros_like(q))
        out, lse = serving.prompt_attention(*x, at, out=to)
        assert out is to and torch.equal(out, want[0]) and torch.equal(lse, want[1])
        got = serving.prompt_attention_grad(dout, *x, out, lse, at, out_dq=lay(torch.zeros_like(q)), out_dk=lay(torch.zeros_like(k)),
                                            out_dv=lay(torch.zeros_like(v)))
        assert all(torch.equal(a, b) for a, b in zip(got, grads))


def test_rows_of_no_sequence():
    """Zeros where the call makes the results, left alone where it is given them."""
    lens, H, KV, D = [40, 0, 77], 8, 2, 64
    q, k, v, starts = problem(5, lens, H, KV, D, "float16", before=3, after=200)
    at, dout = ints(starts), rand(gen(9), *q.shape, dtype="float16")
    rest = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
    rest[3:starts[-1]] = False
    out, lse = serving.prompt_attention(q, k, v, at)
    assert (out[rest] == 0).all() and (lse[rest] == float("-inf")).all() and torch.isfinite(out).all()
    mine, sums = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    serving.prompt_attention(q, k, v, at, out=mine, lse=sums)
    assert (mine[rest] == 7).all() and (sums[rest] == 7).all()
    assert torch.equal(mine[~rest], out[~rest]) and torch.equal(sums[~rest], lse[~rest])
    _, l = serving.prompt_attention(q, k, v, at, out=mine)
    assert (mine[rest] == 7).all() and torch.equal(l, lse)
    got = serving.prompt_attention_grad(dout, q, k, v, out, lse, at)
    assert all((x[rest] == 0).all() and torch.isfinite(x).all() for x in got)
    to = [torch.full_like(x, 7.0) for x in got]
    serving.prompt_attention_grad(dout, q, k, v, out, lse, at, out_dq=to[0], out_dk=to[1], out_dv=to[2])
    for x, y in zip(to, got):
        assert (x[rest] == 7).all() and torch.equal(x[~rest], y[~rest])
    none = ints([5])                                                            # no sequences at all
    out, lse = serving.prompt_attention(q, k, v, none)
    assert (out == 0).all() and (lse == float("-inf")).all()
    assert all((x == 0).all() for x in serving.prompt_attention_grad(dout, q, k, v, out, lse, none))
    empty = q[:0], k[:0], v[:0]
    out, lse = serving.prompt_attention(*empty, ints([0, 0]))
    assert out.shape == (0, H, D) and lse.shape == (0, H)
    assert [x.shape[0] for x in serving.prompt_attention_grad(out, *empty, out, lse, ints([0, 0]))] == [0, 0, 0]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("D", [64, 128])
def test_values_out_of_sight(D, bad):
    """Infinite and NaN keys and values: rows that do not see them are what they were."""
    lens, H, KV = [100, 200, 300], 8, 2
    q, k, v, starts = problem(D, lens, H, KV, D, "bfloat16")
    at, dout = ints(starts), rand(gen(2), *q.shape, dtype="bfloat16")
    out, lse = serving.prompt_attention(q, k, v, at)
    grads = serving.prompt_attention_grad(dout, q, k, v, out, lse, at)
    # a whole sequence
    k2, v2, q2, dout2 = (x.clone() for x in (k, v, q, dout))
    for x in (k2, v2, q2, dout2):
        x[100:300] = bad
    o, l = serving.prompt_attention(q2, k2, v2, at)
    got = serving.prompt_attention_grad(dout2, q2, k2, v2, o, l, at)
    keep = torch.ones(600, dtype=torch.bool, device="cuda")
    keep[100:300] = False
    for x, y in zip((o, l, *got), (out, lse, *grads)):
        assert torch.equal(x[keep], y[keep])
    # later values and keys of the same one
    for row, head in ((450, 0), (599, 1), (428, 0), (511, 1), (310, 1)):
        for which in (k, v):
            x = which.clone()
            x[row, head, 5] = bad
            o, l = serving.prompt_attention(q, x if which is k else k, x if which is v else v, at)
            keep = torch.ones(600, H, dtype=torch.bool, device="cuda")
            keep[row:, head * (H // KV):(head + 1) * (H // KV)] = False
            assert torch.equal(o[keep], out[keep]) and torch.equal(l[keep], lse[keep])
            if which is v:                                                      # and the others have it in that one place
                assert torch.equal(l, lse)
                there = torch.zeros_like(keep)
                there[row:, head * (H // KV):(head + 1) * (H // KV)] = True
                seen, was = o[there], out[there]
                assert not torch.isfinite(seen[:, 5]).any() or bad == float("-inf") and not torch.isfinite(seen[:, 5]).any()
                assert torch.equal(seen[:, :5], was[:, :5]) and torch.equal(seen[:, 6:], was[:, 6:])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("D,group", [(64, 4), (128, 4), (128, 3)])
def test_gradients_out_of_sight(D, group, bad):
    """One infinite or NaN value of a sequence: gradients that it has no part in are what they were."""
    lens, KV = [100, 200, 300], 2
    H = KV * group
    q, k, v, starts = problem(D, lens, H, KV, D, "bfloat16")
    at, dout = ints(starts), rand(gen(2), *q.shape, dtype="bfloat16")

    def grads(q, k, v, dout):
        out, lse = serving.prompt_attention(q, k, v, at)
        return serving.prompt_attention_grad(dout, q, k, v, out, lse, at)
    want = grads(q, k, v, dout)
    for row in (300, 427, 428, 450, 511, 599):
        for name in ("q", "k", "v", "dout"):
            x = {"q": q, "k": k, "v": v, "dout": dout}
            x[name] = x[name].clone()
            x[name][row, 0, 5] = bad
            got = grads(**x)
            keep = [torch.ones(600, n, dtype=torch.bool, device="cuda") for n in (H, KV, KV)]
            if name in ("q", "dout"):                            # that query's own, and those of the keys it sees
                keep[0][row, 0] = keep[1][300:row + 1, 0] = keep[2][300:row + 1, 0] = False
            else:                                                # those of the queries that see it, and of all their keys
                keep[0][row:, :group] = keep[1][300:, 0] = False
                if name == "k":
                    keep[2][300:, 0] = False
            for a, b, m in zip(got, want, keep):
                assert torch.equal(a[m], b[m]), (name, row)
            if name == "dout":
                assert not torch.isfinite(got[2][300:row + 1, 0, 5]).any()
            if bad != bad:                                       # (an infinite key may weigh nothing)
                assert torch.isnan(got[0][row, 0]).all(), (name, row)


@pytest.mark.parametrize("lens", [[100], [3000], [40, 2500, 7]])
@pytest.mark.parametrize("D", [64, 128])
def test_a_query_of_nan(D, lens):
    """Its row is NaN, cut or whole, wherever it is; the others are what they were."""
    q, k, v, starts = problem(D, lens, 4, 1, D, "bfloat16")
    at = ints(starts)
    out, lse = serving.prompt_attention(q, k, v, at)
    rows = sorted({0, 1, 63, 64, starts[-1] // 2, starts[-1] - 1} & set(range(starts[-1])))
    x = q.clone()
    x[rows, 2, 7] = float("nan")
    o, l = serving.prompt_attention(x, k, v, at)
    keep = torch.ones(starts[-1], 4, dtype=torch.bool, device="cuda")
    keep[rows, 2] = False
    assert torch.isnan(o[~keep]).all() and torch.isnan(l[~keep]).all()
    assert torch.equal(o[keep], out[keep]) and torch.equal(l[keep], lse[keep])


def test_large_and_equal_scores():
    """Scores of thousands, and rows whose scores are all alike."""
    D, H, n = 128, 4, 300
    g = gen(6)
    q, k, v = (rand(g, n, H, D, dtype="bfloat16") for _ in range(3))
    at = ints([0, n])
    for scale, kk in ((40.0, k), (1.0, torch.zeros_like(k)), (1e-3, k)):
        out, lse = serving.prompt_attention(q, kk, v, at, scale=scale)
        (want, w_lse), (bound, b_lse), _, _ = R.packed(f64(q), f64(kk), f64(v), [0, n], scale, True, "bfloat16")
        check(out, want, bound, ("out", scale))
        check(lse, w_lse, b_lse, ("lse", scale))


def test_starts_at_the_ends_of_their_type():
    """Sequences stay within the call whatever the numbers are; the ones whose starts are good are worked out as ever."""
    low, high = -2**31, 2**31 - 1
    q, k, v, _ = problem(2, [30, 50], 4, 2, 64, "bfloat16")
    want = serving.prompt_attention(q, k, v, ints([0, 30, 80]))
    for bad, rows in (([0, 30, low], slice(0, 30)), ([low, 30, 80], slice(30, 80)), ([high, low, low], slice(0, 0)), ([0, 30, high], slice(0, 80))):
        status = ints([0])
        out, lse = serving.prompt_attention(q, k, v, ints(bad), status=status)
        assert int(status) == gts.GTS_ERR_INVALID_PARAMS, bad
        assert torch.equal(out[rows], want[0][rows]) and torch.equal(lse[rows], want[1][rows]), bad
        got = serving.prompt_attention_grad(out, q, k, v, out, lse, ints(bad))
        assert all(torch.isfinite(x).all() for x in got), bad


def test_starts_out_of_range_are_clamped():
    q, k, v, starts = problem(1, [30, 50], 4, 2, 64, "bfloat16")
    for bad, good in (([-5, 30, 80], [0, 30, 80]), ([0, 30, 1 << 30], [0, 30, 80]), ([0, 30, 20], [0, 30, 30])):
        status = ints([0])
        out, lse = serving.prompt_attention(q, k, v, ints(bad), status=status)
        assert int(status) == gts.GTS_ERR_INVALID_PARAMS
        want = serving.prompt_attention(q, k, v, ints(good))
        assert torch.equal(out[:30], want[0][:30])
        status = ints([0])
        got = serving.prompt_attention_grad(out, q, k, v, out, lse, ints(bad), status=status)
        assert int(status) == gts.GTS_ERR_INVALID_PARAMS and all(torch.isfinite(x).all() for x in got)
        serving.prompt_attention(q, k, v, ints(bad))


def test_refusals():
    q, k, v, starts = problem(1, [30, 50], 4, 2, 64, "bfloat16")
    at = ints(starts)
    out, lse = serving.prompt_attention(q, k, v, at)
    bad = [dict(q=q.float(), k=k.float(), v=v.float()), dict(q=q.half()), dict(q=q[0]), dict(q=q[:7]), dict(k=k[:, :, :32]), dict(v=v[:, :1]),
           dict(q=q[..., :48], k=k[..., :48], v=v[..., :48]), dict(starts=at.long()), dict(starts=at.cpu()), dict(starts=at[None]),
           dict(starts=at[:0]), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(q=q[:, :3]),
           dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(status=ints([0, 0])), dict(workspace=torch.zeros(0, dtype=torch.uint8, device="cuda"))]
    for kw in bad:
        with pytest.raises(gts.GtsError):
            serving.prompt_attention(**{**dict(q=q, k=k, v=v, starts=at), **kw})
        with pytest.raises(gts.GtsError):
            serving.prompt_attention_grad(**{**dict(dout=out, q=q, k=k, v=v, out=out, lse=lse, starts=at), **kw})
    for kw in (dict(out=out[:5]), dict(lse=lse[:5]), dict(lse=lse.double()), dict(low=out[:5]), dict(low=lse)):
        with pytest.raises(gts.GtsError):
            serving.prompt_attention(q, k, v, at, **kw)
    for kw in (dict(dout=out[:5]), dict(dout=out.float()), dict(dlse=lse[:5]), dict(lse=lse[:4]), dict(out_dq=k), dict(out_dk=q)):
        with pytest.raises(gts.GtsError):
            serving.prompt_attention_grad(**{**dict(dout=out, q=q, k=k, v=v, out=out, lse=lse, starts=at), **kw})


# ---------------------------------------------------------------- chunks
def paged(seed, new, lens, H, KV, D, page, order, dtype, before=0, after=0, columns=0, fill=float("nan")):
    """Queries of `new` tokens of each sequence, whose first `lens` tokens are in pages; all else in the cache is `fill`."""
    g = gen(seed)
    starts = rows_of(new, before)
    q = rand(g, starts[-1] + after, H, D, dtype=dtype)
    rubbish(q[:before]), rubbish(q[starts[-1]:])
    held = [-(-max(n, 0) // page) for n in lens]
    ids = torch.randperm(sum(held) + 2, generator=g).tolist()
    cache = serving.PagedCache.empty(len(ids), page, KV, D, DT[dtype], order=order)
    cache.k.fill_(fill), cache.v.fill_(fill)
    table = np.full((len(lens), max(max(held, default=0), columns)), -1, np.int32)
    keys = []
    for b, n in enumerate(lens):
        table[b, :held[b]] = [ids.pop() for _ in range(held[b])]
        k, v = rand(g, max(n, 0), KV, D, dtype=dtype) * 2, rand(g, max(n, 0), KV, D, dtype=dtype)
        for j in range(held[b]):
            part = slice(j * page, min((j + 1) * page, n))
            cache.k[table[b, j], :part.stop - part.start] = k[part]
            cache.v[table[b, j], :part.stop - part.start] = v[part]
        keys.append((f64(k), f64(v)))
    return dict(q=q, starts=ints(starts), cache=cache, page_table=torch.from_numpy(table).cuda(), lens=ints(list(lens))), starts, keys


def chunk_reference(p, starts, keys, dtype):
    q = f64(p["q"])
    T, H, D = q.shape
    res = np.zeros(q.shape), np.full((T, H), -np.inf), np.zeros(q.shape), np.zeros((T, H))
    for (a, b), (k, v) in zip(zip(starts[:-1], starts[1:]), keys):
        got = R.attention(q[a:b], k, v, D ** -0.5, True, dtype)
        for to, x in zip(res, (*got[0], *got[1])):
            to[a:b] = x
    return res


def check_chunk(got, want):
    check(got[0], want[0], want[2], "out")
    lost = np.isinf(want[1])
    assert np.array_equal(f64(got[1])[lost], want[1][lost])
    check(got[1][torch.from_numpy(~lost).cuda()], want[1][~lost], want[3][~lost], "lse")


# new tokens, lengths, heads, key heads, head, page
CHUNKS = [([1], [1], 1, 1, 64, 16), ([17], [1000], 32, 8, 128, 16), ([3, 0, 5, 1], [3, 40, 0, 2], 4, 2, 64, 48),
          ([130, 70], [130, 500], 8, 2, 128, 64), ([64, 1, 1, 200], [700, 333, 1, 201], 14, 2, 128, 100), ([40], [20], 6, 3, 64, 7),
          ([33, 90], [2000, 128], 8, 1, 128, 1), ([256, 129], [256, 1029], 4, 4, 64, 128), ([5] * 40, list(range(3, 203, 5)), 8, 4, 128, 32),
          ([300], [3000], 2, 1, 128, 256), ([2, 9], [-3, 5], 4, 2, 128, 16), ([20, 30], [600, 77], 100, 1, 64, 24)]


@pytest.mark.parametrize("order", ["tokens", "heads"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(CHUNKS)))
def test_chunk(case, dtype, order):
    p, starts, keys = paged(case, *CHUNKS[case], order, dtype, before=case % 2, after=case % 3, columns=case)
    status = ints([0])
    got = serving.chunk_attention(**p, status=status)
    assert int(status) == 0
    check_chunk(got, chunk_reference(p, starts, keys, dtype))
    again = serving.chunk_attention(**p)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("shift", [1, 8])
def test_chunk_strides(shift):
    """Caches and queries off the 16-byte grid, pages with room between them."""
    new, lens, H, KV, D, page = [130, 20], [200, 333], 4, 2, 128, 32
    p, starts, keys = paged(3, new, lens, H, KV, D, page, "tokens", "bfloat16")
    want = serving.chunk_attention(**p)
    check_chunk(want, chunk_reference(p, starts, keys, "bfloat16"))
    c = p["cache"]
    wide = [torch.zeros(c.n_pages, page, KV * D + 24, dtype=torch.bfloat16, device="cuda")[
            :, :, shift:shift + KV * D].unflatten(2, (KV, D)) for _ in range(2)]
    wide[0].copy_(c.k), wide[1].copy_(c.v)
    q = torch.zeros(p["q"].shape[0], H * D + 16, dtype=torch.bfloat16, device="cuda")[:, shift:shift + H * D].unflatten(1, (H, D))
    q.copy_(p["q"])
    got = serving.chunk_attention(**{**p, "q": q, "cache": serving.PagedCache(*wide)}, out=torch.zeros_like(q))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_chunk_is_prefix_attention_without_a_prefix():
    """The same numbers to their bounds as the decode operator's, on the calls that both take."""
    for new in (1, 4, 40):
        lens = [new + 13 * b for b in range(9)]
        p, starts, keys = paged(new, [new] * 9, lens, 8, 2, 128, 16, "tokens", "bfloat16")
        want = chunk_reference(p, starts, keys, "bfloat16")
        check_chunk(serving.chunk_attention(**p), want)
        q = p["q"].view(9, new, 8, 128)
        out, lse = serving.prefix_attention(q, p["cache"], ints([]), 0, p["page_table"], p["lens"])
        check_chunk((out.flatten(0, 1), lse.flatten(0, 1)), want)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_chunk_values_out_of_sight(value):
    """Later tokens' values of the same chunk, pages' rests and unused pages: rows before them are what they were."""
    new, lens = [200], [333]
    p, starts, _ = paged(3, new, lens, 4, 2, 128, 32, "tokens", "bfloat16", fill=0.0)
    want = serving.chunk_attention(**p)
    q, _, _ = paged(3, new, lens, 4, 2, 128, 32, "tokens", "bfloat16", fill=value)
    got = serving.chunk_attention(**q)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for key in (332, 300, 270, 255, 256):
        c = p["cache"]
        k, v = c.k.clone(), c.v.clone()
        v[int(p["page_table"][0, key // 32]), key % 32, 1, 77] = value
        got = serving.chunk_attention(**{**p, "cache": serving.PagedCache(k, v)})
        i = key - 133
        assert torch.equal(got[0][:i], want[0][:i]) and torch.equal(got[0][i:, :2], want[0][i:, :2])
        assert torch.equal(got[1], want[1]) and not torch.isfinite(got[0][i:, 2:, 77]).any()
        assert torch.equal(got[0][i:, 2:, 78:], want[0][i:, 2:, 78:])


def test_chunk_reports_what_is_out_of_range():
    for what in ("high", "low", "lens", "starts"):
        p, starts, keys = paged(5, [20, 30], [100, 130], 4, 2, 64, 16, "tokens", "bfloat16", fill=0.0)
        want = serving.chunk_attention(**p)
        if what == "high":
            p["page_table"][1, 2] = p["cache"].n_pages
        elif what == "low":
            p["page_table"][1, 2] = -(1 << 31)
        elif what == "lens":
            p["lens"][1] = 1 << 30
        else:
            p["starts"][2] = 1 << 30
        status = ints([0])
        out, lse = serving.chunk_attention(**p, status=status)
        assert int(status) == gts.GTS_ERR_INVALID_PARAMS, what
        assert torch.equal(out[:20], want[0][:20]) and torch.equal(lse[:20], want[1][:20])
        serving.chunk_attention(**p)


def test_chunk_refusals():
    p, _, _ = paged(5, [20, 30], [100, 130], 4, 2, 64, 16, "tokens", "bfloat16", fill=0.0)
    q = p["q"]
    for kw in (dict(q=q.half()), dict(q=q[0]), dict(q=q[:, :3]), dict(q=torch.zeros(50, 4, 128, dtype=q.dtype, device="cuda")), dict(starts=p["starts"][:2]),
               dict(starts=p["starts"].long()), dict(page_table=p["page_table"][:1]), dict(page_table=p["page_table"].long()), dict(lens=p["lens"][:1]),
               dict(lens=p["lens"].long()), dict(scale=0.0), dict(out=q[:3]), dict(lse=torch.zeros(3)), dict(status=ints([0, 0])),
               dict(workspace=torch.zeros(0, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(gts.GtsError):
            serving.chunk_attention(**{**p, **kw})
    wide = serving.PagedCache.empty(4, 16, 2, 256, torch.bfloat16)
    with pytest.raises(gts.GtsError):
        serving.chunk_attention(torch.zeros(50, 4, 256, dtype=q.dtype, device="cuda"), p["starts"], wide, p["page_table"], p["lens"])


# ---------------------------------------------------------------- streams, graphs, sizes
def test_streams_side_by_side():
    p, _, _ = paged(5, [200, 30], [1000, 130], 8, 2, 128, 16, "tokens", "bfloat16", fill=0.0)
    q, k, v, starts = problem(3, [400, 300], 8, 2, 128, "bfloat16")
    at = ints(starts)
    want = serving.chunk_attention(**p), serving.prompt_attention(q, k, v, at)
    grads = serving.prompt_attention_grad(q, q, k, v, *want[1], at)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [(serving.chunk_attention(**p, stream=s), serving.prompt_attention(q, k, v, at, stream=s),
            serving.prompt_attention_grad(q, q, k, v, *want[1], at, stream=s)) for s in streams for _ in range(2)]
    torch.cuda.synchronize()
    for a, b, c in got:
        assert all(torch.equal(x, y) for x, y in zip((*a, *b, *c), (*want[0], *want[1], *grads)))


def test_graphs_follow_starts_and_lengths():
    """Starts, lengths and pages are read on the device; two graphs with a workspace of their own run side by side."""
    p, _, _ = paged(5, [200, 30, 70], [1000, 130, 70], 8, 2, 128, 16, "tokens", "bfloat16", fill=0.0)
    q, k, v, starts = problem(3, [400, 300, 200], 8, 2, 128, "bfloat16")
    at = ints(starts)
    out, lse = serving.prompt_attention(q, k, v, at)
    graphs, side = [], torch.cuda.Stream()
    for _ in range(2):
        ws = serving.chunk_workspace(p["q"], p["starts"], p["cache"], p["page_table"])
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            got = (serving.chunk_attention(**p, workspace=ws), serving.prompt_attention(q, k, v, at),
                   serving.prompt_attention_grad(q, q, k, v, out, lse, at))
        graphs.append((g, got, ws))                      # (a replay writes to the workspace: it lives as long as the graph)
    for step in (0, 1, 2):
        if step == 1:
            p["lens"].copy_(ints([800, 30, 100])), p["starts"].copy_(ints([0, 100, 110, 300])), at.copy_(ints([0, 10, 600, 900]))
        if step == 2:
            p["starts"].copy_(ints([0, 0, 300, 300])), at.copy_(ints([0, 900, 900, 900]))
        with torch.no_grad():
            o, l = serving.prompt_attention(q, k, v, at)
            out.copy_(o), lse.copy_(l)
        want = serving.chunk_attention(**p), (o, l), serving.prompt_attention_grad(q, q, k, v, out, lse, at)
        torch.cuda.synchronize()
        for (g, _, _), s in zip(graphs, (side, torch.cuda.current_stream())):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for _, got, _ in graphs:
            for x, y in zip(got, want):
                assert all(torch.equal(a, b) for a, b in zip(x, y))


def test_backward_in_a_graph():
    """Forward and backward captured together, while an eager graph of the same leaves lives (made on the stream of the capture, as
    torch's leaves want it)."""
    q, k, v, starts = problem(3, [100, 60], 4, 2, 64, "bfloat16")
    x, at = [t.detach().clone().requires_grad_() for t in (q, k, v)], ints(starts)
    dout = rand(gen(4), *q.shape, dtype="bfloat16")
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        alive, _ = serving.prompt_attention(*x, at)
        want = torch.autograd.grad(alive, x, dout, retain_graph=True)
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        out, _ = serving.prompt_attention(*x, at)
        got = torch.autograd.grad(out, x, dout)
    for _ in range(2):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, alive) and all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):
        again = torch.autograd.grad(alive, x, dout)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, want))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,H,KV,D", [([4096], 32, 8, 128), ([1024] * 8, 16, 4, 64), ([512] * 48, 12, 12, 64), ([70] * 200, 8, 8, 128)])
def test_many_calls_on_end(lens, H, KV, D, causal):
    """Calls one after the other, with memory busy: copies that land out of order change nothing."""
    q, k, v, starts = problem(3, lens, H, KV, D, "bfloat16")
    at, status = ints(starts), ints([0])
    out, lse = serving.prompt_attention(q, k, v, at, causal=causal)
    want = serving.prompt_attention_grad(q, q, k, v, out, lse, at, causal=causal)
    other = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for i in range(150):
        if i % 3 == 0:
            with torch.cuda.stream(side):
                other.add_(1)
        o, l = serving.prompt_attention(q, k, v, at, causal=causal, status=status)
        got = serving.prompt_attention_grad(q, q, k, v, out, lse, at, causal=causal, status=status)
        for x, y in zip((o, l, *got), (out, lse, *want)):
            wrong += (x != y).sum()
    torch.cuda.synchronize()
    assert int(status) == 0 and int(wrong) == 0


def test_beyond_32_bit_offsets():
    """Rows past 2^31 values and pages past 2^31 values, the same numbers as near ones."""
    H, KV, D, n = 64, 8, 128, 150
    T = (1 << 31) // (H * D) + 1000
    q = torch.zeros(T, H, D, dtype=torch.bfloat16, device="cuda")
    near = [rand(gen(7), n, h, D, dtype="bfloat16") for h in (H, KV, KV)]
    k, v = (torch.zeros(T, KV, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for x, y in zip((q, k, v), near):
        x[-n:] = y
    at, small = ints([T - n, T]), ints([0, n])
    want = serving.prompt_attention(*near, small)
    out, lse = torch.zeros_like(q), torch.zeros(T, H, device="cuda")
    serving.prompt_attention(q, k, v, at, out=out, lse=lse)
    assert torch.equal(out[-n:], want[0]) and torch.equal(lse[-n:], want[1]) and not out[:-n].any()
    grads = serving.prompt_attention_grad(near[0], *near, *want, small)
    to = [torch.zeros_like(x) for x in (q, k, v)]
    serving.prompt_attention_grad(q, q, k, v, out, lse, at, out_dq=to[0], out_dk=to[1], out_dv=to[2])
    for x, y in zip(to, grads):
        assert torch.equal(x[-n:], y) and not x[:-n].any()
    del q, k, v, out, lse, to, x
    page = 64
    pages = (1 << 31) // (page * KV * D) + 8
    cache, few = (serving.PagedCache.empty(c, page, KV, D, torch.bfloat16) for c in (pages, 4))
    ids = [pages - 1, pages - 3, pages - 2]
    src, dst = ints([0, 1, 2]), ints(ids)
    for c, x in ((few.k, near[1]), (few.v, near[2])):
        c.zero_()
        c[:3].view(-1, KV, D)[:n] = x
    serving.copy_pages(few, src, dst, into=cache)
    assert torch.equal(cache.k[ids], few.k[:3]) and torch.equal(cache.v[ids], few.v[:3])
    got = serving.chunk_attention(near[0][:40], ints([0, 40]), cache, dst[None], ints([n]))
    want = serving.chunk_attention(near[0][:40], ints([0, 40]), few, src[None], ints([n]))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_many_sequences():
    """As many as a call takes, of one token: each is its own value."""
    n = 65535
    g = gen(1)
    q, k, v = (rand(g, n, 2, 64, dtype="bfloat16") for _ in range(3))
    at = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    out, lse = serving.prompt_attention(q, k, v, at)
    assert torch.equal(out, v)
    assert ((lse.double() - (q.double() * k.double()).sum(-1) / 8).abs() <= 1e-5).all()      # (of scores below 8, in 32 bits)
    dq, dk, dv = serving.prompt_attention_grad(q, q, k, v, out, lse, at)
    # p = 1 to 2^-20 (lse and the score are 32-bit sums of one magnitude), dp - e is 0 to 128 2^-24 of terms below 30
    assert torch.equal(dv, q) and float(dq.abs().max()) < 1e-2 and float(dk.abs().max()) < 1e-2
    cache = serving.PagedCache(k[:, None], v[:, None])                                         # a page for each
    got = serving.chunk_attention(q, at, cache, at[:-1, None].contiguous(), torch.ones(n, dtype=torch.int32, device="cuda"))
    assert torch.equal(got[0], v)


def test_chunks_without_keys():
    """No pages at all, no lengths, no tokens."""
    cache = serving.PagedCache.empty(0, 16, 2, 64, torch.bfloat16)
    q = rand(gen(1), 7, 4, 64, dtype="bfloat16")
    out, lse = serving.chunk_attention(q, ints([0, 3, 7]), cache, torch.zeros(2, 0, dtype=torch.int32, device="cuda"), ints([0, 0]))
    assert (out == 0).all() and (lse == float("-inf")).all()
    out, lse = serving.chunk_attention(q[:0], ints([0]), cache, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), ints([]))
    assert out.shape == (0, 4, 64)
    out, lse = serving.chunk_attention(q, ints([0]), cache, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), ints([]))
    assert (out == 0).all() and (lse == float("-inf")).all()


def test_a_long_sequence():
    """Keys by the tens of thousands: the sums' own value (every value row is its token's number / 2^16), and a cut in every way."""
    n, H, KV, D = 40000, 4, 2, 64
    q = torch.zeros(n, H, D, dtype=torch.float16, device="cuda")
    k = rand(gen(1), n, KV, D, dtype="float16")
    at = torch.arange(n, device="cuda", dtype=torch.float64)
    v = (at / 65536).half()[:, None, None].expand(n, KV, D).contiguous()
    out, lse = serving.prompt_attention(q, k, v, ints([0, n]))
    mean = torch.cumsum(v[:, 0, 0].double(), 0) / (at + 1)
    # equal weights: 1 exactly; the sum of n values in 32 bits, 2^-24 n relative at worst, and the rounding of the result
    assert ((out.double() - mean[:, None, None]).abs() <= mean[:, None, None] * (2.0 ** -11 + n * 2.0 ** -24) + 2.0 ** -25).all()
    assert ((lse.double() - torch.log(at + 1)[:, None]).abs() <= 2.0 ** -20 + n * 2.0 ** -24).all()


# ---------------------------------------------------------------- copies of pages
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("order,into_order", [("tokens", None), ("heads", None), ("tokens", "heads"), ("heads", "tokens")])
@pytest.mark.parametrize("page,KV,D", [(16, 8, 128), (1, 1, 64), (100, 3, 80), (7, 2, 20), (64, 8, 256), (33, 1, 1)])
def test_copy(page, KV, D, order, into_order, dtype):
    g = gen(page + D)
    n = 40
    cache = serving.PagedCache.empty(n, page, KV, D, DT[dtype], order=order)
    cache.k.copy_(rand(g, n, page, KV, D, dtype=dtype)), cache.v.copy_(rand(g, n, page, KV, D, dtype=dtype))
    into = None
    if into_order:
        into = serving.PagedCache.empty(n + 5, page, KV, D, DT[dtype], order=into_order)
        into.k.fill_(3.0), into.v.fill_(4.0)
    to = into or cache
    src, dst = [0, 3, 3, 7, -1, 9, 11, -5, 2, 1], [20, 21, 22, 23, 24, -2, 26, 27, 28, 29]
    tokens = [page, 1, 0, page // 2, 3, 3, page + 100, 5, -4, max(1, page - 1)]
    for t in (None, tokens):
        want = [x.clone() for x in (to.k, to.v)]
        for i, (a, b) in enumerate(zip(src, dst)):
            if a >= 0 and b >= 0:
                m = page if t is None else max(0, min(page, t[i]))
                want[0][b, :m], want[1][b, :m] = cache.k[a, :m], cache.v[a, :m]
        status = ints([0])
        serving.copy_pages(cache, ints(src), ints(dst), None if t is None else ints(t), into=into, status=status)
        assert int(status) == 0 and torch.equal(to.k, want[0]) and torch.equal(to.v, want[1])
        to.k[20:30] = 0.5


@pytest.mark.parametrize("shift", [1, 3])
def test_copy_off_the_grid(shift):
    page, KV, D = 16, 2, 64
    whole = torch.zeros(2, 30, page, KV * D + 8, dtype=torch.bfloat16, device="cuda")
    views = [x[:, :, shift:shift + KV * D].unflatten(2, (KV, D)) for x in whole]
    for x in views:
        x.copy_(rand(gen(1), 30, page, KV, D, dtype="bfloat16"))
    before = whole.clone()
    serving.copy_pages(serving.PagedCache(*views), ints([1, 2]), ints([11, 12]), ints([16, 5]))
    before[:, 11, :, shift:shift + KV * D] = before[:, 1, :, shift:shift + KV * D]
    before[:, 12, :5, shift:shift + KV * D] = before[:, 2, :5, shift:shift + KV * D]
    assert torch.equal(whole, before)


def test_copy_out_of_range_and_refusals():
    cache = serving.PagedCache.empty(10, 16, 2, 64, torch.bfloat16)
    cache.k.copy_(rand(gen(1), 10, 16, 2, 64, dtype="bfloat16")), cache.v.copy_(cache.k)
    was = cache.k.clone()
    for src, dst in ((10, 1), (1, 10), (1 << 30, 0), (0, (1 << 31) - 1)):
        status = ints([0])
        serving.copy_pages(cache, ints([src]), ints([dst]), status=status)
        assert int(status) == gts.GTS_ERR_INVALID_PARAMS
        serving.copy_pages(cache, ints([src]), ints([dst]))
        assert torch.equal(cache.k, was)
    serving.copy_pages(cache, ints([]), ints([]))
    serving.copy_pages(cache, ints([4]), ints([4]))
    assert torch.equal(cache.k, was)
    other = serving.PagedCache.empty(10, 16, 2, 64, torch.float16)
    small = serving.PagedCache.empty(10, 8, 2, 64, torch.bfloat16)
    for kw in (dict(src=ints([1]).long()), dict(dst=ints([1, 2])), dict(tokens=ints([])), dict(into=other), dict(into=small),
               dict(status=ints([1, 2])), dict(src=ints([1]).cpu())):
        with pytest.raises(gts.GtsError):
            serving.copy_pages(**{**dict(cache=cache, src=ints([1]), dst=ints([2])), **kw})


# ---------------------------------------------------------------- together
def test_a_prompt_in_chunks_and_a_fork():
    """A prompt appended and attended in chunks has the results of the whole prompt at once; a fork of it (full pages shared, the
    last one copied) goes on with other tokens, and neither disturbs the other."""
    H, KV, D, page, n = 8, 2, 128, 16, 300
    g = gen(12)
    rotary = serving.Rotary(D)
    rows = rand(g, n, H + 2 * KV, D, dtype="bfloat16")
    q, k, v = rows.split([H, KV, KV], 1)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    rq, rk = serving.rope(q, k, pos, rotary)
    whole, lse = serving.prompt_attention(rq, rk, v, ints([0, n]))
    _, (bound, b_lse), _, _ = R.packed(f64(rq), f64(rk), f64(v), [0, n], D ** -0.5, True, "bfloat16")
    cache = serving.PagedCache.empty(60, page, KV, D, torch.bfloat16)
    cache.k.fill_(float("nan")), cache.v.fill_(float("nan"))
    pages = torch.randperm(60, generator=g).to(torch.int32).cuda()
    table = pages[:30][None].contiguous()

    def put(part, table, first):
        p = torch.arange(first, first + len(part[0]), dtype=torch.int32, device="cuda")
        slots = table[0].long()[p.long() // page] * page + p % page
        return serving.append_kv(*part, p, slots, rotary, cache)
    done = 0
    for size in (100, 1, 150, 49):
        part = [x[done:done + size] for x in (q, k, v)]
        aq = put(part, table, done)
        done += size
        out, l = serving.chunk_attention(aq, ints([0, size]), cache, table, ints([done]))
        at = slice(done - size, done)
        assert (np.abs(f64(out) - f64(whole[at])) <= 2 * bound[at]).all()
        assert (np.abs(f64(l) - f64(lse[at])) <= 2 * b_lse[at]).all()
    full = n // page
    fork = table.clone()
    fork[0, full:] = pages[30:30 + fork.shape[1] - full]
    serving.copy_pages(cache, table[0, full:full + 1].contiguous(), fork[0, full:full + 1].contiguous(), ints([n - full * page]))
    more = [rand(g, 20, x, D, dtype="bfloat16") for x in (H, KV, KV)]
    other = [rand(g, 20, x, D, dtype="bfloat16") for x in (H, KV, KV)]
    a, b = put(more, table, n), put(other, fork, n)
    both = serving.chunk_attention(torch.cat([a, b]), ints([0, 20, 40]), cache, torch.cat([table, fork]), ints([n + 20] * 2))
    p2 = torch.arange(n + 20, dtype=torch.int32, device="cuda")
    for i, tail in enumerate((more, other)):
        x = [torch.cat([s, t]) for s, t in zip((q, k, v), tail)]
        xq, xk = serving.rope(x[0], x[1], p2, rotary)
        (want, w_lse), (bo, bl), _, _ = R.packed(f64(xq), f64(xk), f64(x[2]), [0, n + 20], D ** -0.5, True, "bfloat16")
        check(both[0][i * 20:(i + 1) * 20], want[n:], bo[n:], "fork")
        check(both[1][i * 20:(i + 1) * 20], w_lse[n:], bl[n:], "fork")


def test_a_training_step_through_the_rotation():
    """Gradients through rope and prompt_attention to one projection's rows."""
    lens, H, KV, D = [60, 90], 4, 2, 64
    g = gen(30)
    rotary = serving.Rotary(D)
    rows = rand(g, 150, H + 2 * KV, D, dtype="bfloat16").requires_grad_()
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).cuda()
    q, k, v = rows.split([H, KV, KV], 1)
    rq, rk = serving.rope(q, k, pos, rotary)
    out, _ = serving.prompt_attention(rq, rk, v, ints(rows_of(lens)))
    dout = rand(g, *out.shape, dtype="bfloat16")
    out.backward(dout)
    d = [rq.detach(), rk.detach(), v.detach()]
    low = torch.empty_like(d[0])
    o, l = serving.prompt_attention(*d, ints(rows_of(lens)), low=low)
    dq, dk, dv = serving.prompt_attention_grad(dout, *d, o, l, ints(rows_of(lens)), low=low)
    dq, dk = serving.rope_grad(dq, dk, pos, rotary)
    assert torch.equal(rows.grad, torch.cat([dq, dk, dv], 1))
