"""Gradients in float16 over its range: ds is held times a power of two of what bounds it, so neither a gradient of lse that outweighs
dout, nor one by itself, nor large values overflow or vanish."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests import prompt_reference as R  # noqa: E402
from tests.test_gpu_prompt import ints, problem  # noqa: E402
from tests.test_gpu_serving import check, f64, gen, rand  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()


def rest(q, k, v, starts, scale, causal, dout, dlse):
    """What rounding takes from a ds below 2^-14 in its units: with B = 2 max |dout_i| max |v_j| + max |dlse_i| over all sequences (norms
    of rows) ds is held times f >= 2^14 / B, in steps of 2^-24: each is off by 2^-25 / f <= 2^-39 B.  Summed over the keys (rows) seen."""
    rows = slice(starts[0], starts[-1])
    B = 2 * np.linalg.norm(dout[rows], axis=-1).max() * np.linalg.norm(v[rows], axis=-1).max() + np.abs(dlse[rows]).max()
    g, got = q.shape[1] // k.shape[1], [np.zeros(q.shape), np.zeros(k.shape), 0.0]
    for a, b in zip(starts[:-1], starts[1:]):
        seen = np.tril(np.ones((b - a, b - a))) if causal else np.ones((b - a, b - a))
        for h in range(q.shape[1]):
            got[0][a:b, h] += scale * 2.0 ** -39 * B * seen @ np.abs(k[a:b, h // g])
            got[1][a:b, h // g] += scale * 2.0 ** -39 * B * seen.T @ np.abs(q[a:b, h])
    return got


def check_gradients(q, k, v, starts, causal, dout, dlse, got):
    x = [f64(t) for t in (q, k, v, dout, dlse)]
    scale = q.shape[2] ** -0.5
    want, bound = R.packed(*x[:3], starts, scale, causal, "float16", *x[3:])[2:]
    assert max(np.abs(w).max() for w in want) < 60000          # (they are numbers of the type)
    for name, a, w, b, more in zip(("dq", "dk", "dv"), got, want, bound, rest(*x[:3], starts, scale, causal, *x[3:])):
        assert torch.isfinite(a).all(), name
        check(a, w, b + more, name)


SHAPES = [([1], 4, 2, 64), ([70, 1, 300], 4, 2, 128), ([500, 200], 6, 2, 64), ([3, 129] * 4, 2, 2, 128)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("of_dout,of_dlse", [(1e-6, 1.0), (1e-5, 30.0), (1.0, 1e-6), (0.0, 1.0), (0.0, 2.0 ** 16), (0.0, 2.0 ** -16), (0.0, 1e-30), (0.0, 0.0),
                                             (2.0 ** -13, 300.0), (300.0, 2.0 ** -13)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_gradients_of_lse_and_out_of_any_size(shape, of_dout, of_dlse, causal):
    lens, H, KV, D = SHAPES[shape]
    q, k, v, starts = problem(shape, lens, H, KV, D, "float16", before=2, after=3)
    if of_dlse == 2.0 ** 16:                                   # (gradients as large as the type's numbers)
        q, k = q / 16, k / 16
    g, at = gen(shape), ints(starts)
    dout = (rand(g, *q.shape, dtype="float32") * of_dout).half()
    dlse = rand(g, *q.shape[:2], dtype="float32") * of_dlse
    for x in (dout, dlse):                                     # rows of no sequence hold anything
        x[:2], x[starts[-1]:] = float("nan"), 60000.0
    out, lse = serving.prompt_attention(q, k, v, at, causal=causal)
    got = serving.prompt_attention_grad(dout, q, k, v, out, lse, at, causal=causal, dlse=dlse)
    check_gradients(q, k, v, starts, causal, dout, dlse, got)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("size,of_dout", [(2000.0, 0.05), (60000.0, 1e-4), (2000.0, 1e-6), (1e-3, 300.0)])
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_any_size(D, size, of_dout, causal):
    """Values that all point dout's way or all the other one: dout . v is as large as it can be."""
    q, k, v, starts = problem(D, [300, 40], 4, 2, D, "float16")
    g, at = gen(D), ints(starts)
    sign = torch.where(rand(g, v.shape[0], v.shape[1], 1, dtype="float32") < 0, -1.0, 1.0)
    v = (sign * size * (1 + 0.01 * rand(g, *v.shape, dtype="float32").clamp(-5, 5))).half()
    dout = (of_dout * (1 + 0.01 * rand(g, *q.shape, dtype="float32"))).half()
    dlse = torch.zeros(q.shape[:2], device="cuda")
    out, lse = serving.prompt_attention(q, k, v, at, causal=causal)
    got = serving.prompt_attention_grad(dout, q, k, v, out, lse, at, causal=causal)
    check_gradients(q, k, v, starts, causal, dout, dlse, got)


def test_a_loss_of_lse_alone():
    """Through autograd, with a loss's scale of 65536."""
    q, k, v, starts = problem(1, [200, 1, 77], 4, 2, 64, "float16")
    q, k = q / 16, k / 16
    x = [t.detach().requires_grad_() for t in (q, k, v)]
    _, lse = serving.prompt_attention(*x, ints(starts))
    (lse.sum() * 65536.0).backward()
    zero, dlse = torch.zeros_like(q), torch.full(q.shape[:2], 65536.0, device="cuda")
    check_gradients(q, k, v, starts, True, zero, dlse, [t.grad for t in x])


def test_a_row_of_infinities_does_not_set_the_units():
    """Infinite dout, values and gradients of lse of one sequence: the others' gradients are what they were."""
    q, k, v, starts = problem(3, [50, 60, 70], 4, 2, 64, "float16")
    g, at = gen(3), ints(starts)
    dout, dlse = rand(g, *q.shape, dtype="float16"), rand(g, *q.shape[:2], dtype="float32")
    out, lse = serving.prompt_attention(q, k, v, at)
    want = serving.prompt_attention_grad(dout, q, k, v, out, lse, at, dlse=dlse)
    for bad in (float("inf"), float("nan")):
        for which in range(3):
            d, w, l = dout.clone(), v.clone(), dlse.clone()
            (d, w, l)[which][60] = bad
            o, s = serving.prompt_attention(q, k, w, at)
            got = serving.prompt_attention_grad(d, q, k, w, o, s, at, dlse=l)
            for a, b in zip(got, want):
                others = [i for i in range(180) if not 50 <= i < 110]
                check(a[others], f64(b[others]), 2.0 ** -10 * np.abs(f64(b[others])) + 2.0 ** -20, (bad, which))
