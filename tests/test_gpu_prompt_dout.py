"""Values of dout that are not finite: in dv they are in their column of the keys that their row sees, and nowhere else."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests.test_gpu_prompt import ints, problem  # noqa: E402
from tests.test_gpu_serving import f64, gen, rand  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,H,KV,D", [([100, 200, 300], 8, 2, 64), ([100, 200, 300], 8, 2, 128), ([70, 130], 6, 2, 128), ([3000], 4, 4, 64),
                                         ([1500, 33], 4, 1, 128), ([150], 128, 1, 64), ([5, 128, 129, 1] * 30, 4, 4, 128)])
def test_infinite_values_of_dout(lens, H, KV, D, causal, dtype):
    q, k, v, starts = problem(D + H, lens, H, KV, D, dtype)
    at, dout, G = ints(starts), rand(gen(2), *q.shape, dtype=dtype), H // KV
    out, lse = serving.prompt_attention(q, k, v, at, causal=causal)
    want = serving.prompt_attention_grad(dout, q, k, v, out, lse, at, causal=causal)
    rng, bad = np.random.default_rng(D), dout.clone()
    for i, (a, b) in enumerate(zip(starts[:-1], starts[1:])):
        if i % 2 and len(lens) > 3:
            continue
        rows = sorted({a, b - 1, (a + b) // 2, min(a + 127, b - 1), min(a + 128, b - 1)} | set(rng.integers(a, b, 3).tolist()))
        for n, row in enumerate(rows):
            column = int(rng.integers(0, D))
            bad[row, int(rng.integers(0, H)), [column, (column + 40) % D]] = [float("inf"), float("-inf"), float("nan")][(n + i) % 3]
    # the sum of the values that are not finite, for each key and column (weights are positive), and the gradients without a part in them
    odd, same = np.zeros(v.shape), [np.ones(x.shape[:2], bool) for x in (q, k)]
    for row, head, c in torch.nonzero(~torch.isfinite(bad)).tolist():
        a, b = max(s for s in starts if s <= row), min(s for s in starts if s > row)
        seen = slice(a, row + 1 if causal else b)
        with np.errstate(invalid="ignore"):
            odd[seen, head // G, c] += float(bad[row, head, c])
        same[0][row, head] = same[1][seen, head // G] = False
    got = serving.prompt_attention_grad(bad, q, k, v, out, lse, at, causal=causal)
    there = torch.from_numpy(odd != 0).cuda()                                      # (NaN != 0)
    assert torch.equal(got[2][~there], want[2][~there])
    assert np.array_equal(f64(got[2])[odd != 0], odd[odd != 0], equal_nan=True)
    for x, y, m in zip(got[:2], want[:2], same):
        m = torch.from_numpy(m).cuda()
        if dtype == "bfloat16":                                                    # (float16's units are from the finite values)
            assert torch.equal(x[m], y[m])
        assert torch.isfinite(x[m]).all() and not torch.isfinite(x[~m]).all(-1).any()
    again = serving.prompt_attention_grad(bad, q, k, v, out, lse, at, causal=causal)
    assert all(torch.equal(torch.nan_to_num(x, 3.0, 5.0, 7.0), torch.nan_to_num(y, 3.0, 5.0, 7.0)) for x, y in zip(again, got))
