"""The gradient's kernels start while the one before ends: each sees what that has written, not what an earlier call left in the
workspace."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests.test_gpu_prompt import ints, problem  # noqa: E402
from tests.test_gpu_serving import gen, rand  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("lens,H,KV,D", [([40], 4, 2, 64), ([1000], 8, 2, 128), ([300, 5, 700] * 8, 4, 4, 64), ([129] * 100, 2, 1, 128)])
def test_one_workspace_for_call_after_call(lens, H, KV, D, dtype):
    """Two problems in turn over one workspace, with dout of very different size: results are those of calls by themselves."""
    at, sides = None, []
    for seed, size in ((1, 1.0), (2, 2.0 ** -9)):
        q, k, v, starts = problem(seed, lens, H, KV, D, dtype)
        at = ints(starts)
        dout = (rand(gen(seed + 5), *q.shape, dtype="float32") * size).to(q.dtype)
        out, lse = serving.prompt_attention(q, k, v, at)
        sides.append(((dout, q, k, v, out, lse, at), serving.prompt_attention_grad(dout, q, k, v, out, lse, at)))
    torch.cuda.synchronize()
    workspace = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(60):
        got = [serving.prompt_attention_grad(*x, workspace=workspace) for x, _ in sides for _ in range(2)]
        for i, g in enumerate(got):
            for a, b in zip(g, sides[i // 2][1]):
                wrong += (a != b).sum()
    assert int(wrong) == 0
