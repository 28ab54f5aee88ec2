"""Prompts' attention where a block goes from item to item: what one of them holds stays out of the one before."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests.test_gpu_prompt import ints, problem  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,H,KV", [([256, 130, 200, 140] * 100, 4, 4), ([64, 40, 100, 50] * 150, 8, 2), ([128, 129, 300, 100] * 60, 14, 2)])
def test_values_of_the_next_item(lens, H, KV, D, bad):
    """Many items to a block, every other sequence with values that are not finite in its first tile, which some of its rows do not
    see: the rows that do have them in their column, all else is what it was, bit for bit and time after time."""
    q, k, v, starts = problem(D + H, lens, H, KV, D, "bfloat16")
    at = ints(starts)
    out, lse = serving.prompt_attention(q, k, v, at)
    x, hit = v.clone(), torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    for b in range(1, len(lens), 2):
        for head in range(KV):
            key, column = starts[b] + (b * 7 + head) % min(39, lens[b]), (b * 13 + head * 29) % D
            x[key, head, column] = bad
            hit[key:starts[b + 1], head * (H // KV):(head + 1) * (H // KV), column] = True
    for _ in range(20):
        o, l = serving.prompt_attention(q, k, x, at)
        assert torch.equal(l, lse)
        assert torch.equal(o[~hit], out[~hit])
        assert not torch.isfinite(o[hit]).any()
