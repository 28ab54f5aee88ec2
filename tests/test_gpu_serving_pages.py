"""Attention and page numbers that are none."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests.test_gpu_serving import problem  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()


@pytest.mark.parametrize("page", [16, 100])
@pytest.mark.parametrize("low", [-2 ** 31, -2 ** 31 + 5, -2 ** 30])
@pytest.mark.parametrize("B,prefix", [(2, 200), (48, 700), (3, 0)])
def test_the_lowest_page_numbers_are_out_of_range(B, prefix, low, page):
    """No negative number is a page, however low: the status says so, and the rows that do not see it are what they were."""
    for what in ("prefix_pages", "page_table"):
        if what == "prefix_pages" and not prefix:
            continue
        p = problem(8, 8, 2, 128, page, "tokens", "bfloat16", prefix, [150] * B, 1, rubbish=0.0)
        want = serving.prefix_attention(**p)
        p[what][(1,) if what == "prefix_pages" else (1, 1)] = low
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = serving.prefix_attention(**p, status=status)
        assert int(status) == gts.GTS_ERR_INVALID_PARAMS, what
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        if what == "page_table":
            others = torch.arange(B, device="cuda") != 1
            assert torch.equal(out[others], want[0][others]) and torch.equal(lse[others], want[1][others])
