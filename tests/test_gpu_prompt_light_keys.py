"""float16: many keys of so little weight that each alone would vanish beside the largest one."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests.test_gpu_prompt import ints  # noqa: E402
from tests.test_gpu_serving import check, f64, gen, rand  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()


def scores(q, k, gap, heavy):
    """q = 8 in one place; keys there so that the heavy ones lie `gap` (log 2) above the others, in steps that are numbers of the type."""
    q.zero_(), k.zero_()
    q[..., 0] = 8.0
    k[..., 0] = -round(gap * np.log(2) * 128 / 8) / 128
    k[heavy, ..., 0] = 0.0


@pytest.mark.parametrize("heavy", [0, 5000, 39999])
@pytest.mark.parametrize("gap", [20.0, 25.5, 27.0])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_that_add_up(D, gap, heavy):
    """out is the light keys' share of values of 1 (to 1.25), the heavy key's value being 0.  A weight is off by half a step of its type and,
    held times 2^7 against a maximum that is not above the largest score, by 2^-32 of the largest one; p |v| sums to A, the weights to 1
    or more.  So |out error| <= (2^-11 + 4 ds + (64 + n) 2^-24) A + 2^-11 |out| + 2^-25 + 2^-32 sum |v|."""
    n, page = 40000, 64
    g = gen(D)
    cache = serving.PagedCache.empty(-(-n // page), page, 1, D, torch.float16)
    q, k = torch.zeros(3, 2, D, dtype=torch.float16, device="cuda"), torch.zeros(cache.k.numel() // D, 1, D, dtype=torch.float16, device="cuda")
    scores(q, k, gap, heavy)
    v = (1 + 0.25 * torch.rand(k.shape, generator=g, dtype=torch.float32).cuda()).half()
    v[heavy] = 0
    cache.k.copy_(k.view(cache.k.shape)), cache.v.copy_(v.view(cache.v.shape))
    table = torch.arange(cache.n_pages, dtype=torch.int32, device="cuda")[None]
    out, lse = serving.chunk_attention(q, ints([0, 3]), cache, table, ints([n]), scale=1.0)
    s = 8 * f64(k[:n, 0, 0])
    p, z = np.exp(s), f64(v[:n, 0])
    ds = (D + 4) * 2.0 ** -24 * np.abs(s).max() + 4 * 2.0 ** -24 * np.abs(s).max()
    for i in range(3):
        m = n - 2 + i
        if heavy >= m:
            continue
        total = p[:m].sum()
        assert total >= 1
        want = p[:m] @ z[:m] / total
        bound = (2.0 ** -11 + 4 * ds + (64 + m) * 2.0 ** -24) * want + 2.0 ** -11 * want + 2.0 ** -25 + 2.0 ** -32 * z[:m].sum(0)
        check(out[i], np.stack([want] * 2), np.stack([bound] * 2), (i, "out"))
        check(lse[i], np.full(2, np.log(total)), np.full(2, 2 * ds + (16 + m) * 2.0 ** -24), (i, "lse"))


def test_weights_that_add_up_in_a_prompt():
    """The same for packed sequences, causal: the first key is the heavy one of each."""
    n, D = 9000, 64
    q, k = (torch.zeros(2 * n, 1, D, dtype=torch.float16, device="cuda") for _ in range(2))
    scores(q, k, 25.5, [0, n])
    v = (1 + 0.25 * rand(gen(1), 2 * n, 1, D, dtype="float32").abs().clamp(max=1.0)).half()
    v[[0, n]] = 0
    out, lse = serving.prompt_attention(q, k, v, ints([0, n, 2 * n]), scale=1.0)
    for a in (0, n):
        p, z = np.exp(8 * f64(k[a:a + n, 0, 0])), f64(v[a:a + n, 0])
        total, some = np.cumsum(p)[:, None], np.cumsum(p[:, None] * z, 0)
        want, m = some / total, np.arange(1, n + 1)[:, None]
        ds = (D + 8) * 2.0 ** -24 * 25.5
        bound = (2.0 ** -10 + 4 * ds + (64 + m) * 2.0 ** -24) * want + 2.0 ** -25 + 2.0 ** -32 * np.cumsum(z, 0)
        check(out[a:a + n, 0], want, bound, "out")
        check(lse[a:a + n], np.log(total), 2 * ds + (16 + m) * 2.0 ** -24 * (1 + np.abs(np.log(total))), "lse")
