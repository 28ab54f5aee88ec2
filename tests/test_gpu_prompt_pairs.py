"""Prompts' attention when waits run out at an item's end: the two warps of a row leave together, whatever the next item has for
them."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests import short_waits_prompt  # noqa: E402
from tests.test_gpu_prompt import ints, problem  # noqa: E402
from tests.test_gpu_prompt_waits import either, scribbled  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def short(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()
    return short_waits_prompt.build(str(tmp_path_factory.mktemp("short_waits_prompt")))


# as many key heads as query heads: items of 256 queries, of which a sequence of 100 leaves the second half without rows
@pytest.mark.parametrize("lens", [[200, 100] * 60, [100] * 150, [700, 100, 300] * 30])
@pytest.mark.parametrize("tries", [0, 3, 10, 30, 60, 100, 200, 400, 800])
@pytest.mark.parametrize("D", [64, 128])
def test_items_without_rows_for_a_half(short, monkeypatch, D, tries, lens):
    q, k, v, starts = problem(D, lens, 4, 4, D, "bfloat16")
    at = ints(starts)
    assert short.set_tries(tries) == 0
    for causal in (True, False):
        want = serving.prompt_attention(q, k, v, at, causal=causal)
        need = serving.prompt_workspace(q, k, at).numel()
        with monkeypatch.context() as m:
            m.setattr(serving, "_lib", short)
            for seed in range(5):
                status = ints([0])
                got = serving.prompt_attention(q, k, v, at, causal=causal, workspace=scribbled(need, seed), status=status)
                lost = [either(x, y) for x, y in zip(got, want)]
                assert lost[0] == lost[1] and (not lost[0] or int(status) == gts.GTS_ERR_STEP_LIMIT)
                if tries == 0:
                    assert int(status) == gts.GTS_ERR_STEP_LIMIT and lost[0]
        again = serving.prompt_attention(q, k, v, at, causal=causal)
        assert all(torch.equal(x, y) for x, y in zip(again, want))


@pytest.mark.parametrize("tries", [0, 10, 60, 200, 800])
@pytest.mark.parametrize("D", [64, 128])
def test_infinite_values_when_waits_run_out(short, monkeypatch, D, tries):
    """Where values are added by hand: rows of out and dv have them, as they should, or are NaN throughout."""
    lens = [200, 100, 300, 64] * 30
    q, k, v, starts = problem(D, lens, 4, 2, D, "bfloat16")
    at, dout = ints(starts), q.clone()
    for b in range(1, len(lens), 2):
        v[starts[b] + 7 + b % 50, :, (b * 13) % D] = float("inf")
    out, lse = serving.prompt_attention(q, k, v, at)
    finite = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    plain = serving.prompt_attention(q, k, finite, at)
    for b in range(0, len(lens), 2):
        dout[starts[b] + 9 + b % 50, :, (b * 29) % D] = float("inf")
    dv = serving.prompt_attention_grad(dout, q, k, finite, *plain, at)[2]
    assert not torch.isnan(out).any() and not torch.isnan(dv).any()
    need = serving.prompt_workspace(q, k, at).numel()
    assert short.set_tries(tries) == 0
    with monkeypatch.context() as m:
        m.setattr(serving, "_lib", short)
        for seed in range(5):
            status = ints([0])
            got = serving.prompt_attention(q, k, v, at, workspace=scribbled(need, seed), status=status)
            lost = [either(x, y) for x, y in zip(got, (out, lse))]
            assert lost[0] == lost[1] and (not lost[0] or int(status) == gts.GTS_ERR_STEP_LIMIT)
            status = ints([0])
            got = serving.prompt_attention_grad(dout, q, k, finite, *plain, at, status=status)[2]
            assert not either(got, dv) or int(status) == gts.GTS_ERR_STEP_LIMIT
    again = serving.prompt_attention(q, k, v, at)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
