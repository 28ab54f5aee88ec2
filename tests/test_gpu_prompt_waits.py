"""Prompts' attention when its waits run out (tests/short_waits_prompt.py): every block ends, its copies and products with it, the status
says so, rows that miss a part are NaN, nothing outside the results is written, and the calls after it are what they were."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests import short_waits_prompt  # noqa: E402
from tests.test_gpu_prompt import ints, paged, problem, rand, gen  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def short(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()
    return short_waits_prompt.build(str(tmp_path_factory.mktemp("short_waits_prompt")))


def either(got, want):
    """Rows of a head are what they should be or NaN throughout; whether any are lost."""
    lost = torch.isnan(got).flatten(2).all(-1) if got.dim() == 3 else torch.isnan(got)
    assert torch.equal(got[~lost], want[~lost])
    return bool(lost.any())


def scribbled(x, seed):
    return torch.randint(-1 << 31, (1 << 31) - 1, (-(-x // 4),), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


# lengths, heads, key heads
CASES = [([2000], 8, 2), ([300, 40, 700, 1], 4, 4), ([130] * 40, 6, 2), ([64] * 100, 2, 1)]


@pytest.mark.parametrize("tries", [0, 30, 300])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_prompt_blocks_end_and_say_so(short, monkeypatch, case, D, tries):
    q, k, v, starts = problem(D + case, *CASES[case], D, "bfloat16", before=3, after=5)
    at, dout = ints(starts), rand(gen(3), *q.shape, dtype="bfloat16")
    assert short.set_tries(tries) == 0
    for causal in (True, False):
        want = serving.prompt_attention(q, k, v, at, causal=causal)
        grads = serving.prompt_attention_grad(dout, q, k, v, *want, at, causal=causal)
        need = serving.prompt_workspace(q, k, at).numel()
        with monkeypatch.context() as m:
            m.setattr(serving, "_lib", short)
            for seed in range(3):
                out, lse, status = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device="cuda"), ints([0])
                serving.prompt_attention(q, k, v, at, causal=causal, out=out, lse=lse, workspace=scribbled(need, seed), status=status)
                torch.cuda.synchronize()
                assert (out[:3] == 9).all() and (out[-5:] == 9).all() and (lse[:3] == 9).all() and (lse[-5:] == 9).all()
                lost = [either(x[3:-5], y[3:-5]) for x, y in zip((out, lse), want)]
                assert lost[0] == lost[1] and int(status) == (gts.GTS_ERR_STEP_LIMIT if tries == 0 or lost[0] else int(status))
                assert not lost[0] or int(status) == gts.GTS_ERR_STEP_LIMIT
                to, status = [torch.full_like(x, 9.0) for x in (q, k, v)], ints([0])
                serving.prompt_attention_grad(dout, q, k, v, *want, at, causal=causal, out_dq=to[0], out_dk=to[1], out_dv=to[2], status=status)
                torch.cuda.synchronize()
                assert all((x[:3] == 9).all() and (x[-5:] == 9).all() for x in to)
                lost = [either(x[3:-5], y[3:-5]) for x, y in zip(to, grads)]
                assert not any(lost) or int(status) == gts.GTS_ERR_STEP_LIMIT
                if tries == 0:
                    assert int(status) == gts.GTS_ERR_STEP_LIMIT and all(lost)
        again = serving.prompt_attention(q, k, v, at, causal=causal)
        assert all(torch.equal(x, y) for x, y in zip(again, want))
        again = serving.prompt_attention_grad(dout, q, k, v, *want, at, causal=causal)
        assert all(torch.equal(x, y) for x, y in zip(again, grads))


@pytest.mark.parametrize("tries", [0, 30, 300])
@pytest.mark.parametrize("page", [64, 100])
@pytest.mark.parametrize("D", [64, 128])
def test_chunk_blocks_end_and_say_so(short, monkeypatch, D, page, tries):
    p, _, _ = paged(D, [200, 1, 40, 0, 90], [1500, 300, 40, 10, 777], 8, 2, D, page, "heads", "bfloat16", fill=0.0)
    want = serving.chunk_attention(**p)
    assert short.set_tries(tries) == 0
    with monkeypatch.context() as m:
        m.setattr(serving, "_lib", short)
        for _ in range(3):
            status = ints([0])
            got = serving.chunk_attention(**p, status=status)
            lost = [either(x, y) for x, y in zip(got, want)]
            assert lost[0] == lost[1] and (not lost[0] or int(status) == gts.GTS_ERR_STEP_LIMIT)
            if tries == 0:
                assert int(status) == gts.GTS_ERR_STEP_LIMIT and lost[0]
    again = serving.chunk_attention(**p)
    assert all(torch.equal(x, y) for x, y in zip(again, want))
