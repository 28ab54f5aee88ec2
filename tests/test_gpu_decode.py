"""The decode step as a serving program runs it: append with rotation, attention over a shared prompt and each sequence's
own tokens, against attention without a cache; and its tile graph, simulated."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("case", [dict(seqs=1, prefix=40, own=3), dict(seqs=5, prefix=300, own=1), dict(seqs=33, prefix=1000, own=70)])
def test_step_is_attention_without_a_cache(case):
    """Both sides hold rotated values in 16 bits; the step's weights are rounded to 16 bits too (2^-8 of each, independent) and
    so are the results: a few 2^-8 of the largest values, which are under 6 root mean squares."""
    from paper_2607_11262_gb300 import decode
    step = decode.Step(**case, page=16)
    assert step.check() < 6 * 4 * 2.0 ** -8


def test_study_runs_and_simulates():
    from paper_2607_11262_gb300 import study
    rows = study.run_decode_study([dict(seqs=48, prefix=2048, own=64)])
    assert rows[0]["cycles"] > 0 and rows[0]["attend_us"] > 0 and "prefix" in study.format_decode_table(rows)
