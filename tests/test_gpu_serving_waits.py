"""Attention when its waits run out (tests/short_waits.py): every block ends, its copies and products with it, the status says
so, rows that miss a part are NaN, nothing outside the results is written, and the calls after it are what they were."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests import short_waits  # noqa: E402
from tests.test_gpu_serving import problem  # noqa: E402
from tests.test_gpu_serving_paths import widen_table  # noqa: E402

pytestmark = pytest.mark.gpu

GUARD = 64


@pytest.fixture(scope="module")
def short(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()
    return short_waits.build(str(tmp_path_factory.mktemp("short_waits")))


def call(p, seed):
    """(out, lse, status) of a call into the middle of larger buffers, with a workspace of whatever it was."""
    B, new, H, D = p["q"].shape
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = torch.full((B + 2 * GUARD, new, H, D), 9.0, dtype=p["q"].dtype, device="cuda")
    sums = torch.full((B + 2 * GUARD, new, H), 9.0, device="cuda")
    need = serving.attention_workspace(p["cache"], p["q"], p["prefix_len"], p["page_table"]).numel()
    workspace = torch.randint(-1 << 31, (1 << 31) - 1, (-(-need // 4),), dtype=torch.int32, device="cuda", generator=g)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = serving.prefix_attention(**p, out=rows[GUARD:-GUARD], lse=sums[GUARD:-GUARD], workspace=workspace, status=status)
    torch.cuda.synchronize()
    for x in (rows, sums):
        assert torch.all(x[:GUARD] == 9.0) and torch.all(x[-GUARD:] == 9.0)
    return out, lse, int(status)


WITH_PREFIX = [dict(lens=[40 + b % 90 for b in range(64)], prefix=3000), dict(lens=[300, 0, 77] * 10, prefix=100),
               dict(lens=[60 + b for b in range(40)], prefix=1500, new=5), dict(lens=[500] * 6, prefix=400, page=100),
               dict(lens=[0] * 200, prefix=2000), dict(lens=[200] * 30, prefix=700, kv=4, columns=40)]
WITHOUT = [dict(lens=[300 + 11 * b for b in range(40)], prefix=0), dict(lens=[700] * 30, prefix=0, kv=4, columns=20),
           dict(lens=[0, 400, 90, 0] * 20, prefix=0, new=5), dict(lens=[2000] * 3, prefix=0, page=100),
           dict(lens=[900] * 20, prefix=0, new=16)]
CASES = WITH_PREFIX + WITHOUT


def make(D, lens, prefix, new=1, page=64, kv=2, columns=0):
    p = problem(D + prefix, 8, kv, D, page, "heads", "bfloat16", prefix, lens, new, rubbish=0.0)
    return widen_table(p, columns) if columns else p


@pytest.mark.parametrize("tries", [0, 30, 300])
@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_blocks_end_and_say_so(short, monkeypatch, case, D, tries):
    p = make(D, **CASES[case])
    want = serving.prefix_attention(**p)
    assert short.set_tries(tries) == 0
    with monkeypatch.context() as m:
        m.setattr(serving, "_lib", short)
        for seed in range(3):
            out, lse, status = call(p, seed)
            # a row is either what it should be or NaN throughout, lse and all
            lost = torch.isnan(lse)
            assert torch.equal(torch.isnan(out), lost[..., None].expand_as(out))
            assert torch.equal(out[~lost], want[0][~lost]) and torch.equal(lse[~lost], want[1][~lost])
            if tries == 0:  # no tile arrives that soon
                assert status == gts.GTS_ERR_STEP_LIMIT and lost.any()
            if status == gts.GTS_OK:
                assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    again = call(p, 7)
    assert again[2] == gts.GTS_OK and torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
