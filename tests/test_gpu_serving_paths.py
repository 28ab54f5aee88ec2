"""Attention of a decode step where the kernels' ways part: heads taken by fours or one by one, more row tiles than SMs, values
that are not finite behind a causal mask, and gathers beside boxes (bounds: tests/serving_reference.py)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests import serving_reference as R  # noqa: E402
from tests.test_gpu_serving import check, check_attention, f64, problem  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    gts.load()


def widen_table(p, pages):
    """The same problem with a page table of more columns than any sequence needs."""
    t = torch.full((p["page_table"].shape[0], pages), -7, dtype=torch.int32, device="cuda")
    t[:, :p["page_table"].shape[1]] = p["page_table"]
    return {**p, "page_table": t}


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("heads", [(8, 4), (32, 8), (12, 12), (6, 3)])
@pytest.mark.parametrize("page", [16, 100])
def test_heads_by_fours_and_by_ones(D, heads, page):
    for prefix in (0, 90):
        p = problem(D + page, *heads, D, page, "heads", "bfloat16", prefix, [0, 5, 64, 200, 17, 0, 33, 130], 1)
        check_attention(p, "bfloat16")
        check_attention(widen_table(p, -(-2100 // page)), "bfloat16")


@pytest.mark.parametrize("lens", [[0] * 9, [1] * 7 + [0], [3000, 1, 1, 1], [700] * 3])
@pytest.mark.parametrize("heads", [(8, 8), (8, 1)])
def test_cuts_anywhere(lens, heads):
    """Few or no keys, one sequence that takes all blocks, equal ones."""
    for prefix in (0, 257):
        check_attention(problem(len(lens), *heads, 64, 16, "tokens", "float16", prefix, lens, 1), "float16")
        check_attention(problem(len(lens), *heads, 64, 16, "tokens", "float16", prefix, lens, 3), "float16")


def test_more_row_tiles_than_sms():
    p = problem(1, 4, 1, 64, 32, "tokens", "bfloat16", 130, [41 + b % 3 for b in range(246)], 40)
    check_attention(p, "bfloat16")


@pytest.mark.parametrize("heads", [(4, 4), (4, 1), (32, 2)])
@pytest.mark.parametrize("new", [2, 5])
@pytest.mark.parametrize("B", [2, 60])
def test_a_value_behind_the_mask_does_not_reach_those_who_do_not_see_it(heads, new, B):
    """The newest token's values hold an infinity and a NaN: only the newest query is touched, and only in their columns."""
    p = problem(9, *heads, 64, 16, "tokens", "bfloat16", 500, [20 + 13 * (b % 5) for b in range(B)], new, rubbish=0.0)
    clean = serving.prefix_attention(**p)
    n = int(p["lens"][1]) - 1
    page = int(p["page_table"][1, n // 16])
    p["cache"].v[page, n % 16, 0, 3] = float("inf")
    p["cache"].v[page, n % 16, 0, 7] = float("nan")
    out, lse = serving.prefix_attention(**p)
    assert torch.equal(lse, clean[1])
    g = heads[0] // heads[1]
    touched = torch.zeros_like(out, dtype=torch.bool)
    touched[1, new - 1, :g, 3] = touched[1, new - 1, :g, 7] = True
    assert not torch.isfinite(out[touched]).any() and torch.isfinite(out[~touched]).all()
    # the others as before, up to the order in which a key is added
    off = (out.float() - clean[0].float()).abs()[~touched].max()
    assert float(off) <= 2.0 ** -7 * float(clean[0].abs().max())
    # and the same for keys: a NaN score belongs to those who see it
    p["cache"].v[page, n % 16, 0, 3] = p["cache"].v[page, n % 16, 0, 7] = 0.0
    p["cache"].k[page, n % 16, 0, 0] = float("nan")
    out, lse = serving.prefix_attention(**p)
    bad = torch.zeros_like(lse, dtype=torch.bool)
    bad[1, new - 1, :g] = True
    assert torch.equal(torch.isnan(lse), bad) and torch.equal(torch.isnan(out).any(-1), bad)


@pytest.mark.parametrize("page", [8, 24, 40, 64, 256])
@pytest.mark.parametrize("B", [3, 50])
def test_a_fused_cache(page, B):
    """Keys and values in one buffer of pages, as [page][2][token][head][dim], a prefix that ends inside a box."""
    p = problem(page, 8, 4, 128, page, "tokens", "float16", 411, [9 + 21 * (b % 7) for b in range(B)], 1)
    c = p["cache"]
    both = torch.stack([c.k, c.v], 1)
    p["cache"] = serving.PagedCache(both[:, 0], both[:, 1])
    check_attention(p, "float16")


def test_graph_of_a_whole_step_with_a_prefix():
    """Kernels that start beside each other, captured and replayed with other lengths."""
    p = problem(8, 16, 4, 128, 16, "tokens", "bfloat16", 1700, [100 + 3 * b for b in range(40)], 1)
    ws = serving.attention_workspace(p["cache"], p["q"], 1700, p["page_table"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serving.prefix_attention(**p, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = serving.prefix_attention(**p, workspace=ws)
    for step in (0, 99, 1):
        p["lens"].sub_(step)
        for _ in range(3):
            g.replay()
        torch.cuda.synchronize()
        w_out, w_lse, b_out, b_lse = R.attention(f64(p["q"]), f64(p["cache"].k), f64(p["cache"].v), p["prefix_pages"].cpu().numpy(),
                                                 1700, p["page_table"].cpu().numpy(), p["lens"].cpu().numpy(), 128 ** -0.5, "bfloat16")
        check(out, w_out, b_out, "out")
        assert np.all(np.abs(f64(lse) - w_lse) <= b_lse)


def test_calls_in_a_row_share_a_workspace():
    """Calls of different inputs behind each other on one stream, and nothing waited for between them."""
    ps = [problem(s, 16, 4, 128, 16, "tokens", "bfloat16", 900, [50 + 7 * (b % 9) + s for b in range(40)], 1) for s in range(3)]
    ws = serving.attention_workspace(ps[0]["cache"], ps[0]["q"], 900, widen_table(ps[0], 9)["page_table"])
    want = [serving.prefix_attention(**p) for p in ps]
    torch.cuda.synchronize()
    got = [serving.prefix_attention(**ps[i % 3], workspace=ws) for i in range(9)]
    for i, (o, l) in enumerate(got):
        assert torch.equal(o, want[i % 3][0]) and torch.equal(l, want[i % 3][1])


def test_what_is_on_another_device_is_refused():
    q, pos = torch.zeros(3, 2, 64, device="cuda", dtype=torch.float16), torch.zeros(3, dtype=torch.int32, device="cuda")
    elsewhere = serving.Rotary(64, device="cpu")
    cache = serving.PagedCache.empty(2, 16, 2, 64, torch.float16)
    for call in (lambda: serving.rope(q, None, pos, elsewhere), lambda: serving.rope_grad(q, None, pos, elsewhere),
                 lambda: serving.append_kv(q, q, q, pos, torch.arange(3, device="cuda"), elsewhere, cache)):
        with pytest.raises(gts.GtsError) as e:
            call()
        assert e.value.status == gts.GTS_ERR_INVALID_ARG


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("prefix", [256, 257, 272, 300, 383, 1000])
@pytest.mark.parametrize("kw", [dict(), dict(spread=60.0), dict(rubbish=float("inf"))])
def test_prefix_ends_anywhere_in_a_tile(D, prefix, kw):
    """Many rows, so that the tensor cores' kernel takes the prefix; its last tile of any length, scores that keep raising the
    maximum, rubbish in the rest of the pages."""
    for scale in (None, -0.1):
        check_attention(problem(prefix, 16, 4, D, 16, "tokens", "float16", prefix, [3 + b % 40 for b in range(70)], 1, **kw), "float16",
                        scale=scale)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_few_key_heads_and_a_long_prefix(D):
    """One pair of rows cut over all blocks, and pairs that begin and end inside a block."""
    check_attention(problem(1, 33, 1, D, 32, "heads", "bfloat16", 9000, [5, 0, 17], 1), "bfloat16")
    check_attention(problem(2, 40, 40, D, 32, "tokens", "bfloat16", 400, [5, 0, 17] * 14, 1), "bfloat16")


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 5, 16])
@pytest.mark.parametrize("prefix", [0, 100])
def test_many_short_pairs_to_a_block(D, new, prefix):
    """Some 20 tiles to a block, most pairs of one to three: one pair's rows are written while the next one's keys arrive, and
    stretches end between pairs as well as inside of them; a few long sequences among them."""
    rng = np.random.default_rng(D + new)
    lens = [new + int(x) for x in rng.integers(0, 150, 700)]
    lens[::50] = [1500 + int(x) for x in rng.integers(0, 300, 14)]
    lens[3] = lens[77] = 0
    p = problem(D, 16, 4, D, 64, "heads", "bfloat16", prefix, lens, new)
    check_attention(widen_table(p, 40), "bfloat16")
    if new == 1:
        check_attention(p, "bfloat16")
