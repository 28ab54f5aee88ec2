"""The operators of a decode step without a GPU: descriptors, frequencies, refusals of the C entries."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import build as B  # noqa: E402
from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests import serving_reference as R  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCALINGS = [None, {"kind": "linear", "factor": 4.0}, {"kind": "ntk", "factor": 8.0},
            {"kind": "by_parts", "factor": 8.0, "original_len": 8192, "low": 1.0, "high": 32.0}]


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB):
        B.build()


def test_descriptors_have_the_headers_layout():
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    structs = {"gts_heads": serving.HeadsDesc, "gts_cache": serving.CacheDesc, "gts_rotary": serving.RotaryDesc,
               "gts_rope_desc": serving.RopeDesc, "gts_append_desc": serving.AppendDesc,
               "gts_attention_desc": serving.AttentionDesc}
    body = "".join(f'printf("%zu\\n", sizeof({n}));' + "".join(
        f'printf("%zu\\n", offsetof({n}, {f[0]}));' for f in s._fields_) for n, s in structs.items())
    out_dir = os.path.join(B.BUILD_DIR, "c_client")
    os.makedirs(out_dir, exist_ok=True)
    src, exe = os.path.join(out_dir, f"layout_{os.getpid()}.c"), os.path.join(out_dir, f"layout_{os.getpid()}")
    with open(src, "w") as f:
        f.write('#include <stdio.h>\n#include "gts_serving.h"\nint main(void) {' + body + "return 0; }\n")
    try:
        subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I",
                               os.path.join(ROOT, "include"), "-o", exe, src])
        got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    finally:
        for p in (src, exe):
            if os.path.exists(p):
                os.remove(p)
    want = [x for s in structs.values() for x in [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]]
    assert got == want


def test_packed_descriptors_are_the_structures():
    """Each field's value comes back from its place in the structure."""
    for packed, struct in ((serving._ROPE, serving.RopeDesc), (serving._APPEND, serving.AppendDesc),
                           (serving._ATTENTION, serving.AttentionDesc)):
        flat = []

        def leaves(s, at):
            for name, kind in s._fields_:
                if issubclass(kind, ctypes.Structure):
                    leaves(kind, at + getattr(s, name).offset)
                else:
                    flat.append((at + getattr(s, name).offset, kind))
        leaves(struct, 0)
        assert packed.size == ctypes.sizeof(struct)
        raw = packed.pack(*range(1, len(flat) + 1))
        assert [int(kind.from_buffer_copy(raw, at).value) for at, kind in flat] == list(range(1, len(flat) + 1))


@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("rot", [2, 16, 96, 128])
def test_frequencies(rot, scaling):
    r = serving.Rotary(128, rot_dim=rot, base=5000.0, scaling=scaling, device="cpu")
    theta, factor = R.frequencies(rot, 5000.0, scaling)
    assert np.allclose(r.theta, theta, rtol=1e-13, atol=0) and r.factor == factor
    # the phase of a far position, in wrapping integers, against the angle in long doubles
    units = r.units.numpy().view(np.uint64)
    pos = 1_000_003
    with np.errstate(over="ignore"):
        phase = (np.uint64(pos) * units).astype(np.float64) / 2.0 ** 64
    angle = np.longdouble(pos) * theta.astype(np.longdouble) / (2 * np.longdouble(np.pi))
    off = np.abs(phase - (angle - np.floor(angle)).astype(np.float64))
    assert np.all(np.minimum(off, 1 - off) < 1e-9)


def test_rotary_refusals():
    for kw in (dict(rot_dim=3), dict(rot_dim=130), dict(layout="other"), dict(base=0.0),
               dict(scaling={"kind": "linear"}), dict(scaling={"kind": "other", "factor": 2.0}),
               dict(scaling={"kind": "by_parts", "factor": 2.0}),
               dict(scaling={"kind": "linear", "factor": 2.0, "extra": 1})):
        with pytest.raises(gts.GtsError) as e:
            serving.Rotary(128, device="cpu", **kw)
        assert e.value.status == gts.GTS_ERR_INVALID_ARG


def test_cpu_tensors_are_refused():
    r = serving.Rotary(64, device="cpu")
    q = torch.zeros(1, 2, 64)
    with pytest.raises(gts.GtsError, match="CUDA"):
        serving.rope(q, None, torch.zeros(1, dtype=torch.int32), r)
    with pytest.raises(gts.GtsError, match="CUDA"):
        serving.PagedCache(torch.zeros(1, 1, 1, 64), torch.zeros(1, 1, 1, 64))


PTR = 4096  # an address that a refused call never looks at


def _rope(**kw):
    rot = serving.RotaryDesc(PTR, kw.pop("rot_dim", 128), kw.pop("layout", 0), 1.0, kw.pop("transposed", 0))
    h = serving.HeadsDesc(kw.pop("data", PTR), 1024, 128)
    d = serving.RopeDesc(4, 8, 8, 128, serving.GTS_BF16, PTR, rot, h, h, h, h)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("kw", [dict(dtype=7), dict(dtype=-1), dict(head_dim=0), dict(head_dim=5000), dict(rot_dim=130),
                                dict(rot_dim=3), dict(layout=2), dict(transposed=2), dict(positions=None),
                                dict(positions=PTR + 2), dict(data=None), dict(data=PTR + 1), dict(n_tokens=2 ** 31),
                                dict(q_heads=2 ** 17)])
def test_rope_refusals(kw):
    with pytest.raises(gts.GtsError) as e:
        serving.gts_rope(_rope(**kw))
    assert e.value.status == gts.GTS_ERR_INVALID_ARG


def _cache(**kw):
    d = serving.CacheDesc(PTR, PTR, 1 << 16, 1024, 128, 1 << 16, 1024, 128, 10, 64, 8, 128, serving.GTS_BF16)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("kw", [dict(slots=None), dict(slots=PTR + 4), dict(positions=None), dict(d_status=PTR + 1),
                                dict(cache=dict(page_size=0)), dict(cache=dict(k=None)), dict(cache=dict(v=PTR + 1)),
                                dict(cache=dict(dtype=9)), dict(transposed=1)])
def test_append_refusals(kw):
    h = serving.HeadsDesc(PTR, 1024, 128)
    d = serving.AppendDesc(4, 8, PTR, PTR, serving.RotaryDesc(PTR, 128, 0, 1.0, kw.pop("transposed", 0)), h, h, h, h,
                           _cache(**kw.pop("cache", {})), None)
    for k, v in kw.items():
        setattr(d, k, v)
    with pytest.raises(gts.GtsError) as e:
        serving.gts_append_kv(d)
    assert e.value.status == gts.GTS_ERR_INVALID_ARG


def _attention(**kw):
    d = serving.AttentionDesc(2, 1, 32, 0.1, PTR, 4096, 4096, 128, PTR, 4096, 4096, 128, PTR, _cache(**kw.pop("cache", {})),
                              PTR, 100, PTR, 4, PTR, PTR, 1 << 40, None)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(lens=None), dict(prefix_pages=None),
                                dict(page_table=None), dict(workspace=None), dict(workspace=PTR + 8), dict(q_heads=12),
                                dict(q_heads=0), dict(n_seqs=70000), dict(prefix_len=2 ** 31), dict(max_pages=2 ** 26),
                                dict(cache=dict(k=None)), dict(cache=dict(dtype=2)), dict(cache=dict(head_dim=80)),
                                dict(cache=dict(page_size=0)), dict(cache=dict(page_size=70000))])
def test_attention_refusals(kw):
    with pytest.raises(gts.GtsError) as e:
        serving.gts_prefix_attention(_attention(**kw))
    assert e.value.status == gts.GTS_ERR_INVALID_ARG


def test_attention_workspace():
    d = _attention()
    need = serving.gts_attention_workspace_bytes(d)
    assert need >= 16
    d.workspace_bytes = need - 1
    with pytest.raises(gts.GtsError) as e:
        serving.gts_prefix_attention(d)
    assert e.value.status == gts.GTS_ERR_NOMEM
    assert serving.gts_attention_workspace_bytes(_attention(q_heads=12)) == 0


def test_null_descriptors():
    lib = serving._load()
    for f in (lib.gts_rope, lib.gts_append_kv, lib.gts_prefix_attention):
        assert f(None, None) == gts.GTS_ERR_INVALID_ARG and "null" in gts.gts_last_error()
    assert lib.gts_attention_workspace_bytes(None) == 0


def test_divisor_method():
    """attention.cu's division by a multiplication: m = floor(2^(31 + l) / d) + 1, x m >> (31 + l), for every 31-bit x."""
    rng = np.random.default_rng(3)
    ds = sorted({*range(1, 300), 65535, 65536, 1000, *(int(d) for d in rng.integers(1, 65537, 300))})
    for d in ds:
        bits = (d - 1).bit_length()
        if bits == 0:
            continue
        m = (1 << (31 + bits)) // d + 1
        assert m < 1 << 32
        q = np.array([0, 1, d - 1, d, d + 1, 2 ** 31 - 1, *(k * d + e for k in (1, 7, (2 ** 31 - 1) // d) for e in (-1, 0) if k * d + e < 2 ** 31),
                      *rng.integers(0, 2 ** 31, 50)], np.int64)
        got = np.array([(int(x) * m) >> 32 >> (bits - 1) for x in q])
        assert np.array_equal(got, q // d), d


@pytest.mark.parametrize("kw", [dict(q=PTR + 1), dict(out=PTR + 1), dict(lse=PTR + 2), dict(lens=PTR + 1), dict(page_table=PTR + 2),
                                dict(prefix_pages=PTR + 2), dict(d_status=PTR + 2), dict(cache=dict(k=PTR + 1)),
                                dict(n_seqs=60000, q_heads=32768, cache=dict(kv_heads=8))])
def test_attention_refuses_misaligned_tensors_and_too_many_rows(kw):
    with pytest.raises(gts.GtsError) as e:
        serving.gts_prefix_attention(_attention(**kw))
    assert e.value.status == gts.GTS_ERR_INVALID_ARG
