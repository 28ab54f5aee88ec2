"""The operators of prompts without a GPU: descriptors and refusals of the C entries."""
import ctypes
import os
import shutil
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import build as B  # noqa: E402
from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests.test_serving import PTR, ROOT, _cache  # noqa: E402

STRUCTS = {"gts_prompt_desc": (serving.PromptDesc, serving._PROMPT), "gts_prompt_grad_desc": (serving.PromptGradDesc, serving._PROMPT_GRAD),
           "gts_chunk_desc": (serving.ChunkDesc, serving._CHUNK), "gts_copy_pages_desc": (serving.CopyPagesDesc, serving._COPY_PAGES)}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB):
        B.build()


def test_descriptors_have_the_headers_layout(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    body = "".join(f'printf("%zu\\n", sizeof({n}));' + "".join(
        f'printf("%zu\\n", offsetof({n}, {f[0]}));' for f in s._fields_) for n, (s, _) in STRUCTS.items())
    src, exe = str(tmp_path / "layout.c"), str(tmp_path / "layout")
    with open(src, "w") as f:
        f.write('#include <stdio.h>\n#include "gts_serving.h"\nint main(void) {' + body + "return 0; }\n")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), "-o",
                           exe, src])
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [x for s, _ in STRUCTS.values() for x in [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]]


@pytest.mark.parametrize("name", list(STRUCTS))
def test_packed_descriptors_are_the_structures(name):
    struct, packed = STRUCTS[name]
    flat = []

    def leaves(s, at):
        for field, kind in s._fields_:
            if issubclass(kind, ctypes.Structure):
                leaves(kind, at + getattr(s, field).offset)
            else:
                flat.append((at + getattr(s, field).offset, kind))
    leaves(struct, 0)
    assert packed.size == ctypes.sizeof(struct)
    raw = packed.pack(*range(1, len(flat) + 1))
    assert [int(kind.from_buffer_copy(raw, at).value) for at, kind in flat] == list(range(1, len(flat) + 1))


def _set(d, kw):
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _heads(at=PTR):
    return serving.HeadsDesc(at, 1024, 128)


def _prompt(**kw):
    kw = {k: _heads(v) if k in ("q", "k", "v", "out", "low") else v for k, v in kw.items()}
    return _set(serving.PromptDesc(3, 100, 8, 2, 128, serving.GTS_BF16, 1, 0, 0.1, PTR, _heads(), _heads(), _heads(), _heads(), _heads(), PTR, PTR,
                                   1 << 40, None), kw)


PROMPT = [dict(dtype=serving.GTS_F32), dict(dtype=-1), dict(head_dim=80), dict(head_dim=256), dict(head_dim=0), dict(q_heads=7),
          dict(q_heads=0), dict(kv_heads=0), dict(q_heads=260, kv_heads=2), dict(kv_heads=2048, q_heads=2048), dict(causal=2),
          dict(zero_rest=8), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(starts=None),
          dict(starts=PTR + 2), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=PTR + 1), dict(k=PTR + 1),
          dict(v=PTR + 1), dict(out=PTR + 1), dict(low=PTR + 1), dict(lse=PTR + 2), dict(workspace=None), dict(workspace=PTR + 8), dict(d_status=PTR + 1),
          dict(n_seqs=1 << 16), dict(n_tokens=(1 << 28) + 1), dict(n_tokens=1 << 28, q_heads=16)]


@pytest.mark.parametrize("kw", PROMPT)
def test_prompt_refusals(kw):
    for call, d in ((serving.gts_prompt_attention, _prompt(**kw)),
                    (serving.gts_prompt_attention_grad, serving.PromptGradDesc(_prompt(**kw), _heads(), None, _heads(), _heads(), _heads()))):
        with pytest.raises(gts.GtsError) as e:
            call(d)
        assert e.value.status == gts.GTS_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dout=PTR + 1), dict(dq=PTR + 1),
                                dict(dk=PTR + 1), dict(dv=PTR + 1), dict(dlse=PTR + 2), dict(lse=None)])
def test_prompt_grad_refusals(kw):
    d = serving.PromptGradDesc(_prompt(**{k: v for k, v in kw.items() if k == "lse"}), _heads(), None, _heads(), _heads(), _heads())
    _set(d, {k: v if k == "dlse" else _heads(v) for k, v in kw.items() if k != "lse"})
    with pytest.raises(gts.GtsError) as e:
        serving.gts_prompt_attention_grad(d)
    assert e.value.status == gts.GTS_ERR_INVALID_ARG


def _chunk(**kw):
    kw = {k: _heads(v) if k in ("q", "out") else _cache(**v) if k == "cache" else v for k, v in kw.items()}
    return _set(serving.ChunkDesc(3, 100, 32, 0, 0.1, PTR, _heads(), _heads(), PTR, _cache(), PTR, 4, PTR, PTR, 1 << 40, None), kw)


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(lens=None), dict(page_table=None), dict(starts=None),
                                dict(workspace=None), dict(workspace=PTR + 8), dict(q_heads=12), dict(q_heads=0), dict(n_seqs=70000),
                                dict(max_pages=2 ** 26), dict(scale=0.0), dict(scale=float("nan")), dict(zero_rest=4), dict(q=PTR + 1),
                                dict(out=PTR + 1), dict(lse=PTR + 1), dict(lens=PTR + 1), dict(starts=PTR + 1), dict(page_table=PTR + 2),
                                dict(d_status=PTR + 1), dict(cache=dict(k=None)), dict(cache=dict(dtype=2)), dict(cache=dict(head_dim=80)),
                                dict(cache=dict(page_size=0)), dict(cache=dict(page_size=70000)), dict(cache=dict(v=PTR + 1))])
def test_chunk_refusals(kw):
    with pytest.raises(gts.GtsError) as e:
        serving.gts_chunk_attention(_chunk(**kw))
    assert e.value.status == gts.GTS_ERR_INVALID_ARG


def _copy(**kw):
    kw = {k: _cache(**v) if k in ("cache", "into") else v for k, v in kw.items()}
    return _set(serving.CopyPagesDesc(5, PTR, PTR, PTR, _cache(), _cache(), None), kw)


@pytest.mark.parametrize("kw", [dict(src=None), dict(dst=None), dict(src=PTR + 1), dict(dst=PTR + 2), dict(tokens=PTR + 1), dict(d_status=PTR + 1),
                                dict(n_copies=2 ** 31), dict(cache=dict(dtype=9), into=dict(dtype=9)), dict(cache=dict(dtype=1)),
                                dict(cache=dict(page_size=32)), dict(into=dict(kv_heads=4)), dict(into=dict(head_dim=64)),
                                dict(cache=dict(page_size=0), into=dict(page_size=0)), dict(cache=dict(k=None)), dict(into=dict(v=None)),
                                dict(into=dict(v=PTR + 1)), dict(cache=dict(page_size=65536, kv_heads=4096), into=dict(page_size=65536, kv_heads=4096))])
def test_copy_refusals(kw):
    with pytest.raises(gts.GtsError) as e:
        serving.gts_copy_pages(_copy(**kw))
    assert e.value.status == gts.GTS_ERR_INVALID_ARG


def test_workspaces():
    for make, size, call, at in ((_prompt, serving.gts_prompt_workspace_bytes, serving.gts_prompt_attention, lambda d: d),
                                 (_chunk, serving.gts_chunk_workspace_bytes, serving.gts_chunk_attention, lambda d: d),
                                 (lambda **kw: serving.PromptGradDesc(_prompt(**kw), _heads(), None, _heads(), _heads(), _heads()),
                                  serving.gts_prompt_grad_workspace_bytes, serving.gts_prompt_attention_grad, lambda d: d.forward)):
        d = make()
        need = size(d)
        assert need >= 16
        at(d).workspace_bytes = need - 1
        with pytest.raises(gts.GtsError) as e:
            call(d)
        assert e.value.status == gts.GTS_ERR_NOMEM
        assert size(make(q_heads=7)) == 0


def test_null_descriptors():
    lib = serving._load()
    for f in (lib.gts_prompt_attention, lib.gts_prompt_attention_grad, lib.gts_chunk_attention, lib.gts_copy_pages):
        assert f(None, None) == gts.GTS_ERR_INVALID_ARG and "null" in gts.gts_last_error()
    for f in (lib.gts_prompt_workspace_bytes, lib.gts_prompt_grad_workspace_bytes, lib.gts_chunk_workspace_bytes):
        assert f(None) == 0


def test_cpu_tensors_are_refused():
    q, starts = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.tensor([0, 3], dtype=torch.int32)
    with pytest.raises(gts.GtsError, match="CUDA"):
        serving.prompt_attention(q, q, q, starts)
    with pytest.raises(gts.GtsError, match="CUDA"):
        serving.prompt_attention_grad(q, q, q, q, q, torch.zeros(3, 2), starts)
