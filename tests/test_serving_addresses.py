"""Rotary and PagedCache hold addresses of their tensors: these cannot go stale."""
import copy

import pytest

torch = pytest.importorskip("torch")

from paper_2607_11262_gb300 import gts, serving  # noqa: E402


def refused(x, name, value):
    with pytest.raises(gts.GtsError, match=name) as e:
        setattr(x, name, value)
    assert e.value.status == gts.GTS_ERR_INVALID_ARG
    with pytest.raises(gts.GtsError):
        delattr(x, name)


def test_a_rotarys_attributes_are_fixed():
    r = serving.Rotary(64, device="cpu")
    for name in ("units", "factor", "theta", "layout", "head_dim", "rot_dim", "device"):
        before = getattr(r, name)
        refused(r, name, before)
        assert getattr(r, name) is before


def test_a_copied_rotary_has_its_own_frequencies():
    r = serving.Rotary(64, device="cpu")
    c = copy.deepcopy(r)
    assert c.units.data_ptr() != r.units.data_ptr()
    for t in (0, 1):
        assert c._descriptor(t)[0] == c.units.data_ptr() and r._descriptor(t)[0] == r.units.data_ptr()
        assert c._descriptor(t)[1:] == r._descriptor(t)[1:]
    c.units.data = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(gts.GtsError):
        c._descriptor(0)


def _filled(page=16):
    cache = serving.PagedCache.empty(2, page, 1, 64, torch.float16)
    cache.k.fill_(3.0)
    cache.v.fill_(3.0)
    return cache


def _append(cache):
    x = torch.ones(1, 1, 64, dtype=torch.float16, device="cuda")
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    serving.append_kv(x, x, x, at, at.long() + 17, serving.Rotary(64), cache)


def _written(t):
    return bool((t[1, 1] == 1.0).all()) and int((t == 3.0).sum()) == t.numel() - 64


@pytest.mark.gpu
def test_a_caches_tensors_are_fixed():
    cache = _filled()
    for name in ("k", "v", "dtype", "device", "n_pages", "page_size", "kv_heads", "head_dim"):
        before = getattr(cache, name)
        refused(cache, name, before)
        assert getattr(cache, name) is before


@pytest.mark.gpu
def test_a_copied_cache_is_written_itself():
    cache = _filled()
    other = copy.deepcopy(cache)
    _append(other)
    assert _written(other.k) and _written(other.v) and bool((cache.k == 3.0).all()) and bool((cache.v == 3.0).all())


@pytest.mark.gpu
def test_a_tensor_given_other_memory_is_written_there():
    cache = _filled()
    old, larger = [cache.k.detach(), cache.v.detach()], [torch.full((5, 16, 1, 64), 3.0, dtype=torch.float16, device="cuda") for _ in range(2)]
    cache.k.data, cache.v.data = larger
    _append(cache)
    assert cache._descriptor()[8:12] == (5, 16, 1, 64) and cache.n_pages == 5
    for o, n in zip(old, larger):
        assert bool((o == 3.0).all()) and _written(n)
    cache.v.data = torch.zeros(4, 16, 1, 64, dtype=torch.float16, device="cuda")
    with pytest.raises(gts.GtsError):
        _append(cache)
