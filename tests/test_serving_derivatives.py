"""Derivatives of the rotation beyond the first backward pass: second order, tangents, and gradients of single inputs."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from torch.autograd import forward_ad  # noqa: E402

from paper_2607_11262_gb300 import gts, serving  # noqa: E402
from tests import serving_reference as R  # noqa: E402

T, H, KV, D, ROT = 3, 2, 1, 10, 8


def _plain(calls):
    """The kernel's call worked out on the host, off the autograd graph like it."""
    def call(q, k, positions, rotary, transposed, out_q, out_k, stream):
        calls.append((transposed, q.shape[1], None if k is None else k.shape[1]))

        def one(x):
            if x is None:
                return None
            assert x.stride(-1) == 1
            y, _ = R.rotate(x.detach().double().numpy(), positions.numpy(), rotary.theta, rotary.factor, rotary.layout, bool(transposed))
            return torch.from_numpy(np.ascontiguousarray(y)).to(x.dtype)
        return one(q), one(k)
    return call


@pytest.fixture
def calls(monkeypatch):
    got = []
    monkeypatch.setattr(serving, "_rope_call", _plain(got))
    return got


def inputs(dtype=torch.float64, device="cpu"):
    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn(T, n, D, generator=g, dtype=torch.float64).to(dtype).to(device).requires_grad_() for n in (H, KV))
    return q, k, torch.tensor([0, 5, 70001], dtype=torch.int32, device=device), serving.Rotary(
        D, rot_dim=ROT, scaling={"kind": "by_parts", "factor": 4.0, "original_len": 4096}, device=device)


@pytest.mark.parametrize("call", [serving.rope, serving.rope_grad])
def test_derivatives_against_differences(calls, call):
    """float64, central differences: gradcheck's own tolerances."""
    q, k, pos, rotary = inputs()
    f = lambda x, y: call(x, y, pos, rotary)  # noqa: E731
    only = lambda x: call(x, None, pos, rotary)[0]  # noqa: E731
    assert torch.autograd.gradcheck(f, (q, k), check_forward_ad=True)
    assert torch.autograd.gradcheck(only, (q,), check_forward_ad=True)
    square = lambda x, y: tuple(z.square() for z in call(x, y, pos, rotary))  # noqa: E731
    assert torch.autograd.gradgradcheck(square, (q, k))


@pytest.mark.parametrize("call", [serving.rope, serving.rope_grad])
def test_a_penalty_of_the_gradient_counts(calls, call):
    """loss = sum |A x|^4 / 4, penalty = sum |its gradient|^2: the penalty's own gradient is not nothing."""
    q, k, pos, rotary = inputs()
    a, _ = call(q, k, pos, rotary)
    grad, = torch.autograd.grad(a.pow(4).sum() / 4, q, create_graph=True)
    assert grad.requires_grad
    got, = torch.autograd.grad(grad.square().sum(), q)
    # A^T is the other call: grad = A^T (A q)^3, its square's gradient 2 A^T (3 (A q)^2 A grad)
    back = serving.rope_grad if call is serving.rope else serving.rope
    with torch.no_grad():
        want = back(6 * a * a * call(grad.detach(), None, pos, rotary)[0], None, pos, rotary)[0]
    assert torch.allclose(got, want, rtol=1e-12, atol=1e-12) and float(got.abs().max()) > 0.1


def test_tangents(calls):
    q, k, pos, rotary = inputs()
    tq, tk = torch.ones_like(q), torch.randn_like(k)
    with torch.no_grad():
        want = serving.rope(tq, tk, pos, rotary)
    with forward_ad.dual_level():
        a, b = serving.rope(forward_ad.make_dual(q.detach(), tq), forward_ad.make_dual(k.detach(), tk), pos, rotary)
        assert torch.equal(forward_ad.unpack_dual(a).tangent, want[0]) and torch.equal(forward_ad.unpack_dual(b).tangent, want[1])
        a, b = serving.rope(q.detach(), forward_ad.make_dual(k.detach(), tk), pos, rotary)
        assert torch.equal(forward_ad.unpack_dual(b).tangent, want[1])
        plain = serving.rope(q.detach(), k.detach(), pos, rotary)
        assert forward_ad.unpack_dual(plain[0]).tangent is None
        with pytest.raises(gts.GtsError):
            serving.rope(forward_ad.make_dual(q.detach(), tq), None, pos, rotary, out_q=torch.empty_like(q))


def test_only_the_gradients_asked_for(calls):
    q, k, pos, rotary = inputs()
    for x, want in ((q, (1, H, None)), (k, (1, KV, None))):
        a, b = serving.rope(q.detach().requires_grad_(x is q), k.detach().requires_grad_(x is k), pos, rotary)
        calls.clear()
        (a.sum() + b.sum()).backward()                     # gradients of stride 0
        assert calls == [want]
    a, none = serving.rope(q, None, pos, rotary)
    assert none is None
    a.sum().backward()
    with torch.no_grad():
        assert torch.equal(q.grad, serving.rope_grad(torch.ones_like(q), None, pos, rotary)[0])


def test_outputs_of_the_callers_take_no_gradients(calls):
    q, k, pos, rotary = inputs()
    for call, kw in ((serving.rope, "out_q"), (serving.rope_grad, "out_dq"), (serving.rope_grad, "out_dk")):
        with pytest.raises(gts.GtsError) as e:
            call(q, k, pos, rotary, **{kw: torch.empty_like(k if kw == "out_dk" else q)})
        assert e.value.status == gts.GTS_ERR_INVALID_ARG
        with torch.no_grad():
            call(q, k, pos, rotary, **{kw: torch.empty_like(k if kw == "out_dk" else q)})


@pytest.mark.gpu
def test_derivatives_on_the_gpu():
    """The kernel's second order and tangents are the calls of the formulas above, bit for bit; a gradient of stride 0 is its
    copy's."""
    gts.load()
    q, k, pos, rotary = inputs(torch.float32, "cuda")
    a, b = serving.rope(q, k, pos, rotary)
    gq, gk = torch.autograd.grad(a.square().sum() + b.square().sum(), (q, k), create_graph=True)
    got = torch.autograd.grad(gq.sum() + gk.sum(), (q, k))
    one = [torch.ones_like(x) for x in (q, k)]
    with torch.no_grad():
        there = serving.rope(*one, pos, rotary)
        want = serving.rope_grad(2 * there[0], 2 * there[1], pos, rotary)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    with forward_ad.dual_level():
        t = serving.rope(forward_ad.make_dual(q.detach(), one[0]), None, pos, rotary)[0]
        assert torch.equal(forward_ad.unpack_dual(t).tangent, there[0])
    for x in (q, k):
        got, = torch.autograd.grad(serving.rope(q, k, pos, rotary)[0 if x is q else 1].sum(), x)
        with torch.no_grad():
            assert torch.equal(got, serving.rope_grad(torch.ones_like(x), None, pos, rotary)[0])
