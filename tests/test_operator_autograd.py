"""The operators' autograd forms: their backward passes are kernels that autograd does not record, so a second derivative has to raise
and not leave the operator out.  On stand-ins for the kernels and on the kernels, in a graph whose other parts are recorded."""
import pytest
import torch
import torch.nn.functional as F

from paper_2502_11058_amd import operators as O


def _gradients(forward, grad, inputs):
    """What a backward call of the plain form gives: new tensors that autograd knows nothing of."""
    x = [t.detach().requires_grad_(True) for t in inputs]
    with torch.enable_grad():
        return torch.autograd.grad(forward(*x), x, grad)


def _norm(x, w):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5) * w


def _turn(x):
    return torch.cat([-x[..., 2:], x[..., :2]], -1)


def _attend(q, k, v):
    p = torch.softmax(torch.einsum("bihd,bjhd->bhij", q, k), -1)
    return torch.einsum("bhij,bjhd->bihd", p, v)


def _entropy(x, w):
    return torch.logsumexp(x @ w.t(), -1)


@pytest.fixture
def stand_ins(monkeypatch):
    put = {"norm_forward": lambda x, w, b, kind, eps: (_norm(x, w), None, x[..., 0]),
           "norm_backward": lambda dy, x, w, mean, rstd, kind, bias: (*_gradients(_norm, dy, (x, w)), None),
           "rotary_forward": lambda q, k, table, positions, layout: (_turn(q), _turn(k)),
           "rotary_backward": lambda dq, dk, table, positions, layout: (-_turn(dq), -_turn(dk)),
           "attention_forward": lambda q, k, v, **kw: (_attend(q, k, v), q[..., 0]),
           "attention_backward": lambda do, q, k, v, o, lse, **kw: _gradients(_attend, do, (q, k, v)),
           "linear_cross_entropy_forward": lambda x, w, t: (_entropy(x, w), x[..., 0]),
           "linear_cross_entropy_backward": lambda g, x, w, t, lse, **kw: _gradients(_entropy, g, (x, w))}
    for name, f in put.items():
        monkeypatch.setattr(O, name, f)


def _calls(w, table=None):
    """name -> a scalar of the operator between a linear map and a square, whose gradients autograd records."""
    t = torch.zeros(3, 4, dtype=torch.int64, device=w.device)
    return {"norm": lambda h: O.norm(h, w[0], kind="rms").square().sum(),
            "rotary": lambda h: sum(x.square().sum() for x in O.rotary(h[:, :, None], h[:, :, None], table)),
            "attention": lambda h: O.attention(h[:, :, None], h[:, :, None], h[:, :, None]).square().sum(),
            "linear_cross_entropy": lambda h: O.linear_cross_entropy(h, w, t, reduction="none").square().sum()}


def _check(name, device, table=None):
    g = torch.Generator().manual_seed(1)
    x, m, w = (torch.randn(s, generator=g).to(device).requires_grad_(True) for s in ((3, 4, 4), (4, 4), (4, 4)))
    f = _calls(w, table)[name]
    plain, = torch.autograd.grad(f(F.linear(x, m)), x)
    first, = torch.autograd.grad(f(F.linear(x, m)), x, create_graph=True)
    assert torch.equal(first, plain)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.square().sum().backward()


NAMES = ["norm", "rotary", "attention", "linear_cross_entropy"]


@pytest.mark.parametrize("name", NAMES)
def test_a_second_derivative_raises(stand_ins, name):
    _check(name, "cpu")


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_a_second_derivative_through_the_kernels_raises(name):
    _check(name, "cuda", O.rotary_table(4, 4))
