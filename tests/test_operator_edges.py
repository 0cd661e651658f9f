"""Shapes at the edge of the torch calls' checks, on the host: what reaches the library, or is refused."""
import pytest
import torch

from paper_2502_11058_amd import binding as B
from paper_2502_11058_amd import operators as O


@pytest.mark.parametrize("shape,cols", [((5, 1), 1), ((2, 3, 1), 1), ((4, 7), 7)])
def test_one_row_for_all(shape, cols):
    """A row expanded over many has a stride of zero, also where it has one column."""
    x = torch.arange(1.0, cols + 1).expand(shape)
    r, rows, stride = O._rows("x", x)
    assert rows == x.numel() // cols and stride >= cols and r.reshape(x.shape).equal(x)


@pytest.mark.gpu
def test_one_column_expanded():
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x, w, dy = torch.randn(1, 1, generator=g, device="cuda").expand(5, 1), torch.randn(1, generator=g, device="cuda"), torch.randn(5, 1, generator=g, device="cuda")
    y, mean, rstd = O.norm_forward(x, w, kind="rms")
    want = O.norm_forward(x.contiguous(), w, kind="rms")
    assert torch.equal(y, want[0]) and torch.equal(rstd, want[2])
    for a, b in zip(O.norm_backward(dy[:1].expand(5, 1), x, w, None, rstd, kind="rms"), O.norm_backward(dy[:1].repeat(5, 1), x.contiguous(), w, None, rstd, kind="rms")):
        assert a is b is None or torch.equal(a, b)


def test_heads_without_channels(monkeypatch):
    """Refused by the library, as other sizes that it does not take are."""
    B.lib()
    monkeypatch.setattr(O, "_typed", lambda first: 0)
    q = torch.zeros(1, 3, 2, 0)
    with pytest.raises(B.DdpError) as e:
        O.attention_forward(q, q, q)
    assert e.value.code == 1 and "head_dim" in str(e.value)
