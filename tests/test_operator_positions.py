"""Positions of rotary calls go with their tokens: a tensor of as many in another order is refused."""
import pytest
import torch

from paper_2502_11058_amd import binding as B
from paper_2502_11058_amd import operators as O


@pytest.fixture
def called(monkeypatch):
    """The checks alone: tensors on the host pass as the GPU's, and what reaches the library is kept."""
    seen = []
    monkeypatch.setattr(O, "_typed", lambda first: 0)
    monkeypatch.setattr(B, "ddp_rotary", lambda shape, q, k, table, positions, q_out, k_out: seen.append(positions))
    return seen


@pytest.mark.parametrize("lead,positions,fits", [((2, 6), (2, 6), True), ((2, 6), (12,), True), ((2, 6), (6, 2), False), ((2, 6), (3, 4), False), ((2, 6), (6,), False),
                                                 ((6,), (6,), True), ((6,), (1, 6), True), ((6,), (2, 3), False), ((1, 6), (6,), True), ((1, 6), (6, 1), True),
                                                 ((1, 1), (), True), ((3, 2, 2), (3, 4), False), ((3, 2, 2), (3, 2, 2), True), ((4, 4), (4, 4), True), ((), (1,), True)])
def test_shapes(called, lead, positions, fits):
    q, table = torch.zeros(*lead, 2, 8), torch.zeros(4, 4, 2)
    p = torch.zeros(positions, dtype=torch.int64)
    if fits:
        O.rotary_forward(q, q, table, p)
        assert called[0] is p
    else:
        with pytest.raises(ValueError, match="positions"):
            O.rotary_forward(q, q, table, p)
        assert not called


@pytest.mark.gpu
def test_positions_of_a_batch():
    """[batch, tokens], a transposed tensor of them, and all in one row: the same; [tokens, batch] is refused."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q, table = torch.randn(3, 5, 2, 32, generator=g, device="cuda"), O.rotary_table(64, 32)
    p = torch.randint(0, 64, (3, 5), generator=g, device="cuda")
    want, _ = O.rotary_forward(q, None, table, p)
    for b in range(3):
        assert torch.equal(O.rotary_forward(q[b], None, table, p[b])[0], want[b])
    for same in (p.flatten(), p.t().contiguous().t(), p.int()):
        assert torch.equal(O.rotary_forward(q, None, table, same)[0], want)
    with pytest.raises(ValueError):
        O.rotary_forward(q, None, table, p.t())
