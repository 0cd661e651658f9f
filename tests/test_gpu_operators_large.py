"""Calls whose launches come near 2^32 threads, which no grid has, and pass it."""
import pytest
import torch

from operator_bounds import EPS, generator

pytestmark = pytest.mark.gpu


def test_rotary_of_more_tokens_than_a_grid_has_wavefronts():
    """2^28 tokens, four a workgroup with a wavefront each, are a grid of 2^26 x 64 threads."""
    from paper_2502_11058_amd import operators as O
    n = (1 << 28) + 9
    g = generator(1)
    q = torch.empty(n, 1, 4, device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    p = torch.randint(0, 512, (n,), generator=g, device="cuda", dtype=torch.int32)
    table = O.rotary_table(512, 4)
    got, _ = O.rotary_forward(q, None, table, p)
    for a in range(0, n, 1 << 25):
        x, y, t = q[a:a + (1 << 25), 0].float(), got[a:a + (1 << 25), 0].float(), table[p[a:a + (1 << 25)].long()]
        c, s, u, v = t[..., 0], t[..., 1], x[:, :2], x[:, 2:]
        # two products and a sum in fp32, rounded to bf16
        room = 4 * EPS * (u.abs() + v.abs())
        for part, want in ((y[:, :2], u * c - v * s), (y[:, 2:], u * s + v * c)):
            assert ((part - want).abs() <= room + 2.0 ** -8 * want.abs()).all(), a


def test_a_table_of_more_pairs_than_a_grid_has_threads():
    """2^25 positions of 128 pairs: 2^32 pairs, 32 GiB."""
    from paper_2502_11058_amd import operators as O
    rows = (1 << 25) + 3
    table = O.rotary_table(rows, 256, base=500000.0)
    at = torch.tensor([0, 1, 12345678, (1 << 24) + 1, (1 << 25) - 1, 1 << 25, rows - 1], device="cuda")
    a = at.double()[:, None] * 500000.0 ** (-torch.arange(128, dtype=torch.float64, device="cuda") * 2 / 256)
    # half a unit of fp32, and the angle's own rounding in 64 bits: angles up to 2^25, two units of them
    assert ((table[at].double() - torch.stack([a.cos(), a.sin()], -1)).abs() <= 2.0 ** -24 + 2.0 ** -26).all()
