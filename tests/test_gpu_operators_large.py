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


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_of_rows_of_2_to_the_27(kind):
    """The weight's gradient has 32 columns a workgroup of 1024 threads."""
    from paper_2502_11058_amd import operators as O
    cols = (1 << 27) + 7
    g = generator(3)
    x, dy = (torch.empty(2, cols, device="cuda", dtype=torch.bfloat16).normal_(generator=g) for _ in range(2))
    w = torch.ones(cols, device="cuda", dtype=torch.bfloat16)
    y, mean, rstd = O.norm_forward(x, w, kind=kind)
    dx, dw, db = O.norm_backward(dy, x, w, mean, rstd, kind=kind, bias=True)
    for a in range(0, cols, 1 << 24):
        at = slice(a, a + (1 << 24))
        h, d = (x[:, at].float() - (mean[:, None] if kind == "layer" else 0.0)) * rstd[:, None], dy[:, at].float()
        # from the mean and rstd that the call gave: a few units of fp32, rounded to bf16
        for got, terms in ((dw[at], d * h), (db[at], d)):
            assert ((got.float() - terms.sum(0)).abs() <= 8 * EPS * (terms.abs().sum(0) + d.abs().sum(0)) + 2.0 ** -8 * terms.sum(0).abs()).all(), a
        assert ((y[:, at].float() - h).abs() <= 8 * EPS * (h.abs() + 1) + 2.0 ** -8 * h.abs()).all(), a


@pytest.mark.parametrize("dtype,batch,dim", [(torch.float32, (1 << 20) + 1, 8), (torch.bfloat16, (1 << 20) + 1, 72), (torch.bfloat16, (1 << 21) + 1, 8)])
def test_attention_of_more_heads_than_a_grid_has_workgroups(dtype, batch, dim):
    """8 heads of so many sequences with one query and key each, a workgroup of 256 or 512 threads a head: o is v, dv is do, and nothing is left
    for dq and dk."""
    from paper_2502_11058_amd import operators as O
    g = generator(batch + dim)
    q, k, v, do = (torch.empty(batch, 1, 8, dim, device="cuda", dtype=dtype).normal_(generator=g) for _ in range(4))
    o, lse = O.attention_forward(q, k, v)
    dq, dk, dv = O.attention_backward(do, q, k, v, o, lse)
    fine = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -18
    for a in range(0, batch, 1 << 18):
        at = slice(a, a + (1 << 18))
        x, y, u, w = (t[at, 0].double() for t in (q, k, v, do))
        z, terms = (x * y).sum(-1) * dim ** -0.5, (x * y).abs().sum(-1) * dim ** -0.5
        # the score's products and sum in fp32, and the logarithm's base changed both ways; that much of p, which is 1, is off
        assert ((lse[at, :, 0].double() - z).abs() <= 64 * EPS * (terms + 1)).all(), a
        off = (fine + 64 * EPS * (terms + 1))[..., None]
        assert ((o[at, 0].double() - u).abs() <= off * u.abs()).all() and ((dv[at, 0].double() - w).abs() <= off * w.abs()).all(), a
        # do . v and do . o differ by what o was rounded and by fp32
        off = 2 * off * (w * u).abs().sum(-1, keepdim=True) * dim ** -0.5
        assert (dq[at, 0].double().abs() <= off * y.abs()).all() and (dk[at, 0].double().abs() <= off * x.abs()).all(), a
