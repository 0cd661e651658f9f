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


# ---- offsets beyond 2^31 elements ----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_of_more_than_2_to_the_31_elements(dtype):
    from paper_2502_11058_amd import operators as O
    rows, cols = (1 << 20) + 5, 2056
    g = generator(5)
    x, dy = (torch.empty(rows, cols, device="cuda", dtype=dtype).normal_(generator=g) for _ in range(2))
    w, b = (torch.empty(cols, device="cuda", dtype=dtype).normal_(generator=g) for _ in range(2))
    y, mean, rstd = O.norm_forward(x, w, b)
    dx, dw, db = O.norm_backward(dy, x, w, mean, rstd, bias=True)
    sums = torch.zeros(2, cols, device="cuda", dtype=torch.float64)
    squares = torch.zeros_like(sums)
    fine = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -23
    for a in range(0, rows, 1 << 16):
        at = slice(a, a + (1 << 16))
        u, d = x[at].double(), dy[at].double()
        m = u.mean(1, keepdim=True)
        r = 1 / torch.sqrt(((u - m) ** 2).mean(1, keepdim=True) + 1e-5)
        h = (u - m) * r
        # fp32 knows the mean, h and what they are multiplied with to a few units
        assert ((y[at].double() - (h * w.double() + b.double())).abs() <= 16 * EPS * ((h.abs() + 1) * w.double().abs() + b.double().abs()) + fine * y[at].double().abs()).all(), a
        e = d * w.double()
        want = r * (e - e.mean(1, keepdim=True) - h * (e * h).mean(1, keepdim=True))
        assert ((dx[at].double() - want).abs() <= 16 * EPS * r * (e.abs() + e.abs().mean(1, keepdim=True) * (1 + h.abs()) * 2) + fine * want.abs()).all(), a
        for i, t in enumerate((d * h, d)):
            sums[i] += t.sum(0)
            squares[i] += (t * t).sum(0)
    # a thousand partial sums of a thousand terms each, in fp32: each off by some units of its root-mean-square size, at random
    for got, want, sq in ((dw, sums[0], squares[0]), (db, sums[1], squares[1])):
        assert ((got.double() - want).abs() <= 64 * EPS * sq.sqrt() + fine * want.abs()).all()


def test_rotary_of_more_than_2_to_the_31_elements():
    from paper_2502_11058_amd import operators as O
    n, heads, dim = (1 << 20) + 5, 16, 136
    g = generator(6)
    q = torch.empty(n, heads, dim, device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    p = torch.randint(0, 512, (n,), generator=g, device="cuda")
    table = O.rotary_table(512, 128)
    got, _ = O.rotary_forward(q, None, table, p, layout="interleaved")
    for a in range(0, n, 1 << 17):
        x, y, t = q[a:a + (1 << 17)].float(), got[a:a + (1 << 17)].float(), table[p[a:a + (1 << 17)]][:, None]
        c, s, u, v = t[..., 0], t[..., 1], x[..., 0:128:2], x[..., 1:128:2]
        room = 4 * EPS * (u.abs() + v.abs())
        for part, want in ((y[..., 0:128:2], u * c - v * s), (y[..., 1:128:2], u * s + v * c)):
            assert ((part - want).abs() <= room + 2.0 ** -8 * want.abs()).all(), a
        assert torch.equal(x[..., 128:], y[..., 128:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_to_a_cache_of_more_than_2_to_the_31_elements(dtype):
    """The last five tokens of a million, 17 heads of 124 channels."""
    from test_gpu_operators_attention import _check
    g = generator(7)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    q, do = (torch.empty(1, 5, 17, 124, device="cuda", dtype=t).normal_(generator=g) for _ in range(2))
    k, v = (torch.empty(1, (1 << 20) + 77, 17, 124, device="cuda", dtype=t).normal_(generator=g) for _ in range(2))
    _check(q, k, v, do)


@pytest.mark.parametrize("dtype,tokens", [(torch.float32, 40), (torch.float32, 70), (torch.bfloat16, 70)])
def test_a_head_of_more_than_2_to_the_31_elements(dtype, tokens):
    from operator_bounds import TINY, near, over
    from paper_2502_11058_amd import operators as O
    vocab, hidden, step = (1 << 19) + 77, 4160, 1 << 15
    g = generator(tokens)
    x = torch.empty(tokens, hidden, device="cuda", dtype=dtype).normal_(generator=g)
    w = torch.empty(vocab, hidden, device="cuda", dtype=dtype).normal_(0, 1.5 / hidden ** 0.5, generator=g)
    t = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    t[0], t[1], grad = vocab - 1, -100, torch.rand(tokens, generator=g, device="cuda") + 0.5
    loss, lse = O.linear_cross_entropy_forward(x, w, t)
    dx, dw = O.linear_cross_entropy_backward(grad, x, w, t, lse)
    # as in the tests of small sizes, the weight taken in pieces
    u, xd = (2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -24), x.double()
    pieces = [slice(a, a + step) for a in range(0, vocab, step)]
    z, terms = (torch.cat([f(xd, w[p].double()) for p in pieces], 1) for f in (lambda a, b: a @ b.t(), lambda a, b: a.abs() @ b.t().abs()))
    valid, gd = t >= 0, torch.where(t >= 0, grad.double(), 0.0)
    want_lse, at = torch.logsumexp(z, 1), t.clamp(min=0)[:, None]
    p = torch.exp(z - want_lse[:, None])
    off_z = over(hidden) * terms + 4 * EPS * z.abs()
    off_lse = 2 * (p * off_z).sum(1) + 4 * EPS * want_lse.abs() + over(vocab)
    near(lse, want_lse, off_lse, "lse")
    near(loss, torch.where(valid, want_lse - z.gather(1, at)[:, 0], 0.0), off_lse + off_z.gather(1, at)[:, 0] + 4 * EPS * z.gather(1, at)[:, 0].abs(), "loss")
    hot = torch.zeros_like(p).scatter_(1, at, 1.0)
    dz = (p - hot) * gd[:, None]
    off = (p * (off_z + off_lse[:, None]) + (u + 8 * EPS) * (p - hot).abs() + 4 * EPS * p + TINY) * gd[:, None]
    want, room = (torch.zeros(tokens, hidden, device="cuda", dtype=torch.float64) for _ in range(2))
    for i in pieces:
        wd = w[i].double()
        want += dz[:, i] @ wd
        room += (off[:, i] + over(vocab) * dz[:, i].abs()) @ wd.abs()
        near(dw[i], dz[:, i].t() @ xd, off[:, i].t() @ xd.abs() + over(tokens) * (dz[:, i].abs().t() @ xd.abs()), f"dweight from {i.start}")
    near(dx, want, room, "dx")


def test_several_pieces_of_the_vocabulary_in_fp32():
    """dz is three planes there, whose distance is another in the last piece, which is shorter."""
    from test_gpu_operators_cross_entropy import _check, _inputs
    _check(*_inputs(23, "f32", 9000, 20011, 64))
