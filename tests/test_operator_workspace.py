"""Workspaces of the norm's backward pass: as many partial rows as its kernels write, and not more."""
import pytest
import torch

from paper_2502_11058_amd import binding as B

# rows, columns, type, partial rows: one of four rows a wavefront's workgroup up to 4 KiB a row, one a row up to 16 KiB, 64 beyond
SHAPES = [(1, 5, B.DDP_F32, 1), (9, 64, B.DDP_BF16, 3), (4096, 1024, B.DDP_F32, 1024), (1001, 2048, B.DDP_BF16, 251), (5000, 2048, B.DDP_BF16, 1024), (700, 4096, B.DDP_BF16, 512),
          (300, 4096, B.DDP_F32, 300), (4096, 4097, B.DDP_F32, 64), (600, 8193, B.DDP_BF16, 64), (30, 40000, B.DDP_F32, 30), (0, 64, B.DDP_F32, 0)]


def _shape(rows, cols, dtype):
    return B.ddp_norm(B.DDP_NORM_LAYER, dtype, rows, cols, cols, cols, 1e-5)


@pytest.mark.parametrize("rows,cols,dtype,parts", SHAPES)
def test_size(rows, cols, dtype, parts):
    B.lib()
    assert B.ddp_norm_backward_workspace(_shape(rows, cols, dtype)) == 2 * -(-parts * cols * 4 // 256) * 256


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype,parts", [s for s in SHAPES if s[0]])
def test_nothing_is_written_behind_it(rows, cols, dtype, parts):
    t = torch.bfloat16 if dtype == B.DDP_BF16 else torch.float32
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + cols)
    x, dy, w = (torch.randn(s, generator=g, device="cuda").to(t) for s in ((rows, cols), (rows, cols), (cols,)))
    shape, n = _shape(rows, cols, dtype), B.ddp_norm_backward_workspace(_shape(rows, cols, dtype))
    mean, rstd = (torch.empty(rows, device="cuda") for _ in range(2))
    B.ddp_norm_forward(shape, x, w, None, torch.empty_like(x), mean, rstd)
    ws = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    B.ddp_norm_backward(shape, dy, x, w, mean, rstd, dx, dw, db, ws, n)
    assert (ws[n:] == 0x5a).all()
    d, h = dy.double(), (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    # sums of `rows` terms in fp32, at random off by some units of their root-mean-square sum; then rounded
    for got, want, terms in ((dw, (d * h).sum(0), d * h), (db, d.sum(0), d)):
        room = 2.0 ** -20 * terms.square().sum(0).sqrt() * (1 + rows ** 0.5 / 16) + (2.0 ** -8 if t is torch.bfloat16 else 2.0 ** -23) * want.abs() + 1e-30
        assert ((got.double() - want).abs() <= room).all()
