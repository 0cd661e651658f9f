"""Sizes of the cross entropy whose launches would have 2^32 threads or more, of which a part would run without an error, are refused on the
host: by the calls that say what workspace they need, as by the others."""
import pytest

from paper_2502_11058_amd import binding as B

TILES = (1 << 23) - 1          # of 256 x 256, 512 threads each


@pytest.mark.parametrize("tokens,vocab,hidden,refused", [
    (1 << 22, 1 << 17, 64, True), (TILES * 256, 256, 64, True), ((1 << 22) - 256, 1 << 17, 64, False), (1 << 17, (1 << 22) - 256, 64, False), (1 << 28, 100, 64, True),
    ((1 << 28) - 16, 100, 64, False), ((1 << 28) - 16, 2049, 64, True), (64, (1 << 30) - 64, 1, False), (64, (1 << 30) - 63, 1, True), (8192, 128256, 4096, False)])
@pytest.mark.parametrize("dtype", [B.DDP_F32, B.DDP_BF16])
def test_cross_entropy(tokens, vocab, hidden, refused, dtype):
    B.lib()
    head = B.ddp_head(dtype, tokens, vocab, hidden, hidden, hidden, hidden, hidden)
    for call in (B.ddp_cross_entropy_forward_workspace, B.ddp_cross_entropy_backward_workspace):
        if refused:
            with pytest.raises(B.DdpError) as e:
                call(head, None, None)
            assert e.value.code == 1 and len(str(e.value)) > 20
        else:
            assert call(head, None, None) > 0
