"""The norms around a block: bounds for each row, and weights that are still being written."""
import pytest

from paper_2307_11339_amd import rnn
from test_block_norm import BF16, F32, LAYER, RMS, G_SILU, Case, gpu  # noqa: F401  (the fixture)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_weights_that_another_stream_is_still_writing(gpu, dtype):
    """The vectors are written on a side stream behind some milliseconds of other work; the norm is created without waiting."""
    torch = gpu
    c = Case(5, 3, 1024, dtype, after=LAYER, groups=4, gate=G_SILU, before=RMS)
    assert c.forward() == rnn.RNN_OK
    torch.cuda.synchronize()
    y, out = c.y.clone(), c.out.clone()
    late = {n: None if t is None else torch.full_like(t, 3.0) for n, t in c.vec.items()}
    m = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            m = m @ m * 1e-2
        for n, t in late.items():
            if t is not None:
                t.copy_(c.vec[n])
    handle = rnn.rnn_block_norm_create(1024, dtype, LAYER, 4, late["aw"], late["ab"], G_SILU, late["sc"], RMS, late["bw"], late["bb"],
                                       c.eps, 1)
    rnn.rnn_block_norm_destroy(c.handle)
    c.handle = handle
    assert c.forward() == rnn.RNN_OK
    torch.cuda.synchronize()
    assert torch.equal(c.y, y) and torch.equal(c.out, out)
