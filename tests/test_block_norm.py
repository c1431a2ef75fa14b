"""The norms around a block with its gate and residual scale, through the C ABI, against the formula in 64 bits.

Tolerances (u = 2^-24, the rounding of fp32).  With m = the largest absolute value of a row and n = its width, a sum of n
products is off by at most (n + 2) u of the sum of absolute values; the sum of squares has no cancellation, so a norm's factor
is off by (n + 8) u relatively, and its mean by (n + 2) u m.  Every further product or sum adds one u of what it handles, the
gate's function 2^-20 (a bf16 path uses the fast exponential and reciprocal; fp32 paths are closer).  A norm scales what went
in before by its factor, so a first error is carried on multiplied by factor * (1 + |normed value|^2 of a row, at most n).
The tests take inputs of order one and eps such that the factors stay below F, computed from the reference, and allow
    16 (n + 8) u (1 + |value|) F + 2^-20 |value| + own rounding,   own = 2^-8 (bf16) or 2^-24 (fp32) of the value.
"""
import ctypes

import numpy as np
import pytest

from paper_2307_11339_amd import rnn

F32, BF16 = rnn.RNN_F32, rnn.RNN_BF16
NONE, RMS, LAYER = rnn.RNN_NORM_NONE, rnn.RNN_NORM_RMS, rnn.RNN_NORM_LAYER
G_NONE, G_LINEAR, G_SIGMOID, G_SILU = rnn.RNN_GATE_NONE, rnn.RNN_GATE_LINEAR, rnn.RNN_GATE_SIGMOID, rnn.RNN_GATE_SILU


def _create_status(width=64, dtype=F32, after=RMS, groups=1, gate=G_NONE, before=NONE, eps=1e-5):
    lib = rnn.load_library()
    out = ctypes.c_void_p(1)
    rc = lib.rnn_block_norm_create(ctypes.byref(out), width, dtype, after, groups, None, None, gate, None, before, None, None, eps, 0)
    if rc == rnn.RNN_OK:
        lib.rnn_block_norm_destroy(out)
    else:
        assert not out.value
    return rc


@pytest.mark.parametrize("change", [dict(width=0), dict(groups=0), dict(groups=3), dict(dtype=2), dict(after=3), dict(after=-1),
                                    dict(before=3), dict(gate=4), dict(gate=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
                                    dict(eps=float("inf"))])
def test_create_refuses(change):
    assert _create_status(**change) == rnn.RNN_EINVAL


@pytest.mark.parametrize("change", [dict(width=16388), dict(width=66), dict(width=68, dtype=BF16), dict(width=64, groups=4),
                                    dict(width=88, groups=2, dtype=BF16), dict(width=132, groups=2)])
def test_create_says_what_is_not_supported(change):
    assert _create_status(**change) == rnn.RNN_EUNSUPPORTED


def test_null_handles_are_refused():
    lib = rnn.load_library()
    assert lib.rnn_block_norm_create(None, 64, 0, 1, 1, None, None, 0, None, 0, None, None, 1e-5, 0) == rnn.RNN_EINVAL
    assert rnn.rnn_block_norm_forward(None, 16, None, None, None, 16, None, 1, 1) == rnn.RNN_EINVAL
    rnn.rnn_block_norm_destroy(None)


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _norm64(a, kind, groups, w, b, eps):
    g = a.reshape(a.shape[:-1] + (groups, -1))
    if kind == LAYER:
        g = g - g.mean(-1, keepdims=True)
    factor = 1.0 / np.sqrt((g * g).mean(-1, keepdims=True) + eps)
    out = (g * factor).reshape(a.shape)
    if w is not None:
        out = out * w
    return (out if b is None else out + b), factor


class Case:
    def __init__(self, T, B, W, dtype, after=NONE, groups=1, gate=G_NONE, residual=True, before=RMS, vectors=True, lengths=None,
                 layout="time", eps=1e-5, host_weights=False, seed=0):
        import torch
        self.torch = torch
        rng = np.random.default_rng(seed + W + 131 * T + after + 7 * before)
        self.T, self.B, self.W, self.dtype, self.eps, self.layout = T, B, W, dtype, eps, layout
        self.after, self.groups, self.gate_kind, self.before = after, groups, gate, before
        self.tdt = tdt = torch.bfloat16 if dtype == BF16 else torch.float32

        def tensor(*shape):
            return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(tdt)

        if layout == "packed":
            buf = tensor(B, T, 2 * W + 8).cuda()
            self.x, self.gate = buf[..., 8:8 + W].transpose(0, 1), buf[..., 8 + W:].transpose(0, 1)
        else:
            self.x, self.gate = self.place(tensor(T, B, W)), self.place(tensor(T, B, W))
        if gate == G_NONE:
            self.gate = None
        self.residual = self.place(tensor(T, B, W)) if residual else None
        self.vec = {}
        for name, mean in (("aw", 1.0), ("ab", 0.0), ("sc", 0.5), ("bw", 1.0), ("bb", 0.0)):
            self.vec[name] = (tensor(W).float() * 0.2 + mean).to(tdt).cuda() if vectors else None
        if after == RMS:
            self.vec["ab"] = None
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.clamped = np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
        self.y, self.out = self.place(torch.full((T, B, W), 7.0, dtype=tdt)), self.place(torch.full((T, B, W), 7.0, dtype=tdt))
        torch.cuda.synchronize()
        v = dict(self.vec)
        if host_weights:
            v = {n: None if t is None else (t.cpu().view(torch.int16) if dtype == BF16 else t.cpu()).numpy() for n, t in v.items()}
        self.handle = rnn.rnn_block_norm_create(W, dtype, after, groups, v["aw"], v["ab"], gate, v["sc"], before, v["bw"], v["bb"],
                                                eps, 0 if host_weights else 1)

    def place(self, x):
        if self.layout == "time":
            return x.cuda()
        return x.transpose(0, 1).contiguous().cuda().transpose(0, 1)

    def forward(self, stream=None, **other):
        a = dict(x=self.x, gate=self.gate, residual=self.residual, out=self.out, y=self.y, lengths=self.lengths, T=self.T, B=self.B)
        a.update(other)
        return rnn.rnn_block_norm_forward(self.handle, a["x"], a["gate"], a["residual"], a["out"], a["y"], a["lengths"], a["T"], a["B"],
                                          stream or self.torch.cuda.current_stream())

    def reference(self):
        h = lambda t: None if t is None else t.detach().float().cpu().numpy().astype(np.float64)
        v = {n: h(t) for n, t in self.vec.items()}
        a, F = h(self.x), 1.0
        with np.errstate(all="ignore"):
            if self.after:
                a, f = _norm64(a, self.after, self.groups, v["aw"], v["ab"], self.eps)
                F = max(F, float(np.nanmax(f)))
            if self.gate is not None:
                z = h(self.gate)
                a = a * {G_LINEAR: z, G_SIGMOID: 1 / (1 + np.exp(-z)), G_SILU: z / (1 + np.exp(-z))}[self.gate_kind]
            if v["sc"] is not None:
                a = a * v["sc"]
            r = a if self.residual is None else a + h(self.residual)
            y = r
            if self.before:
                y, f = _norm64(r, self.before, 1, v["bw"], v["bb"], self.eps)
                F = max(F, F * float(np.nanmax(f)))
        dead = np.arange(self.T)[:, None] >= self.clamped[None, :]
        return np.where(dead[..., None], 0.0, r), np.where(dead[..., None], 0.0, y), F

    def check(self):
        self.torch.cuda.synchronize()
        r, y, F = self.reference()
        own = 2.0 ** -8 if self.dtype == BF16 else 2.0 ** -24
        for got, want in ((self.out, r), (self.y, y)):
            got = got.float().cpu().numpy().astype(np.float64)
            tol = 16 * (self.W + 8) * 2.0 ** -24 * (1 + abs(want)) * F + 2.0 ** -20 * abs(want) + own * abs(want)
            worst = (abs(got - want) / tol).max()
            assert worst <= 1, worst
        bits = self.torch.int16 if self.dtype == BF16 else self.torch.int32
        for b in range(self.B):
            for t in (self.out, self.y):
                assert not bool((t[int(self.clamped[b]):, b].contiguous().view(bits) != 0).any())

    def __del__(self):
        if getattr(self, "handle", None):
            self.torch.cuda.synchronize()
            rnn.rnn_block_norm_destroy(self.handle)


SHAPES = [(1, 1, 8), (1, 3, 64), (5, 2, 256), (3, 7, 504), (2, 130, 1024), (7, 3, 1280), (2, 2, 2048), (3, 1, 4104), (1, 2, 8192), (2, 1, 16384)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("before", [RMS, LAYER], ids=["rms", "layer"])
@pytest.mark.parametrize("shape", SHAPES, ids=["T%d_B%d_W%d" % s for s in SHAPES])
def test_sum_and_norm(gpu, shape, before, dtype):
    c = Case(*shape, dtype, before=before)
    assert c.forward() == rnn.RNN_OK
    c.check()


GROUPED = [(2, 3, 64, 2), (4, 2, 400, 5), (3, 2, 1280, 5), (2, 2, 1024, 16), (2, 2, 2048, 16), (1, 3, 1056, 33), (3, 1, 4096, 2),
           (2, 2, 8192, 64), (1, 2, 16384, 512), (2, 1, 14400, 400), (2, 1, 16320, 4)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("before", [NONE, LAYER], ids=["after_only", "sandwich"])
@pytest.mark.parametrize("shape", GROUPED, ids=["T%d_B%d_W%d_g%d" % s for s in GROUPED])
def test_norm_by_groups_with_gate(gpu, shape, before, dtype):
    T, B, W, groups = shape
    if dtype == BF16 and (W // groups) % 8:
        pytest.skip("groups of this width are fp32 only")
    for after, gate in ((RMS, G_SILU), (LAYER, G_SIGMOID)):
        c = Case(T, B, W, dtype, after=after, groups=groups, gate=gate, before=before, layout="batch")
        assert c.forward() == rnn.RNN_OK
        c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("after,gate,residual,before,vectors", [
    (NONE, G_NONE, True, NONE, True), (NONE, G_NONE, False, RMS, True), (NONE, G_LINEAR, False, NONE, False),
    (RMS, G_NONE, False, NONE, False), (LAYER, G_NONE, True, NONE, True), (LAYER, G_LINEAR, True, LAYER, False),
    (NONE, G_SILU, True, LAYER, True), (RMS, G_SIGMOID, True, RMS, True)])
def test_parts_that_may_be_absent(gpu, after, gate, residual, before, vectors, dtype):
    for T, B, lengths in ((1, 1, None), (9, 4, [9, 0, 4, 100])):
        c = Case(T, B, 320, dtype, after=after, groups=5, gate=gate, residual=residual, before=before, vectors=vectors, lengths=lengths,
                 layout="packed", host_weights=True)
        assert c.forward() == rnn.RNN_OK
        c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_one_output_or_both_and_in_place(gpu, dtype):
    torch = gpu
    c = Case(5, 3, 512, dtype, after=RMS, groups=4, gate=G_SILU, before=LAYER, lengths=[5, 3, 0])
    assert c.forward() == rnn.RNN_OK
    c.check()
    y, out = c.y.clone(), c.out.clone()
    c.y.fill_(5.0)
    c.out.fill_(5.0)
    assert c.forward(out=None) == rnn.RNN_OK
    torch.cuda.synchronize()
    assert torch.equal(c.y, y) and bool((c.out == 5).all())
    c.y.fill_(5.0)
    assert c.forward(y=None) == rnn.RNN_OK
    torch.cuda.synchronize()
    assert torch.equal(c.out, out) and bool((c.y == 5).all())
    assert c.forward(out=c.residual, y=c.x) == rnn.RNN_OK          # the stream and the block's output updated in place
    torch.cuda.synchronize()
    assert torch.equal(c.residual, out) and torch.equal(c.x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_rows_that_are_hard_to_norm(gpu, dtype):
    """Rows of zeros, rows far from zero, rows of large values; NaN and infinities only in their own rows."""
    torch = gpu
    c = Case(6, 2, 256, dtype, after=LAYER, before=LAYER, residual=False, vectors=False, eps=1e-3)
    c.x[0] = 0
    c.x[1] += 64.0
    c.x[2] *= 2.0 ** 40
    c.x[3] *= 2.0 ** -40
    assert c.forward() == rnn.RNN_OK
    c.check()
    y = c.y.clone()
    c.x[4, 0, 17] = float("nan")
    c.x[5, 1, 3] = float("inf")
    assert c.forward() == rnn.RNN_OK
    torch.cuda.synchronize()
    same = torch.ones((6, 2), dtype=torch.bool, device="cuda")
    same[4, 0] = same[5, 1] = False
    assert torch.equal(c.y[same], y[same])
    assert bool(c.y[~same].isnan().all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_padding_is_not_read_and_gates_saturate(gpu, dtype):
    torch = gpu
    c = Case(8, 3, 192, dtype, after=RMS, groups=3, gate=G_SIGMOID, lengths=[8, 2, 0])
    c.gate[0, 0, :64] = 200.0
    c.gate[0, 0, 64:128] = -200.0
    assert c.forward() == rnn.RNN_OK
    c.check()
    y, out = c.y.clone(), c.out.clone()
    for b, n in enumerate((8, 2, 0)):
        for t in (c.x, c.gate, c.residual):
            t[n:, b] = float("nan")
    assert c.forward() == rnn.RNN_OK
    torch.cuda.synchronize()
    assert torch.equal(c.y, y) and torch.equal(c.out, out)


@pytest.mark.gpu
def test_many_rows_and_nothing_outside(gpu):
    """More rows than workgroups at once; outputs as slices of wider buffers."""
    torch = gpu
    c = Case(300, 50, 128, BF16, before=RMS, lengths=[300 - 5 * b for b in range(50)])
    ybuf, obuf = (torch.full((300, 50, 128 + 24), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.y, c.out = ybuf[..., 16:144], obuf[..., :128]
    assert c.forward() == rnn.RNN_OK
    c.check()
    assert bool((ybuf[..., :16] == 7).all()) and bool((ybuf[..., 144:] == 7).all()) and bool((obuf[..., 128:] == 7).all())


@pytest.mark.gpu
def test_rows_more_than_two_to_the_31_elements_apart(gpu):
    torch = gpu
    T, B, W, far = 2, 3, 64, (1 << 30) + 8
    c = Case(T, B, W, BF16)
    bufs = [torch.empty(2 * far + T * W, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    views = [torch.as_strided(b, (T, B, W), (W, far, 1)) for b in bufs]
    views[0].copy_(c.x)
    c.x, c.y = views
    assert c.forward() == rnn.RNN_OK
    c.check()


@pytest.mark.gpu
def test_calls_are_refused(gpu):
    torch = gpu
    c = Case(4, 2, 64, BF16, after=RMS, gate=G_SILU)
    assert c.forward(x=None) == rnn.RNN_EINVAL
    assert c.forward(gate=None) == rnn.RNN_EINVAL
    assert c.forward(y=None, out=None) == rnn.RNN_EINVAL
    assert c.forward(T=0) == rnn.RNN_EINVAL and c.forward(B=-1) == rnn.RNN_EINVAL
    for name in ("x", "gate", "residual", "out", "y"):
        assert c.forward(**{name: getattr(c, name).data_ptr() + 2}) == rnn.RNN_EINVAL
        odd = torch.zeros((4, 2, 68), dtype=torch.bfloat16, device="cuda")[..., :64]
        assert c.forward(**{name: odd}) == rnn.RNN_EINVAL
    assert c.forward(y=c.y[:1].expand(4, -1, -1)) == rnn.RNN_EINVAL
    assert c.forward(out=torch.zeros(1024, dtype=torch.bfloat16, device="cuda").as_strided((4, 2, 64), (64, 128, 1))) == rnn.RNN_EINVAL
    assert c.forward(T=1 << 20, B=1 << 11) == rnn.RNN_EUNSUPPORTED
    assert c.forward() == rnn.RNN_OK
    c.check()


@pytest.mark.gpu
def test_recorded_and_replayed_on_a_side_stream(gpu):
    torch = gpu
    c = Case(33, 5, 640, BF16, after=LAYER, groups=5, gate=G_SILU, before=RMS)
    stream_of_residuals = c.residual.clone()
    want = []
    for _ in range(3):
        assert c.forward(residual=stream_of_residuals, out=stream_of_residuals) == rnn.RNN_OK
        torch.cuda.synchronize()
        want.append((c.y.clone(), stream_of_residuals.clone()))
    state = c.residual.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            rc = c.forward(side, residual=state, out=state)
        assert rc == rnn.RNN_OK
    torch.cuda.synchronize()
    for y, r in want:
        c.y.fill_(3.0)
        torch.randn(1000, 1000, device="cuda").sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.y, y) and torch.equal(state, r)
