"""The norms around a block: bounds for each row and value, and weights that are still being written.

Bounds (u = 2^-24, first order, 5 % more for the rest).  A term of a sum passes through D additions at most: those of a thread's
elements, six across a wave, those across waves.
  - a mean of n values is off by D u mean|x|; a sum of squares by D u of itself, a norm's factor f by half of that and 8 u;
  - what a value was off by before a norm (e), with the mean's error, is d; the factor moves by f^2 mean(|x| d) of itself, x the
    values that it is taken of (behind their mean), and a value by f d and by what the factor moves;
  - every other product or sum: u of its result; the gate's function (2 |z| + 6) u of itself.
An output's own rounding is 2^-8 (bf16) or u of it.  In bf16 it hides what the rest of a row does wrong alike, so two numbers of each
row are looked at besides, where roundings of 0.42 2^-8 (root mean square) average out: its mean and its product with what is
wanted, six deviations.  Values that are alike are rounded alike: n of them are off by n times one rounding, not by sqrt(n).
Rows without weights are left out of this: a bf16 number times a factor, less a mean, is off by what its eight bits say, the
same in every binade (a factor near 1 and a mean shift all 128 of a binade by the same part of a step), so that roundings
do not average out at all.  The tests without a GPU plant mistakes and see them out of bounds.
"""
import numpy as np
import pytest

from paper_2307_11339_amd import rnn
from test_block_norm import BF16, F32, GROUPED, LAYER, NONE, RMS, SHAPES, G_NONE, G_SIGMOID, G_SILU, Case, gpu  # noqa: F401  (the fixture)

U = 2.0 ** -24


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


def _depth(W, dtype):
    """More additions than any value passes through on its way into a sum over a row: slots are at most twice as many as there are
    pieces of 16 bytes, and eight waves take them in turn; rows of two or three pieces a thread, whatever their number."""
    n = 8 if dtype == BF16 else 4
    return n * max(3, -(-2 * W // n // 512)) + 24


def _norm_stage(x, e, kind, groups, w, b, eps, depth, drop="", piece=4):
    """A norm of rows x [R, W] that are off by e at most: the result and what it is off by.  drop: a mistake to make."""
    shape = x.shape
    x, e = (a.reshape(shape[0], groups, -1) for a in (x, e))
    n = x.shape[-1]
    d = e
    if kind == LAYER:
        mean = (x[..., :n - piece] if drop == "mean" else x).sum(-1, keepdims=True) / n
        d = e + e.mean(-1, keepdims=True) + depth * U * abs(x).mean(-1, keepdims=True)
        if drop == "one pass":
            f32 = x.astype(np.float32)
            var = ((f32 * f32).sum(-1, keepdims=True) / np.float32(n) - (f32.sum(-1, keepdims=True) / np.float32(n)) ** 2).astype(np.float64)
        x = x - mean
        d = d + U * abs(x)
    sq = ((x[..., :n - piece] if drop == "squares" else x) ** 2).sum(-1, keepdims=True) / n
    if drop == "one pass":
        sq = np.maximum(var, 0)
    f = 1 / np.sqrt(sq + eps)
    if drop == "skip":
        f = np.ones_like(f)
    moved = f * f * (abs(x) * d).mean(-1, keepdims=True) + (depth / 2 + 8) * U
    y, e = x * f, f * d + abs(x) * f * moved
    y, e = (a.reshape(shape) for a in (y, e))
    if w is not None:
        y, e = y * w, e * abs(w)
    e = e + 2 * U * abs(y)
    if b is not None:
        y = y + b
        e = e + U * abs(y)
    return y, e


def _expected(x, gate, residual, vec, after, groups, kind, before, eps, dtype, drop=("", "")):
    """(r, bound, y, bound) of rows [R, W] in 64 bits."""
    depth, piece = _depth(x.shape[1], dtype), 8 if dtype == BF16 else 4
    a, e = x, np.zeros_like(x)
    if after:
        a, e = _norm_stage(a, e, after, groups, vec["aw"], vec["ab"], eps, depth, drop[0], piece)
    if kind != G_NONE:
        z = gate
        act = 1 / (1 + np.exp(-z))
        act = act * z if kind == G_SILU else act
        a, e = a * act, e * abs(act)
        e = e + (2 * abs(z) + 7) * U * abs(a)
    if vec["sc"] is not None:
        a, e = a * vec["sc"], e * abs(vec["sc"])
        e = e + U * abs(a)
    if residual is not None:
        a = a + residual
        e = e + U * abs(a)
    y, ey = a, e
    if before:
        y, ey = _norm_stage(a, e, before, 1, vec["bw"], vec["bb"], eps, depth, drop[1], piece)
    return a, 1.05 * e, y, 1.05 * ey


def _worst(got, want, e, dtype, rows=True):
    """The largest part of its bound that a value, a row's mean or a row's scale is off by."""
    own, W = (2.0 ** -8 if dtype == BF16 else U), want.shape[1]
    off = got - want
    worst = (abs(off) / (e + own * abs(want) + 1e-38)).max()
    for o, w, b in zip(off, want, e) if rows else ():
        value, count = np.unique(abs(w), return_counts=True) if dtype == BF16 else (abs(w), 1)
        noise = 6 * 0.42 * own
        mean = abs(o.sum()) / (b.sum() + noise * np.sqrt(((count * value) ** 2).sum()) + 1e-38)
        scale = abs((o * w).sum()) / ((b * abs(w)).sum() + noise * np.sqrt(((count * value ** 2) ** 2).sum()) + 1e-38)
        worst = max(worst, mean, scale)
    return worst


def _round(x, dtype):
    import torch
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16 if dtype == BF16 else torch.float32).double().numpy()


WIDTHS = sorted({(W, 1) for _, _, W in SHAPES} | {(W, g) for _, _, W, g in GROUPED})


def _rows(W, dtype, seed, offset=0.0):
    rng = np.random.default_rng(seed + W)
    new = lambda *s, mean=0.0, by=1.0: _round(rng.standard_normal(s) * by + mean, dtype)
    vec = {"aw": new(W, mean=1, by=0.2), "ab": new(W, by=0.2), "sc": new(W, mean=0.5, by=0.2), "bw": new(W, mean=1, by=0.2), "bb": new(W, by=0.2)}
    return new(4, W, mean=1 + offset), new(4, W), new(4, W, mean=1), vec


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("W,groups", WIDTHS)
def test_the_bounds_notice_mistakes(W, groups, dtype):
    """A piece of 16 bytes left out of a mean or of the squares, a norm left out: each shows, in either norm, while results that
    are only rounded are far inside."""
    if (W // groups) % (8 if dtype == BF16 else 4):
        pytest.skip("groups of this width are not taken in this type")
    x, gate, residual, vec = _rows(W, dtype, 1)
    if groups > 1:            # the norm behind the block, by groups
        setup = (LAYER, groups, G_SILU, NONE)
        places = [0]
    else:                     # the norm before the next block, of the sum
        setup = (NONE, 1, G_NONE, LAYER)
        places = [1]
    args = (x, gate if groups > 1 else None, None if groups > 1 else residual, vec) + setup + (1e-5, dtype)
    r, er, y, ey = _expected(*args)
    assert _worst(_round(r, dtype), r, er, dtype) <= 1 and _worst(_round(y, dtype), y, ey, dtype) <= 1
    for place in places:
        for mistake in ("mean", "squares", "skip"):
            drop = ["", ""]
            drop[place] = mistake
            _, _, bad, _ = _expected(*args, drop=drop)
            assert _worst(_round(bad, dtype), y, ey, dtype) > 1, (mistake, _worst(_round(bad, dtype), y, ey, dtype))


@pytest.mark.parametrize("W", sorted({W for _, _, W in SHAPES}))
def test_the_bounds_notice_a_variance_in_one_pass(W):
    x, _, _, vec = _rows(W, F32, 2, offset=1024.0)
    args = (x, None, None, dict(vec, sc=None), NONE, 1, G_NONE, LAYER, 1e-5, F32)
    _, _, y, ey = _expected(*args)
    _, _, bad, _ = _expected(*args, drop=("", "one pass"))
    assert _worst(bad, y, ey, F32) > 1, _worst(bad, y, ey, F32)


def _hold(torch, c):
    """A Case against the bounds: every row by itself."""
    torch.cuda.synchronize()
    h = lambda t: None if t is None else t.detach().double().cpu().numpy().reshape(-1, c.W)
    vec = {n: None if t is None else t.detach().double().cpu().numpy() for n, t in c.vec.items()}
    live = (np.arange(c.T)[:, None] < c.clamped[None, :]).reshape(-1)
    some = np.flatnonzero(live)
    some = some[np.unique(np.linspace(0, some.size - 1, min(some.size, 300)).astype(int))]        # of many rows 300
    pick = lambda a: None if a is None else a[some]
    r, er, y, ey = _expected(pick(h(c.x)), pick(h(c.gate)), pick(h(c.residual)), vec, c.after, c.groups, c.gate_kind, c.before, c.eps, c.dtype)
    got_r, got_y = h(c.out), h(c.y)
    off = [_worst(pick(g), w, b, c.dtype, c.dtype == F32 or c.vec["sc"] is not None) for g, w, b in ((got_r, r, er), (got_y, y, ey))]
    assert max(off) <= 1, off
    assert not got_r[~live].any() and not got_y[~live].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("before", [RMS, LAYER], ids=["rms", "layer"])
@pytest.mark.parametrize("shape", SHAPES + [(60, 50, 1280), (40, 33, 2048), (70, 40, 504), (1030, 2, 4104)], ids=["T%d_B%d_W%d" % s for s in SHAPES + [(60, 50, 1280), (40, 33, 2048), (70, 40, 504), (1030, 2, 4104)]])
def test_each_row_of_sum_and_norm(gpu, shape, before, dtype):
    torch = gpu
    c = Case(*shape, dtype, before=before)
    c.x += 1.0
    assert c.forward() == rnn.RNN_OK
    _hold(torch, c)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("before", [NONE, RMS, LAYER], ids=["after_only", "rms", "sandwich"])
@pytest.mark.parametrize("shape", GROUPED + [(100, 30, 1280, 5), (130, 20, 2080, 26), (1100, 2, 4096, 32)], ids=["T%d_B%d_W%d_g%d" % s for s in GROUPED + [(100, 30, 1280, 5), (130, 20, 2080, 26), (1100, 2, 4096, 32)]])
def test_each_row_by_groups_with_gate(gpu, shape, before, dtype):
    torch = gpu
    T, B, W, groups = shape
    if dtype == BF16 and (W // groups) % 8:
        pytest.skip("groups of this width are fp32 only")
    for after, gate in ((RMS, G_SIGMOID), (LAYER, G_SILU)):
        c = Case(T, B, W, dtype, after=after, groups=groups, gate=gate, before=before, layout="batch",
                 lengths=[max(0, T - b) for b in range(B)])
        c.x += 1.0
        assert c.forward() == rnn.RNN_OK
        _hold(torch, c)


@pytest.mark.gpu
@pytest.mark.parametrize("row", ["zeros", "far", "large", "small", "one value"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("W", [256, 1000, 8192])
def test_rows_that_are_hard_to_norm_one_by_one(gpu, W, dtype, row):
    torch = gpu
    c = Case(3, 2, W, dtype, after=LAYER, before=LAYER, residual=False, vectors=False, eps=1e-3)
    if row == "zeros":
        c.x.zero_()
    elif row == "far":
        c.x += 1024.0 if dtype == F32 else 16.0
    elif row == "large":
        c.x *= 2.0 ** 40
    elif row == "small":
        c.x *= 2.0 ** -40
    else:
        c.x.zero_()
        c.x[..., W // 2] = 3.0
    assert c.forward() == rnn.RNN_OK
    _hold(torch, c)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,W,groups", [(F32, 16384, 1), (F32, 15860, 61), (F32, 7540, 29), (BF16, 15080, 29), (BF16, 16384, 1)])
def test_wide_rows_over_their_own_inputs(gpu, dtype, W, groups):
    """Inputs that are read late are still read before anything is written over them."""
    torch = gpu
    c = Case(5, 3, W, dtype, after=LAYER, groups=groups, gate=G_SILU, before=RMS, lengths=[5, 0, 3])
    assert c.forward() == rnn.RNN_OK
    _hold(torch, c)
    inputs = {n: getattr(c, n).clone() for n in ("x", "gate", "residual")}
    y, out = c.y.clone(), c.out.clone()
    for to_y, to_out in (("x", "residual"), ("gate", "x"), ("residual", "gate"), ("gate", "residual")):
        for n, t in inputs.items():
            getattr(c, n).copy_(t)
        assert c.forward(y=getattr(c, to_y), out=getattr(c, to_out)) == rnn.RNN_OK
        torch.cuda.synchronize()
        assert torch.equal(getattr(c, to_y), y) and torch.equal(getattr(c, to_out), out)
