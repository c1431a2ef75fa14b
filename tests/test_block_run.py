"""Two blocks of a residual network run together, as a program uses them: an LSTM layer reads the normed stream and gives q, k, v
and a gate as slices of its output, linear attention reads them in place, and the norms around the block norm its heads, apply
the gate, add to the residual stream in place and norm the sum for the next block.  Everything is enqueued before anything is
looked at.  Each call's outputs are then held against its formula in 64 bits, on what the call before left in device memory:
    LSTM       1e-4 (fp32), 2e-2 (bf16), as for the layer alone
    attention  as in test_linear_attention
    norms      as in test_block_norm; eps = 0.01 keeps each norm's factor at 10 or less, so F <= 100
"""
import numpy as np
import pytest

from paper_2307_11339_amd import rnn
from test_linear_attention import _reference, _tolerances

pytestmark = pytest.mark.gpu

F32, BF16 = rnn.RNN_F32, rnn.RNN_BF16
H, HKV, DK, DV = 4, 2, 16, 40
W = H * DV                                        # the residual stream
PARTS = [H * DK, HKV * DK, HKV * DV, H * DV]      # q, k, v, gate
UNITS = sum(PARTS)
EPS = 0.01
DECAY = [1.0, 0.99, 0.75, 0.0]
BLOCKS = 2


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _host(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


class Net:
    """The handles of the blocks and their weights."""

    def __init__(self, torch, dtype):
        self.torch, self.dtype = torch, dtype
        self.tdt = torch.bfloat16 if dtype == BF16 else torch.float32
        gen = torch.Generator().manual_seed(11)

        def w(*shape, by=1.0, plus=0.0):
            return (torch.randn(shape, generator=gen) * by + plus).to(self.tdt).cuda()

        self.weights, self.lstm, self.attention, self.vectors, self.norm = [], [], [], [], []
        for _ in range(BLOCKS):
            self.weights.append([w(4 * UNITS, W, by=0.15), w(4 * UNITS, UNITS, by=0.05), w(4 * UNITS, by=0.3), None])
            self.vectors.append([w(W, by=0.2, plus=1.0), w(W, by=0.2, plus=0.5), w(W, by=0.2, plus=1.0), w(W, by=0.2)])
            aw, sc, bw, bb = self.vectors[-1]
            torch.cuda.synchronize()
            self.lstm.append(rnn.rnn_model_create(0, 1, W, UNITS, 1, dtype, self.weights[-1], 1))
            self.attention.append(rnn.rnn_linear_attention_create(H, HKV, DK, DV, dtype, DECAY, 0.5))
            self.norm.append(rnn.rnn_block_norm_create(W, dtype, rnn.RNN_NORM_RMS, H, aw, None, rnn.RNN_GATE_SILU, sc,
                                                       rnn.RNN_NORM_LAYER, bw, bb, EPS, 1))

    def states(self, B):
        """h, c and the attention's state of each block, for B live streams."""
        zeros = lambda *s: self.torch.zeros(s, device="cuda")
        return [(zeros(1, B, UNITS), zeros(1, B, UNITS), zeros(B, H, DK, DV)) for _ in range(BLOCKS)]

    def buffers(self, T, B):
        """What a run writes: the LSTM's output, the attention's, the normed stream, for each block."""
        new = lambda *s: self.torch.full(s, 7.0, dtype=self.tdt, device="cuda")
        return [(new(T, B, UNITS), new(T, B, H, DV), new(T, B, W)) for _ in range(BLOCKS)]

    def run(self, x, stream, buffers, states, lengths, T, B, s=None, streams_after=None):
        """x: the normed stream that the first block reads; stream: the residual stream, updated in place."""
        for i in range(BLOCKS):
            z, o, n = buffers[i]
            h, c, S = states[i]
            assert rnn.rnn_forward(self.lstm[i], x, lengths, h, c, z, h, c, T, B, s) == rnn.RNN_OK
            q, k, v, gate = z.split(PARTS, -1)
            q, k, v = q.unflatten(-1, (H, DK)), k.unflatten(-1, (HKV, DK)), v.unflatten(-1, (HKV, DV))
            assert rnn.rnn_linear_attention_forward(self.attention[i], q, k, v, lengths, S, o, S, T, B, s) == rnn.RNN_OK
            assert rnn.rnn_block_norm_forward(self.norm[i], o.view(T, B, W), gate, stream, stream, n, lengths, T, B, s) == rnn.RNN_OK
            if streams_after is not None:
                streams_after.append(stream.clone())
            x = n

    def close(self):
        self.torch.cuda.synchronize()
        for i in range(BLOCKS):
            rnn.rnn_model_destroy(self.lstm[i])
            rnn.rnn_linear_attention_destroy(self.attention[i])
            rnn.rnn_block_norm_destroy(self.norm[i])

    # ---- the formulas in 64 bits ----

    def lstm64(self, i, x, live):
        wi, wh, b = (_host(w) for w in self.weights[i][:3])
        T, B = x.shape[:2]
        h, c, y = np.zeros((B, UNITS)), np.zeros((B, UNITS)), np.zeros((T, B, UNITS))
        sig = lambda a: 1 / (1 + np.exp(-a))
        for t in range(T):
            gi, gf, gg, go = np.split(x[t] @ wi.T + h @ wh.T + b, 4, -1)
            new_c = sig(gf) * c + sig(gi) * np.tanh(gg)
            new_h = sig(go) * np.tanh(new_c)
            on = live[t][:, None]
            h, c = np.where(on, new_h, h), np.where(on, new_c, c)
            y[t] = np.where(on, new_h, 0.0)
        return y, h, c

    def norms64(self, i, o, gate, stream):
        aw, sc, bw, bb = (_host(v) for v in self.vectors[i])
        g = o.reshape(o.shape[:2] + (H, DV))
        f1 = 1 / np.sqrt((g * g).mean(-1, keepdims=True) + EPS)
        a = (g * f1).reshape(o.shape) * aw * (gate / (1 + np.exp(-gate))) * sc
        r = stream + a
        d = r - r.mean(-1, keepdims=True)
        f2 = 1 / np.sqrt((d * d).mean(-1, keepdims=True) + EPS)
        return r, d * f2 * bw + bb, max(1.0, f1.max()) * max(1.0, f2.max())

    def check(self, x, streams, buffers, states, lengths):
        """streams: the residual stream before the first block and after each."""
        self.torch.cuda.synchronize()
        T, B = x.shape[:2]
        live = np.arange(T)[:, None] < lengths[None, :]
        own, tol_lstm = (2.0 ** -8, 2e-2) if self.dtype == BF16 else (2.0 ** -24, 1e-4)
        for i in range(BLOCKS):
            (z, o, n), (h, c, S) = ([_host(t) for t in part] for part in (buffers[i], states[i]))
            y, want_h, want_c = self.lstm64(i, _host(x) if i == 0 else _host(buffers[i - 1][2]), live)
            assert abs(z - y).max() <= tol_lstm and abs(h[0] - want_h).max() <= tol_lstm and abs(c[0] - want_c).max() <= tol_lstm
            q, k, v, gate = np.split(z, np.cumsum(PARTS)[:-1], -1)
            args = [a.reshape(T, B, heads, -1) for a, heads in ((q, H), (k, HKV), (v, HKV))] + [DECAY, 0.5, lengths, None]
            want_o, want_S = _reference(*args)
            tol_o, tol_S = _tolerances(self.dtype, *args, want_o)
            assert (abs(o - want_o) <= tol_o).all() and (abs(S - want_S) <= tol_S).all()
            r, want_n, F = self.norms64(i, o.reshape(T, B, W), gate, _host(streams[i]))
            for got, want in ((_host(streams[i + 1]), r), (n, want_n)):
                want = np.where(live[..., None], want, 0.0)
                tol = 16 * (W + 8) * 2.0 ** -24 * (1 + abs(want)) * F + 2.0 ** -20 * abs(want) + own * abs(want)
                assert (abs(got - want) <= tol).all()
                assert not got[~live].any()


def _inputs(torch, net, T, B, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(100 + seed)
    new = lambda: torch.randn(T, B, W, device="cuda", generator=gen).to(net.tdt)
    return new(), new()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,B,lengths", [(1, 3, None), (7, 2, [7, 0]), (150, 3, [150, 64, 1]), (1100, 1, None)],
                         ids=["token", "few", "padded", "prompt"])
def test_blocks_together(gpu, T, B, lengths, dtype):
    torch = gpu
    net = Net(torch, dtype)
    x, stream = _inputs(torch, net, T, B)
    streams, after = [stream.clone()], []
    buffers, states = net.buffers(T, B), net.states(B)
    ends = np.full(B, T) if lengths is None else np.asarray(lengths)
    on_device = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    net.run(x, stream, buffers, states, on_device, T, B, torch.cuda.current_stream(), after)
    net.check(x, streams + after, buffers, states, ends)
    net.close()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_a_prompt_then_token_by_token_recorded(gpu, dtype):
    """A prompt in one call, then one token a call with the states updated in place: eagerly, and as replays of one recorded
    token on a second set of states, which gives the same bits; both together are the sequence's formulas."""
    torch = gpu
    net = Net(torch, dtype)
    B, prompt, T = 3, 80, 90
    x, stream = _inputs(torch, net, T, B, 1)
    first = stream.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        states, after = net.states(B), []
        whole = net.buffers(prompt, B)
        net.run(x[:prompt], stream[:prompt], whole, states, None, prompt, B, s, after)
        other = [tuple(t.clone() for t in block) for block in states]
        xt, st, token = x[0:1].clone(), stream[0:1].clone(), net.buffers(1, B)
        net.run(xt, st, token, [tuple(t.clone() for t in block) for block in states], None, 1, B, s)      # workspaces
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        net.run(xt, st, token, other, None, 1, B, s)
    torch.cuda.synchronize()
    parts = [[whole[i]] for i in range(BLOCKS)]
    middle = [after[0]]                           # the stream between the blocks
    for t in range(prompt, T):
        out, between = net.buffers(1, B), []
        with torch.cuda.stream(s):
            live = stream[t:t + 1].clone()
            net.run(x[t:t + 1], live, out, states, None, 1, B, s, between)
            xt.copy_(x[t:t + 1])
            st.copy_(stream[t:t + 1])
            graph.replay()
            stream[t:t + 1] = live
        torch.cuda.synchronize()
        assert torch.equal(st, live)
        for i in range(BLOCKS):
            assert all(torch.equal(a, b) for a, b in zip(token[i], out[i]))
            assert all(torch.equal(a, b) for a, b in zip(other[i], states[i]))
            parts[i].append(out[i])
        middle.append(between[0])
    buffers = [tuple(torch.cat(p) for p in zip(*parts[i])) for i in range(BLOCKS)]
    net.check(x, [first, torch.cat(middle), stream], buffers, states, np.full(B, T))
    del graph
    net.close()
