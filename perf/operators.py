"""Linear attention with a decay for each head, and the norms around a block, as a list of calls to measure: listed(), and
draw() for more of the same.  Where `own` is false, run() computes them from elementary torch operations.

A case with op = "attention" is one call of a linear-attention layer:
    dtype        "bf16" | "f32"       type of q, k, v and o
    T, B         steps and sequences of the call
    H, Hkv       heads, heads of k and v (head h reads k and v of head h // (H // Hkv))
    Dk, Dv       width of a head's q and k, of its v and o
    len_min      0: every sequence has T steps; else lengths are uniform in [len_min, T]
    state        whether a state is handed in and the new one wanted
    layout       "time" [T, B, heads, .] | "batch" [B, T, heads, .]
    packed       q, k and v are slices of one projection's output
A case with op = "norm" is one call of the norms around a block:
    dtype, T, B, len_min, layout      likewise
    W, groups    row width; parts of a row that the norm behind the block treats alone (heads)
    after        "" | "rms" | "layer"     norm of the block's output
    gate         "" | "linear" | "sigmoid" | "silu"
    residual     whether there is a residual stream to add to (with a scale for each channel), whose new value is wanted
    before       "" | "rms" | "layer"     norm of the sum, for the next block
    packed       x and gate are slices of one projection's output
"""
import math

import torch

own = False

EPS = 1e-5


def _attention(name, dtype, T, B, H, Hkv, Dk, Dv, len_min=0, state=False, layout="time", packed=False):
    c = dict(op="attention", dtype=dtype, T=T, B=B, H=H, Hkv=Hkv, Dk=Dk, Dv=Dv, len_min=len_min, state=state,
             layout=layout, packed=packed)
    return dict(c, name=name) if name else c


def _norm(name, dtype, T, B, W, groups=1, after="", gate="", residual=False, before="", len_min=0, layout="time", packed=False):
    c = dict(op="norm", dtype=dtype, T=T, B=B, W=W, groups=groups, after=after, gate=gate, residual=residual, before=before,
             len_min=len_min, layout=layout, packed=packed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token of a live stream: the state of the call before comes in, the new one goes out.  All latency.
        _attention("token", "bf16", 1, 1, 8, 8, 128, 128, state=True),
        # One new token of each of many streams served together: as fast as states can be read and written.
        _attention("token_batch", "bf16", 1, 128, 16, 16, 128, 128, state=True, packed=True),
        # A few tokens of each of some streams at once, in fp32: too few for a chunk.
        _attention("few_tokens_f32", "f32", 6, 24, 8, 8, 64, 64, state=True),
        # One prompt of ordinary length: few heads, so the steps have to be split.
        _attention("prompt", "bf16", 4096, 1, 16, 16, 128, 128, state=True),
        # One very long document whose heads share their keys and values.
        _attention("long_document", "bf16", 65536, 1, 16, 2, 128, 128, state=True),
        # An acoustic batch: padded batch-first slices of one projection, sizes that fit nothing.
        _attention("ragged", "bf16", 301, 57, 5, 5, 80, 160, len_min=75, layout="batch", packed=True),
        # Offline encoding of a full batch, the largest call.
        _attention("offline", "bf16", 2048, 32, 16, 16, 128, 128),
        # A batch of an fp32 model, as it comes out of training without conversion.
        _attention("batch_f32", "f32", 512, 16, 8, 8, 64, 64, state=True),
        # One token's row between two blocks.
        _norm("row", "bf16", 1, 1, 1024, residual=True, before="rms"),
        # Behind the recurrence of a large batch: every head's output normed and gated, slices of one tensor each.
        _norm("heads_gated", "bf16", 2048, 32, 2048, groups=16, after="rms", gate="silu", packed=True),
        # Between the layers of a residual stack at the size of the offline LSTM encoder: sum and next norm.
        _norm("residual", "bf16", 512, 256, 1024, residual=True, before="rms"),
        # Everything at once on a padded fp32 batch: norm of the block, gate, scaled residual, norm for the next block.
        _norm("sandwich_f32", "f32", 301, 57, 1280, groups=5, after="layer", gate="sigmoid", residual=True, before="layer",
              len_min=75, layout="batch"),
    ]


def _log(rng, lo, hi, step=1):
    """A size in [lo, hi], even over its logarithm, a multiple of `step`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))
    return min(hi - hi % step, max(lo + -lo % step, int(v / step + 0.5) * step))


def _one(rng):
    """One draw: a kind of use as in listed(), its sizes spread over that use's range."""
    use = rng.choice(("token", "few_tokens", "prompt", "batch", "batch", "heads", "between", "sandwich"))
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    layout, packed = rng.choice(("time", "batch")), rng.random() < 0.5
    step = 8 if dtype == "bf16" else 4
    if use in ("heads", "between", "sandwich"):
        T, B = (1, _log(rng, 1, 256)) if rng.random() < 0.3 else (_log(rng, 16, 2048), _log(rng, 1, 64))
        len_min = max(1, T // 4) if T > 1 and rng.random() < 0.5 else 0
        kind = rng.choice(("rms", "layer"))
        if use == "heads":
            groups = rng.randint(1, 32)
            return _norm("", dtype, T, B, groups * _log(rng, 32, 256, step), groups, kind, rng.choice(("", "sigmoid", "silu")),
                         len_min=len_min, layout=layout, packed=packed)
        if use == "between":
            return _norm("", dtype, T, B, _log(rng, 64, 8192, step), residual=True, before=kind, len_min=len_min, layout=layout)
        groups = rng.choice((1, 1, 2, 4, 5, 8))
        return _norm("", dtype, T, B, groups * _log(rng, 64, 1024, step), groups, kind, rng.choice(("", "linear", "sigmoid", "silu")),
                     residual=True, before=rng.choice(("rms", "layer")), len_min=len_min, layout=layout, packed=packed)
    Dk, Dv = (rng.choice((64, 128)),) * 2 if rng.random() < 0.5 else (_log(rng, 32, 256, step), _log(rng, 32, 256, step))
    Hkv = rng.randint(1, 16)
    H = Hkv * rng.choice((1, 1, 1, 2)) if Hkv <= 8 else Hkv
    len_min, state = 0, True
    if use == "token":
        T, B = 1, _log(rng, 1, 128)
    elif use == "few_tokens":
        T, B = rng.randint(2, 24), _log(rng, 1, 64)
        len_min = 1 if rng.random() < 0.5 else 0
    elif use == "prompt":
        T, B = _log(rng, 256, 16384), rng.randint(1, 4)
    else:
        T, B, state = _log(rng, 64, 2048), _log(rng, 4, 64), rng.random() < 0.5
        len_min = max(1, T // 4) if rng.random() < 0.6 else 0
    return _attention("", dtype, T, B, H, Hkv, Dk, Dv, len_min, state, layout, packed)


def draw(rng):
    while True:
        c = _one(rng)
        w = work(dict(c, len_min=0))
        # half of the largest listed call: odd sizes run at a fraction of its rate
        if w["bytes"] <= 5e8 and w["flops"] <= (3.5e10 if c["dtype"] == "bf16" else 1e10):
            return c


class _State:
    """The inputs of one user, and with `own` the handle that the program keeps."""
    handle = None

    def __del__(self):
        if self.handle is not None:
            from paper_2307_11339_amd import rnn
            torch.cuda.synchronize()
            (rnn.rnn_linear_attention_destroy if self.c["op"] == "attention" else rnn.rnn_block_norm_destroy)(self.handle)


def _inputs(c, seed):
    """The tensors of a case, from its seed alone: [T, B, ...] views, whatever their layout."""
    s = _State()
    s.c = c
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    T, B = c["T"], c["B"]
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rows(widths):
        """One tensor of rows for each width, or one tensor for all when packed."""
        lead = (T, B) if c["layout"] == "time" else (B, T)
        parts = ([torch.randn(lead + (sum(widths),), device="cuda", generator=g).to(dt).split(widths, -1)] if c["packed"]
                 else [[torch.randn(lead + (w,), device="cuda", generator=g).to(dt) for w in widths]])[0]
        return [p if c["layout"] == "time" else p.transpose(0, 1) for p in parts]

    if c["op"] == "attention":
        H, Hkv, Dk, Dv = c["H"], c["Hkv"], c["Dk"], c["Dv"]
        q, k, v = rows([H * Dk, Hkv * Dk, Hkv * Dv])
        s.q, s.k, s.v = q.unflatten(-1, (H, Dk)), k.unflatten(-1, (Hkv, Dk)), v.unflatten(-1, (Hkv, Dv))
        # the first head forgets over some 16 steps, the last over a thousand
        s.decay = [1.0 - 2.0 ** -(4.0 + 6.0 * h / max(H - 1, 1)) for h in range(H)]
        s.scale = Dk ** -0.5
        s.s0 = torch.randn((B, H, Dk, Dv), device="cuda", generator=g) if c["state"] else None
    else:
        W = c["W"]
        s.x, s.gate = (rows([W, W]) if c["gate"] else rows([W]) + [None])
        s.residual = None
        if c["residual"]:
            lead = (T, B, W) if c["layout"] == "time" else (B, T, W)
            s.residual = torch.randn(lead, device="cuda", generator=g).to(dt)
            s.residual = s.residual if c["layout"] == "time" else s.residual.transpose(0, 1)

        def vector(mean):
            return (mean + 0.2 * torch.randn(W, device="cuda", generator=g)).to(dt)

        s.after_weight = vector(1.0) if c["after"] else None
        s.after_bias = vector(0.0) if c["after"] == "layer" else None
        s.scale = vector(0.5) if c["residual"] else None
        s.before_weight = vector(1.0) if c["before"] else None
        s.before_bias = vector(0.0) if c["before"] == "layer" else None
    s.lengths = None
    if c["len_min"]:
        s.lengths = torch.randint(c["len_min"], T + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
    return s


def prepare(case, seed):
    c, s = case, _inputs(case, seed)
    T, B = c["T"], c["B"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32

    def out(width):
        return (torch.empty((T, B, width), dtype=dt, device="cuda") if c["layout"] == "time"
                else torch.empty((B, T, width), dtype=dt, device="cuda").transpose(0, 1))

    if c["op"] == "attention":
        s.decay_t = torch.tensor(s.decay, dtype=torch.float32, device="cuda")
    if not own:
        return s
    from paper_2307_11339_amd import rnn
    dtype = rnn.RNN_BF16 if c["dtype"] == "bf16" else rnn.RNN_F32
    torch.cuda.synchronize()
    if c["op"] == "attention":
        s.handle = rnn.rnn_linear_attention_create(c["H"], c["Hkv"], c["Dk"], c["Dv"], dtype, s.decay, s.scale)
        s.o = out(c["H"] * c["Dv"]).unflatten(-1, (c["H"], c["Dv"]))
        s.sT = torch.empty((B, c["H"], c["Dk"], c["Dv"]), device="cuda") if c["state"] else None
        rc = rnn.rnn_linear_attention_reserve(s.handle, T, B)
        if rc != rnn.RNN_OK:
            raise rnn.RnnError(rc, "rnn_linear_attention_reserve")
    else:
        norms = {"": rnn.RNN_NORM_NONE, "rms": rnn.RNN_NORM_RMS, "layer": rnn.RNN_NORM_LAYER}
        gates = {"": rnn.RNN_GATE_NONE, "linear": rnn.RNN_GATE_LINEAR, "sigmoid": rnn.RNN_GATE_SIGMOID, "silu": rnn.RNN_GATE_SILU}
        s.handle = rnn.rnn_block_norm_create(c["W"], dtype, norms[c["after"]], c["groups"], s.after_weight, s.after_bias,
                                             gates[c["gate"]], s.scale, norms[c["before"]], s.before_weight, s.before_bias, EPS, 1)
        s.y = out(c["W"])
        s.residual_out = out(c["W"]) if c["residual"] else None
    return s


def run(s):
    if own:
        return _run_own(s)
    return _plain_attention(s) if s.c["op"] == "attention" else _plain_norm(s)


def _run_own(s):
    from paper_2307_11339_amd import rnn
    c = s.c
    if c["op"] == "attention":
        rc = rnn.rnn_linear_attention_forward(s.handle, s.q, s.k, s.v, s.lengths, s.s0, s.o, s.sT, c["T"], c["B"],
                                              torch.cuda.current_stream())
        if rc != rnn.RNN_OK:
            raise rnn.RnnError(rc, "rnn_linear_attention_forward")
        return [s.o] if s.sT is None else [s.o, s.sT]
    rc = rnn.rnn_block_norm_forward(s.handle, s.x, s.gate, s.residual, s.residual_out, s.y, s.lengths, c["T"], c["B"],
                                    torch.cuda.current_stream())
    if rc != rnn.RNN_OK:
        raise rnn.RnnError(rc, "rnn_block_norm_forward")
    return [s.y] if s.residual_out is None else [s.y, s.residual_out]


CHUNK = 128   # steps that the plain form takes at once


def _plain_attention(s):
    """Chunks of steps: the products inside a chunk under the decayed triangle, the rest through the state."""
    c = s.c
    T, B, H, Hkv, Dk, Dv = (c[n] for n in ("T", "B", "H", "Hkv", "Dk", "Dv"))
    C = min(CHUNK, T)
    dev = s.q.device
    rep = H // Hkv
    S = s.s0.clone() if s.s0 is not None else torch.zeros((B, H, Dk, Dv), device=dev)
    lengths = None if s.lengths is None else s.lengths.long()
    # powers of the decays in 64 bits: the exponent of a far pair would lose them in 32
    powers = (s.decay_t.double()[:, None] ** torch.arange(C + 1, device=dev, dtype=torch.float64)).float()   # [H, C + 1]
    i = torch.arange(C, device=dev)
    apart = i[:, None] - i[None, :]
    triangle = torch.where(apart >= 0, powers[:, apart.clamp(min=0)], torch.zeros((), device=dev))             # [H, C, C]
    o = torch.empty((T, B, H, Dv), dtype=s.q.dtype, device=dev)
    for t0 in range(0, T, C):
        n = min(C, T - t0)
        q = s.q[t0:t0 + n].float().permute(1, 2, 0, 3)      # [B, H, n, Dk]
        k = s.k[t0:t0 + n].float().permute(1, 2, 0, 3)
        v = s.v[t0:t0 + n].float().permute(1, 2, 0, 3)
        if rep > 1:
            k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
        if lengths is None:
            left, here = None, powers[None, :, n].expand(B, H)
            weight = powers[None, :, (n - 1 - i[:n])].expand(B, H, n)
        else:
            left = (lengths - t0).clamp(0, n)                                              # valid steps of each sequence
            valid = (i[None, :n] < left[:, None])[:, None, :, None]
            k, v = k * valid, v * valid
            here = powers[:, left].transpose(0, 1)                                         # [B, H]
            behind = (left[:, None] - 1 - i[None, :n]).clamp(min=0)
            weight = powers[:, behind].transpose(0, 1)                                     # [B, H, n]
        scores = torch.matmul(q, k.transpose(-1, -2).contiguous()) * triangle[None, :, :n, :n]
        out = torch.matmul(scores, v) + torch.matmul(q, S) * powers[None, :, 1:n + 1, None]
        out = out * s.scale
        if left is not None:
            out = torch.where(valid, out, torch.zeros((), device=dev))
        o[t0:t0 + n] = out.permute(2, 0, 1, 3).to(o.dtype)
        S = S * here[..., None, None] + torch.matmul((k * weight[..., None]).transpose(-1, -2).contiguous(), v)
    return [o] if s.s0 is None else [o, S]


def _normed(a, kind, groups, weight, bias):
    shape = a.shape
    a = a.unflatten(-1, (groups, shape[-1] // groups))
    if kind == "layer":
        a = a - a.mean(-1, keepdim=True)
    a = a * torch.rsqrt((a * a).mean(-1, keepdim=True) + EPS)
    a = a.reshape(shape) * weight.float()
    return a if bias is None else a + bias.float()


def _plain_norm(s):
    c = s.c
    a = s.x.float()
    if c["after"]:
        a = _normed(a, c["after"], c["groups"], s.after_weight, s.after_bias)
    if s.gate is not None:
        z = s.gate.float()
        if c["gate"] != "linear":
            p = 1.0 / (1.0 + torch.exp(-z))
            z = p if c["gate"] == "sigmoid" else z * p
        a = a * z
    if s.residual is not None:
        a = s.residual.float() + s.scale.float() * a
    y = _normed(a, c["before"], 1, s.before_weight, s.before_bias) if c["before"] else a
    if s.lengths is not None:
        t = torch.arange(c["T"], device=a.device)
        valid = (t[:, None] < s.lengths[None, :])[..., None]
        zero = torch.zeros((), device=a.device)
        y, a = torch.where(valid, y, zero), torch.where(valid, a, zero)
    y = y.to(s.x.dtype)
    return [y] if s.residual is None else [y, a.to(s.x.dtype)]


def exact(case, seed):
    """The definitions in 64 bits: the recurrence step by step; the norms row by row."""
    c, s = case, _inputs(case, seed)
    T, B = c["T"], c["B"]
    lengths = torch.full((B,), T, device="cuda") if s.lengths is None else s.lengths
    if c["op"] == "attention":
        H, Hkv, Dk, Dv = c["H"], c["Hkv"], c["Dk"], c["Dv"]
        # the decays as the operator is given them, in 32 bits
        lam = torch.tensor(s.decay, dtype=torch.float32, device="cuda").double().view(1, H, 1, 1)
        owner = torch.arange(H, device="cuda") // (H // Hkv)
        S = torch.zeros((B, H, Dk, Dv), dtype=torch.float64, device="cuda")
        if s.s0 is not None:
            S += s.s0
        o = torch.zeros((T, B, H, Dv), dtype=torch.float64, device="cuda")
        for t in range(T):
            k, v = s.k[t].double()[:, owner], s.v[t].double()[:, owner]
            new = lam * S
            new.addcmul_(k[..., :, None], v[..., None, :])
            got = torch.matmul(s.q[t].double()[:, :, None, :], new)[:, :, 0] * s.scale
            if s.lengths is None:
                S, o[t] = new, got
            else:
                live = (t < lengths).view(B, 1, 1)
                S = torch.where(live[..., None], new, S)
                o[t] = torch.where(live, got, torch.zeros_like(got))
        return [o] if s.s0 is None else [o, S]

    outs = [torch.zeros((T, B, c["W"]), dtype=torch.float64, device="cuda") for _ in range(2 if c["residual"] else 1)]

    def norm64(a, kind, weight, bias):
        mean = a.sum(-1, keepdim=True) / a.shape[-1] if kind == "layer" else 0.0
        var = ((a - mean) ** 2).sum(-1, keepdim=True) / a.shape[-1]
        a = (a - mean) / torch.sqrt(var + EPS) * weight.double()
        return a if bias is None else a + bias.double()

    for b0 in range(0, B, 16):          # some sequences at a time: 64-bit copies of the whole batch would be large
        b = slice(b0, min(B, b0 + 16))
        a = s.x[:, b].double()
        if c["after"]:
            size = c["W"] // c["groups"]
            a = torch.cat([norm64(a[..., j * size:(j + 1) * size], c["after"], s.after_weight[j * size:(j + 1) * size],
                                  None if s.after_bias is None else s.after_bias[j * size:(j + 1) * size])
                           for j in range(c["groups"])], -1)
        if c["gate"]:
            z = s.gate[:, b].double()
            a = a * {"linear": lambda: z, "sigmoid": lambda: 1 / (1 + torch.exp(-z)), "silu": lambda: z / (1 + torch.exp(-z))}[c["gate"]]()
        if c["residual"]:
            a = s.residual[:, b].double() + s.scale.double() * a
        y = norm64(a, c["before"], s.before_weight, s.before_bias) if c["before"] else a
        live = torch.arange(T, device="cuda")[:, None, None] < lengths[b].view(1, -1, 1)
        outs[0][:, b] = torch.where(live, y, torch.zeros_like(y))
        if c["residual"]:
            outs[1][:, b] = torch.where(live, a, torch.zeros_like(a))
    return outs


def work(case):
    """Every input that a sequence really has read once, every output written once; the update of the state and its
    read-out, 2 Dk Dv multiplications and additions each a step and head; some ten operations for each value of a norm."""
    c = case
    size = 2 if c["dtype"] == "bf16" else 4
    T, B = c["T"], c["B"]
    live = B * ((T + c["len_min"]) / 2 if c["len_min"] else T)     # half the padding of uniform lengths is nobody's work
    if c["op"] == "attention":
        H, Hkv, Dk, Dv = c["H"], c["Hkv"], c["Dk"], c["Dv"]
        return {"bytes": size * (live * (H * Dk + Hkv * (Dk + Dv)) + T * B * H * Dv) + (8 * B * H * Dk * Dv if c["state"] else 0),
                "flops": 4.0 * live * H * Dk * Dv}
    reads = 1 + bool(c["gate"]) + bool(c["residual"])
    writes = 1 + bool(c["residual"])
    return {"bytes": size * c["W"] * (live * reads + T * B * writes), "flops": 10.0 * live * c["W"]}
