"""Timing cases for the operators of the layers that lie between two coded maps.

A residual block on the pixel (token) vectors of a map: a norm whose output leaves as 8-bit floating-point codes with
a scale for each block of 128, products of such codes (a 1 x 1 convolution, a linear layer), and a norm of the
products' result that is gated, scaled and added to the residual; in training the gradients of all of it.  Tensors
are dense NCHW like the codec's: a list of tokens is (T, C, 1, 1), maps have H * W pixels.

`run` computes an operator in its plain form, from elementary torch operations in 32 bits, or (`own`) by the
library's call.  Activations have channels of unequal spread and a few large ones; maps are ReLU outputs.
"""
import math

import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0
SMALLEST = 2.0 ** -100
EPS = 1e-6
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # decoding: the codes of a single token's hidden state, latency
        dict(name="codes of one token", op="quantize", n=1, c=4096, hw=1, dtype="bf16", rows="pixels", square=False),
        # a training step's activations: by pixels for the forward product, by channels for the weights' gradient
        dict(name="codes both ways 8192x4096", op="quantize", n=8192, c=4096, hw=1, dtype="bf16", rows="both", square=False),
        # maps of the benchmark's layer between two coded layers
        dict(name="codes of maps 256x14x14", op="quantize", n=1024, c=256, hw=196, dtype="bf16", rows="pixels", square=False),
        # weights after an optimizer step: fp32 masters, 128 x 128 tiles, for the forward and the backward product
        dict(name="codes of weights 8192x4096", op="quantize", n=8192, c=4096, hw=1, dtype="f32", rows="both", square=True),
        # decoding: one token through a linear layer, bound by the weights' bytes
        dict(name="one token 4096 to 4096", op="matmul", n=1, hw=1, c=4096, o=4096, form="forward", dtype="bf16", bias=False, relu=False),
        # an expansion of an inverted-residual network: 7 x 7 maps, sizes off the tiles, bias and ReLU
        dict(name="1x1 conv 320 to 960 7x7", op="matmul", n=37, hw=49, c=320, o=960, form="forward", dtype="bf16", bias=True, relu=True),
        # a prompt (or a training batch) through a wide linear layer
        dict(name="prompt 8192x4096 to 8192", op="matmul", n=8192, hw=1, c=4096, o=8192, form="forward", dtype="bf16", bias=False, relu=False),
        # the same step's gradient of the weights, summed over the tokens
        dict(name="weight gradient 4096x4096", op="matmul", n=16384, hw=1, c=4096, o=4096, form="weights", dtype="f32", bias=False, relu=False),
        # decoding: between two blocks, latency
        dict(name="norms of one token", op="norms", n=1, c=4096, hw=1, dtype="bf16", gate="channel", out="codes"),
        # the same for a training batch
        dict(name="norms 16384x4096", op="norms", n=16384, c=4096, hw=1, dtype="bf16", gate="channel", out="codes"),
        # its gradient
        dict(name="norms backward 16384x4096", op="backward", n=16384, c=4096, hw=1, dtype="bf16", gate="channel"),
        # fp32 maps with a gate for each value, a small batch
        dict(name="norms backward 256x14x14", op="backward", n=37, c=256, hw=196, dtype="f32", gate="tensor"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case: 1 to 32768 tokens or maps of 7 x 7 to 56 x 56 pixels, 16 to 8192 channels, no more bytes than the
    largest listed case of the operator."""
    op = rng.choice(["quantize", "quantize", "matmul", "matmul", "matmul", "norms", "norms", "backward", "backward"])
    most = max((work(c) for c in listed() if c["op"] == op), key=lambda w: w["bytes"] + w["flops"] / 400)
    while True:
        maps = rng.random() < 0.35
        hw = rng.choice([7, 8, 14, 19, 28, 56]) ** 2 if maps else 1
        n = _log_int(rng, 1, 512 if maps else 32768)
        c = _log_int(rng, 16, 1024 if maps else 8192)
        if rng.random() < 0.6:
            c = max(16, c // 16 * 16)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        case = dict(op=op, n=n, c=c, hw=hw, dtype=dtype)
        if op == "quantize":
            case.update(rows=rng.choice(["pixels", "pixels", "channels", "both"]), square=rng.random() < 0.25)
        elif op == "matmul":
            o = _log_int(rng, 16, 1024 if maps else 8192)
            form = rng.choice(["forward", "forward", "forward", "input", "weights"])
            case.update(o=max(16, o // 16 * 16) if rng.random() < 0.6 else o, form=form,
                        bias=form == "forward" and rng.random() < 0.5, relu=form == "forward" and rng.random() < 0.5)
        elif op == "norms":
            case.update(gate=rng.choice(["none", "channel", "tensor"]), out=rng.choice(["codes", "tensor"]))
        else:
            case.update(gate=rng.choice(["none", "channel", "tensor"]))
        w = work(case)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return case


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    p = case["n"] * case["hw"]
    c = case["c"]
    blocks = lambda n: -(-n // BLOCK)                                            # noqa: E731
    if case["op"] == "quantize":
        scales = {"pixels": blocks(c) * (blocks(p) if case["square"] else p), "channels": blocks(p) * (blocks(c) if case["square"] else c)}
        kinds = ["pixels", "channels"] if case["rows"] == "both" else [case["rows"]]
        return {"bytes": p * c * e + sum(p * c + 4 * scales[k] for k in kinds), "flops": 3 * p * c}
    if case["op"] == "matmul":
        o = case["o"]
        m, n, k = {"forward": (p, o, c), "input": (p, c, o), "weights": (o, c, p)}[case["form"]]
        scales = blocks(k) * (m + (n if case["form"] == "weights" else blocks(n)))
        return {"bytes": m * k + n * k + 4 * scales + m * n * e, "flops": 2 * m * n * k}
    if case["op"] == "norms":
        moved = 2 * e + e + (e if case["gate"] == "tensor" else 0) + (e if case["out"] == "tensor" else 1 + 4 / BLOCK)
        return {"bytes": p * c * moved, "flops": 10 * p * c}
    return {"bytes": p * c * e * (6 + (2 if case["gate"] == "tensor" else 0)), "flops": 25 * p * c}


# ---- inputs --------------------------------------------------------------------------------

def _rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(g, n, c, hw, dtype, relu=False):
    """(n, c, h, w): channels of unequal spread, one in a hundred ten times as large; ReLU outputs for maps."""
    spread = torch.exp(0.7 * torch.randn(c, generator=g, device="cuda"))
    spread = torch.where(torch.rand(c, generator=g, device="cuda") < 0.01, spread * 10, spread)
    side = math.isqrt(hw)
    x = torch.randn(n, c, side, side, generator=g, device="cuda") * spread[None, :, None, None]
    return (x.relu_() if relu else x).to(dtype)


def _rows(x, kind):
    """The tensor as a matrix: a row for each pixel, or for each channel."""
    n, c, h, w = x.shape
    return x.permute(0, 2, 3, 1).reshape(-1, c) if kind == "pixels" else x.permute(1, 0, 2, 3).reshape(c, -1)


def _codes(m, square):
    """Codes [R][C] and scales [C / 128][R], or [C / 128][R / 128] of 128 x 128 tiles, of a matrix in 32 bits."""
    r, c = m.shape
    pad_c = -c % BLOCK
    pad_r = -r % BLOCK if square else 0
    v = torch.nn.functional.pad(m, (0, pad_c, 0, pad_r)).reshape((r + pad_r) // (BLOCK if square else 1), BLOCK if square else 1, -1, BLOCK)
    amax = v.abs().amax(dim=(1, 3)).clamp_min(SMALLEST)
    scale = amax * (1.0 / E4M3_MAX)
    q = (v * scale.reciprocal()[:, None, :, None]).reshape(r + pad_r, c + pad_c)[:r, :c]
    return q.to(torch.float8_e4m3fn), scale.t().contiguous()


def _padded(codes, scale, square):
    """As the library keeps them: rows of a multiple of 16 codes, scales of a multiple of 128 rows."""
    r, c = codes.shape
    wide = torch.zeros(r, -(-c // 16) * 16, dtype=torch.uint8, device="cuda")
    wide[:, :c] = codes.view(torch.uint8)
    if not square:
        scale = torch.nn.functional.pad(scale, (0, -r % BLOCK))
    return wide.view(torch.float8_e4m3fn), scale.contiguous()


def prepare(case, seed):
    g = _rng(seed)
    dtype = DTYPES[case["dtype"]]
    n, c, hw = case["n"], case["c"], case["hw"]
    st = dict(case=case)
    if case["op"] == "quantize":
        x = _activations(g, n, c, hw, torch.float32, relu=hw > 1)
        st["x"] = (x * 0.02 if case["square"] else x).to(dtype)
    elif case["op"] == "matmul":
        o, form = case["o"], case["form"]
        side = math.isqrt(hw)
        st["shape"] = (n, side, side)
        if form == "weights":
            a, b = (_codes(_rows(_activations(g, n, k, hw, torch.float32, relu=r), "channels"), False) for k, r in ((o, False), (c, hw > 1)))
            st["shape"] = (o, 1, 1)
        else:
            k, m = (c, o) if form == "forward" else (o, c)
            a = _codes(_rows(_activations(g, n, k, hw, torch.float32, relu=hw > 1 and form == "forward"), "pixels"), False)
            b = _codes(torch.randn(m, k, generator=g, device="cuda") / math.sqrt(k), True)
        st["a"], st["b"] = _padded(*a, False), _padded(*b, form != "weights")
        st["bias"] = torch.randn(o, generator=g, device="cuda") if case["bias"] else None
    else:
        st["h"] = _activations(g, n, c, hw, dtype)
        st["y"] = _activations(g, n, c, hw, dtype)
        vector = lambda at: at + 0.2 * torch.randn(c, generator=g, device="cuda")  # noqa: E731
        st["after"], st["before"] = vector(1.0), vector(1.0)
        st["gate"] = {"none": lambda: None, "channel": lambda: vector(0.3),
                      "tensor": lambda: torch.sigmoid(_activations(g, n, c, hw, torch.float32)).to(dtype)}[case["gate"]]()
        st["scale"] = torch.rand(1, generator=g, device="cuda") + 0.2
        if case["op"] == "backward":
            st["dx"], st["ds"] = ((torch.randn(st["h"].shape, generator=g, device="cuda") * 1e-2).to(dtype) for _ in range(2))
    return st


# ---- the library's calls -------------------------------------------------------------------

_contexts = {}


def _context():
    import paper_1905_10830_b200 as tc
    device = torch.cuda.current_device()
    if device not in _contexts:
        _contexts[device] = tc.tc_create(device)
    return tc, _contexts[device]


def _values(b):
    """Codes and scales of a block matrix without the padding of its rows."""
    return [b.codes[:, :b.cols], b.scales if b.square else b.scales[:, :b.rows]]


def _run_own(st):
    tc, ctx = _context()
    case = st["case"]
    if case["op"] == "quantize":
        got = tc.tc_quantize_blocks(ctx, st["x"], rows=case["rows"], square=case["square"])
        return [v for b in (got if case["rows"] == "both" else [got]) for v in _values(b)]
    if case["op"] == "matmul":
        k = {"forward": case["c"], "input": case["o"], "weights": case["n"] * case["hw"]}[case["form"]]
        a = tc.Blocks(*st["a"], cols=k, square=False)
        b = tc.Blocks(*st["b"], cols=k, square=case["form"] != "weights")
        return tc.tc_matmul_blocks(ctx, a, b, shape=st["shape"], dtype=DTYPES[case["dtype"]], bias=st["bias"], relu=case["relu"])
    vectors = dict(after=st["after"], gate=st["gate"], scale=st["scale"], before=st["before"], eps=EPS)
    if case["op"] == "norms":
        s, x = tc.tc_residual_norms(ctx, st["h"], st["y"], blocks=case["out"] == "codes", **vectors)
        return [s] + (_values(x) if case["out"] == "codes" else [x])
    return tc.tc_residual_norms_backward(ctx, st["h"], st["y"], st["dx"], st["ds"], **vectors)._asdict()


# ---- plain forms ---------------------------------------------------------------------------

def _run_plain(st):
    case = st["case"]
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "quantize":
        x = st["x"].float()
        kinds = ["pixels", "channels"] if case["rows"] == "both" else [case["rows"]]
        return [v for kind in kinds for v in _codes(_rows(x, kind), case["square"])]
    if case["op"] == "matmul":
        k = {"forward": case["c"], "input": case["o"], "weights": case["n"] * case["hw"]}[case["form"]]
        tiles = case["form"] != "weights"
        spread = lambda s, rows, tall: (s.repeat_interleave(BLOCK, 1) if tall else s)[:, :rows].t().repeat_interleave(BLOCK, 1)[:, :k]  # noqa: E731
        (a, sa), (b, sb) = st["a"], st["b"]
        va = a[:, :k].float() * spread(sa, a.shape[0], False)
        vb = b[:, :k].float() * spread(sb, b.shape[0], tiles)
        out = va @ vb.t()
        if st["bias"] is not None:
            out = out + st["bias"]
        if case["relu"]:
            out = out.relu()
        n, h, w = st["shape"]
        return out.to(dtype).reshape(n, h, w, -1).permute(0, 3, 1, 2).contiguous()
    h, y = st["h"].float(), st["y"].float()
    after, before, scale = st["after"][None, :, None, None], st["before"][None, :, None, None], st["scale"]
    gate = 1.0 if st["gate"] is None else st["gate"][None, :, None, None] if case["gate"] == "channel" else st["gate"].float()
    norm = lambda v: torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)          # noqa: E731
    n = y * norm(y)
    if case["op"] == "norms":
        s = h + scale * gate * (n * after)
        x = s * norm(s) * before
        return [s.to(dtype)] + (list(_codes(_rows(x, "pixels"), False)) if case["out"] == "codes" else [x.to(dtype)])
    dx, r = st["dx"].float(), norm(h)
    t = dx * before
    d = st["ds"].float() + r * t - h * (r ** 3 * (t * h).mean(1, keepdim=True))
    v = scale * d * gate * after
    dy = norm(y) * (v - n * (v * n).mean(1, keepdim=True))
    dgate = scale * d * n * after
    return dict(h=d.to(dtype), y=dy.to(dtype), after=(scale * d * gate * n).sum((0, 2, 3)),
                gate={"none": lambda: None, "channel": lambda: dgate.sum((0, 2, 3)), "tensor": lambda: dgate.to(dtype)}[case["gate"]](),
                scale=(d * gate * n * after).sum().reshape(1), before=(dx * h * r).sum((0, 2, 3)))


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definitions in 64 bits ------------------------------------------------------------

def _exact_codes(m, square):
    """Block by block: the largest magnitude over 448 is the scale, a code the nearest e4m3 value of x / scale."""
    r, c = m.shape
    values, scales = torch.empty(r, c, dtype=torch.float8_e4m3fn, device=m.device), []
    for c0 in range(0, c, BLOCK):
        part = m[:, c0:c0 + BLOCK]
        a = part.abs().max(1).values
        if square:
            a = torch.stack([t.max() for t in a.split(BLOCK)])
        s = torch.clamp(a, min=SMALLEST) / E4M3_MAX
        values[:, c0:c0 + BLOCK] = (part / (s.repeat_interleave(BLOCK)[:r] if square else s)[:, None]).to(torch.float8_e4m3fn)
        scales.append(s)
    return [values, torch.stack(scales)]


def _channels_last(t):
    return t.double().flatten(2).transpose(1, 2).reshape(-1, t.shape[1])


def exact(case, seed):
    st = prepare(case, seed)
    n, hw, c = case["n"], case["hw"], case["c"]
    side = math.isqrt(hw)
    maps = lambda m: m.reshape(n, hw, -1).transpose(1, 2).reshape(n, -1, side, side)  # noqa: E731
    if case["op"] == "quantize":
        x = _channels_last(st["x"])
        got = []
        if case["rows"] != "channels":
            got += _exact_codes(x, case["square"])
        if case["rows"] != "pixels":
            got += _exact_codes(x.t(), case["square"])
        return got
    if case["op"] == "matmul":
        (a, sa), (b, sb) = st["a"], st["b"]
        k = {"forward": c, "input": case["o"], "weights": n * hw}[case["form"]]
        out = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
        for i, k0 in enumerate(range(0, k, BLOCK)):
            k1 = min(k, k0 + BLOCK)
            rows = sa[i].double()[:a.shape[0]]
            cols = sb[i].double()
            cols = (cols if case["form"] == "weights" else cols.repeat_interleave(BLOCK))[:b.shape[0]]
            out += rows[:, None] * (a[:, k0:k1].double() @ b[:, k0:k1].double().t()) * cols[None, :]
        if case["bias"]:
            out += st["bias"].double()
        if case["relu"]:
            out.clamp_(min=0)
        return out[:, :, None, None] if case["form"] == "weights" else maps(out)
    s, y = _channels_last(st["h"]), _channels_last(st["y"])
    after, before, scale = st["after"].double(), st["before"].double(), st["scale"].double()
    gate = _channels_last(st["gate"]) if case["gate"] == "tensor" else st["gate"].double() if case["gate"] == "channel" else torch.ones(c, dtype=torch.float64, device="cuda")
    q = 1.0 / torch.sqrt((y ** 2).sum(1, keepdim=True) / c + EPS)
    if case["op"] == "norms":
        s = s + scale * (gate * (y * q * after))
        x = s / torch.sqrt((s ** 2).sum(1, keepdim=True) / c + EPS) * before
        return [maps(s)] + (_exact_codes(x, False) if case["out"] == "codes" else [maps(x)])
    dx, ds = _channels_last(st["dx"]), _channels_last(st["ds"])
    r = 1.0 / torch.sqrt((s ** 2).sum(1, keepdim=True) / c + EPS)
    # x_c = s_c r b_c, dr/ds_c = -r^3 s_c / C
    d = ds + r * before * dx - (r ** 3 / c) * s * (before * dx * s).sum(1, keepdim=True)
    u = y * q * after
    grads = dict(h=maps(d), scale=(d * gate * u).sum().reshape(1), before=(dx * s * r).sum(0))
    grads["gate"] = {"none": lambda: None, "channel": lambda: (scale * d * u).sum(0), "tensor": lambda: maps(scale * d * u)}[case["gate"]]()
    du = scale * d * gate
    grads["after"] = (du * y * q).sum(0)
    dn = du * after
    grads["y"] = maps(q * dn - (q ** 3 / c) * y * (dn * y).sum(1, keepdim=True))
    return grads
