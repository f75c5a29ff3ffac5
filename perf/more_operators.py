"""Timing cases for more operators of the layers that lie between two coded maps, and of their training.

A layer on 8-bit integers: codes of a tensor with one scale for each row (a pixel or token, or a channel), products of such
codes (a 1 x 1 convolution, a linear layer, and both gradients), the group norm with its activation that stands before it,
on maps whose channels are neighbours in memory, with its gradient, and the clipping of all gradients by their common norm.

`run` computes an operator in its plain form, from elementary torch operations in 32 bits (64 for quotients next to a
rounding's border and the sum over all gradients), or (`own`) by the library's call.
"""
import math
import random

import torch

own = False

SMALLEST = 2.0 ** -100
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # decoding: the codes of a single token's hidden state, latency
        dict(name="codes of one token", op="quantize", n=1, c=4096, hw=1, dtype="bf16", rows="pixels"),
        # a training step's activations: by pixels for the forward product, by channels for the weights' gradient
        dict(name="codes both ways 8192x4096", op="quantize", n=8192, c=4096, hw=1, dtype="bf16", rows="both"),
        # decoding: one token through a linear layer, bound by the weights' bytes
        dict(name="one token 4096 to 4096", op="matmul", n=1, hw=1, c=4096, o=4096, form="forward", dtype="bf16", bias=False, relu=False),
        # an expansion of an inverted-residual network: 7 x 7 maps, sizes off the tiles, bias and ReLU
        dict(name="1x1 conv 320 to 960 7x7", op="matmul", n=37, hw=49, c=320, o=960, form="forward", dtype="bf16", bias=True, relu=True),
        # a prompt (or a training batch) through a wide linear layer
        dict(name="prompt 8192x4096 to 8192", op="matmul", n=8192, hw=1, c=4096, o=8192, form="forward", dtype="bf16", bias=False, relu=False),
        # the same step's gradient of the weights, summed over the tokens
        dict(name="weight gradient 4096x4096", op="matmul", n=16384, hw=1, c=4096, o=4096, form="weights", dtype="f32", bias=False, relu=False),
        # one map of the benchmark's layer, latency
        dict(name="group norm of one map", op="norm", n=1, c=256, hw=196, groups=32, dtype="bf16", act="silu"),
        # a training batch of large maps
        dict(name="group norm 256x56x56", op="norm", n=128, c=256, hw=3136, groups=32, dtype="bf16", act="relu"),
        # a small batch in fp32
        dict(name="norm backward 256x14x14", op="backward", n=37, c=256, hw=196, groups=32, dtype="f32", act="silu"),
        # a training batch of large maps
        dict(name="norm backward 128x56x56", op="backward", n=128, c=128, hw=3136, groups=32, dtype="bf16", act="silu"),
        # a residual network's gradients: 62 tensors of 64 to some million values, packed one behind the other
        dict(name="clip 62 tensors", op="clip", tensors=62, values=11_700_000, dtype="f32", packed=True, over=True),
        # a large model's: 290 tensors, of both types
        dict(name="clip 290 tensors", op="clip", tensors=290, values=700_000_000, dtype="mixed", packed=False, over=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case: 1 to 32768 tokens or maps of 7 x 7 to 128 x 128 pixels, 16 to 8192 channels, 1 to 600 gradients of together up to
    700 million values; no more bytes and operations than the largest listed case of the operator."""
    op = rng.choice(["quantize", "matmul", "matmul", "norm", "norm", "backward", "backward", "clip"])
    most = max((work(c) for c in listed() if c["op"] == op), key=lambda w: w["bytes"] + w["flops"] / 400)
    while True:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op == "clip":
            case = dict(op=op, tensors=_log_int(rng, 1, 600), values=_log_int(rng, 1000, 700_000_000), dtype=rng.choice(["f32", "bf16", "mixed"]),
                        packed=rng.random() < 0.5, over=rng.random() < 0.7)
        elif op in ("norm", "backward"):
            hw = rng.choice([7, 8, 14, 19, 28, 56, 64, 128]) ** 2
            case = dict(op=op, n=_log_int(rng, 1, 512), hw=hw, dtype=dtype)
            groups = rng.choice([1, 4, 8, 16, 32, 32, 32])
            c = groups * _log_int(rng, max(1, 16 // groups), 1024 // groups)
            case.update(c=c, groups=c if rng.random() < 0.1 else groups, act=rng.choice(["none", "relu", "silu"] if op == "norm" else ["none", "silu"]))
        else:
            maps = rng.random() < 0.35
            case = dict(op=op, n=_log_int(rng, 1, 512 if maps else 32768), hw=rng.choice([7, 8, 14, 19, 28, 56]) ** 2 if maps else 1, dtype=dtype)
            size = lambda: (lambda v, even: max(16, v // 16 * 16) if even else v)(_log_int(rng, 16, 1024 if maps else 8192), rng.random() < 0.6)  # noqa: E731
            case["c"] = size()
            if op == "quantize":
                case.update(rows=rng.choice(["pixels", "pixels", "channels", "both"]))
            else:
                form = rng.choice(["forward", "forward", "forward", "input", "weights"])
                case.update(o=size(), form=form, bias=form == "forward" and rng.random() < 0.5, relu=form == "forward" and rng.random() < 0.5)
        w = work(case)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return case


def work(case):
    if case["op"] == "clip":
        return {"bytes": sum(n * (4 if t == "f32" else 2) for n, t in _sizes(case)) * 2, "flops": 3 * case["values"]}
    e = 4 if case["dtype"] == "f32" else 2
    p = case["n"] * case["hw"]
    c = case["c"]
    if case["op"] == "quantize":
        scales = {"pixels": p, "channels": c, "both": p + c}[case["rows"]]
        return {"bytes": p * c * (e + (2 if case["rows"] == "both" else 1)) + 4 * scales, "flops": 3 * p * c}
    if case["op"] == "matmul":
        o = case["o"]
        m, n, k = {"forward": (p, o, c), "input": (p, c, o), "weights": (o, c, p)}[case["form"]]
        return {"bytes": m * k + n * k + 4 * (m + n) + m * n * e, "flops": 2 * m * n * k}
    if case["op"] == "norm":
        return {"bytes": 2 * p * c * e + 8 * case["n"] * case["groups"], "flops": 10 * p * c}
    return {"bytes": 3 * p * c * e + 8 * case["n"] * case["groups"], "flops": 25 * p * c}


# ---- inputs --------------------------------------------------------------------------------

def _rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _spread(g, c):
    """Channels of unequal spread, one in a hundred ten times as large."""
    spread = torch.exp(0.7 * torch.randn(c, generator=g, device="cuda"))
    return torch.where(torch.rand(c, generator=g, device="cuda") < 0.01, spread * 10, spread)


def _activations(g, n, c, hw, relu=False):
    """(n, c, h, w); ReLU outputs for maps."""
    side = math.isqrt(hw)
    x = torch.randn(n, c, side, side, generator=g, device="cuda") * _spread(g, c)[None, :, None, None]
    return x.relu_() if relu else x


def _channels_last(g, case, scale=None):
    """(n, c, h, w) whose channels are neighbours in memory: a convolution's output, with means off zero."""
    side = math.isqrt(case["hw"])
    x = torch.randn(case["n"], side, side, case["c"], generator=g, device="cuda")
    if scale is None:
        x = x.mul_(_spread(g, case["c"])).add_(0.5 * torch.randn(case["c"], generator=g, device="cuda"))
    else:
        x = x.mul_(scale)
    return x.to(DTYPES[case["dtype"]]).permute(0, 3, 1, 2)


def _sizes(case):
    """The tensors' numbers of values, some vectors, most of the values in few large ones, and their types."""
    rng = random.Random(case["tensors"])
    share = [math.exp(rng.uniform(0.0, 9.0)) for _ in range(case["tensors"])]
    sizes = [max(1, int(case["values"] * s / sum(share))) for s in share]
    return [(n, ("bf16" if i % 3 else "f32") if case["dtype"] == "mixed" else case["dtype"]) for i, n in enumerate(sizes)]


def _views(case, fill):
    """(buffers by type, the gradients as views of them), one behind the other or each at a multiple of 512 bytes; between them zeros."""
    at, places = {"f32": 0, "bf16": 0}, []
    for n, t in _sizes(case):
        places.append((t, at[t], n))
        at[t] += n if case["packed"] else (n + 255) // 256 * 256
    flat = {t: torch.zeros(n, dtype=DTYPES[t], device="cuda") for t, n in at.items() if n}
    views = [flat[t][i:i + n] for t, i, n in places]
    for v in views:
        fill(v)
    return flat, views


def _rows(x, kind):
    """The tensor as a matrix: a row for each pixel, or for each channel."""
    n, c, h, w = x.shape
    return x.permute(0, 2, 3, 1).reshape(-1, c) if kind == "pixels" else x.permute(1, 0, 2, 3).reshape(c, -1)


def _codes(m):
    """Codes [R][C] and scales [R] of a matrix: scale = max|x| / 127 rounded to 32 bits, code = the integer nearest to x / scale."""
    m = m.float()
    scale = (m.abs().amax(1).clamp_min(SMALLEST).double() / 127.0).float()     # (a quotient of 32 bits by a constant is a product)
    return (m.double() / scale.double()[:, None]).round().to(torch.int8), scale


def _padded(codes, scale):
    """As the library keeps them: rows of a multiple of 16 codes."""
    r, c = codes.shape
    wide = torch.zeros(r, -(-c // 16) * 16, dtype=torch.int8, device="cuda")
    wide[:, :c] = codes
    return wide, scale


def prepare(case, seed):
    g = _rng(seed)
    st = dict(case=case)
    if case["op"] == "clip":
        st["flat"], st["grads"] = _views(case, lambda v: v.normal_(generator=g).mul_(1e-2))
        st["flat_out"], st["out"] = _views(case, lambda v: None)
        norm = 1e-2 * math.sqrt(case["values"])
        st["max_norm"] = 0.3 * norm if case["over"] else 10 * norm + 1
        return st
    dtype = DTYPES[case["dtype"]]
    n, c, hw = case["n"], case["c"], case["hw"]
    if case["op"] == "quantize":
        st["x"] = _activations(g, n, c, hw, relu=hw > 1).to(dtype)
    elif case["op"] == "matmul":
        o, form = case["o"], case["form"]
        side = math.isqrt(hw)
        st["shape"] = (n, side, side)
        if form == "weights":
            a, b = (_codes(_rows(_activations(g, n, k, hw, relu=r), "channels")) for k, r in ((o, False), (c, hw > 1)))
            st["shape"] = (o, 1, 1)
        else:
            k, m = (c, o) if form == "forward" else (o, c)
            a = _codes(_rows(_activations(g, n, k, hw, relu=hw > 1 and form == "forward"), "pixels"))
            b = _codes(torch.randn(m, k, generator=g, device="cuda") / math.sqrt(k))
        st["a"], st["b"] = _padded(*a), _padded(*b)
        st["bias"] = torch.randn(o, generator=g, device="cuda") if case["bias"] else None
    else:
        st["x"] = _channels_last(g, case)
        st["weight"], st["bias"] = (at + 0.2 * torch.randn(c, generator=g, device="cuda") for at in (1.0, 0.0))
        if case["op"] == "backward":
            st["dy"] = _channels_last(g, case, 1e-2)
            mean, rstd, _ = _moments(st["x"], case["groups"])
            st["stats"] = torch.stack([mean.flatten(1), rstd.flatten(1)], 2)
    return st


# ---- the library's calls -------------------------------------------------------------------

_contexts = {}


def _context():
    import paper_1905_10830_b200 as tc
    device = torch.cuda.current_device()
    if device not in _contexts:
        _contexts[device] = tc.tc_create(device)
    return tc, _contexts[device]


def _run_own(st):
    tc, ctx = _context()
    case = st["case"]
    if case["op"] == "quantize":
        got = tc.tc_quantize_rows(ctx, st["x"], rows=case["rows"])
        return [v for r in (got if case["rows"] == "both" else [got]) for v in (r.codes[:, :r.cols], r.scales)]
    if case["op"] == "matmul":
        k = {"forward": case["c"], "input": case["o"], "weights": case["n"] * case["hw"]}[case["form"]]
        a, b = (tc.Rows(*st[name], cols=k) for name in ("a", "b"))
        return tc.tc_matmul_rows(ctx, a, b, shape=st["shape"], dtype=DTYPES[case["dtype"]], bias=st["bias"], relu=case["relu"])
    act = None if case.get("act") == "none" else case.get("act")
    if case["op"] == "norm":
        return list(tc.tc_group_norm(ctx, st["x"], case["groups"], weight=st["weight"], bias=st["bias"], eps=EPS, activation=act))
    if case["op"] == "backward":
        return tc.tc_group_norm_backward(ctx, st["x"], st["dy"], st["stats"], weight=st["weight"], bias=st["bias"], activation=act)._asdict()
    norm = tc.tc_clip_gradients(ctx, st["grads"], st["max_norm"], out=st["out"])
    return dict(norm=norm, **st["flat_out"])


# ---- plain forms ---------------------------------------------------------------------------

def _grouped(x, groups):
    """(n, groups, channels of a group, h, w) in 32 bits."""
    n, c, h, w = x.shape
    return x.float().reshape(n, groups, c // groups, h, w)


def _moments(x, groups):
    """Mean and 1 / deviation of each map's groups, and the values as they are grouped."""
    v = _grouped(x, groups)
    mean = v.mean((2, 3, 4), keepdim=True)
    return mean, torch.rsqrt((v - mean).square().mean((2, 3, 4), keepdim=True) + EPS), v


def _run_plain(st):
    case = st["case"]
    if case["op"] == "quantize":
        kinds = ["pixels", "channels"] if case["rows"] == "both" else [case["rows"]]
        return [v for kind in kinds for v in _codes(_rows(st["x"], kind))]
    if case["op"] == "matmul":
        k = {"forward": case["c"], "input": case["o"], "weights": case["n"] * case["hw"]}[case["form"]]
        (a, sa), (b, sb) = st["a"], st["b"]
        out = (a[:, :k].float() @ b[:, :k].float().t()) * sa[:, None] * sb
        if st["bias"] is not None:
            out = out + st["bias"]
        if case["relu"]:
            out = out.relu()
        n, h, w = st["shape"]
        return out.to(DTYPES[case["dtype"]]).reshape(n, h, w, -1).permute(0, 3, 1, 2).contiguous()
    if case["op"] == "clip":
        norm = torch.stack([g.float().square().sum() for g in st["grads"]]).double().sum().sqrt().float()
        factor = (st["max_norm"] / norm).clamp(max=1.0)
        for g, o in zip(st["grads"], st["out"]):
            o.copy_(g.float() * factor)
        return dict(norm=norm.reshape(1), **st["flat_out"])
    shape, groups = st["x"].shape, case["groups"]
    dtype = DTYPES[case["dtype"]]
    weight, bias = (st[name].reshape(1, groups, -1, 1, 1) for name in ("weight", "bias"))
    last = lambda v: v.reshape(shape).to(dtype).contiguous(memory_format=torch.channels_last)  # noqa: E731
    if case["op"] == "norm":
        mean, rstd, v = _moments(st["x"], groups)
        y = (v - mean) * rstd * weight + bias
        y = y.relu() if case["act"] == "relu" else y * torch.sigmoid(y) if case["act"] == "silu" else y
        return [last(y), torch.stack([mean.flatten(1), rstd.flatten(1)], 2)]
    mean, rstd = (st["stats"][:, :, i].reshape(shape[0], groups, 1, 1, 1) for i in (0, 1))
    n = (_grouped(st["x"], groups) - mean) * rstd
    d = _grouped(st["dy"], groups)
    if case["act"] == "silu":
        z = n * weight + bias
        s = torch.sigmoid(z)
        d = d * (s * (1.0 + z * (1.0 - s)))
    dn = d * weight
    dx = rstd * (dn - dn.mean((2, 3, 4), keepdim=True) - n * (dn * n).mean((2, 3, 4), keepdim=True))
    return dict(x=last(dx), weight=(d * n).sum((0, 3, 4)).flatten(), bias=d.sum((0, 3, 4)).flatten())


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definitions in 64 bits ------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "clip":
        total = sum(float((g.double() ** 2).sum()) for g in st["grads"])
        factor = min(1.0, st["max_norm"] / math.sqrt(total))
        return dict(norm=torch.tensor([math.sqrt(total)], dtype=torch.float64), **{t: f.double() * factor for t, f in st["flat"].items()})
    n, hw, c = case["n"], case["hw"], case["c"]
    side = math.isqrt(hw)
    if case["op"] == "quantize":
        by_pixel = st["x"].double().flatten(2).transpose(1, 2).reshape(-1, c)
        got = []
        for kind, m in (("pixels", by_pixel), ("channels", by_pixel.t())):
            if case["rows"] in (kind, "both"):
                a = torch.clamp(m.abs().max(1).values, min=SMALLEST)
                held = (a / 127).float().double()                          # what the codes are counted in is the scale as it is kept
                got += [torch.round(m / held[:, None]).to(torch.int8), a / 127]
        return got
    if case["op"] == "matmul":
        (a, sa), (b, sb) = st["a"], st["b"]
        out = (a.double() * sa.double()[:, None]) @ (b.double() * sb.double()[:, None]).t()
        if case["bias"]:
            out += st["bias"].double()
        if case["relu"]:
            out.clamp_(min=0)
        maps, _, _ = st["shape"]
        return out[:, :, None, None] if case["form"] == "weights" else out.reshape(maps, hw, -1).transpose(1, 2).reshape(maps, -1, side, side)
    groups = case["groups"]
    x = st["x"].double().permute(0, 2, 3, 1).reshape(n, hw, groups, c // groups)
    weight, bias = (st[name].double().reshape(groups, -1) for name in ("weight", "bias"))
    mean = x.mean((1, 3))
    var = ((x - mean[:, None, :, None]) ** 2).mean((1, 3))
    deviation = torch.sqrt(var + EPS)
    q = (x - mean[:, None, :, None]) / deviation[:, None, :, None]
    maps = lambda v: v.reshape(n, side, side, c).permute(0, 3, 1, 2)            # noqa: E731
    z = q * weight + bias
    if case["op"] == "norm":
        y = {"none": lambda: z, "relu": lambda: z.clamp(min=0), "silu": lambda: z / (1 + torch.exp(-z))}[case["act"]]()
        return [maps(y), torch.stack([mean, 1 / deviation], 2)]
    d = st["dy"].double().permute(0, 2, 3, 1).reshape(n, hw, groups, c // groups)
    if case["act"] == "silu":
        s = 1 / (1 + torch.exp(-z))
        d = d * (s + z * s * (1 - s))
    # with u = dL/dq and m values a group: dL/dx = (u - sum u / m - q sum(u q) / m) / deviation
    u, m = d * weight, hw * (c // groups)
    dx = (u - u.sum((1, 3), keepdim=True) / m - q * ((u * q).sum((1, 3), keepdim=True) / m)) / deviation[:, None, :, None]
    return dict(x=maps(dx), weight=(d * q).sum((0, 1)).flatten(), bias=d.sum((0, 1)).flatten())
