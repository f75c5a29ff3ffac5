"""The group norm, its gradient and their tolerances in 64 bits, for tensors (N, C, H, W)."""
import torch

U = 2.0 ** -24                                    # half a step of fp32
# Additions that follow one another in a sum of a group: 128 of a thread's, 8 of its channels, 128 of a lane's and 5 of a warp's, the parts of a
# map (up to 8, or 32 lanes' shares of them and 5), some roundings of means.
DEPTH = 300


def grouped(x, groups):
    n, c, h, w = x.shape
    return x.double().reshape(n, groups, c // groups, h, w)


def per_channel(v, groups):
    return v.double().reshape(1, groups, -1, 1, 1)


def stats(x, groups, eps):
    v = grouped(x, groups)
    mean = v.mean((2, 3, 4))
    var = ((v - mean[:, :, None, None, None]) ** 2).mean((2, 3, 4))
    return mean, 1 / torch.sqrt(var + eps)


def act(z, kind):
    return {None: lambda: z, "relu": lambda: z.clamp(min=0), "silu": lambda: z / (1 + torch.exp(-z))}[kind]()


def slope(z, kind):
    if kind is None:
        return torch.ones_like(z)
    if kind == "relu":
        return (z > 0).double()
    s = torch.sigmoid(z)
    return s + z * s * (1 - s)


def forward(x, groups, weight, bias, eps, kind, mean=None, rstd=None):
    """(y, z) grouped."""
    if mean is None:
        mean, rstd = stats(x, groups, eps)
    n = (grouped(x, groups) - mean[:, :, None, None, None]) * rstd[:, :, None, None, None]
    z = n * per_channel(weight, groups) + per_channel(bias, groups)
    return act(z, kind), z


def stats_tolerance(x, groups, eps):
    """Bounds of the errors of mean, and of rstd relative to it."""
    v = grouped(x, groups)
    mean, rstd = stats(x, groups, eps)
    off = DEPTH * U * v.abs().mean((2, 3, 4)) + 4 * U * mean.abs()
    sigma = 1 / rstd
    # squares about a mean that is `off` away, joined about another; half of what the variance is off
    rel = 0.5 * (2 * DEPTH * U + 6 * off / sigma + (off / sigma) ** 2) + 8 * U
    return off, rel


def sigmoid_error(z):
    """Relative error of 1 / (1 + e^-z): the exponential (2 + 1.2 |z| steps of 2^-23), an addition, a quotient of two steps."""
    return (6 + 1.2 * z.abs()) * 2.0 ** -23


def forward_tolerance(x, groups, weight, bias, eps, kind):
    """Bound of y's error before it is rounded."""
    mean, rstd = stats(x, groups, eps)
    off, rel = (t[:, :, None, None, None] for t in stats_tolerance(x, groups, eps))
    y, z = forward(x, groups, weight, bias, eps, kind)
    w, b = per_channel(weight, groups).abs(), per_channel(bias, groups).abs()
    n = ((grouped(x, groups) - mean[:, :, None, None, None]) * rstd[:, :, None, None, None]).abs()
    tol = w * (off * rstd[:, :, None, None, None] * (1 + rel) + n * (rel + 4 * U)) + (n * w + b) * 2 * U
    if kind == "silu":
        tol = 1.1 * tol + y.abs() * sigmoid_error(z) + 2.0 ** -120
    return tol


def backward(x, dy, groups, mean, rstd, weight, bias, kind):
    """(dx, dweight, dbias) from the statistics given, dx grouped."""
    m, r = (t.double()[:, :, None, None, None] for t in (mean, rstd))
    n = (grouped(x, groups) - m) * r
    w = per_channel(weight, groups)
    dz = grouped(dy, groups) * slope(n * w + per_channel(bias, groups), kind)
    u = dz * w
    dx = r * (u - u.mean((2, 3, 4), keepdim=True) - n * (u * n).mean((2, 3, 4), keepdim=True))
    return dx, (dz * n).sum((0, 3, 4)).flatten(), dz.sum((0, 3, 4)).flatten()


def backward_tolerance(x, dy, groups, mean, rstd, weight, bias, kind):
    """Bounds of the errors of backward's results, dx before it is rounded."""
    m, r = (t.double()[:, :, None, None, None] for t in (mean, rstd))
    n = ((grouped(x, groups) - m) * r)
    w, b = per_channel(weight, groups), per_channel(bias, groups)
    z = n * w + b
    d = grouped(dy, groups).abs()
    dz = d * slope(z, kind).abs()
    off_z = 4 * U * ((n * w).abs() + b.abs())
    if kind == "silu":                            # the derivative's slope is at most 1/2; s + z s (1 - s) of terms each a few roundings
        s = torch.sigmoid(z)
        off = d * (0.5 * off_z + (s + 2 * (z * s).abs()) * (sigmoid_error(z) + 4 * U)) + dz * U
    elif kind == "relu":                          # on the other side of 0 where z is that near it
        off = d * (z.abs() <= off_z).double()
    else:
        off = torch.zeros_like(d)
    n = n.abs()
    w = w.abs()
    off_n = 2 * U * n
    u, off_u = dz * w, off * w + dz * w * U
    depth = DEPTH * U
    mean_of = lambda t: t.mean((2, 3, 4), keepdim=True)                         # noqa: E731
    off_1 = mean_of(off_u) + depth * mean_of(u)
    off_2 = mean_of(off_u * n + u * off_n) + depth * mean_of(u * n)
    dx = r * (off_u + off_1 + n * off_2 + off_n * mean_of(u * n) + 8 * U * (u + mean_of(u) + n * mean_of(u * n)))
    total = lambda t: t.sum((0, 3, 4)).flatten()                                # noqa: E731
    return dx, total(off * n + dz * off_n) + (depth + 4 * U) * total(dz * n), total(off) + (depth + 4 * U) * total(dz)
