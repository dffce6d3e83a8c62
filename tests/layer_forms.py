"""The operators beside the attention in 64 bits, with the error that their arithmetic in 32 bits may have.

Every form returns (values, bounds), both float64: ``bounds`` is how far an fp32 computation of the value may be off
before it is rounded to its type.  u = 2^-24 is half a step of fp32, relative to the value; what is counted:

* an angle: reduced in fp64, then fp32, off by less than u / 2; sine and cosine 4 u (2 steps), scale u, products and
  sum 2 u: 8 u times scale (|x1| + |x2|) for a rotated pair;
* a norm: sum of squares over a row (at most 20 additions one after the other) 20 u, halved by the root, root, quotient
  and products 4 u: 16 u times the value;
* a decay: exp 2 u (1 step), a quotient 2 u; a product of decays u a factor; a fused multiply-add u: 8 u a token of the
  recurrence taken with absolute values.  Below 2^-126 a step is no longer relative but 2^-149: 1 - a of a logit of 90 is
  exp(-90) = 8e-40, and exp and the product with the quotient may each be off by a step there, which what it is then
  multiplied by multiplies; and so may that product, which the next factor multiplies.
"""
import torch

U = 2.0 ** -24
TINY = 2 * 2.0 ** -149


def half_step(ref, dtype):
    """Half a step of ``dtype`` at values ``ref``: subnormal steps included."""
    info = torch.finfo(dtype)
    return (info.eps / 2) * ref.abs() + info.smallest_normal * info.eps / 2


def close(got, form, dtype=None):
    """Whether ``got`` is within the bound and the rounding of its type; non-finite values have to be the same."""
    ref, bound = form
    dtype = dtype or got.dtype
    got = got.detach().double().cpu()
    fine = torch.isfinite(ref)
    same = torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(got[torch.isinf(ref)], ref[torch.isinf(ref)])
    # 1.01: the value that is rounded is itself off by the bound
    off = (got[fine] - ref[fine]).abs() - (1.01 * bound + 1.01 * half_step(ref, dtype))[fine]
    return same and got.shape == ref.shape and bool((off <= 0).all())


def rotate(x, freq, positions, layout, scale=1.0, transposed=False):
    """x [B, H, N, d] in float64, positions [B, N]."""
    rot = 2 * freq.numel()
    theta = positions.double()[:, None, :, None] * freq.double()
    c, s = theta.cos() * scale, theta.sin() * scale * (-1.0 if transposed else 1.0)
    y, bound = x.clone(), torch.zeros_like(x)
    one, two = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == 0 else (slice(0, rot, 2), slice(1, rot, 2))
    x1, x2 = x[..., one], x[..., two]
    y[..., one], y[..., two] = x1 * c - x2 * s, x2 * c + x1 * s
    bound[..., one] = bound[..., two] = 8 * U * scale * (x1.abs() + x2.abs())
    return y, bound


def spread(x, freq, layout, scale):
    """scale (|x1| + |x2|) for the pairs of x, |x| for the rest: what an error of x may become by the rotation."""
    rot, y = 2 * freq.numel(), x.abs().clone()
    one, two = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == 0 else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., one] = y[..., two] = scale * (x[..., one].abs() + x[..., two].abs())
    return y


def norm_rope(x, w, freq, positions, layout, scale=1.0, eps=1e-6):
    u = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w
    y, bound = rotate(u, freq, positions, layout, scale)
    return y, bound + 16 * U * spread(u, freq, layout, scale)


def norm_rope_backward(dy, x, w, freq, positions, layout, scale=1.0, eps=1e-6):
    """((dx, bound), (dw, bound)).  dw: at most 64 additions one after the other at the sizes that are tested."""
    r = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    n = x * r
    du, _ = rotate(dy, freq, positions, layout, scale, transposed=True)
    wide = spread(dy, freq, layout, scale)
    mean = (w * du * n).mean(-1, keepdim=True)
    dx = r * (w * du - n * mean)
    bound = 40 * U * r * (w.abs() * wide + n.abs() * (w.abs() * wide * n.abs()).mean(-1, keepdim=True))
    return (dx, bound), ((du * n).sum((0, 1, 2)), 96 * U * (wide * n.abs()).sum((0, 1, 2)))


def gates(z, x, mode):
    """a, b and 1 - a (of use with mode 2)."""
    if mode == 0:
        return z, x, torch.ones_like(z)
    if mode == 1:
        return z.exp(), x, torch.ones_like(z)
    return torch.sigmoid(z), torch.sigmoid(-z) * x, torch.sigmoid(-z)


def scan(z, x, mode, state=None):
    """One sequence per batch entry: ((h, bound), (state after it, bound)); z, x [B, N, C] in float64."""
    B, N, C = x.shape
    a, b, _ = gates(z, x, mode)
    h = torch.zeros(B, C, dtype=torch.float64) if state is None else state.double()
    wide, off = h.abs(), torch.zeros_like(h)
    out, bound = torch.zeros_like(x), torch.zeros_like(x)
    for t in range(N):
        h = a[:, t] * h + b[:, t]
        wide = a[:, t].abs() * wide + b[:, t].abs()
        off = a[:, t].abs() * off + 8 * U * wide
        out[:, t], bound[:, t] = h, off
    return (out, bound), (h, off)


def scan_backward(dh, z, x, h, mode, state=None, dstate=None):
    """((dx, bound), (dgate, bound), (dstate_in, bound)); h as the forward call left it."""
    B, N, C = h.shape
    a, _, rest = gates(z, h, mode)
    g = torch.zeros(B, C, dtype=torch.float64) if dstate is None else dstate.double()
    first = torch.zeros(B, C, dtype=torch.float64) if state is None else state.double()
    wide, off = g.abs(), torch.zeros_like(g)
    dx, dgate = torch.zeros_like(h), torch.zeros_like(h)
    bx, bg = torch.zeros_like(h), torch.zeros_like(h)
    for t in range(N - 1, -1, -1):
        before = h[:, t - 1] if t else first
        D, Dw, Do = dh[:, t] + g, dh[:, t].abs() + wide, off + U * (dh[:, t].abs() + wide)
        g, wide = a[:, t] * D, a[:, t].abs() * Dw
        off = a[:, t].abs() * Do + 8 * U * wide
        dx[:, t], bx[:, t] = rest[:, t] * D, rest[:, t] * (Do + 8 * U * Dw) + TINY * Dw
        if mode == 0:
            dgate[:, t], bg[:, t] = D * before, (Do + 2 * U * Dw) * before.abs()
        elif mode == 1:
            dgate[:, t], bg[:, t] = g * before, (off + 2 * U * wide) * before.abs()
        else:
            apart, both = before - x[:, t], before.abs() + x[:, t].abs()
            dgate[:, t] = g * rest[:, t] * apart
            bg[:, t] = rest[:, t] * (off * apart.abs() + 8 * U * wide * both) + TINY * (1 + wide) * both
    return (dx, bx), (dgate, bg), (g, off)
