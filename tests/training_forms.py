"""The operators of a training step in 64 bits, with the error that their arithmetic may have (see layer_forms.py, whose
``close`` compares): every form returns (values, bounds), both float64.

Attention's gradients: u = 2^-24, and v half a step of a 16-bit input type.  An output is a sum of products over tokens of
scores and of what the state gives; with all factors taken absolutely (W) its error is at most

* in 16 bits 3 v W: a score is rounded once as an operand, the state twice (its summands, itself);
* D u W for a score of D products, 64 u W for the sum over a chunk, for the state 64 u W for a chunk's own sum and, for each
  chunk that it is carried on, 20 u W (16 additions of a chunk's four-token products, decays, the decay's own rounding):
  (D + 140 + 20 chunks) u W; also of dstate_in, whose summands are formed to 2^-24 whatever the type.

Where operands of fp16 fall under its normal range a rounding is 2^-25 instead: every operand of a product may be off by that.

Norms of rows, u as above: a row's sum of squares, or of products, of up to 50 additions one after the other (sixteen
elements of a thread, six steps of a wave, sixteen waves) 50 u, halved by the root; the sum x + residual u; quotient, root and
products 5 u: 36 u times the value.  Its gradient: the norm's 36 u on each factor r and n (three of them in the second term), 50 u
of the mean, 8 u of products: 160 u of the terms taken absolutely, u of the sum with what comes along.  The weight's gradient: 36 u
of n, at most 64 additions one after the other at the sizes that are tested: 110 u of its summands taken absolutely.
"""
import torch

U = 2.0 ** -24


def powers(gamma, n):
    """gamma^n, 0^0 = 1; gamma [H] float64, n whole numbers of any shape."""
    return gamma.view((-1,) + (1,) * n.dim()) ** n.double()


def attention(q, k, v, gamma, state=None):
    """(out, state after the last token) of [B, H, N, .] tensors in float64."""
    N = q.shape[2]
    i = torch.arange(N)
    M = powers(gamma, (i[:, None] - i[None, :]).clamp(min=0)) * (i[:, None] >= i[None, :])
    out = (q @ k.transpose(-1, -2) * M) @ v
    left = (powers(gamma, N - 1 - i)[..., None] * k).transpose(-1, -2) @ v
    if state is not None:
        out = out + powers(gamma, i + 1)[..., None] * (q @ state)
        left = left + powers(gamma, torch.tensor(N)).view(-1, 1, 1) * state
    return out, left


def _gradients(dout, q, k, v, gamma, state, dstate):
    B, H, N, r = q.shape
    i = torch.arange(N)
    M = powers(gamma, (i[:, None] - i[None, :]).clamp(min=0)) * (i[:, None] >= i[None, :])
    P, dP = q @ k.transpose(-1, -2) * M, dout @ v.transpose(-1, -2) * M
    dq, dk, dv = dP @ k, dP.transpose(-1, -2) @ q, P.transpose(-1, -2) @ dout
    late, behind = powers(gamma, i + 1)[..., None], powers(gamma, N - 1 - i)[..., None]
    left = (late * q).transpose(-1, -2) @ dout
    if state is not None:
        dq = dq + late * (dout @ state.transpose(-1, -2))
    if dstate is not None:
        dk = dk + behind * (v @ dstate.transpose(-1, -2))
        dv = dv + behind * (k @ dstate)
        left = left + powers(gamma, torch.tensor(N)).view(-1, 1, 1) * dstate
    return dq, dk, dv, left


def attention_backward(dout, q, k, v, gamma, state=None, dstate=None, dtype=torch.float32):
    """((dq, bound), (dk, bound), (dv, bound), (dstate_in, bound)) of float64 tensors; ``dtype``: the type they came in."""
    def wide(t):
        return None if t is None else t.abs()
    got = _gradients(dout, q, k, v, gamma, state, dstate)
    most = _gradients(wide(dout), wide(q), wide(k), wide(v), gamma, wide(state), wide(dstate))
    fine = (max(q.shape[3], v.shape[3]) + 140 + 20 * (q.shape[2] // 64 + 1)) * U
    rough = 0.0 if dtype == torch.float32 else 3 * torch.finfo(dtype).eps / 2
    bounds = [(rough + fine) * m for m in most[:3]] + [fine * most[3]]
    if dtype == torch.float16:
        # a score (off by 2^-25) meets a row of the third operand; the state, its summands off by 2^-25 a token, the first's
        small = 2.0 ** -25
        def row(t):
            return t.abs().sum(2, keepdim=True)
        def each(t):
            return t.abs().sum(3, keepdim=True)
        bounds[0] = bounds[0] + small * (row(k) + each(dout) * (1 + row(v).amax(-1, keepdim=True)))
        bounds[1] = bounds[1] + small * (row(q) + each(v) * (1 + row(dout).amax(-1, keepdim=True)))
        bounds[2] = bounds[2] + small * (row(dout) + each(k) * (1 + row(q).amax(-1, keepdim=True)))
        bounds[3] = bounds[3] + small * row(q).transpose(-1, -2)
    return tuple(zip(got, bounds))


def add_norm(x, residual, w, eps):
    """((y, bound), (s, bound)) of float64 tensors."""
    s = x if residual is None else x + residual
    y = s / (s.square().mean(-1, keepdim=True) + eps).sqrt() * w
    return (y, 36 * U * y.abs()), (s, U * s.abs())


def add_norm_backward(dy, h, w, eps, along=None):
    """((gradient of the sum, bound), (gradient of the weight, bound))."""
    r = 1 / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    n, u = h * r, dy * w
    g = r * (u - n * (u * n).mean(-1, keepdim=True))
    bound = 160 * U * r * (u.abs() + n.abs() * (u * n).abs().mean(-1, keepdim=True))
    if along is not None:
        g = g + along
        bound = bound + U * g.abs()
    rows = tuple(range(dy.dim() - 1))
    return (g, bound), ((dy * n).sum(rows), 110 * U * (dy * n).abs().sum(rows))


def eight_bits(y, scale, bound):
    """How far a value of 8 bits times its scale may be off y: half a step (2^-4 of the value, the smallest step 2^-9), and y's
    and the scale's own errors."""
    return 1.01 * torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * scale) + 2 * bound + 8 * U * y.abs()
