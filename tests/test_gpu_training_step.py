"""The operators of a training step together, as a layer of linear attention runs them: norm of the residual sum, a
projection, norms and rotation of heads, the decayed attention, a loss; all of it back to the gradients, which are clipped."""
import pytest
import torch

import training_forms as forms

pytestmark = pytest.mark.gpu

B, H, N, D, EPS = 2, 3, 150, 64, 1e-6
C = H * D


def draw(dtype):
    g = torch.Generator().manual_seed(5)
    x, res, target = (torch.randn((B, N, C), generator=g) for _ in range(3))
    proj = torch.randn((C, 3 * C), generator=g) * C ** -0.5
    w, wq, wk = 1 + 0.2 * torch.randn(C, generator=g), 1 + 0.2 * torch.randn(D, generator=g), 1 + 0.2 * torch.randn(D, generator=g)
    gamma = (1 - 2.0 ** -torch.linspace(3.0, 7.0, H)).float()
    return [t.to(dtype) for t in (x, res, target, proj, w, wq / 8, wk / 8)] + [gamma]


def step64(x, res, target, proj, w, wq, wk, gamma, freq):
    """Gradients of half the squared distance of attention and residual stream from their targets."""
    leaves = [t.double().requires_grad_() for t in (x, res, proj, w, wq, wk)]
    x, res, proj, w, wq, wk = leaves
    (y, _), (s, _) = forms.add_norm(x, res, w, EPS)
    at = (y @ proj).view(B, N, 3 * H, D).transpose(1, 2)
    q, k, v = at[:, :H], at[:, H:2 * H], at[:, 2 * H:]
    theta = torch.arange(N).double()[:, None] * freq

    def turned(t, weight):
        t = t / (t.square().mean(-1, keepdim=True) + EPS).sqrt() * weight
        a, b = t.chunk(2, -1)
        return torch.cat((a * theta.cos() - b * theta.sin(), b * theta.cos() + a * theta.sin()), -1)

    o, _ = forms.attention(turned(q, wq), turned(k, wk), v, gamma.double())
    out = o.transpose(1, 2).reshape(B, N, C)
    loss = 0.5 * (out - target.double()).square().sum() + 0.5 * (s - target.double()).square().sum()
    return torch.autograd.grad(loss, leaves)


def step(leet, x, res, target, proj, w, wq, wk, gamma, freq, limit=None):
    """The same by the library's calls."""
    y, s = leet.leet_attn_add_rms_norm(x, res, w, eps=EPS)
    at = (y.view(B * N, C) @ proj).view(B, N, 3 * H, D).transpose(1, 2)
    q, k = leet.leet_attn_qk_norm_rope(at[:, :H], at[:, H:2 * H], wq, wk, freq, eps=EPS)
    v = at[:, 2 * H:].contiguous()
    o = leet.leet_attn_forward_v2(q, k, v, gamma, out_dtype=q.dtype)
    do = o - target.view(B, N, H, D).transpose(1, 2)
    dat = torch.empty((B, N, 3 * C), dtype=x.dtype, device="cuda")
    to = dat.view(B, N, 3 * H, D).transpose(1, 2)
    dq, dk, dv = leet.leet_attn_backward(do.contiguous(), q, k, v, gamma)
    _, _, dwq, dwk = leet.leet_attn_qk_norm_rope_backward(dq, dk, at[:, :H], at[:, H:2 * H], wq, wk, freq, eps=EPS, dx_q=to[:, :H],
                                                          dx_k=to[:, H:2 * H])
    to[:, 2 * H:].copy_(dv)
    dy = (dat.view(B * N, 3 * C) @ proj.t()).view(B, N, C)
    dproj = y.view(B * N, C).t() @ dat.view(B * N, 3 * C)
    dx, _, dw = leet.leet_attn_add_rms_norm_backward(dy, s, w, eps=EPS, dresidual=s - target)
    grads = [dx, dx, dproj, dw, dwq, dwk]
    if limit is None:
        return grads
    return [dx.clone()], leet.leet_attn_clip_gradients(grads[2:], limit), grads[2:]


# fp32: some two hundred roundings of 2^-24 on the way to each value, of numbers up to a hundred times the gradient's typical
# one; 16 bits: some ten of half a step, independent of one another
@pytest.mark.parametrize("dtype,most", [(torch.float32, 200 ** 0.5 * 100 * 2.0 ** -24), (torch.bfloat16, 10 ** 0.5 * 2.0 ** -8)])
def test_gradients_of_a_layer(dtype, most):
    from paper_2501_02573_amd import binding as leet
    t = draw(dtype)
    freq = leet.rope_frequencies(D)[0]
    want = step64(*t, freq)
    got = step(leet, *(a.cuda() for a in t), freq.cuda())
    for a, b in zip(got, want):
        assert float((a.double().cpu() - b).norm() / b.norm()) < most


def test_captured_beside_an_eager_one():
    from paper_2501_02573_amd import binding as leet
    t = [a.cuda() for a in draw(torch.bfloat16)]
    freq = leet.rope_frequencies(D)[0].cuda()

    def call():
        a, norm, grads = step(leet, *t, freq, limit=1.0)
        return a + [norm] + grads

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = call()
    for i in range(4):
        t[0].mul_(-0.5 if i % 2 else -2.0)
        eager = call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, kept))
        assert float(kept[1]) > 1.0


def test_eight_bit_rows_before_a_product():
    """For serving: the norm's 8-bit rows, times their scales, in the place of 16-bit ones."""
    from paper_2501_02573_amd import binding as leet
    t = [a.cuda() for a in draw(torch.bfloat16)]
    x, res, proj, w = t[0], t[1], t[3], t[4]
    y, s = leet.leet_attn_add_rms_norm(x, res, w, eps=EPS)
    y8, scales, s8 = leet.leet_attn_add_rms_norm_q8(x, res, w, eps=EPS, group=64)
    assert torch.equal(s, s8)
    back = (y8.float().unflatten(-1, (-1, 64)) * scales[..., None]).flatten(-2)
    a, b = back.view(-1, C) @ proj.float(), y.float().view(-1, C) @ proj.float()
    # values of three bits of mantissa are off by at most 2^-4, 2^-4 / sqrt(3) in the mean, independently
    assert float((a - b).norm() / b.norm()) < 2.0 ** -4
