"""The operators of a training step as far as a machine without a GPU goes: the 64-bit forms against differences and
refusals of bad arguments before any device call."""
import pytest
import torch

import training_forms as forms


@pytest.fixture(scope="module")
def leet():
    from paper_2501_02573_amd import binding
    return binding


def by_differences(f, x, at, step=1e-6):
    """Derivative of the scalar f along each coordinate in ``at`` of x."""
    out = []
    for i in at:
        d = torch.zeros_like(x).view(-1)
        d[i] = step
        d = d.view_as(x)
        out.append((f(x + d) - f(x - d)) / (2 * step))
    return torch.stack(out)


@pytest.mark.parametrize("gamma", [0.0, 0.7, 1.0])
def test_attention_backward_form_against_differences(gamma):
    g = torch.Generator().manual_seed(0)
    B, H, N, r, w = 1, 2, 7, 3, 4
    def normal(*shape):
        return torch.randn(shape, generator=g, dtype=torch.float64)
    q, k, v, do = normal(B, H, N, r), normal(B, H, N, r), normal(B, H, N, w), normal(B, H, N, w)
    s, ds = normal(B, H, r, w), normal(B, H, r, w)
    gam = torch.tensor([gamma, 0.9], dtype=torch.float64)

    def loss(q, k, v, s):
        out, left = forms.attention(q, k, v, gam, s)
        return (out * do).sum() + (left * ds).sum()

    got = [x for x, _ in forms.attention_backward(do, q, k, v, gam, s, ds)]
    leaves = [t.clone().requires_grad_() for t in (q, k, v, s)]
    for a, b in zip(got, torch.autograd.grad(loss(*leaves), leaves)):
        assert torch.allclose(a, b, rtol=1e-12, atol=1e-12)
    for n, x in enumerate((q, k, v, s)):
        at = range(0, x.numel(), 3)
        args = [q, k, v, s]
        def f(y):
            return loss(*args[:n], y, *args[n + 1:])
        assert torch.allclose(by_differences(f, x, at), got[n].reshape(-1)[::3], rtol=1e-7, atol=1e-7)


# ---- refusals at the C boundary: nothing here reaches a device ----

P = 0x1000000   # aligned, never touched


def backward(leet, **change):
    step = 1 << 26
    a = dict(dout=P, q=P + step, k=P + 2 * step, v=P + 3 * step, gamma=P + 4 * step, dq=P + 5 * step, dk=P + 6 * step,
             dv=P + 7 * step, s=P + 8 * step, ds=P + 9 * step, left=P + 10 * step, ws=P + 11 * step, wsb=1 << 25, segments=2, B=2,
             H=4, N=300, r=128, w=128, dtype=1, mask=0)
    a.update(change)
    return leet.lib.leet_attn_backward(*(a[n] for n in ("dout", "q", "k", "v", "gamma", "dq", "dk", "dv", "s", "ds", "left", "ws",
                                                       "wsb", "segments", "B", "H", "N", "r", "w", "dtype", "mask")), None)


def test_backward_arguments_that_are_fine_reach_the_device(leet):
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")
    assert backward(leet) in (leet.LEET_ERR_LAUNCH, leet.LEET_ERR_UNSUPPORTED)
    assert backward(leet, s=None, ds=None, left=None) in (leet.LEET_ERR_LAUNCH, leet.LEET_ERR_UNSUPPORTED)
    assert backward(leet, gamma=None, mask=1) in (leet.LEET_ERR_LAUNCH, leet.LEET_ERR_UNSUPPORTED)
    assert backward(leet, segments=1, ws=None, wsb=0) in (leet.LEET_ERR_LAUNCH, leet.LEET_ERR_UNSUPPORTED)


@pytest.mark.parametrize("bad", [dict(**{n: None}) for n in ("dout", "q", "k", "v", "gamma", "dq", "dk", "dv")]
                         + [dict(**{n: P + 40 * (1 << 26) + 8}) for n in ("dout", "q", "k", "v", "dq", "dk", "dv", "s", "ds", "left", "ws")]
                         + [dict(gamma=P + 2), dict(mask=2), dict(mask=-1), dict(segments=-1), dict(B=0), dict(H=-1), dict(N=-1),
                            dict(ws=None), dict(wsb=1000), dict(ws=P + 11 * (1 << 26) + 16)])
def test_backward_invalid(leet, bad):
    assert backward(leet, **bad) == leet.LEET_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(r=32, w=32), dict(r=64, w=128), dict(r=128, w=64),
                                 dict(r=128, w=256, dtype=0), dict(r=256, w=128)])
def test_backward_unsupported(leet, bad):
    assert backward(leet, **bad) == leet.LEET_ERR_UNSUPPORTED


def test_backward_too_large(leet):
    assert backward(leet, B=1 << 20, H=1 << 10) == leet.LEET_ERR_TOO_LARGE
    assert backward(leet, N=(1 << 30) + 1) == leet.LEET_ERR_TOO_LARGE


def test_backward_outputs_over_other_arguments(leet):
    step = 1 << 26
    places = dict(dout=0, q=1, k=2, v=3, gamma=4, dq=5, dk=6, dv=7, s=8, ds=9, left=10, ws=11)
    for out in ("dq", "dk", "dv", "left", "ws"):
        for other in places:
            if other != out:
                assert backward(leet, **{out: P + places[other] * step}) == leet.LEET_ERR_INVALID_ARG, (out, other)


def test_backward_workspace(leet):
    assert leet.backward_workspace_bytes(2, 3, 300, 128, 256, leet.LEET_BF16, 2) == 2 * 6 * 128 * 256 * 4
    assert leet.backward_workspace_bytes(2, 3, 300, 128, 128, leet.LEET_BF16, 1) == 0
    assert leet.backward_workspace_bytes(2, 3, 0, 128, 128, leet.LEET_BF16, 3) == 0
    assert leet.backward_workspace_bytes(2, 3, 300, 96, 96, leet.LEET_BF16, 3) == 0


def test_backward_binding_refuses(leet):
    q = torch.zeros(1, 2, 5, 64)
    with pytest.raises(ValueError):   # not on a GPU
        leet.leet_attn_backward(q, q, q, q, torch.ones(2))
    with pytest.raises(TypeError):
        leet.leet_attn_backward(q.bfloat16(), q, q, q, torch.ones(2))
    with pytest.raises(ValueError):
        leet.leet_attn_backward(q[:, :, :4], q, q, q, torch.ones(2))
    with pytest.raises(ValueError):
        leet.leet_attn_backward(q, q, q, q, torch.ones(3))
    with pytest.raises(ValueError):
        leet.leet_attn_backward(q, q, q, q, torch.ones(2), state_in=torch.zeros(1, 2, 64, 32))
    with pytest.raises(TypeError):
        leet.leet_attn_backward(q, q, q, q, torch.ones(2), dk=q.half())
