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
    assert backward(leet, B=1 << 10, H=1 << 9, segments=2, wsb=1 << 62) == leet.LEET_ERR_TOO_LARGE   # the scan's threads


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


# ---- norms ----

@pytest.mark.parametrize("along", [False, True])
def test_add_norm_backward_form_against_differences(along):
    g = torch.Generator().manual_seed(0)
    def normal(*shape):
        return torch.randn(shape, generator=g, dtype=torch.float64)
    h, w, dy, a = normal(2, 3, 5), normal(5), normal(2, 3, 5), normal(2, 3, 5) if along else None

    def loss(h, w):
        (y, _), (s, _) = forms.add_norm(h, None, w, 1e-3)
        return (y * dy).sum() + ((s * a).sum() if along else 0)

    (dh, _), (dw, _) = forms.add_norm_backward(dy, h, w, 1e-3, a)
    assert torch.allclose(by_differences(lambda t: loss(t, w), h, range(30)), dh.reshape(-1), rtol=1e-7, atol=1e-7)
    assert torch.allclose(by_differences(lambda t: loss(h, t), w, range(5)), dw, rtol=1e-7, atol=1e-7)


STEP = 1 << 26


def rows(leet, at, batch=1 << 16, token=4096):
    return leet._pack_rows(P + at * STEP, batch, token)


def norm(leet, which, **change):
    a = dict(x=rows(leet, 0), res=rows(leet, 1), out=rows(leet, 2), sum=rows(leet, 3), grad=rows(leet, 4), w=P + 5 * STEP, dw=P + 6 * STEP,
             scales=P + 7 * STEP, ws=P + 8 * STEP, wsb=1 << 25, group=128, wd=1, eps=1e-6, B=2, N=16, C=4096, dtype=1, rd=1)
    a.update(change)
    lib = leet.lib
    if which == "forward":
        return lib.leet_attn_add_rms_norm(a["x"], a["res"], a["out"], a["sum"], a["w"], a["wd"], a["eps"], a["B"], a["N"], a["C"],
                                          a["dtype"], a["rd"], None)
    if which == "q8":
        return lib.leet_attn_add_rms_norm_q8(a["x"], a["res"], a["out"], a["scales"], a["group"], a["sum"], a["w"], a["wd"], a["eps"],
                                             a["B"], a["N"], a["C"], a["dtype"], a["rd"], None)
    return lib.leet_attn_add_rms_norm_backward(a["x"], a["res"], a["grad"], a["out"], a["sum"] if a["rd"] != a["dtype"] else None,
                                               a["w"], a["dw"], a["wd"], a["eps"], a["ws"], a["wsb"], a["B"], a["N"], a["C"],
                                               a["dtype"], a["rd"], None)


WHICH = ("forward", "q8", "backward")


@pytest.mark.parametrize("which", WHICH)
def test_norm_arguments_that_are_fine_reach_the_device(leet, which):
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")
    there = (leet.LEET_ERR_LAUNCH, leet.LEET_ERR_UNSUPPORTED)
    assert norm(leet, which) in there and norm(leet, which, w=None, dw=None, ws=None, wsb=0) in there
    assert norm(leet, which, rd=0, res=rows(leet, 1), sum=rows(leet, 3)) in there
    assert norm(leet, which, out=rows(leet, 0) if which != "q8" else rows(leet, 2)) in there
    assert norm(leet, which, out=rows(leet, 1) if which != "q8" else rows(leet, 2), grad=None) in there
    if which != "backward":
        assert norm(leet, which, res=None, sum=None) in there and norm(leet, which, sum=rows(leet, 1)) in there
        assert norm(leet, which, sum=rows(leet, 0)) in there and norm(leet, which, sum=None) in there
    else:
        assert norm(leet, which, dw=P + 5 * STEP) in there   # in the weight's place


@pytest.mark.parametrize("which", WHICH)
@pytest.mark.parametrize("bad", [dict(x=None), dict(out=None), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(B=0),
                                 dict(N=-1), dict(C=0), dict(w=P + 1), dict(B=2, out=None)])
def test_norm_invalid(leet, which, bad):
    assert norm(leet, which, **bad) == leet.LEET_ERR_INVALID_ARG


def test_norm_invalid_of_one_call(leet):
    def at(off, batch=1 << 16, token=4096):
        return leet._pack_rows(P + off, batch, token)
    bad = leet.LEET_ERR_INVALID_ARG
    for which in ("forward", "backward"):
        assert norm(leet, which, x=at(1)) == bad and norm(leet, which, out=at(2 * STEP + 1)) == bad
        assert norm(leet, which, out=at(2 * STEP, 4096, 4096)) == bad      # rows over one another
        assert norm(leet, which, out=at(2 * STEP, 1 << 16, 4095)) == bad
    assert norm(leet, "forward", res=None) == bad                          # a sum without a residual
    assert norm(leet, "backward", res=None) == bad
    assert norm(leet, "q8", scales=None) == bad and norm(leet, "q8", scales=P + 2) == bad and norm(leet, "q8", C=4100, group=64) == bad
    assert norm(leet, "backward", ws=None) == bad and norm(leet, "backward", wsb=100) == bad and norm(leet, "backward", ws=P + 8 * STEP + 16) == bad
    assert norm(leet, "backward", dw=P + 1) == bad


@pytest.mark.parametrize("which", WHICH)
def test_norm_unsupported_and_too_large(leet, which):
    for bad in (dict(dtype=3), dict(rd=2), dict(wd=2), dict(dtype=0, rd=1)):
        assert norm(leet, which, **bad) == leet.LEET_ERR_UNSUPPORTED
    for bad in (dict(C=16385), dict(B=1 << 20, N=1 << 12), dict(B=1, N=1 << 23)):
        assert norm(leet, which, group=0, **bad) == leet.LEET_ERR_TOO_LARGE
    if which == "q8":
        assert norm(leet, which, group=16) == leet.LEET_ERR_UNSUPPORTED and norm(leet, which, group=-1) == leet.LEET_ERR_UNSUPPORTED


def test_norm_outputs_over_other_arguments(leet):
    def near(at):   # four rows further on, so neither in place nor apart
        return leet._pack_rows(P + at * STEP + 4 * 8192, 1 << 16, 4096)
    bad = leet.LEET_ERR_INVALID_ARG
    for which in WHICH:
        for other in (0, 1) + ((4, 6, 8) if which == "backward" else (3,)) + (5,) + ((7,) if which == "q8" else ()):
            assert norm(leet, which, out=near(other)) == bad if other < 5 else norm(leet, which, out=rows(leet, other)) == bad, (which, other)
    for which in ("forward", "q8"):
        for other in (0, 1):
            assert norm(leet, which, sum=near(other)) == bad
        assert norm(leet, which, sum=rows(leet, 2)) == bad and norm(leet, which, sum=rows(leet, 5)) == bad
    for other in (0, 1, 2, 3, 5):
        assert norm(leet, "q8", scales=P + other * STEP) == bad
    assert norm(leet, "q8", out=rows(leet, 0)) == bad   # a byte an element is not in place of two
    for other in (0, 1, 2, 4, 5, 6):
        assert norm(leet, "backward", ws=P + other * STEP) == bad
    assert norm(leet, "backward", rd=0, sum=rows(leet, 2)) == bad and norm(leet, "backward", rd=0, sum=rows(leet, 0)) == bad


def test_norm_no_rows(leet):
    assert norm(leet, "forward", N=0, x=None, out=None) == leet.LEET_OK
    assert norm(leet, "q8", N=0, x=None, out=None, scales=None) == leet.LEET_OK
    assert norm(leet, "backward", N=0, x=None, dw=None) == leet.LEET_OK
    assert leet.add_rms_norm_workspace_bytes(2, 0, 64) == 0
    assert leet.add_rms_norm_workspace_bytes(1, 10, 1024) == 10 * 1024 * 4 and leet.add_rms_norm_workspace_bytes(1, 10, 512) == 3 * 512 * 4


def test_norm_binding_refuses(leet):
    x = torch.zeros(2, 3, 8)
    for call in (leet.leet_attn_add_rms_norm, leet.leet_attn_add_rms_norm_q8):
        with pytest.raises(ValueError):   # not on a GPU
            call(x)
        with pytest.raises(ValueError):
            call(torch.zeros(8))
        with pytest.raises(ValueError):
            call(x, weight=torch.ones(7))
        with pytest.raises(TypeError):
            call(x, weight=torch.ones(8).half())
        with pytest.raises(TypeError):
            call(x, x.half())
        with pytest.raises(ValueError):
            call(x, residual_out=x)
    with pytest.raises(ValueError):
        leet.leet_attn_add_rms_norm_q8(x, group=32)
    with pytest.raises(ValueError):
        leet.leet_attn_add_rms_norm_backward(x, x, dweight=torch.ones(8))
    with pytest.raises(TypeError):
        leet.leet_attn_add_rms_norm_backward(x, x.half())


# ---- clipping ----

def clip(leet, grads, limit=1.0, norm=P + 60 * STEP, ws=P + 61 * STEP, wsb=8192):
    packed = b"".join(leet._gradient.pack(*(v or 0 for v in g)) for g in grads)
    return leet.lib.leet_attn_clip_gradients(packed or None, len(grads), limit, norm, ws, wsb, None)


def test_clip_refuses(leet):
    def g(at=0, out=None, count=1000, dtype=0):
        return (P + at * STEP, P + (at if out is None else out) * STEP, count, dtype)
    bad = leet.LEET_ERR_INVALID_ARG
    there = (leet.LEET_ERR_LAUNCH, leet.LEET_ERR_UNSUPPORTED)
    assert leet.clip_gradients_workspace_bytes() == 8192
    if not torch.cuda.is_available():
        assert clip(leet, [g(), g(1, 2)]) in there and clip(leet, [g(), g(0)], float("inf")) in there and clip(leet, [], norm=None) in there
        assert clip(leet, [(P + i * 4000, P + i * 4000, 1000, 0) for i in range(500)]) in there
        assert clip(leet, [(None, None, 0, 0), g()]) in there
    for limit in (-1.0, float("nan")):
        assert clip(leet, [g()], limit) == bad
    assert clip(leet, [g()], ws=None) == bad and clip(leet, [g()], wsb=8000) == bad and clip(leet, [g()], ws=P + 61 * STEP + 8) == bad
    assert clip(leet, [g()], norm=P + 2) == bad
    assert clip(leet, [(None, P, 5, 0)]) == bad and clip(leet, [(P, None, 5, 0)]) == bad and clip(leet, [g(count=-1)]) == bad
    assert clip(leet, [(P + 2, P + 2, 5, 0)]) == bad and clip(leet, [(P, P + STEP + 1, 5, 1)]) == bad
    assert clip(leet, [g(dtype=3)]) == leet.LEET_ERR_UNSUPPORTED
    assert clip(leet, [g(count=(1 << 40) + 1)]) == leet.LEET_ERR_TOO_LARGE
    # outputs over other arguments, the same tensor twice
    assert clip(leet, [g(), g()]) == bad and clip(leet, [g(0, 2), g(1, 2)]) == bad and clip(leet, [g(0, 1), g(1, 2)]) == bad
    assert clip(leet, [(P, P + 8, 100, 0)]) == bad
    assert clip(leet, [g(60)]) == bad and clip(leet, [g(0, 61)]) == bad and clip(leet, [g(61)], float("inf")) == bad
    assert clip(leet, [(P + i * 4000, P + i * 4000, 1001 if i == 77 else 1000, 0) for i in range(500)]) == bad


def test_clip_binding_refuses(leet):
    x = torch.zeros(4, 6)
    with pytest.raises(ValueError):
        leet.leet_attn_clip_gradients([])
    with pytest.raises(ValueError):   # not on a GPU
        leet.leet_attn_clip_gradients([x], 1.0)
    with pytest.raises(ValueError):
        leet.leet_attn_clip_gradients([x], 1.0, outs=[])
    for limit in (None, float("inf")):
        with pytest.raises(ValueError):   # nothing would be written
            leet.leet_attn_clip_gradients([x], limit, outs=[x.clone()])
