"""Norms of residual sums, their 8-bit output and their gradient on the GPU against 64 bits."""
import pytest
import torch

import training_forms as forms
from layer_forms import close, half_step

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32), (F32, F32)]
CHANNELS = [1, 7, 8, 64, 129, 511, 512, 513, 1000, 1024, 1025, 2048, 2051, 4096, 4100, 8192, 8200, 16384]
EPS = 1e-5


@pytest.fixture(scope="module")
def leet():
    from paper_2501_02573_amd import binding
    return binding


def normal(shape, dtype, seed, sigma=1.0, mean=0.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * sigma + mean).to(dtype)


def held(name, got, form, dtype=None):
    if not close(got, form, dtype):
        ref, bound = form
        off = (got.double().cpu() - ref).abs() / (bound + half_step(ref, dtype or got.dtype))
        raise AssertionError(f"{name}: {float(off.max()):.3g} of the bound at {int(off.argmax())}")


def d(t):
    return None if t is None else t.double()


def cu(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("C", CHANNELS)
@pytest.mark.parametrize("dtype,stream", TYPES)
def test_forward(leet, C, dtype, stream):
    for rows, weights in (((2, 3), dtype), ((1, 1), F32), ((5, 1), None)):
        x, res = normal((*rows, C), dtype, 1), normal((*rows, C), stream, 2, 2.0)
        w = None if weights is None else normal((C,), weights, 3, 0.2, 1.0)
        w64 = torch.ones(C, dtype=torch.float64) if w is None else w.double()
        y, s = leet.leet_attn_add_rms_norm(cu(x), cu(res), cu(w), eps=EPS)
        want = forms.add_norm(d(x), d(res), w64, EPS)
        held("y", y, want[0])
        held("sum", s, want[1])
        y, none = leet.leet_attn_add_rms_norm(cu(x), None, cu(w), eps=EPS)
        assert none is None
        held("y alone", y, forms.add_norm(d(x), None, w64, EPS)[0])


@pytest.mark.parametrize("C", CHANNELS)
@pytest.mark.parametrize("dtype,stream", TYPES)
def test_backward(leet, C, dtype, stream):
    for rows, weights, along in (((2, 3), dtype, True), ((1, 1), F32, False), ((7, 1), None, True)):
        dy, h = normal((*rows, C), dtype, 1), normal((*rows, C), stream, 2, 2.0)
        a = normal((*rows, C), stream, 4) if along else None
        w = None if weights is None else normal((C,), weights, 3, 0.2, 1.0)
        w64 = torch.ones(C, dtype=torch.float64) if w is None else w.double()
        dx, dh, dw = leet.leet_attn_add_rms_norm_backward(cu(dy), cu(h), cu(w), eps=EPS, dresidual=cu(a))
        g, gw = forms.add_norm_backward(d(dy), d(h), w64, EPS, d(a))
        held("dx", dx, g)
        held("dh", dh, g)
        assert (dh is dx) == (dtype == stream) and dh.dtype == stream
        if w is None:
            assert dw is None
        else:
            held("dw", dw, gw)


def groups_of(y8, scales, group):
    C = y8.shape[-1]
    return (y8.float().cpu().double().unflatten(-1, (-1, group or C)) * scales.cpu().double()[..., None]).flatten(-2)


@pytest.mark.parametrize("C,group", [(1, 0), (7, 0), (513, 0), (1000, 0), (2048, 0), (4100, 0), (8200, 0), (32, 32), (96, 32), (544, 32),
                                     (64, 64), (1088, 64), (128, 128), (640, 128), (4096, 128), (8320, 128), (16384, 64)])
@pytest.mark.parametrize("dtype,stream", TYPES)
def test_eight_bits(leet, C, group, dtype, stream):
    x, res, w = normal((2, 5, C), dtype, 1), normal((2, 5, C), stream, 2, 2.0), normal((C,), dtype, 3, 0.2, 1.0)
    if C > 100:
        x[0, 0], res[0, 0] = 0, 0   # a row of zeros
        x[1, 1, :C // 2] *= 2.0 ** -12
    y8, scales, s = leet.leet_attn_add_rms_norm_q8(cu(x), cu(res), cu(w), eps=EPS, group=group)
    assert y8.dtype == torch.float8_e4m3fn and scales.shape == (2, 5, C // group if group else 1)
    (y, bound), sums = forms.add_norm(d(x), d(res), d(w), EPS)
    held("sum", s, sums)
    most = y.unflatten(-1, (-1, group or C)).abs().amax(-1).clamp(min=2.0 ** -100) / 448
    assert float(((scales.cpu().double() - most).abs() / most).max()) < 40 * forms.U
    off = (groups_of(y8, scales, group) - y).abs()
    spread = most[..., None].expand(*most.shape, group or C).flatten(-2)
    assert bool((off <= forms.eight_bits(y, spread, bound)).all())
    # the largest of a group is the largest value of 8 bits
    assert bool((y8.float().abs().unflatten(-1, (-1, group or C)).amax(-1).cpu()[most > 2.0 ** -100 / 448] == 448).all())
    y8, scales, none = leet.leet_attn_add_rms_norm_q8(cu(x), weight=cu(w), eps=EPS, group=group)
    assert none is None
    (y, bound), _ = forms.add_norm(d(x), None, d(w), EPS)
    spread = scales.cpu().double()[..., None].expand(*scales.shape, group or C).flatten(-2)
    assert bool(((groups_of(y8, scales, group) - y).abs() <= forms.eight_bits(y, spread, bound)).all())


@pytest.mark.parametrize("dtype,stream", TYPES)
def test_many_rows(leet, dtype, stream):
    """More rows than workgroups are launched at once; a weight's gradient over all of them."""
    for rows, C in (((3, 2001), 72), ((1, 3001), 600)):
        x, res, w = normal((*rows, C), dtype, 1), normal((*rows, C), stream, 2), normal((C,), dtype, 3, 0.2, 1.0)
        y, s = leet.leet_attn_add_rms_norm(cu(x), cu(res), cu(w), eps=EPS)
        want = forms.add_norm(d(x), d(res), d(w), EPS)
        held("y", y, want[0])
        held("sum", s, want[1])
        dx, dh, dw = leet.leet_attn_add_rms_norm_backward(cu(x), cu(res), cu(w), eps=EPS)
        g, gw = forms.add_norm_backward(d(x), d(res), d(w), EPS)
        held("dx", dx, g)
        held("dh", dh, g)
        held("dw", dw, gw)
        again = leet.leet_attn_add_rms_norm_backward(cu(x), cu(res), cu(w), eps=EPS)
        assert all(torch.equal(a, b) for a, b in zip((dx, dh, dw), again))


def test_rows_beyond_the_cache(leet):
    """Streamed past the last-level cache: the same bits as the same rows a few at a time."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x, res = (torch.randn((1, 30000, 2048), generator=g, device="cuda").to(BF16) for _ in range(2))
    w = torch.randn(2048, generator=g, device="cuda")
    y, s = leet.leet_attn_add_rms_norm(x, res, w)
    y8, scales, _ = leet.leet_attn_add_rms_norm_q8(x, res, w, group=64)
    dx, _, _ = leet.leet_attn_add_rms_norm_backward(x, res, w, dresidual=y)
    for at in (slice(0, 500), slice(29500, 30000)):
        a, b = leet.leet_attn_add_rms_norm(x[:, at], res[:, at], w)
        c, e, _ = leet.leet_attn_add_rms_norm_q8(x[:, at], res[:, at], w, group=64)
        f, _, _ = leet.leet_attn_add_rms_norm_backward(x[:, at], res[:, at], w, dresidual=y[:, at])
        for full, part in ((y, a), (s, b), (y8.view(torch.uint8), c.view(torch.uint8)), (scales, e), (dx, f)):
            assert torch.equal(full[:, at], part)


def test_offsets_beyond_two_to_the_31(leet):
    x = torch.randn((1, 300000, 8192), device="cuda", dtype=BF16)
    w = torch.randn(8192, device="cuda")
    y, _ = leet.leet_attn_add_rms_norm(x, None, w)
    dx, _, dw = leet.leet_attn_add_rms_norm_backward(y, x, w)
    at = slice(299990, 300000)
    assert torch.equal(y[:, at], leet.leet_attn_add_rms_norm(x[:, at], None, w)[0])
    assert torch.equal(dx[:, at], leet.leet_attn_add_rms_norm_backward(y[:, at], x[:, at], w)[0])
    y8, scales, _ = leet.leet_attn_add_rms_norm_q8(x, None, w)
    part = leet.leet_attn_add_rms_norm_q8(x[:, at], None, w)
    assert torch.equal(y8[:, at].view(torch.uint8), part[0].view(torch.uint8)) and torch.equal(scales[:, at], part[1])


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("C", [96, 129, 1031])
def test_strides_and_what_lies_between(leet, dtype, stream, C):
    """Rows out of wider buffers, batches in the inner dimension, at addresses that suit one element; nothing else is written."""
    B, N = 3, 5

    def place(dt, seed, fill=None):
        buf = normal((N, B, C + 9), dt, seed).cuda() if fill is None else torch.full((N, B, C + 9), fill, dtype=dt, device="cuda")
        return buf, buf[:, :, 3:3 + C].transpose(0, 1)

    (_, x), (_, res), (_, a) = place(dtype, 1), place(stream, 2), place(stream, 3)
    w = normal((C + 1,), dtype, 4).cuda()[1:]
    bufs = [place(dtype, 0, 5.0), place(stream, 0, 5.0)]
    y, s = leet.leet_attn_add_rms_norm(x, res, w, eps=EPS, out=bufs[0][1], residual_out=bufs[1][1])
    want = leet.leet_attn_add_rms_norm(x.contiguous(), res.contiguous(), w.clone(), eps=EPS)
    assert torch.equal(y, want[0]) and torch.equal(s, want[1])
    grads = [place(dtype, 0, 5.0), place(stream, 0, 5.0)]
    dx, dh, dw = leet.leet_attn_add_rms_norm_backward(x, res, w, eps=EPS, dresidual=a, dx=grads[0][1],
                                                      dh=grads[1][1] if dtype != stream else None)
    want = leet.leet_attn_add_rms_norm_backward(x.contiguous(), res.contiguous(), w.clone(), eps=EPS, dresidual=a.contiguous())
    assert all(torch.equal(p, q) for p, q in zip((dx, dh, dw), want))
    for buf, view in bufs + grads[:1] + (grads[1:] if dtype != stream else []):
        assert bool((buf[:, :, :3] == 5.0).all()) and bool((buf[:, :, 3 + C:] == 5.0).all())
    raw = torch.full((N, B, C + 9), 7, dtype=torch.uint8, device="cuda")
    y8 = raw[:, :, 3:3 + C].transpose(0, 1).view(torch.float8_e4m3fn)
    leet.leet_attn_add_rms_norm_q8(x, res, w, eps=EPS, out=y8)
    plain = leet.leet_attn_add_rms_norm_q8(x.contiguous(), res.contiguous(), w.clone(), eps=EPS)[0]
    assert torch.equal(y8.contiguous().view(torch.uint8), plain.view(torch.uint8))
    assert bool((raw[:, :, :3] == 7).all()) and bool((raw[:, :, 3 + C:] == 7).all())


def test_two_dimensions_and_a_broadcast_residual(leet):
    x, res, w = normal((6, 300), BF16, 1).cuda(), normal((300,), BF16, 2).cuda().expand(6, 300), normal((300,), F32, 3).cuda()
    y, s = leet.leet_attn_add_rms_norm(x, res, w)
    want = leet.leet_attn_add_rms_norm(x[None], res[None].contiguous(), w)
    assert torch.equal(y, want[0][0]) and torch.equal(s, want[1][0]) and s.is_contiguous()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place(leet, dtype):
    for C in (200, 700, 2100):
        x, res, w = normal((2, 9, C), dtype, 1).cuda(), normal((2, 9, C), dtype, 2).cuda(), normal((C,), dtype, 3).cuda()
        y, s = leet.leet_attn_add_rms_norm(x, res, w)
        x1, r1 = x.clone(), res.clone()
        assert leet.leet_attn_add_rms_norm(x1, r1, w, out=x1, residual_out=r1)[0] is x1
        assert torch.equal(x1, y) and torch.equal(r1, s)
        x1, r1 = x.clone(), res.clone()
        leet.leet_attn_add_rms_norm(x1, r1, w, out=r1, residual_out=x1)
        assert torch.equal(r1, y) and torch.equal(x1, s)
        want = leet.leet_attn_add_rms_norm_backward(x, s, w, dresidual=res)
        for n in range(3):
            t = [x.clone(), s.clone(), res.clone()]
            w1 = w.clone()
            got = leet.leet_attn_add_rms_norm_backward(t[0], t[1], w1, dresidual=t[2], dx=t[n], dweight=w1)
            assert torch.equal(t[n], want[0]) and torch.equal(w1, want[2])


@pytest.mark.parametrize("dtype,stream", [(BF16, BF16), (F16, F32), (F32, F32)])
@pytest.mark.parametrize("C", [200, 700, 16384])
def test_large_and_small_rows(leet, dtype, stream, C):
    scale = torch.tensor([1.0, 2.0 ** 120, 2.0 ** -110, 2.0 ** 60, 2.0 ** -60, 2.0 ** 63], dtype=torch.float64).view(1, 6, 1)
    res = (normal((1, 6, C), F32, 1).double() * scale).to(stream)
    x, w = torch.zeros((1, 6, C), dtype=dtype), normal((C,), F32, 3, 0.2, 1.0)
    y, s = leet.leet_attn_add_rms_norm(cu(x), cu(res), cu(w), eps=0.0)
    want = forms.add_norm(d(x), d(res), d(w), 0.0)
    held("y", y, want[0])
    assert torch.equal(s.cpu(), res)
    dy = normal((1, 6, C), dtype, 4)
    dx, dh, dw = leet.leet_attn_add_rms_norm_backward(cu(dy), cu(res), cu(w), eps=0.0)
    g, gw = forms.add_norm_backward(d(dy), d(res), d(w), 0.0)
    if stream == dtype or dtype != F16:   # what fits fp16 is the other types' matter
        held("dx", dx, g)
    held("dh", dh, (g[0], g[1] + 2.0 ** -140))
    held("dw", dw, gw)


def test_rows_that_are_not_finite_stay_alone(leet):
    x, w = normal((1, 9, 300), BF16, 1).cuda(), normal((300,), BF16, 2).cuda()
    bad = x.clone()
    bad[0, 2, 7], bad[0, 5, 0] = float("nan"), float("inf")
    y, z = leet.leet_attn_add_rms_norm(x, None, w)[0], leet.leet_attn_add_rms_norm(bad, None, w)[0]
    q, sc, _ = leet.leet_attn_add_rms_norm_q8(bad, None, w)
    q0, sc0, _ = leet.leet_attn_add_rms_norm_q8(x, None, w)
    dx0, dx = leet.leet_attn_add_rms_norm_backward(x, x, w)[0], leet.leet_attn_add_rms_norm_backward(x, bad, w)[0]
    fine = [n for n in range(9) if n not in (2, 5)]
    assert torch.equal(y[:, fine], z[:, fine]) and torch.equal(dx0[:, fine], dx[:, fine])
    assert torch.equal(q[:, fine].float(), q0[:, fine].float()) and torch.equal(sc[:, fine], sc0[:, fine])
    assert bool(z[0, 2].isnan().all()) and bool(dx[0, 2].isnan().all())
    assert bool((q.float() * sc)[0, 2].isnan().all()) and bool((q.float() * sc)[0, 5, 0].isnan())
    zero = torch.zeros((1, 1, 300), device="cuda")
    assert bool(leet.leet_attn_add_rms_norm(zero, eps=0.0)[0].isnan().all()) and not leet.leet_attn_add_rms_norm(zero)[0].any()


def test_no_rows(leet):
    x, w = torch.zeros((2, 0, 64), device="cuda"), torch.ones(64, device="cuda")
    y, s = leet.leet_attn_add_rms_norm(x, x, w)
    assert y.shape == x.shape and s.shape == x.shape
    assert leet.leet_attn_add_rms_norm_q8(x, x, w, group=32)[1].shape == (2, 0, 2)
    dw = torch.full((64,), 3.0, device="cuda")
    leet.leet_attn_add_rms_norm_backward(x, x, w, dweight=dw)
    assert not dw.any()


def test_graph_and_streams(leet):
    sets = [(normal((2, 500, 640), BF16, s).cuda(), normal((2, 500, 640), F32, s + 1).cuda(), normal((640,), F32, s + 2).cuda())
            for s in (1, 4)]

    def call(x, res, w):
        y, s = leet.leet_attn_add_rms_norm(x, res, w)
        return (y, s) + leet.leet_attn_add_rms_norm_backward(y, s, w, dresidual=res) + leet.leet_attn_add_rms_norm_q8(x, res, w)[:2]

    def same(a, b):
        return all(torch.equal(p.float(), q.float()) for p, q in zip(a, b))

    want = [call(*t) for t in sets]
    torch.cuda.synchronize()
    got = []
    for t in sets:
        with torch.cuda.stream(torch.cuda.Stream()):
            got.append(call(*t))
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(want, got))
    graphs, kept = [], []
    for t in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            kept.append(call(*t))
    for i in range(3):
        for t in sets:
            t[0].mul_(-0.5)
        eager = [call(*t) for t in sets]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(eager, kept))
