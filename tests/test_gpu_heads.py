"""Position rotation and the norms of queries and keys on the GPU, against their 64-bit forms."""
import pytest
import torch

import layer_forms as forms

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def leet():
    from paper_2501_02573_amd import binding
    return binding


def _normal(shape, dtype, seed, sigma=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * sigma + mean).to(dtype).cuda()


def _freq(rot, base=10000.0):
    return base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)


def _f64(t):
    return t.detach().double().cpu()


def _fused(B, N, Hq, Hk, d, dtype, seed, shift=0):
    """q and k as parts of a token-major projection; shift: elements by which its storage is off its alignment."""
    width = (Hq + 2 * Hk) * d
    flat = _normal((B * N * width + shift,), dtype, seed)[shift:]
    at = flat.view(B, N, Hq + 2 * Hk, d).transpose(1, 2)
    return at[:, :Hq], at[:, Hq:Hq + Hk]


# (B, N, Hq, Hk, d, rot)
SHAPES = [(1, 1, 1, 1, 64, 64), (2, 65, 4, 2, 64, 32), (1, 300, 3, 1, 128, 128), (3, 33, 5, 5, 128, 64), (2, 17, 2, 1, 256, 256),
          (1, 40, 2, 2, 256, 64), (2, 9, 2, 1, 80, 32), (1, 21, 3, 3, 128, 34), (2, 5, 1, 2, 2, 2), (1, 31, 2, 2, 34, 10),
          (1, 3, 2, 2, 96, 94), (5, 2, 33, 7, 128, 16), (64, 1, 32, 32, 128, 128), (1, 7, 40, 3, 16, 16)]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_rope(leet, shape, dtype, layout):
    B, N, Hq, Hk, d, rot = shape
    q, k = _fused(B, N, Hq, Hk, d, dtype, 1)
    freq = _freq(rot)
    pos = torch.randint(0, 200000, (B, N), generator=torch.Generator().manual_seed(2))
    out_q, out_k = leet.leet_attn_rope(q, freq.cuda(), k=k, positions=pos.cuda(), layout=layout, scale=1.25)
    assert out_q.is_contiguous() and out_k.is_contiguous() and out_q.dtype == dtype
    for x, y in ((q, out_q), (k, out_k)):
        assert forms.close(y, forms.rotate(_f64(x), freq, pos, layout, 1.25))
    back = leet.leet_attn_rope(out_q, freq.cuda(), positions=pos.cuda(), layout=layout, scale=1.25, transposed=True)
    assert forms.close(back, forms.rotate(_f64(out_q), freq, pos, layout, 1.25, transposed=True))


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(2, 37, 3, 2, 128, 128), (1, 50, 2, 1, 64, 16)])
def test_rope_of_rows_off_their_alignment(leet, shape, dtype, layout):
    B, N, Hq, Hk, d, rot = shape
    q, k = _fused(B, N, Hq, Hk, d, dtype, 3, shift=1)
    assert q.data_ptr() % 16
    out_q, out_k = leet.leet_attn_rope(q, _freq(rot).cuda(), k=k, pos0=7, layout=layout)
    pos = (torch.arange(N) + 7).expand(B, N)
    for x, y in ((q, out_q), (k, out_k)):
        assert forms.close(y, forms.rotate(_f64(x), _freq(rot), pos, layout))


def test_rope_far_out_and_before_zero(leet):
    freq = _freq(64)
    x = _normal((1, 2, 6, 64), F32, 4)
    # 2^40: the product with the fastest frequency (1) is exact, with others off by 2^-53 of 2^40: 1e-4 turns of the
    # slowest would show, 2^-13 rad is what the 64-bit form itself is off by; so frequencies that multiply exactly
    exact = torch.tensor([2.0 ** -i for i in range(32)], dtype=torch.float64)
    pos = torch.tensor([[0, -1, -100003, 1 << 20, (1 << 31) + 5, 12345678901]])
    y = leet.leet_attn_rope(x, exact.cuda(), positions=pos.cuda())
    # an angle of 1e10 is off by 2^-53 of itself in 64 bits, 1.4e-6: in turns, in the form and in the kernel alike
    ref, bound = forms.rotate(_f64(x), exact, pos, 0)
    far = 2 * 2.0 ** -53 * pos.abs().double()[:, None, :, None] * (_f64(x)[..., :32].abs() + _f64(x)[..., 32:].abs())
    assert forms.close(y, (ref, bound + torch.cat((far, far), -1)))
    z = leet.leet_attn_rope(x, freq.cuda(), positions=pos[0, :].cuda() * 0, pos0=-3)
    assert forms.close(z, forms.rotate(_f64(x), freq, torch.full((1, 6), -3), 0))


@pytest.mark.parametrize("scale", [1.0, 1.2079441, -0.7])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("d, rot", [(128, 128), (64, 32), (128, 34)])
def test_cosines_and_sines_are_rounded_once(leet, d, rot, layout, scale):
    """Pairs (1, 0) come out as their cosine and sine times the scale, each the nearest fp32 number but for what the 64 bits
    leave out: 2^-32 of the series, and 2^-51 of the angle here and in the form (which adds a rounding of its own)."""
    N = 4000
    pos = torch.randint(-70000, 200000, (1, N), generator=torch.Generator().manual_seed(9))
    freq, x = _freq(rot), torch.zeros((1, 1, N, d), dtype=F32)
    one, two = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == 0 else (slice(0, rot, 2), slice(1, rot, 2))
    x[..., one] = 1.0
    scale = torch.tensor(scale, dtype=F32).double().item()
    theta = pos.double()[0, :, None] * freq
    for transposed in (False, True):
        y = leet.leet_attn_rope(x.cuda(), freq.cuda(), positions=pos.cuda(), layout=layout, scale=scale, transposed=transposed)
        y, sign = _f64(y)[0, 0], -1.0 if transposed else 1.0
        for got, want in ((y[:, one], theta.cos() * scale), (y[:, two], sign * theta.sin() * scale)):
            # half a step at a value is 2^-25 of the power of two above it, at the most
            half = 2.0 ** -25 * torch.exp2(torch.ceil(torch.log2(want.abs().clamp_min(2.0 ** -100))))
            off = half + abs(scale) * (2.0 ** -32 + 2.0 ** -50 * theta.abs())
            assert bool(((got - want).abs() <= off).all())


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("rot", [16, 20])
def test_elements_that_are_not_rotated_keep_clear_of_their_neighbours(leet, rot, layout):
    x = _normal((1, 1, 4, 32), BF16, 5)
    x[0, 0, 1, rot:] = float("inf")
    x[0, 0, 2, rot + 1::2] = float("nan")
    y = leet.leet_attn_rope(x, _freq(rot).cuda(), layout=layout)
    assert torch.equal(y[..., rot:].nan_to_num(7.0), x[..., rot:].nan_to_num(7.0))
    assert forms.close(y, forms.rotate(_f64(x), _freq(rot), torch.arange(4).view(1, 4), layout))


def test_rope_in_place_and_into_a_part(leet):
    freq, pos = _freq(64), torch.arange(19).expand(2, 19)
    q, k = _fused(2, 19, 3, 2, 128, BF16, 6)
    want = [forms.rotate(_f64(t), freq, pos, 0) for t in (q, k)]
    leet.leet_attn_rope(q, freq.cuda(), k=k, out_q=q, out_k=k)
    assert forms.close(q, want[0]) and forms.close(k, want[1])
    wide = torch.full((2, 19, 8, 128), 5.0, dtype=BF16, device="cuda")
    x = _normal((2, 4, 19, 128), BF16, 7)
    leet.leet_attn_rope(x, freq.cuda(), out_q=wide.transpose(1, 2)[:, 2:6])
    assert forms.close(wide.transpose(1, 2)[:, 2:6], forms.rotate(_f64(x), freq, pos, 0))
    assert bool((wide[:, :, :2] == 5).all()) and bool((wide[:, :, 6:] == 5).all())


def test_rope_reads_broadcast_inputs(leet):
    x = _normal((1, 1, 11, 64), F16, 8).expand(2, 3, 11, 64)
    y = leet.leet_attn_rope(x, _freq(64).cuda())
    assert forms.close(y, forms.rotate(_f64(x), _freq(64), torch.arange(11).expand(2, 11), 0))


def test_no_tokens(leet):
    x = torch.empty((2, 3, 0, 64), dtype=BF16, device="cuda")
    assert leet.leet_attn_rope(x, _freq(64).cuda()).shape == x.shape
    w = torch.ones(64, dtype=BF16, device="cuda")
    assert leet.leet_attn_qk_norm_rope(x, x, w, w, _freq(64).cuda())[1].shape == x.shape
    dq, dk, dwq, dwk = leet.leet_attn_qk_norm_rope_backward(x, x, x, x, w, w, _freq(64).cuda())
    assert dq.shape == x.shape and bool((dwq == 0).all()) and bool((dwk == 0).all())


WEIGHTS = ["in", "f32", "none", "q only"]


def _weights(kind, d, dtype):
    if kind == "none":
        return None, None
    wdt = F32 if kind == "f32" else dtype
    wq, wk = _normal((d,), wdt, 11, 0.3, 1.0), _normal((d,), wdt, 12, 0.3, 1.0)
    return wq, None if kind == "q only" else wk


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("i, shape", list(enumerate(SHAPES)))
def test_norm_rope_and_backward(leet, i, shape, dtype, layout):
    B, N, Hq, Hk, d, rot = shape
    shift = 1 if i % 5 == 4 else 0
    q, k = _fused(B, N, Hq, Hk, d, dtype, 13, shift)
    wq, wk = _weights(WEIGHTS[(i + layout) % 4], d, dtype)
    freq = _freq(rot)
    pos = torch.randint(0, 50000, (B, N), generator=torch.Generator().manual_seed(14))
    how = dict(positions=pos.cuda(), layout=layout, scale=0.75, eps=1e-5)
    out_q, out_k = leet.leet_attn_qk_norm_rope(q, k, wq, wk, freq.cuda(), **how)
    ones = torch.ones(d, dtype=torch.float64)
    for x, w, y in ((q, wq, out_q), (k, wk, out_k)):
        assert forms.close(y, forms.norm_rope(_f64(x), ones if w is None else _f64(w), freq, pos, layout, 0.75, 1e-5))

    dy_q, dy_k = _normal((B, Hq, N, d), dtype, 15), _normal((B, Hk, N, d), dtype, 16)
    into = _fused(B, N, Hq, Hk, d, dtype, 17)
    dx_q, dx_k, dwq, dwk = leet.leet_attn_qk_norm_rope_backward(dy_q, dy_k, q, k, wq, wk, freq.cuda(), dx_q=into[0],
                                                                dx_k=into[1], **how)
    assert dx_q is into[0] and (dwk is None) == (wk is None)
    for x, w, dy, dx, dw in ((q, wq, dy_q, dx_q, dwq), (k, wk, dy_k, dx_k, dwk)):
        to_x, to_w = forms.norm_rope_backward(_f64(dy), _f64(x), ones if w is None else _f64(w), freq, pos, layout, 0.75, 1e-5)
        assert forms.close(dx, to_x)
        if w is not None:
            assert dw.dtype == w.dtype and forms.close(dw, to_w)


def test_norm_of_zero_rows_and_large_values(leet):
    freq = _freq(128)
    q = _normal((1, 2, 9, 128), BF16, 20)
    q[0, 0, 3] = 0
    q[0, 1, 4] *= 2.0 ** 40
    k = _normal((1, 1, 9, 128), BF16, 21)
    w = _normal((128,), BF16, 22, 0.3, 1.0)
    y, _ = leet.leet_attn_qk_norm_rope(q, k, w, w, freq.cuda())
    pos = torch.arange(9).view(1, 9)
    assert bool((y[0, 0, 3] == 0).all())
    assert forms.close(y, forms.norm_rope(_f64(q), _f64(w), freq, pos, 0))
    dy = _normal(q.shape, BF16, 23)
    dx, _, dw, _ = leet.leet_attn_qk_norm_rope_backward(dy, k, q, k, w, w, freq.cuda())
    to_x, to_w = forms.norm_rope_backward(_f64(dy), _f64(q), _f64(w), freq, pos, 0)
    assert forms.close(dx, to_x) and forms.close(dw, to_w)
    # a row that is not finite stays by itself
    q[0, 1, 4, 5] = float("nan")
    z, _ = leet.leet_attn_qk_norm_rope(q, k, w, w, freq.cuda())
    assert bool(z[0, 1, 4].isnan().all())
    z[0, 1, 4] = y[0, 1, 4]
    assert torch.equal(z, y)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d, rot", [(128, 128), (64, 32), (256, 64), (34, 10)])
def test_norm_of_rows_whose_squares_leave_the_range(leet, d, rot, dtype, layout):
    """Rows of 2^-100 to 2^120 and more beside ordinary ones: their squares are beyond fp32, their norms are not."""
    freq, eps = _freq(rot), 1e-37          # below the range's end is weighed against eps = 2^-123
    q, k = _normal((1, 3, 40, d), F32, 24), _normal((1, 1, 40, d), F32, 25)
    powers = torch.tensor([0.0, 120.0, 63.0, 90.0, -100.0, -63.0, 55.0, 60.0, -49.0, -55.0]).exp2()
    q, k = q * powers.repeat(4).cuda()[:, None], k * powers.flip(0).repeat(4).cuda()[:, None]
    q[0, 0, 11, 0], q[0, 0, 11, 1:] = 3e38, 0.0
    q, k = q.to(dtype), k.to(dtype)
    w, pos = _normal((d,), dtype, 26, 0.3, 1.0), torch.arange(40).view(1, 40)
    y, z = leet.leet_attn_qk_norm_rope(q, k, w, w, freq.cuda(), eps=eps, layout=layout)
    eps = torch.tensor(eps, dtype=F32).double().item()
    for x, out in ((q, y), (k, z)):
        assert forms.close(out, forms.norm_rope(_f64(x), _f64(w), freq, pos, layout, eps=eps))
    # gradients of inputs go like one over the row's length: those of a row of 2^120 are not below the smallest normal number
    dy, dz = _normal(q.shape, dtype, 27, 2.0 ** 10), _normal(k.shape, dtype, 28, 2.0 ** 10)
    dx, dk, dw, dwk = leet.leet_attn_qk_norm_rope_backward(dy, dz, q, k, w, w, freq.cuda(), eps=eps, layout=layout)
    for x, g, gx, gw in ((q, dy, dx, dw), (k, dz, dk, dwk)):
        to_x, to_w = forms.norm_rope_backward(_f64(g), _f64(x), _f64(w), freq, pos, layout, eps=eps)
        assert forms.close(gw, to_w) and forms.close(gx, to_x)


def test_weight_gradient_over_many_rows(leet):
    """More rows than one round of workgroups takes: dw of ones' gradient is a sum that is known."""
    B, H, N, d = 2, 16, 5000, 64
    q = torch.ones((B, H, N, d), dtype=F32, device="cuda")
    k = torch.ones((B, 1, N, d), dtype=F32, device="cuda")
    w = torch.ones(d, device="cuda")
    freq = torch.zeros(32, dtype=torch.float64, device="cuda")   # nothing turns
    _, _, dwq, dwk = leet.leet_attn_qk_norm_rope_backward(q, k, q, k, w, w, freq, eps=0.0)
    # every term is 1, sums stay whole numbers below 2^24
    assert bool((dwq == B * H * N).all()) and bool((dwk == B * N).all())
    again = leet.leet_attn_qk_norm_rope_backward(q, k, q, k, w, w, freq, eps=0.0)
    assert torch.equal(again[2], dwq)


def test_weight_gradients_are_equal_from_call_to_call(leet):
    q, k = _fused(2, 1000, 8, 2, 128, BF16, 30)
    dq, dk = _normal((2, 8, 1000, 128), BF16, 31), _normal((2, 2, 1000, 128), BF16, 32)
    w = _normal((128,), F32, 33, 0.3, 1.0)
    one, two = (leet.leet_attn_qk_norm_rope_backward(dq, dk, q, k, w, w, _freq(128).cuda()) for _ in range(2))
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    # and with a workspace of the caller's
    ws = torch.empty(leet.qk_norm_rope_workspace_bytes(2, 8, 2, 1000, 128), dtype=torch.uint8, device="cuda")
    three = leet.leet_attn_qk_norm_rope_backward(dq, dk, q, k, w, w, _freq(128).cuda(), workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(one, three))
    with pytest.raises(leet.LeetAttnError):
        leet.leet_attn_qk_norm_rope_backward(dq, dk, q, k, w, w, _freq(128).cuda(), workspace=ws[:256])


def test_gradient_in_place(leet):
    q, k = _fused(1, 70, 4, 2, 128, BF16, 40)
    dq, dk = _normal((1, 4, 70, 128), BF16, 41), _normal((1, 2, 70, 128), BF16, 42)
    w = _normal((128,), BF16, 43, 0.3, 1.0)
    want = leet.leet_attn_qk_norm_rope_backward(dq, dk, q, k, w, w, _freq(64).cuda(), layout=leet.ROPE_INTERLEAVED)
    got = leet.leet_attn_qk_norm_rope_backward(dq, dk, q, k, w, w, _freq(64).cuda(), layout=leet.ROPE_INTERLEAVED,
                                               dx_q=dq, dx_k=dk)
    assert got[0] is dq and all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("d, rot", [(128, 64), (34, 10)])
def test_gradient_over_the_inputs(leet, d, rot):
    """Gradients of inputs and weights in the place of the inputs and weights, parts of one projection."""
    q, k = _fused(2, 333, 6, 3, d, BF16, 44)
    dq, dk = _normal((2, 6, 333, d), BF16, 45), _normal((2, 3, 333, d), BF16, 46)
    wq, wk = _normal((d,), BF16, 47, 0.3, 1.0), _normal((d,), BF16, 48, 0.3, 1.0)
    want = leet.leet_attn_qk_norm_rope_backward(dq, dk, q, k, wq, wk, _freq(rot).cuda())
    got = leet.leet_attn_qk_norm_rope_backward(dq, dk, q, k, wq, wk, _freq(rot).cuda(), dx_q=q, dx_k=k, dq_weight=wq, dk_weight=wk)
    assert got[0] is q and got[3] is wk and all(torch.equal(a, b) for a, b in zip(want, got))


def test_on_another_stream_and_in_a_graph(leet):
    q, k = _fused(2, 300, 4, 4, 128, BF16, 50)
    dq, dk = _normal((2, 4, 300, 128), BF16, 51), _normal((2, 4, 300, 128), BF16, 52)
    w, freq = _normal((128,), BF16, 53, 0.3, 1.0), _freq(128).cuda()

    def both():
        y = leet.leet_attn_qk_norm_rope(q, k, w, w, freq)
        return y + leet.leet_attn_qk_norm_rope_backward(dq, dk, q, k, w, w, freq)

    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = both()
    for sign in (1, -1, 1):
        q.mul_(sign)
        dq.mul_(sign)
        graph.replay()
        eager = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, kept))


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype, d, N", [(BF16, 128, 5000), (F16, 64, 9001), (F32, 256, 1203)])
def test_rows_beyond_the_cache(leet, dtype, d, N, layout):
    """Rows that are streamed give what the same rows give a few tokens at a time."""
    B, Hq, Hk = 4, 16, 12
    q, k = (torch.randn((B, N, H, d), device="cuda").to(dtype).transpose(1, 2) for H in (Hq, Hk))
    assert 2 * (q.numel() + k.numel()) * q.element_size() > 160 << 20
    w, freq = _normal((d,), dtype, 60, 0.3, 1.0), _freq(d // 2).cuda()
    turned = leet.leet_attn_rope(q, freq, k=k, layout=layout)
    y = leet.leet_attn_qk_norm_rope(q, k, w, w, freq, layout=layout)
    dx = leet.leet_attn_qk_norm_rope_backward(y[0], y[1], q, k, w, w, freq, layout=layout)
    sums = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(2)]
    for lo in range(0, N, 400):
        some = slice(lo, min(lo + 400, N))
        part = [t[:, :, some] for t in (q, k)]
        for whole, few in ((turned, leet.leet_attn_rope(part[0], freq, k=part[1], layout=layout, pos0=lo)),
                           (y, leet.leet_attn_qk_norm_rope(*part, w, w, freq, layout=layout, pos0=lo))):
            assert all(torch.equal(a[:, :, some], b) for a, b in zip(whole, few))
        few = leet.leet_attn_qk_norm_rope_backward(y[0][:, :, some], y[1][:, :, some], *part, w.float(), w.float(), freq,
                                                   layout=layout, pos0=lo)
        assert all(torch.equal(a[:, :, some], b) for a, b in zip(dx[:2], few[:2]))
        for s, g in zip(sums, few[2:]):
            s += g.double()
    # with dy = y, u = w n, so terms w n^2 of one sign a column: the sum's error is relative, 96 u of a part's and of the
    # whole's, which the type's rounding is added to (in fp16 to infinity: the sums of 2e5 rows and more are beyond 65504)
    for got, s in zip(dx[2:], sums):
        over = s.abs() > 1.01 * torch.finfo(dtype).max
        assert bool((got[over] == float("inf")).all())
        off = (got.double() - s).abs() - (2 * 96 * forms.U * s.abs() + 1.01 * forms.half_step(s, dtype))
        assert bool((off[~over] <= 0).all())


def test_offsets_beyond_32_bits(leet):
    """Tokens 2^25 elements apart: the last rows are past 2^32 bytes, and past 2^31 elements."""
    N, d, freq = 70, 64, _freq(64)
    wide = torch.empty((N, 1 << 25), dtype=BF16, device="cuda")
    x = wide[:, 128:128 + 2 * d].view(1, N, 2, d).transpose(1, 2)
    x.copy_(_normal((1, 2, N, d), BF16, 61))
    w, pos = _normal((d,), BF16, 62, 0.3, 1.0), torch.arange(N).view(1, N)
    y, z = leet.leet_attn_qk_norm_rope(x[:, :1], x[:, 1:], w, w, freq.cuda())
    want = forms.norm_rope(_f64(x), _f64(w), freq, pos, 0)
    assert forms.close(torch.cat((y, z), 1), want)
    into = wide[:, 1024:1024 + 2 * d].view(1, N, 2, d).transpose(1, 2)
    leet.leet_attn_rope(x, freq.cuda(), out_q=into)
    assert forms.close(into, forms.rotate(_f64(x), freq, pos, 0))
