"""The operators beside the attention, as far as a machine without a GPU goes: frequency tables, refusals of bad
arguments before any device call, and the 64-bit forms that the GPU tests compare with."""
import ctypes
import math

import pytest
import torch

import layer_forms as forms


@pytest.fixture(scope="module")
def leet():
    from paper_2501_02573_amd import binding
    return binding


# ---- frequencies ----

def test_frequencies_unscaled(leet):
    freq, scale = leet.rope_frequencies(8, base=100.0)
    assert scale == 1.0 and freq.dtype == torch.float64
    assert torch.allclose(freq, 100.0 ** (-torch.arange(4, dtype=torch.float64) / 4), rtol=1e-15)


def test_frequencies_linear_and_base(leet):
    plain, _ = leet.rope_frequencies(64)
    linear, scale = leet.rope_frequencies(64, scaling=leet.ROPE_SCALING_LINEAR, factor=4.0)
    assert scale == 1.0 and torch.equal(linear, plain / 4)
    based, scale = leet.rope_frequencies(64, scaling=leet.ROPE_SCALING_BASE, factor=4.0)
    assert scale == 1.0 and based[0] == 1.0
    assert abs(based[-1].item() / (plain[-1].item() / 4) - 1) < 1e-12
    assert torch.equal(leet.rope_frequencies(2, scaling=leet.ROPE_SCALING_BASE, factor=4.0)[0], torch.ones(1, dtype=torch.float64))


@pytest.mark.parametrize("scaling", ["BANDS", "TURNS"])
def test_frequencies_by_bands(leet, scaling):
    rot, trained, factor = 128, 4096, 8.0
    plain, _ = leet.rope_frequencies(rot)
    freq, scale = leet.rope_frequencies(rot, scaling=getattr(leet, "ROPE_SCALING_" + scaling), factor=factor, trained=trained)
    assert abs(scale - (0.1 * math.log(factor) + 1.0 if scaling == "BANDS" else 1.0)) < 1e-7
    turns = trained * plain / (2 * math.pi)
    ratio = plain / freq
    index = [rot * math.log(trained / (t * 2 * math.pi)) / (2 * math.log(10000.0)) for t in (32.0, 1.0)]
    for i in range(rot // 2):
        if scaling == "TURNS":
            share = min(max((32.0 - turns[i].item()) / 31.0, 0.0), 1.0)
        else:
            low, high = math.floor(index[0]), math.ceil(index[1])
            share = min(max((i - low) / (high - low), 0.0), 1.0)
        assert abs(freq[i].item() / (plain[i].item() * ((1 - share) + share / factor)) - 1) < 1e-12
    assert ratio[0] == 1.0 and abs(ratio[-1].item() - factor) < 1e-12
    assert bool((ratio[1:] >= ratio[:-1] - 1e-12).all())


@pytest.mark.parametrize("bad", [dict(rot=7), dict(rot=0), dict(base=1.0), dict(base=math.inf), dict(scaling=9),
                                 dict(factor=0.5), dict(factor=math.nan), dict(scaling=3), dict(scaling=4, trained=-1),
                                 dict(scaling=3, trained=16, slow=0.0), dict(scaling=3, trained=16, slow=4.0, fast=4.0)])
def test_frequencies_refused(leet, bad):
    with pytest.raises((ValueError, leet.LeetAttnError)):
        leet.rope_frequencies(**{"rot": 8, **bad})


# ---- refusals at the C boundary: nothing here reaches a device ----

P = 0x100000   # aligned, never touched


def _heads_args(leet, **change):
    """Arguments of the three calls on heads, by name."""
    H = lambda at=P, b=1 << 20, h=1 << 14, n=128: leet._pack_heads(at, b, h, n)  # noqa: E731
    a = dict(q=H(), out_q=H(2 * P), Hq=2, k=H(3 * P), out_k=H(4 * P), Hk=2, dq=H(5 * P), dk=H(6 * P), wq=P, wk=P, gq=P, gk=2 * P,
             wd=leet.LEET_BF16, eps=1e-6, rot=leet._pack_rotation(P, 64, 0, 0, 0, 0, 1.0), ws=P, wsb=1 << 40, B=2, N=16,
             d=128, dtype=leet.LEET_BF16)
    a.update(change)
    return a


def _rope(leet, a):
    return leet.lib.leet_attn_rope(a["q"], a["out_q"], a["Hq"], a["k"], a["out_k"], a["Hk"], a["rot"], a["B"], a["N"],
                                   a["d"], a["dtype"], 0, None)


def _norm(leet, a):
    return leet.lib.leet_attn_qk_norm_rope(a["q"], a["out_q"], a["Hq"], a["k"], a["out_k"], a["Hk"], a["wq"], a["wk"],
                                           a["wd"], a["eps"], a["rot"], a["B"], a["N"], a["d"], a["dtype"], None)


def _back(leet, a):
    return leet.lib.leet_attn_qk_norm_rope_backward(
        a["out_q"], a["q"], a["dq"], a["Hq"], a["out_k"], a["k"], a["dk"], a["Hk"], a["wq"], a["wk"], a["gq"], a["gk"],
        a["wd"], a["eps"], a["rot"], a["ws"], a["wsb"], a["B"], a["N"], a["d"], a["dtype"], None)


def test_heads_refused(leet):
    H, R = leet._pack_heads, leet._pack_rotation
    INVALID, UNSUPPORTED, LARGE = leet.LEET_ERR_INVALID_ARG, leet.LEET_ERR_UNSUPPORTED, leet.LEET_ERR_TOO_LARGE
    cases = [
        (INVALID, dict(q=None)), (INVALID, dict(out_q=None)), (INVALID, dict(out_k=None)), (INVALID, dict(rot=None)),
        (INVALID, dict(q=H(0, 0, 0, 0))), (INVALID, dict(q=H(P + 1, 1 << 20, 1 << 14, 128))),
        (INVALID, dict(B=0)), (INVALID, dict(N=-1)), (INVALID, dict(Hq=0)), (INVALID, dict(Hk=0)),
        (UNSUPPORTED, dict(d=127)), (UNSUPPORTED, dict(d=258)), (UNSUPPORTED, dict(d=0)), (UNSUPPORTED, dict(dtype=7, wd=7)),
        (INVALID, dict(rot=R(0, 64, 0, 0, 0, 0, 1.0))), (INVALID, dict(rot=R(P + 4, 64, 0, 0, 0, 0, 1.0))),
        (INVALID, dict(rot=R(P, 63, 0, 0, 0, 0, 1.0))), (INVALID, dict(rot=R(P, 130, 0, 0, 0, 0, 1.0))),
        (INVALID, dict(rot=R(P, 0, 0, 0, 0, 0, 1.0))), (INVALID, dict(rot=R(P, 64, 2, 0, 0, 0, 1.0))),
        (INVALID, dict(rot=R(P, 64, 0, P + 4, 0, 0, 1.0))), (INVALID, dict(rot=R(P, 64, 0, 0, 0, 0, math.nan))),
        (INVALID, dict(rot=R(P, 64, 0, 0, 0, 0, math.inf))),
        (LARGE, dict(B=1 << 16, N=1 << 16)),
        # rows that are written must lie apart: a head stride within a row, a stride of zero, tokens over heads
        (INVALID, dict(out_q=H(2 * P, 1 << 20, 64, 128))), (INVALID, dict(out_q=H(2 * P, 0, 1 << 14, 128))),
        (INVALID, dict(out_q=H(2 * P, 1 << 20, 1024, 128))), (INVALID, dict(out_q=H(2 * P, 1 << 20, -(1 << 14), 128))),
    ]
    for want, change in cases:
        assert _rope(leet, _heads_args(leet, **change)) == want, change
        assert _norm(leet, _heads_args(leet, **change)) == want, change
        if "out_q" not in change and "out_k" not in change:
            assert _back(leet, _heads_args(leet, **change)) == want, change
    for call in (_norm, _back):
        assert call(leet, _heads_args(leet, k=None, out_k=None)) == INVALID
        assert call(leet, _heads_args(leet, wd=leet.LEET_F16)) == UNSUPPORTED
        assert call(leet, _heads_args(leet, eps=-1.0)) == INVALID
        assert call(leet, _heads_args(leet, eps=math.inf)) == INVALID
        assert call(leet, _heads_args(leet, wq=P + 1)) == INVALID
    assert _back(leet, _heads_args(leet, out_q=None)) == INVALID
    assert _back(leet, _heads_args(leet, dq=H(5 * P, 0, 1 << 14, 128))) == INVALID
    assert _back(leet, _heads_args(leet, gk=P + 1)) == INVALID
    # two outputs at one place, or one over the other's input
    for call in (_rope, _norm):
        for change in (dict(out_k=H(2 * P, 1 << 20, 1 << 14, 128)), dict(out_q=H(3 * P, 1 << 20, 1 << 14, 128)),
                       dict(out_k=H(P, 1 << 20, 1 << 14, 128))):
            assert call(leet, _heads_args(leet, **change)) == INVALID, change
    for change in (dict(dk=H(5 * P, 1 << 20, 1 << 14, 128)), dict(dq=H(4 * P, 1 << 20, 1 << 14, 128)),
                   dict(dk=H(P, 1 << 20, 1 << 14, 128)), dict(gk=P, gq=P)):
        assert _back(leet, _heads_args(leet, **change)) == INVALID, change
    # no tokens: legal, and nothing to do
    assert _rope(leet, _heads_args(leet, N=0)) == leet.LEET_OK
    assert _norm(leet, _heads_args(leet, N=0)) == leet.LEET_OK
    assert _back(leet, _heads_args(leet, N=0, gq=None, gk=None)) == leet.LEET_OK


def test_norm_backward_workspace(leet):
    need = leet.qk_norm_rope_workspace_bytes(4, 16, 16, 4096, 128)
    assert need > 0 and need % 512 == 0 and need <= 4 << 20
    assert leet.qk_norm_rope_workspace_bytes(4, 16, 0, 4096, 128) == 0
    assert leet.qk_norm_rope_workspace_bytes(4, 16, 16, 0, 128) == 0


def _scan_args(leet, **change):
    R = lambda at=P, b=1 << 20, n=256: leet._pack_rows(at, b, n)  # noqa: E731
    a = dict(x=R(), gate=R(2 * P), out=R(3 * P), h=R(4 * P), dx=R(5 * P), dgate=R(6 * P), s_in=P, s_out=P, ds_in=2 * P,
             offsets=None, S=0, ws=P, wsb=1 << 40, B=2, N=16, C=256, dtype=leet.LEET_BF16, gd=leet.LEET_F32, mode=1)
    a.update(change)
    return a


def _scan(leet, a):
    return leet.lib.leet_attn_gated_scan(a["x"], a["gate"], a["out"], a["s_in"], a["s_out"], a["offsets"], a["S"], a["ws"],
                                         a["wsb"], a["B"], a["N"], a["C"], a["dtype"], a["gd"], a["mode"], None)


def _scan_back(leet, a):
    return leet.lib.leet_attn_gated_scan_backward(a["out"], a["x"], a["gate"], a["h"], a["dx"], a["dgate"], a["s_in"],
                                                  a["s_out"], a["ds_in"], a["offsets"], a["S"], a["ws"], a["wsb"], a["B"],
                                                  a["N"], a["C"], a["dtype"], a["gd"], a["mode"], None)


def _step(leet, a):
    return leet.lib.leet_attn_gated_scan_step(a["x"], a["gate"], a["out"], a["s_out"], a["B"], a["C"], a["dtype"], a["gd"],
                                              a["mode"], None)


def test_scan_refused(leet):
    R = leet._pack_rows
    INVALID, UNSUPPORTED, LARGE = leet.LEET_ERR_INVALID_ARG, leet.LEET_ERR_UNSUPPORTED, leet.LEET_ERR_TOO_LARGE
    both = [(INVALID, dict(gate=None)), (INVALID, dict(out=None)), (INVALID, dict(gate=R(0, 0, 0))),
            (INVALID, dict(gate=R(2 * P + 2, 1 << 20, 256))), (INVALID, dict(B=0)), (INVALID, dict(C=0)),
            (INVALID, dict(mode=3)), (UNSUPPORTED, dict(dtype=5)), (UNSUPPORTED, dict(gd=leet.LEET_F16)),
            (UNSUPPORTED, dict(dtype=leet.LEET_F32, gd=leet.LEET_BF16))]
    seq = [(INVALID, dict(N=-1)), (INVALID, dict(offsets=P)), (INVALID, dict(offsets=P + 2, B=1)),
           (INVALID, dict(offsets=P, B=1, S=-1)), (INVALID, dict(s_in=P + 2)), (INVALID, dict(s_out=P + 2)),
           (LARGE, dict(C=1 << 29)), (LARGE, dict(N=(1 << 30) + 1)), (LARGE, dict(B=1 << 26))]
    for want, change in both + seq:
        assert _scan(leet, _scan_args(leet, **change)) == want, change
        assert _scan_back(leet, _scan_args(leet, **change)) == want, change
    for want, change in both:
        assert _step(leet, _scan_args(leet, **change)) == want, change
    assert _scan(leet, _scan_args(leet, x=None)) == INVALID
    assert _scan(leet, _scan_args(leet, out=R(3 * P, 1 << 20, 255))) == INVALID     # rows over one another
    assert _scan(leet, _scan_args(leet, out=R(3 * P, 0, 256))) == INVALID
    assert _scan(leet, _scan_args(leet, out=R(P, 1 << 20, 256))) == INVALID         # out is x
    assert _scan_back(leet, _scan_args(leet, x=None, mode=2)) == INVALID
    assert _scan_back(leet, _scan_args(leet, h=None)) == INVALID
    assert _scan_back(leet, _scan_args(leet, dx=R(4 * P, 1 << 20, 256))) == INVALID  # dx is h
    assert _scan_back(leet, _scan_args(leet, dgate=R(5 * P, 1 << 20, 256))) == INVALID
    assert _scan_back(leet, _scan_args(leet, ds_in=P)) == INVALID                    # dstate_in is state_in
    assert _scan_back(leet, _scan_args(leet, dgate=R(6 * P, 1 << 20, 128))) == INVALID
    assert _step(leet, _scan_args(leet, s_out=None)) == INVALID
    assert _step(leet, _scan_args(leet, C=1 << 29)) == LARGE
    # nothing to do
    assert _scan(leet, _scan_args(leet, N=0, s_out=None)) == leet.LEET_OK
    assert _scan(leet, _scan_args(leet, N=0)) == leet.LEET_OK                        # state handed on in place
    assert _scan(leet, _scan_args(leet, B=1, offsets=P, S=0)) == leet.LEET_OK
    assert _scan_back(leet, _scan_args(leet, N=0, ds_in=None)) == leet.LEET_OK


def test_binding_refuses_before_the_library(leet):
    q, freq = torch.zeros(1, 2, 3, 8), torch.ones(4, dtype=torch.float64)
    x, s = torch.zeros(2, 3, 8), torch.zeros(2, 8)
    for call in (lambda: leet.leet_attn_rope(q, freq),                                    # no GPU tensors
                 lambda: leet.leet_attn_rope(q[0], freq),
                 lambda: leet.leet_attn_rope(q, freq, out_k=q),
                 lambda: leet.leet_attn_rope(q, freq, k=q[:, :, :2]),
                 lambda: leet.leet_attn_qk_norm_rope(q, q, torch.ones(7), None, freq),
                 lambda: leet.leet_attn_qk_norm_rope_backward(q, q, q, q, None, None, freq, dq_weight=torch.ones(8)),
                 lambda: leet.leet_attn_gated_scan(x, x),
                 lambda: leet.leet_attn_gated_scan(x[0], x[0]),
                 lambda: leet.leet_attn_gated_scan(x, x, state_in=s[:1]),
                 lambda: leet.leet_attn_gated_scan(x, x, offsets=torch.zeros(3, dtype=torch.int32)),
                 lambda: leet.leet_attn_gated_scan(x[:1], x[:1], offsets=torch.zeros(3)),
                 lambda: leet.leet_attn_gated_scan_backward(x, None, x, x, mode=leet.GATE_SIGMOID),
                 lambda: leet.leet_attn_gated_scan_step(s, s, s[:1])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        leet.leet_attn_rope(q, freq, k=q.half())
    with pytest.raises(TypeError):
        leet.leet_attn_qk_norm_rope(q, q, torch.ones(8).half(), None, freq)
    # what a view looks like to the library, without a GPU
    with pytest.raises(ValueError):
        leet._heads_view(q.transpose(2, 3), "q", torch.Size((1, 2, 8, 3)), q.dtype)
    with pytest.raises(TypeError):
        leet._rows_view(x.half(), "x", x.shape, x.dtype)
    with pytest.raises(ValueError):
        leet._rotation(freq.float(), 0, None, 0, 1.0, 1, 3)
    with pytest.raises(ValueError):
        leet._rotation(freq, 0, torch.zeros(4, dtype=torch.int64), 0, 1.0, 1, 3)


def test_sizes_beyond_an_int_are_refused(leet):
    """Sizes whose products pass 32 or 64 bits, and tensors longer than the library counts, never come to a launch."""
    LARGE, most = leet.LEET_ERR_TOO_LARGE, (1 << 31) - 1
    for Hq, Hk in ((most, most), (most, 1), (1, most), (most - 14, most - 15)):
        for call in (_rope, _norm, _back):
            assert call(leet, _heads_args(leet, B=1, N=1, Hq=Hq, Hk=Hk)) == LARGE
        assert leet.qk_norm_rope_workspace_bytes(1, Hq, Hk, 1, 128) == 0
    for B, N, C in ((most, 1 << 30, 1 << 28), (1 << 30, 1 << 30, 1 << 28), (1 << 22, 1, 1), (1 << 10, 1 << 28, 1 << 26)):
        for call, backward in ((_scan, False), (_scan_back, True)):
            assert call(leet, _scan_args(leet, B=B, N=N, C=C)) == LARGE
            assert leet.gated_scan_workspace_bytes(B, N, C, backward) == 0
    for call in (_scan, _scan_back):
        assert call(leet, _scan_args(leet, B=1, offsets=P, S=(1 << 30) + 1)) == LARGE
    wide = torch.zeros(1)
    freq = torch.ones(1, dtype=torch.float64)
    for big in ((1 << 32) + 1, 1 << 31):
        for shape in ((big, 1, 1, 2), (1, big, 1, 2), (1, 1, big, 2)):
            q = wide.expand(shape)
            for call in (lambda: leet.leet_attn_rope(q, freq), lambda: leet.leet_attn_qk_norm_rope(q, q, None, None, freq),
                         lambda: leet.leet_attn_qk_norm_rope_backward(q, q, q, q, None, None, freq)):
                with pytest.raises(leet.LeetAttnError, match="exceed"):
                    call()
        for shape in ((big, 1, 1), (1, big, 1), (1, 1, big)):
            x = wide.expand(shape)
            for call in (lambda: leet.leet_attn_gated_scan(x, x), lambda: leet.leet_attn_gated_scan_backward(x, None, x, x)):
                with pytest.raises(leet.LeetAttnError, match="exceed"):
                    call()
        for shape in ((big, 1), (1, big)):
            x = wide.expand(shape)
            with pytest.raises(leet.LeetAttnError, match="exceed"):
                leet.leet_attn_gated_scan_step(x, x, wide)


def test_an_output_over_its_input_has_its_strides(leet):
    """In place is the same data and strides; the same address with others would be written before it is read."""
    H, INVALID = leet._pack_heads, leet.LEET_ERR_INVALID_ARG
    for strides in ((1 << 20, 128, 256), (1 << 20, 1 << 13, 128), (1 << 19, 1 << 14, 128), (1 << 20, 1 << 14, 256)):
        other = H(P, *strides)
        for call in (_rope, _norm):
            assert call(leet, _heads_args(leet, out_q=other)) == INVALID, strides
        assert _back(leet, _heads_args(leet, dq=other)) == INVALID, strides
        assert _back(leet, _heads_args(leet, dq=H(2 * P, *strides))) == INVALID, strides    # over dout_q
        assert _back(leet, _heads_args(leet, dk=H(4 * P, *strides))) == INVALID, strides    # over dout_k
    R = leet._pack_rows
    assert _step(leet, _scan_args(leet, out=R(P, 1 << 19, 0), s_out=7 * P)) == INVALID        # over x
    assert _step(leet, _scan_args(leet, out=R(2 * P, 1 << 20, 0), s_out=7 * P)) == INVALID    # over a gate of another type
    assert _step(leet, _scan_args(leet, out=R(2 * P, 1 << 19, 0), gd=leet.LEET_BF16, s_out=7 * P)) == INVALID
    assert _step(leet, _scan_args(leet, out=R(7 * P, 1 << 20, 0), s_out=7 * P)) == INVALID    # over the state


# ---- the forms themselves: gradients against differences ----

def _difference(f, x, dx, e=1e-6):
    return (f(x + e * dx) - f(x - e * dx)) / (2 * e)


@pytest.mark.parametrize("layout", [0, 1])
def test_norm_rope_gradient_form_against_differences(layout):
    g = torch.Generator().manual_seed(5)
    x, dy, dx = (torch.randn(2, 3, 4, 10, generator=g, dtype=torch.float64) for _ in range(3))
    w, dw = (torch.randn(10, generator=g, dtype=torch.float64) for _ in range(2))
    freq, pos = torch.tensor([1.0, 0.3, 0.01], dtype=torch.float64), torch.arange(8).view(2, 4)
    (gx, _), (gw, _) = forms.norm_rope_backward(dy, x, w, freq, pos, layout, scale=1.3)
    by_x = _difference(lambda v: (forms.norm_rope(v, w, freq, pos, layout, 1.3)[0] * dy).sum(), x, dx)
    by_w = _difference(lambda v: (forms.norm_rope(x, v, freq, pos, layout, 1.3)[0] * dy).sum(), w, dw)
    assert abs((gx * dx).sum() - by_x) < 1e-7 and abs((gw * dw).sum() - by_w) < 1e-7


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_scan_gradient_form_against_differences(mode):
    g = torch.Generator().manual_seed(6)
    z, x, dh, dz, dx = (torch.randn(2, 7, 3, generator=g, dtype=torch.float64) for _ in range(5))
    s, ds, d_in = (torch.randn(2, 3, generator=g, dtype=torch.float64) for _ in range(3))
    z = 0.5 + 0.2 * z if mode == 0 else -z.abs() if mode == 1 else z

    def value(z, x, s):
        (h, _), (left, _) = forms.scan(z, x, mode, s)
        return (h * dh).sum() + (left * ds).sum()

    (h, _), _ = forms.scan(z, x, mode, s)
    (gx, _), (gz, _), (gs, _) = forms.scan_backward(dh, z, x, h, mode, s, ds)
    for grad, step, f, at in ((gx, dx, lambda v: value(z, v, s), x), (gz, dz, lambda v: value(v, x, s), z),
                              (gs, d_in, lambda v: value(z, x, v), s)):
        assert abs((grad * step).sum() - _difference(f, at, step)) < 1e-7


def test_the_comparison_rejects_what_is_off():
    ref = torch.tensor([1.0, -2.0, 0.0, float("inf"), float("nan")], dtype=torch.float64)
    bound = torch.zeros_like(ref)
    good = ref.to(torch.bfloat16)
    assert forms.close(good, (ref, bound))
    for i, v in ((0, 1.02), (1, 2.0), (2, 1e-3), (3, 1.0), (4, 0.0)):
        bad = good.clone()
        bad[i] = v
        assert not forms.close(bad, (ref, bound))
