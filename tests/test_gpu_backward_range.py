"""The attention's backward pass in fp16 over that type's whole range: gradients of 2^-18, scores and states beyond 65504, states
of any size.  The definition in 64 bits is that of training_forms.py.

Bounds.  v = 2^-11 is half a step of fp16, u = 2^-24.  What is formed inside is brought into fp16's range by powers of two before it
is rounded, so a rounding is v of the value or, of values far below the largest that are scaled together, half of the least number,
2^-25, at that scale.  Scores: the token's largest at 2^14, so 2^-39 of it.  States: their largest at 4 or more, 2^-27 of it.  What is
added to a state: the largest z at 2^8 or more, 2^-33 of it; where dstate_in is wanted at 2^14 or more, 2^-39.  All this comes
beside ``attention_backward``'s bounds in fp32 (u) and its 3 v."""
import pytest
import torch

import training_forms as forms
from test_gpu_backward import decays, held, on, wide

pytestmark = pytest.mark.gpu

F16 = torch.float16
SCORE, STATE, SUMMAND, FINE = 2.0 ** -39, 2.0 ** -27, 2.0 ** -33, 2.0 ** -39


@pytest.fixture(scope="module")
def leet():
    from paper_2501_02573_amd import binding
    return binding


def bounded(dout, q, k, v, gamma, state, dstate):
    """``attention_backward`` with the bounds of the header, and nothing for fp16's least number."""
    form = forms.attention_backward(dout, q, k, v, gamma, state, dstate, dtype=torch.float32)
    most = forms._gradients(*(None if t is None else t.abs() for t in (dout, q, k, v)), gamma,
                            *(None if t is None else t.abs() for t in (state, dstate)))

    def row(t):     # sum over the tokens
        return t.abs().sum(2, keepdim=True)

    def each(t):    # sum over a token's elements
        return t.abs().sum(3, keepdim=True)

    def largest(t):
        return t.abs().amax((2, 3), keepdim=True)

    def state_off(y, z, s):
        """How far an element of a state may be off beside u: what was added to it, and itself as an operand."""
        sums = (y.abs().transpose(-1, -2) @ z.abs()).amax((2, 3), keepdim=True) + (0 if s is None else largest(s))
        return SUMMAND * row(y).amax(-1, keepdim=True) * largest(z) + STATE * sums

    P, dP = (q.abs() @ k.abs().transpose(-1, -2)), (dout.abs() @ v.abs().transpose(-1, -2))
    extra = [SCORE * dP.amax(-1, keepdim=True) * row(k) + each(dout) * state_off(v, k, state),
             SCORE * dP.amax(-2).unsqueeze(-1) * row(q) + each(v) * state_off(dout, q, dstate),
             SCORE * P.amax(-2).unsqueeze(-1) * row(dout) + each(k) * state_off(q, dout, dstate)]
    out = [(g, b + 3 * 2.0 ** -11 * m + e) for (g, b), m, e in zip(form[:3], most, extra)]
    left = FINE * row(q).amax(-1, keepdim=True) * dout.abs().amax((2, 3), keepdim=True)
    # The matrix instructions add products to 2^-24 of the largest one's exponent, and an operand below 2^-14, fp16's least normal
    # number, has that exponent there: of the two, q is an operand as it came.
    least = torch.where(q == 0, q, q.abs().clamp(min=2.0 ** -14))
    wider = forms.attention_backward(dout.abs(), least, k.abs(), v.abs(), gamma, *(None if t is None else t.abs() for t in (state, dstate)))
    return out + [(form[3][0], wider[3][1] + left)]


def inputs(N, r, dv, scales, states=True, seed=0, B=1, H=3):
    """dout, q, k, v with elements of about ``scales``, states of what goes into them."""
    g = torch.Generator().manual_seed(seed)
    sd, sq, sk, sv = scales
    do, q, k, v = (torch.randn((B, H, N, w), generator=g) * s for w, s in ((dv, sd), (r, sq), (r, sk), (dv, sv)))
    s = torch.randn((B, H, r, dv), generator=g) * sk * sv if states else None
    ds = torch.randn((B, H, r, dv), generator=g) * sq * sd if states else None
    return [t.half() for t in (do, q, k, v)] + [s, ds]


def check(leet, ts, gamma, segments, few):
    do, q, k, v, s, ds = ts
    B, H, N, r = q.shape
    mask = leet.LEET_MASK_DECAY if gamma is not None else leet.LEET_MASK_CAUSAL
    left = torch.full((B, H, r, v.shape[3]), float("nan"), device="cuda")
    want = bounded(*wide(do, q, k, v), torch.ones(H, dtype=torch.float64) if gamma is None else gamma.double(), *wide(s, ds))
    args = on(do, q, k, v, gamma)
    for wanted in (left, None):   # the state's gradient is taken to fp32 where it is wanted
        got = leet.leet_attn_backward(*args, state_in=on(s)[0], dstate_out=on(ds)[0], dstate_in=wanted, segments=segments, mask=mask)
        for name, a, b in zip(("dq", "dk", "dv"), got, want):
            held(name, a, b)
            # Independent roundings of up to half a step: the output's, and in longer calls the score's and the state's
            alone = float((b[0].half().double() - b[0]).norm())
            off = float((a.double().cpu() - b[0]).norm())
            if a.numel() > 4096:
                assert off <= (1.1 if few else 3 ** 0.5) * alone, (name, off / alone)
    held("dstate_in", left, want[3])


SHAPES = [(64, 64), (128, 128), (128, 256)]
#          dout       q        k        v
SCALES = [(2.0 ** -10, 0.125, 0.125, 0.125), (2.0 ** -14, 1.0, 1.0, 1.0), (2.0 ** -18, 1.0, 1.0, 1.0),
          (2.0 ** -16, 2.0 ** -8, 8.0, 8.0),
          (2.0 ** 10, 2.0 ** -14, 2.0 ** -13, 2.0 ** 8),    # scores of up to 2^21 for dq and dk, whose other operands are small
          (2.0 ** 10, 2.0 ** 8, 2.0 ** -14, 2.0 ** -14),    # states of 2^20 for dk and dv
          (2.0 ** -13, 2.0 ** -8, 2.0 ** 9, 2.0 ** 9),      # states of 2^20 for dq
          (2.0 ** 13, 2.0 ** -14, 2.0 ** -14, 2.0 ** -14)]


@pytest.mark.parametrize("scales", SCALES)
@pytest.mark.parametrize("r,dv", SHAPES)
@pytest.mark.parametrize("N,segments", [(1, 0), (100, 0), (300, 0), (300, 1), (333, 3)])
def test_small_and_large_values(leet, scales, r, dv, N, segments):
    check(leet, inputs(N, r, dv, scales), decays(3), segments, N <= 128)
    check(leet, inputs(N, r, dv, scales, seed=1), None, segments, N <= 128)


@pytest.mark.parametrize("r,dv", SHAPES)
@pytest.mark.parametrize("segments", [0, 2])
def test_values_of_many_sizes_in_one_sequence(leet, r, dv, segments):
    """Tokens and channels of sizes that lie 2^20 apart."""
    do, q, k, v, s, ds = inputs(400, r, dv, (1.0, 1.0, 1.0, 1.0))
    token = 2.0 ** (torch.arange(400) % 21 - 14.0)[:, None]
    channel = 2.0 ** -(torch.arange(max(r, dv)) % 11.0)
    ts = [(do * token).half(), q * channel[:r].half(), k, (v * channel[:dv]).half(), s, ds]
    want = bounded(*wide(*ts[:4]), decays(3).double(), *wide(s, ds))
    left = torch.empty_like(ds, device="cuda")
    got = leet.leet_attn_backward(*on(*ts[:4], decays(3)), state_in=on(s)[0], dstate_out=on(ds)[0], dstate_in=left, segments=segments)
    for name, a, b in zip(("dq", "dk", "dv", "dstate_in"), got + (left,), want):
        held(name, a, b)


@pytest.mark.parametrize("r,dv", SHAPES)
@pytest.mark.parametrize("size", [1e-30, 1e30])
@pytest.mark.parametrize("N,segments", [(70, 0), (200, 1), (200, 2)])
def test_states_of_any_size(leet, r, dv, size, N, segments):
    """Entering states far beyond fp16 where what they meet is zero: nothing becomes infinite, dstate_in is fp32's."""
    do, q, k, v, s, ds = inputs(N, r, dv, (2.0 ** -12, 1.0, 1.0, 1.0))
    gamma = decays(3)
    left = torch.empty_like(ds, device="cuda")
    zero = torch.zeros_like
    got = leet.leet_attn_backward(*on(do, q, zero(k), zero(v), gamma), dstate_out=on(ds * size)[0], dstate_in=left, segments=segments)
    want = bounded(*wide(do, q, zero(k), zero(v)), gamma.double(), None, (ds * size).double())
    assert not got[0].any() and not got[1].any() and not got[2].any()
    held("dstate_in", left, want[3])
    got = leet.leet_attn_backward(*on(zero(do), q, k, v, gamma), state_in=on(s * size)[0], segments=segments)
    assert not got[0].any() and not got[1].any() and not got[2].any()


@pytest.mark.parametrize("r,dv", SHAPES)
@pytest.mark.parametrize("N,segments", [(70, 0), (300, 1), (300, 2)])
def test_an_infinity_stays_in_its_channel(leet, r, dv, N, segments):
    """An infinite key makes its own channel of dq infinite or NaN behind it, and the others are what they were."""
    do, q, k, v, s, ds = on(*inputs(N, r, dv, (1.0, 1.0, 1.0, 1.0)))
    gamma = decays(3).cuda()
    want = leet.leet_attn_backward(do, q, k, v, gamma, state_in=s, segments=segments)[0]
    k[0, 1, 5, 7] = float("inf")
    got = leet.leet_attn_backward(do, q, k, v, gamma, state_in=s, segments=segments)[0]
    others = [c for c in range(r) if c != 7]
    assert torch.equal(got[..., others], want[..., others]) and not bool(got[0, 1, 64:, 7].isfinite().any())


@pytest.mark.parametrize("N,segments", [(100, 0), (300, 1), (300, 2)])
def test_tokens_without_a_gradient(leet, N, segments):
    """Padding: gradients of zero give zeros, and leave the others what they are without it."""
    do, q, k, v, _, _ = on(*inputs(N, 128, 128, (2.0 ** -14, 1.0, 1.0, 1.0), states=False))
    gamma = decays(3).cuda()
    do[:, :, N // 2:] = 0
    dq, dk, dv = leet.leet_attn_backward(do, q, k, v, gamma, segments=segments)
    assert not dq[:, :, N // 2:].any() and not dk[:, :, N // 2:].any() and not dv[:, :, N // 2:].any()
    assert bool(dq[:, :, :N // 2].any()) and bool(dk.isfinite().all()) and bool(dv.isfinite().all())


@pytest.mark.parametrize("r,dv", SHAPES)
@pytest.mark.parametrize("segments", [0, 1, 3])
def test_states_that_fade(leet, r, dv, segments):
    """Behind what made them states fall below everything that fp32 holds, over many tokens that add nothing."""
    do, q, k, v, _, _ = inputs(900, r, dv, (1.0, 1.0, 1.0, 1.0), states=False)
    gamma = torch.tensor([0.5, 0.75, 0.9])
    late = torch.arange(900)[:, None] >= 64
    early = torch.arange(900)[:, None] < 900 - 64
    for ts in ([do, q, k.masked_fill(late, 0), v.masked_fill(late, 0)], [do.masked_fill(early, 0), q.masked_fill(early, 0), k, v]):
        want = bounded(*wide(*ts), gamma.double(), None, None)
        left = torch.empty((1, 3, r, dv), device="cuda")
        got = leet.leet_attn_backward(*on(*ts, gamma), dstate_in=left, segments=segments)
        for name, a, b in zip(("dq", "dk", "dv", "dstate_in"), got + (left,), want):
            held(name, a, b)


@pytest.mark.parametrize("r,dv", SHAPES)
@pytest.mark.parametrize("decay", [True, False])
@pytest.mark.parametrize("segments", [1, 2])
def test_the_states_gradient_of_small_channels(leet, r, dv, decay, segments):
    """Channels of dout that lie 2^21 apart: those of the state's gradient are off by 2^-39 of the largest, no more."""
    do, q, k, v, _, _ = inputs(300, r, dv, (1.0, 1.0, 1.0, 1.0), states=False)
    do = (do * 2.0 ** (10 - torch.arange(dv) % 22.0)).half()
    gamma = decays(3) if decay else None
    left = torch.empty((1, 3, r, dv), device="cuda")
    leet.leet_attn_backward(*on(do, q, k, v, gamma), dstate_in=left, segments=segments,
                            mask=leet.LEET_MASK_DECAY if decay else leet.LEET_MASK_CAUSAL)
    want = bounded(*wide(do, q, k, v), gamma.double() if decay else torch.ones(3, dtype=torch.float64), None, None)
    held("dstate_in", left, want[3])


@pytest.mark.parametrize("r,dv", SHAPES)
@pytest.mark.parametrize("size", [2.0 ** -60, 1e30])
@pytest.mark.parametrize("N,segments", [(70, 0), (200, 1), (200, 2)])
def test_states_of_any_size_without_decay(leet, r, dv, size, N, segments):
    do, q, k, v, s, ds = inputs(N, r, dv, (2.0 ** -12, 1.0, 1.0, 1.0))
    zero, ones = torch.zeros_like, torch.ones(3, dtype=torch.float64)
    left = torch.empty_like(ds, device="cuda")
    causal = leet.LEET_MASK_CAUSAL
    got = leet.leet_attn_backward(*on(do, q, zero(k), zero(v)), None, dstate_out=on(ds * size)[0], dstate_in=left, segments=segments,
                                  mask=causal)
    want = bounded(*wide(do, q, zero(k), zero(v)), ones, None, (ds * size).double())
    assert not got[0].any() and not got[1].any() and not got[2].any()
    held("dstate_in", left, want[3])
    got = leet.leet_attn_backward(*on(do, q, k, v), None, state_in=on(s * 2.0 ** -20)[0], segments=segments, mask=causal)
    for name, a, b in zip(("dq", "dk", "dv"), got, bounded(*wide(do, q, k, v), ones, (s * 2.0 ** -20).double(), None)):
        held(name, a, b)
    got = leet.leet_attn_backward(*on(zero(do), q, k, v), None, state_in=on(s * size)[0], segments=segments, mask=causal)
    assert not got[0].any() and not got[1].any() and not got[2].any()
