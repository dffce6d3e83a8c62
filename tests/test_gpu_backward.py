"""The attention's backward pass on the GPU against its formula in 64 bits."""
import pytest
import torch

import training_forms as forms
from layer_forms import close

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def leet():
    from paper_2501_02573_amd import binding
    return binding


def inputs(B, H, N, r, dv, dtype, states, seed=0):
    g = torch.Generator().manual_seed(seed)
    q, k = (torch.randn((B, H, N, r), generator=g) * r ** -0.5 for _ in range(2))
    v, do = torch.randn((B, H, N, dv), generator=g) * dv ** -0.5, torch.randn((B, H, N, dv), generator=g)
    s = [torch.randn((B, H, r, dv), generator=g) if states else None for _ in range(2)]
    return [t.to(dtype) for t in (do, q, k, v)] + s


def on(*ts):
    return [None if t is None else t.cuda() for t in ts]


def wide(*ts):
    return [None if t is None else t.double() for t in ts]


def held(name, got, form):
    """Asserts that ``got`` is within its bound; says how far it is off where it is not."""
    if not close(got, form):
        off = (got.double().cpu() - form[0]).abs() / form[1]
        raise AssertionError(f"{name}: {float(off.max()):.3g} of the bound at {int(off.argmax())}, finite {bool(off.isfinite().all())}")


def check(leet, B, H, N, r, dv, dtype, gamma, states=True, segments=0, seed=0):
    do, q, k, v, s, ds = inputs(B, H, N, r, dv, dtype, states, seed)
    mask = leet.LEET_MASK_DECAY if gamma is not None else leet.LEET_MASK_CAUSAL
    left = torch.full((B, H, r, dv), float("nan"), device="cuda")
    args = on(do, q, k, v, gamma)
    got = leet.leet_attn_backward(*args, state_in=on(s)[0], dstate_out=on(ds)[0], dstate_in=left, segments=segments, mask=mask)
    g = torch.ones(H, dtype=torch.float64) if gamma is None else gamma.double()
    want = forms.attention_backward(*wide(do, q, k, v), g, *wide(s, ds), dtype=dtype)
    for name, a, b in zip(("dq", "dk", "dv", "dstate_in"), got + (left,), want):
        held(name, a, b)
    if dtype != F32:
        # without the state's gradient wanted its summands are rounded to 16 bits; over many values the errors are
        # independent, each 0.6 of half a step in the mean: sqrt(4) 0.6 of it with the output's own rounding
        got = leet.leet_attn_backward(*args, state_in=on(s)[0], dstate_out=on(ds)[0], segments=segments, mask=mask)
        for name, a, b in zip(("dq", "dk", "dv"), got, want):
            held(name, a, b)
            if a.numel() > 4096 and float(b[0].norm()) > 1e-3:
                assert float((a.double().cpu() - b[0]).norm() / b[0].norm()) < 1.2 * torch.finfo(dtype).eps / 2, name


def decays(H):
    return (1 - 2.0 ** -torch.linspace(2.0, 9.0, H)).float()


@pytest.mark.parametrize("N", [1, 2, 31, 63, 64, 65, 127, 128, 129, 200, 321])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths(leet, N, dtype, d):
    check(leet, 2, 3, N, d, d, dtype, decays(3))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("N", [1, 65, 400])
def test_rank_and_value_width_apart(leet, N, dtype):
    check(leet, 1, 3, N, 128, 256, dtype, decays(3))
    check(leet, 1, 3, N, 128, 256, dtype, decays(3), segments=3)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("segments", [1, 2, 3, 5, 100])
def test_segments(leet, dtype, segments):
    check(leet, 1, 5, 700, 64, 64, dtype, decays(5), segments=segments)
    check(leet, 3, 1, 449, 128, 128, dtype, decays(1), segments=segments, states=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_no_decay(leet, dtype, d):
    check(leet, 2, 2, 300, d, d, dtype, None)
    check(leet, 2, 2, 300, d, d, dtype, None, segments=2, states=False)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_extreme_decays(leet, dtype):
    gamma = torch.tensor([0.0, 1.0, 1e-30, 0.5, 1 - 2.0 ** -12, 1e-3])
    check(leet, 1, 6, 200, 64, 64, dtype, gamma)
    check(leet, 1, 6, 200, 128, 128, dtype, gamma, segments=3)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_tokens(leet, dtype):
    do, q, k, v, s, ds = on(*inputs(2, 2, 0, 64, 64, dtype, True))
    left = torch.full_like(ds, 7.0)
    got = leet.leet_attn_backward(do, q, k, v, decays(2).cuda(), state_in=s, dstate_out=ds, dstate_in=left)
    assert [t.shape for t in got] == [q.shape] * 3 and torch.equal(left, ds)
    leet.leet_attn_backward(do, q, k, v, decays(2).cuda(), dstate_in=left)
    assert not left.any()


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F16, 64), (F32, 64), (F32, 128)])
def test_writes_its_outputs_and_nothing_else(leet, dtype, d):
    B, H, N = 1, 3, 201
    do, q, k, v, s, ds = on(*inputs(B, H, N, d, d, dtype, True))
    n, guard = B * H * N * d, 64
    bufs = [torch.full((n + 2 * guard,), 5.0, dtype=dtype, device="cuda") for _ in range(3)]
    outs = [b[guard:guard + n].view(B, H, N, d) for b in bufs]
    need = leet.backward_workspace_bytes(B, H, N, d, d, leet._dtype_code(q), 2)
    assert need == 2 * B * H * d * d * 4
    ws = torch.full((need + 512,), 0xff, dtype=torch.uint8, device="cuda")
    kept = [t.clone() for t in (do, q, k, v, s, ds)]
    got = leet.leet_attn_backward(do, q, k, v, decays(H).cuda(), *outs, state_in=s, dstate_out=ds, workspace=ws[256:256 + need],
                                  segments=2)
    want = leet.leet_attn_backward(do, q, k, v, decays(H).cuda(), state_in=s, dstate_out=ds, segments=2)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for b in bufs:
        assert bool((b[:guard] == 5.0).all()) and bool((b[guard + n:] == 5.0).all())
    assert bool((ws[:256] == 0xff).all()) and bool((ws[256 + need:] == 0xff).all())
    assert all(torch.equal(a, b) for a, b in zip(kept, (do, q, k, v, s, ds)))


def test_pieces_give_what_the_whole_gives(leet):
    """A sequence in two pieces, the state handed on by the forward call and its gradient handed back."""
    B, H, N, cut, d = 2, 2, 260, 100, 64
    do, q, k, v, s, ds = on(*inputs(B, H, N, d, d, F32, True))
    gamma = decays(H).cuda()
    left = torch.empty_like(ds)
    whole = leet.leet_attn_backward(do, q, k, v, gamma, state_in=s, dstate_out=ds, dstate_in=left)
    a, b = ([t[:, :, :cut].contiguous() for t in (do, q, k, v)], [t[:, :, cut:].contiguous() for t in (do, q, k, v)])
    mid, dmid, first = torch.empty_like(s), torch.empty_like(s), torch.empty_like(s)
    leet.leet_attn_forward_ex(a[1], a[2], a[3], gamma, state_in=s, state_out=mid)
    late = leet.leet_attn_backward(*b, gamma, state_in=mid, dstate_out=ds, dstate_in=dmid)
    early = leet.leet_attn_backward(*a, gamma, state_in=s, dstate_out=dmid, dstate_in=first)
    # both are fp32 sums of some 300 products, off by a few 2^-24 sqrt(300) of the largest
    for w, x, y in zip(whole, early, late):
        assert float((torch.cat((x, y), 2) - w).abs().max() / w.abs().max()) < 4 * 2.0 ** -24 * 300 ** 0.5
    assert float((first - left).abs().max() / left.abs().max()) < 4 * 2.0 ** -24 * 300 ** 0.5


def test_offsets_beyond_two_to_the_31(leet):
    B, H, N, d = 1, 36, 500000, 128   # 2.3e9 elements a tensor
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, do = (torch.randn((B, H, N, d), generator=g, device="cuda", dtype=torch.bfloat16).mul_(0.1) for _ in range(4))
    gamma = decays(H).cuda()
    got = leet.leet_attn_backward(do, q, k, v, gamma, segments=4)
    for h in (0, H - 1):
        alone = leet.leet_attn_backward(*(t[:, h:h + 1].clone() for t in (do, q, k, v)), gamma[h:h + 1].clone(), segments=4)
        assert all(torch.equal(a[:, h:h + 1], b) for a, b in zip(got, alone))


def test_streams_and_graphs(leet):
    """Two calls at once on streams of their own, and captured ones replayed beside eager ones: the calls share nothing."""
    B, H, N, d = 2, 4, 1500, 128
    sets = [on(*inputs(B, H, N, d, d, BF16, True, seed)) for seed in (1, 2)]
    gamma = decays(H).cuda()

    def call(t):
        left = torch.empty_like(t[5])
        return leet.leet_attn_backward(*t[:4], gamma, state_in=t[4], dstate_out=t[5], dstate_in=left, segments=3) + (left,)

    want = [call(t) for t in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        got = []
        for st, t in zip(streams, sets):
            with torch.cuda.stream(st):
                got.append(call(t))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(want, got) for x, y in zip(a, b))
    graphs, kept = [], []
    for t in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            kept.append(call(t))
    for i in range(3):
        for t in sets:
            t[0].mul_(-0.5)
        eager = [call(t) for t in sets]
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(eager, kept) for x, y in zip(a, b))


def test_gradients_by_a_function_of_the_callers(leet):
    """Wrapped with the forward call for autograd: the gradients of the 64-bit formula."""
    B, H, N, d = 2, 2, 150, 64

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, gamma):
            ctx.save_for_backward(q, k, v, gamma)
            return leet.leet_attn_forward(q, k, v, gamma)

        @staticmethod
        def backward(ctx, do):
            q, k, v, gamma = ctx.saved_tensors
            return leet.leet_attn_backward(do.contiguous(), q, k, v, gamma) + (None,)

    do, q, k, v, _, _ = inputs(B, H, N, d, d, F32, False)
    gamma = decays(H)
    leaves = [t.cuda().requires_grad_() for t in (q, k, v)]
    got = torch.autograd.grad(Attention.apply(*leaves, gamma.cuda()), leaves, do.cuda())
    plain = [t.double().requires_grad_() for t in (q, k, v)]
    want = torch.autograd.grad(forms.attention(*plain, gamma.double())[0], plain, do.double())
    bounds = [b for _, b in forms.attention_backward(*wide(do, q, k, v), gamma.double())]
    for a, w, b in zip(got, want, bounds):
        held("gradient", a, (w, b))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("segments", [0, 1])
def test_more_sequences_than_compute_units(leet, dtype, segments):
    check(leet, 9, 10, 130, 128, 128, dtype, decays(10), segments=segments)
    check(leet, 9, 10, 64, 128, 128, dtype, None, segments=segments, states=False)


def test_offsets_beyond_two_to_the_31_in_one_segment(leet):
    B, H, N, d = 1, 36, 500000, 128   # 2.3e9 elements a tensor
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v, do = (torch.randn((B, H, N, d), generator=g, device="cuda", dtype=torch.bfloat16).mul_(0.1) for _ in range(4))
    gamma = decays(H).cuda()
    got = leet.leet_attn_backward(do, q, k, v, gamma, segments=1)
    for h in (0, H - 1):
        alone = leet.leet_attn_backward(*(t[:, h:h + 1].clone() for t in (do, q, k, v)), gamma[h:h + 1].clone(), segments=1)
        assert all(torch.equal(a[:, h:h + 1], b) for a, b in zip(got, alone))


@pytest.mark.parametrize("dtype,d,dv", [(BF16, 128, 128), (F16, 64, 64), (BF16, 128, 256), (F32, 128, 128)])
def test_calls_repeat_eager_on_streams_and_replayed(leet, dtype, d, dv):
    """The plan is the library's own; every replay is compared with an eager call on the same inputs."""
    sets = [on(*inputs(2, 4, 900, d, dv, dtype, True, seed)) for seed in (1, 2)]
    gamma = decays(4).cuda()

    def call(t):
        return leet.leet_attn_backward(*t[:4], gamma, state_in=t[4], dstate_out=t[5])

    want = [call(t) for t in sets]
    torch.cuda.synchronize()
    got = []
    for t in sets:
        with torch.cuda.stream(torch.cuda.Stream()):
            got.append(call(t))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for a, b in zip(want, got) for x, y in zip(a, b))
    graphs, kept = [], []
    for t in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            kept.append(call(t))
    for _ in range(3):
        for t in sets:
            t[0].mul_(-0.5)
        eager = [call(t) for t in sets]
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(eager, kept) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_value_that_is_not_finite_stays_in_its_sequence(leet, dtype):
    do, q, k, v, _, _ = on(*inputs(1, 3, 150, 128, 128, dtype, False))
    gamma = decays(3).cuda()
    want = leet.leet_attn_backward(do, q, k, v, gamma)
    v[0, 1, 70, 5] = float("nan")
    got = leet.leet_attn_backward(do, q, k, v, gamma)
    for a, b in zip(want, got):
        assert torch.equal(a[:, 0::2], b[:, 0::2])
    assert bool(got[0][0, 1, 70:].isnan().all()) and bool(got[1][0, 1, 70].isnan().all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128), (128, 256)])
def test_a_few_tokens_lose_nothing_but_the_outputs_rounding(leet, dtype, d, dv):
    for N in (1, 2, 3, 17, 64, 65, 128):
        do, q, k, v, s, ds = inputs(1, 2, N, d, dv, dtype, N % 2 == 1, N)
        gamma = decays(2)
        got = leet.leet_attn_backward(*on(do, q, k, v, gamma), state_in=on(s)[0], dstate_out=on(ds)[0])
        want = forms.attention_backward(*wide(do, q, k, v), gamma.double(), *wide(s, ds), dtype=dtype)
        for a, (b, _) in zip(got, want):
            # operands in two terms are off by eps^2 / 4 (fp16: by half of its least number, 2^-25, where values are some 2^-9
            # or more, a sixteenth of eps / 2); all else is the one rounding at the store, a tenth of it let through
            alone = float((b.to(dtype).double() - b).norm())
            assert float((a.double().cpu() - b).norm()) <= 1.1 * alone, N
