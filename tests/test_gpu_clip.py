"""The norm over many tensors and the clipping on the GPU against 64 bits."""
import math

import pytest
import torch

from layer_forms import close

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = 2.0 ** -24


@pytest.fixture(scope="module")
def leet():
    from paper_2501_02573_amd import binding
    return binding


def tensors(sizes, dtypes, seed=0, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * sigma).to(dtypes[i % len(dtypes)]) for i, n in enumerate(sizes)]


def norm_of(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


def check(leet, ts, limit):
    want = norm_of(ts)
    by = min(1.0, limit / want) if want else 1.0
    on = [t.cuda() for t in ts]
    before = [t.clone() for t in on]
    outs = [torch.full_like(t, 9.0) for t in on]
    norm = leet.leet_attn_clip_gradients(on, limit, outs=outs)
    assert abs(float(norm) - want) <= 4 * U * want   # fp64 but for its own rounding, and the reference's square root's
    assert all(torch.equal(a, b) for a, b in zip(on, before))
    for t, o in zip(ts, outs):
        ref = t.double() * by
        assert close(o, (ref, 3 * U * ref.abs()))    # the factor's rounding and the product's
    again = leet.leet_attn_clip_gradients(on, limit)
    assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(on, outs))
    if by == 1.0:
        assert all(torch.equal(a, b) for a, b in zip(on, before))


SIZES = [1, 2, 7, 8, 9, 0, 255, 8191, 8192, 8193, 16384, 0, 100003]


@pytest.mark.parametrize("dtypes", [[F32], [BF16], [F16], [BF16, F32, F16]])
@pytest.mark.parametrize("limit", [0.5, 1e9, 0.0])
def test_types_and_sizes(leet, dtypes, limit):
    check(leet, tensors(SIZES, dtypes), limit)
    check(leet, tensors([1], dtypes), limit)


def test_more_tensors_than_a_launch_takes(leet):
    check(leet, tensors([(37 * i) % 9000 for i in range(150)], [BF16, F32]), 3.0)
    check(leet, tensors([5] * 64, [F32]), 3.0)
    check(leet, tensors([5] * 65, [F32]), 3.0)


def test_more_tiles_than_workgroups(leet):
    check(leet, tensors([20_000_001, 3], [BF16]), 1.0)


def test_norm_alone(leet):
    ts = [t.cuda() for t in tensors(SIZES, [BF16, F32])]
    before = [t.clone() for t in ts]
    norm = leet.leet_attn_clip_gradients(ts)
    assert abs(float(norm) / norm_of(before) - 1) < 4 * U and all(torch.equal(a, b) for a, b in zip(ts, before))
    kept = torch.zeros(1, device="cuda")
    assert leet.leet_attn_clip_gradients(ts, norm=kept) is kept and torch.equal(kept, norm)


def test_zeros_and_none(leet):
    ts = [torch.zeros(1000, device="cuda"), torch.zeros(0, device="cuda")]
    assert float(leet.leet_attn_clip_gradients(ts, 1.0)) == 0.0 and not ts[0].any()
    assert float(leet.leet_attn_clip_gradients([torch.zeros(0, device="cuda")], 1.0)) == 0.0


def test_large_and_small_values(leet):
    check(leet, tensors(SIZES, [BF16, F32], sigma=1e34), 1.0)
    check(leet, tensors(SIZES, [BF16, F32], sigma=1e-30), 1e-29)
    ts = [torch.full((1000,), 3e38, device="cuda"), torch.ones(5, device="cuda")]   # the norm is beyond a float
    assert math.isinf(float(leet.leet_attn_clip_gradients(ts, 1.0)))
    assert abs(float(ts[0][0]) * math.sqrt(1000) - 1) < 1e-6


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_norm_that_is_not_finite_clips_nothing(leet, bad):
    ts = [t.cuda() for t in tensors(SIZES, [BF16, F32])]
    ts[8][77] = bad
    before, outs = [t.clone() for t in ts], [torch.zeros_like(t) for t in ts]
    norm = leet.leet_attn_clip_gradients(ts, 1.0, outs=outs)
    assert not math.isfinite(float(norm))
    leet.leet_attn_clip_gradients(ts, 1.0)
    for a, b, c in zip(before, outs, ts):
        assert torch.equal(a.view(torch.uint8) if a.numel() else a, b.view(torch.uint8) if b.numel() else b)
        assert torch.equal(a.view(torch.uint8) if a.numel() else a, c.view(torch.uint8) if c.numel() else c)


def test_dense_tensors_of_any_order_and_address(leet):
    g = torch.Generator().manual_seed(3)
    a = torch.randn((30, 40), generator=g).cuda().t()
    b = torch.randn((3001,), generator=g).to(BF16).cuda()[1:]
    c = torch.randn((4, 5, 6, 8), generator=g).cuda().contiguous(memory_format=torch.channels_last)
    want = norm_of([a.cpu(), b.cpu(), c.cpu()])
    kept = [t.double().cpu() for t in (a, b, c)]
    norm = leet.leet_attn_clip_gradients([a, b, c], 2.0)
    assert abs(float(norm) / want - 1) < 4 * U
    for t, k in zip((a, b, c), kept):
        assert close(t, (k * 2.0 / want, 3 * U * (k * 2.0 / want).abs()))


def test_writes_nothing_else(leet):
    buf = torch.full((3, 9000), 4.0, device="cuda", dtype=BF16)
    leet.leet_attn_clip_gradients([buf[0, 3:8201], buf[1, 5:6]], 0.25)
    assert bool((buf[0, :3] == 4).all()) and bool((buf[0, 8201:] == 4).all()) and bool((buf[2] == 4).all())
    assert bool((buf[1, :5] == 4).all()) and bool((buf[1, 6:] == 4).all()) and bool((buf[0, 3:8201] < 1).all())


def test_more_than_two_to_the_31_values(leet):
    t = torch.ones(2 ** 31 + 4099, device="cuda", dtype=BF16)
    t[-1] = 3.0
    want = math.sqrt(2 ** 31 + 4098 + 9)
    norm = leet.leet_attn_clip_gradients([t], want / 2)
    assert abs(float(norm) / want - 1) < 4 * U
    assert float(t[-1]) == 1.5 and float(t[0]) == 0.5 and float(t[2 ** 31]) == 0.5


def test_graph_and_streams(leet):
    sets = [[t.cuda() for t in tensors(SIZES + [70000], [BF16, F32], seed)] for seed in (1, 2)]

    def call(ts):
        outs = [torch.empty_like(t) for t in ts]
        return outs + [leet.leet_attn_clip_gradients(ts, 1.0, outs=outs)]

    want = [call(t) for t in sets]
    torch.cuda.synchronize()
    got = []
    for t in sets:
        with torch.cuda.stream(torch.cuda.Stream()):
            got.append(call(t))
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for a, b in zip(want, got) for p, q in zip(a, b))
    graphs, kept = [], []
    for t in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            kept.append(call(t))
    for i in range(3):
        for t in sets:
            t[3].mul_(-0.5)
        eager = [call(t) for t in sets]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for a, b in zip(eager, kept) for p, q in zip(a, b))


@pytest.mark.parametrize("dtypes", [[F32], [BF16], [F16, F32]])
def test_sizes_about_a_tile(leet, dtypes):
    check(leet, tensors([16383, 16385, 32767, 32768, 0, 32769, 16384, 49153], dtypes), 0.7)
    check(leet, tensors([16383], dtypes), 0.7)


def test_unaligned_tensors_past_the_cache(leet):
    n = 70_000_001   # in, out: 280 MB
    buf, to = torch.ones(n + 2, device="cuda", dtype=BF16), torch.full((n + 2,), 7.0, device="cuda", dtype=BF16)
    norm = leet.leet_attn_clip_gradients([buf[1:-1]], n ** 0.5 / 4, outs=[to[1:-1]])
    assert abs(float(norm) / n ** 0.5 - 1) < 4 * U and bool((buf == 1).all())
    assert bool((to[1:-1] == 0.25).all()) and float(to[0]) == 7.0 and float(to[-1]) == 7.0
