"""What the attention's backward pass rounds, by kernel: decays at the ends of their range, and errors over many values.

An output in 16 bits is rounded once.  Beside that a score is rounded once as an operand, and so is the state; the one has the share
of an output that comes from its own chunk, the other the rest, so with independent roundings of one size, relative to what they
round, the variances are 1 (the output's) and 1 (both shares together): errors are 2^0.5 times those of rounding the outputs
alone.  What is added to a state has twice the bits and takes no part; with one term it would be 3^0.5.  A tenth is let
through for outputs whose terms cancel."""
import pytest
import torch

import training_forms as forms
from test_gpu_backward import check, decays, inputs, on, wide

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def leet():
    from paper_2501_02573_amd import binding
    return binding


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("N", [193, 256, 333])
@pytest.mark.parametrize("segments", [0, 1, 2])
def test_extreme_decays_at_width_128(leet, dtype, N, segments):
    """Few sequences of three chunks and more, in one segment: a compute unit each."""
    gamma = torch.tensor([0.0, 1.0, 1e-30, 0.5, 1 - 2.0 ** -12, 1e-3])
    check(leet, 1, 6, N, 128, 128, dtype, gamma, segments=segments)
    check(leet, 1, 6, N, 128, 128, dtype, gamma, segments=segments, states=False)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("gamma", [0.0, 1e-30, 0.5, 1.0])
def test_extreme_decays_at_width_256(leet, dtype, gamma):
    check(leet, 1, 2, 200, 128, 256, dtype, torch.tensor([gamma, 0.9]))
    check(leet, 1, 2, 200, 128, 256, dtype, torch.tensor([gamma, 0.9]), segments=2)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("r,dv", [(64, 64), (128, 128), (128, 256)])
@pytest.mark.parametrize("segments", [1, 3])
@pytest.mark.parametrize("decay", [True, False])
def test_two_roundings(leet, dtype, r, dv, segments, decay):
    H = 4
    do, q, k, v, s, ds = inputs(1, H, 700, r, dv, dtype, True)
    gamma = decays(H) if decay else None
    left = torch.empty((1, H, r, dv), device="cuda")
    want = forms.attention_backward(*wide(do, q, k, v), torch.ones(H, dtype=torch.float64) if gamma is None else gamma.double(),
                                    *wide(s, ds), dtype=dtype)
    for wanted in (None, left):
        got = leet.leet_attn_backward(*on(do, q, k, v, gamma), state_in=on(s)[0], dstate_out=on(ds)[0], dstate_in=wanted,
                                      segments=segments, mask=leet.LEET_MASK_DECAY if decay else leet.LEET_MASK_CAUSAL)
        for name, a, (b, _) in zip(("dq", "dk", "dv"), got, want):
            alone = float((b.to(dtype).double() - b).norm())
            off = float((a.double().cpu() - b).norm())
            assert off <= 1.1 * 2 ** 0.5 * alone, (name, off / alone)
