"""Limits of the clipping that float32 does not hold."""
import pytest
import torch


@pytest.fixture(scope="module")
def leet():
    from paper_2501_02573_amd import binding
    return binding


@pytest.fixture
def limits(leet, monkeypatch):
    """What reaches the library, which takes a float and writes no output where that is infinite."""
    seen = []

    class Library:
        @staticmethod
        def leet_attn_clip_gradients(grads, count, limit, *rest):
            seen.append(leet.ctypes.c_float(limit).value)
            return leet.LEET_OK

        leet_attn_clip_gradients_workspace_bytes = leet.lib.leet_attn_clip_gradients_workspace_bytes

    class Gradient:
        """As much of a GPU tensor as the call looks at."""
        dtype, shape = torch.float32, (4,)
        get_device, is_contiguous, data_ptr, numel = lambda s: 0, lambda s: True, lambda s: 256, lambda s: 4

    monkeypatch.setattr(leet, "lib", Library)
    monkeypatch.setattr(leet, "_call_on", lambda index, fn, *args: fn(*args))
    norm = Gradient()
    norm.numel = lambda: 1
    space = torch.empty(8192, dtype=torch.uint8)
    monkeypatch.setattr(space, "get_device", lambda: 0, raising=False)

    def call(limit, outs):
        leet.leet_attn_clip_gradients([Gradient()], limit, outs=[Gradient()] if outs else None, norm=norm, workspace=space)
        return seen.pop()

    return call


@pytest.mark.parametrize("limit", [3.5e38, 1e39, 1e47, 1.7976931348623157e308])
def test_outs_are_never_left_unwritten(limits, limit):
    with pytest.raises(ValueError):
        limits(limit, True)


@pytest.mark.parametrize("limit", [3.5e38, 1e39, 2.0 ** 156])
def test_limits_that_a_norm_can_exceed_are_not_taken_as_none(limits, limit):
    with pytest.raises(ValueError):
        limits(limit, False)


def test_limits_that_no_norm_reaches_are_none(limits):
    # fewer than 2^64 values below 2^128 have a norm below 2^160
    assert limits(2.0 ** 160, False) == limits(1.7976931348623157e308, False) == limits(None, False) == float("inf")


def test_limits_of_float32_arrive(limits):
    most = torch.finfo(torch.float32).max
    for limit in (0.0, 0.5, 1, most):
        assert limits(limit, True) == limits(limit, False) == limit


@pytest.mark.gpu
@pytest.mark.parametrize("limit", [1e39, 1.7976931348623157e308])
def test_on_the_gpu(leet, limit):
    g = torch.full((1000,), 3e38, device="cuda")   # a norm of 9.5e39
    with pytest.raises(ValueError):
        leet.leet_attn_clip_gradients([g], limit, outs=[torch.empty_like(g)])
    if limit < 2.0 ** 160:
        with pytest.raises(ValueError):
            leet.leet_attn_clip_gradients([g], limit)
    else:
        leet.leet_attn_clip_gradients([g], limit)
    assert bool((g == 3e38).all())
    most, out = torch.finfo(torch.float32).max, torch.zeros_like(g)
    leet.leet_attn_clip_gradients([g], most, outs=[out])
    assert abs(float(out[0]) * 1000 ** 0.5 / most - 1) < 1e-6
