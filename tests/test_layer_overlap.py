"""Outputs of the operators beside the attention that share memory with other arguments are refused, on made-up addresses; and
the search that finds them, against sets of bytes."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2501_02573_amd", "csrc")
A = 1 << 32         # addresses that far apart share nothing at the sizes below
needs_no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses must not reach a device")


@pytest.fixture(scope="module")
def leet():
    from paper_2501_02573_amd import binding
    return binding


@pytest.fixture(scope="module")
def shared(tmp_path_factory):
    """The search as a function of two lists: address, bytes of a row, then size and stride of three dimensions."""
    at = tmp_path_factory.mktemp("overlap")
    (at / "overlap.cpp").write_text(
        '#include "leet_overlap.hpp"\n'
        "static leet::Span span(const long long* a) {\n"
        "    return leet::Span((const void*)a[0], 1, a[1], {{a[2], a[3]}, {a[4], a[5]}, {a[6], a[7]}});\n"
        "}\n"
        'extern "C" int shared(const long long* a, const long long* b) { return overlap(span(a), span(b)); }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", str(at / "overlap.so"),
                    str(at / "overlap.cpp")], check=True)
    f = ctypes.CDLL(str(at / "overlap.so")).shared
    return lambda a, b: bool(f((ctypes.c_longlong * 8)(*a), (ctypes.c_longlong * 8)(*b)))


def _bytes(t):
    at, width, n0, s0, n1, s1, n2, s2 = t
    return {at + i * s0 + j * s1 + k * s2 + w for i in range(n0) for j in range(n1) for k in range(n2) for w in range(width)}


def test_search_against_sets_of_bytes(shared):
    rng, seen = random.Random(1), [0, 0]
    for _ in range(20000):
        a = [1000 + rng.randint(0, 150), rng.randint(1, 6)] + [v for _ in range(3) for v in (rng.randint(1, 3), rng.randint(-3, 40))]
        b = [1000 + rng.randint(0, 150), rng.randint(1, 6)] + [v for _ in range(3) for v in (rng.randint(1, 3), rng.randint(-3, 40))]
        if rng.random() < 0.6:
            b[3::2] = a[3::2]
        want = bool(_bytes(a) & _bytes(b))
        assert shared(a, b) == want and shared(b, a) == want, (a, b)
        seen[want] += 1
    assert min(seen) > 4000


def test_search_of_large_tensors(shared):
    """Parts of one buffer: columns, heads, tokens and batches beside one another and over one another by one element."""
    d, H, N, B = 256, 32, 100000, 64
    row = 3 * H * d
    part = lambda at, h, n=N: [at, d, B, N * row, h, d, n, row]  # noqa: E731
    q, k, v = part(A, H), part(A + H * d, H), part(A + 2 * H * d, H)
    for a, b in ((q, k), (q, v), (k, v), (part(A, H, N // 2), part(A + N // 2 * row, H, N - N // 2))):
        assert not shared(a, b) and not shared(b, a)
    for a, b in ((q, part(A + H * d - 2, H)), (part(A, H + 1), k), (part(A, H, N // 2 + 1), part(A + N // 2 * row, H, N - N // 2)),
                 (q, part(A + row * N, H)), (q, [A + B * N * row - row, 2, 1, 0, 1, 0, 1, 0])):
        assert shared(a, b) and shared(b, a)
    dense = [A, d, B, H * N * d, H, N * d, N, d]
    assert shared(dense, q) and shared(dense, [A + 12345, 7, 1, 0, 1, 0, 1, 0])
    assert not shared(dense, [A + B * H * N * d, 7, 1, 0, 1, 0, 1, 0])
    assert not shared([0] + dense[1:], dense) and not shared([A, d, 0, 0, 1, 0, 1, 0], dense)     # nothing there
    far = (1 << 62) - 1
    assert not shared([A, 4, 9, far, 1, 0, 1, 0], [A + 8, 4, 9, far, 1, 0, 1, 0])


# ---- the entry points ----

def _heads(leet, **change):
    H = lambda i, more=0: leet._pack_heads(i * A + more, 1 << 14, 1 << 12, 128)  # noqa: E731
    a = dict(q=H(1), dy=H(2), out=H(3), k=H(4), dk=H(5), out_k=H(6), wq=7 * A, wk=8 * A, gq=9 * A, gk=10 * A, freq=11 * A,
             pos=12 * A, pos_batch=16, ws=13 * A)
    a.update({n: H(*v) if isinstance(v, tuple) else v for n, v in change.items()})
    a["rot"] = leet._pack_rotation(a["freq"], 64, 0, a["pos"], a["pos_batch"], 0, 1.0)
    return a


def _rope(leet, a):
    return leet.lib.leet_attn_rope(a["q"], a["out"], 2, a["k"], a["out_k"], 2, a["rot"], 2, 16, 128, leet.LEET_BF16, 0, None)


def _norm(leet, a):
    return leet.lib.leet_attn_qk_norm_rope(a["q"], a["out"], 2, a["k"], a["out_k"], 2, a["wq"], a["wk"], leet.LEET_BF16, 1e-6,
                                           a["rot"], 2, 16, 128, leet.LEET_BF16, None)


def _norm_back(leet, a):
    return leet.lib.leet_attn_qk_norm_rope_backward(a["dy"], a["q"], a["out"], 2, a["dk"], a["k"], a["out_k"], 2, a["wq"],
                                                    a["wk"], a["gq"], a["gk"], leet.LEET_BF16, 1e-6, a["rot"], a["ws"], 1 << 20,
                                                    2, 16, 128, leet.LEET_BF16, None)


@needs_no_device
def test_heads(leet):
    """Every change of the call that passes all checks and ends where there is no device."""
    INVALID, PASSED = leet.LEET_ERR_INVALID_ARG, leet.LEET_ERR_LAUNCH
    rows = 256      # bytes of a row
    over = [dict(out=(1, 2)), dict(out=(1, -2)), dict(out=(1, rows)), dict(out=(4,)), dict(out=(4, rows - 2)), dict(out_k=(3, 2)),
            dict(out_k=(1, 4 * rows)), dict(out=(11, 0)), dict(freq=3 * A + 128), dict(pos=6 * A + 256), dict(out_k=(12, -rows + 8))]
    weights = [dict(wq=3 * A), dict(wk=6 * A + 64), dict(wq=6 * A + 2)]
    back = [dict(out=(2, 2)), dict(out=(5,)), dict(out_k=(2, rows)), dict(gq=10 * A + 254), dict(gq=3 * A + 2), dict(gk=6 * A),
            dict(ws=A + 256), dict(ws=2 * A), dict(ws=3 * A), dict(ws=6 * A), dict(ws=7 * A), dict(ws=9 * A), dict(ws=11 * A),
            dict(ws=12 * A)]
    apart = [{}, dict(out=(1,)), dict(out_k=(4,)), dict(out=(1,), out_k=(4,)), dict(pos=0), dict(freq=3 * A + 16 * rows),
             dict(out=(1, 16 * rows + (1 << 14)))]
    for call, refused, fine in ((_rope, over, apart), (_norm, over + weights, apart),
                                (_norm_back, over + weights + back, apart + [dict(out=(2,)), dict(gq=7 * A), dict(gq=0, gk=0, ws=3 * A)])):
        for change in refused:
            assert call(leet, _heads(leet, **change)) == INVALID, (call, change)
        for change in fine:
            assert call(leet, _heads(leet, **change)) == PASSED, (call, change)


def _rows(leet, **change):
    R = lambda i, more=0, token=100, batch=1 << 16: leet._pack_rows(i * A + more, batch, token)  # noqa: E731
    a = dict(x=R(1), gate=R(2), out=R(3), h=R(4), dh=R(5), dx=R(6), dgate=R(7), s_in=8 * A, s_out=9 * A, ds_out=10 * A,
             ds_in=11 * A, offsets=None, S=0, ws=12 * A, B=2, N=500, C=100, mode=2)
    a.update({n: R(*v) if isinstance(v, tuple) else v for n, v in change.items()})
    return a


def _scan(leet, a):
    return leet.lib.leet_attn_gated_scan(a["x"], a["gate"], a["out"], a["s_in"], a["s_out"], a["offsets"], a["S"], a["ws"],
                                         1 << 24, a["B"], a["N"], a["C"], leet.LEET_BF16, leet.LEET_BF16, a["mode"], None)


def _scan_back(leet, a):
    return leet.lib.leet_attn_gated_scan_backward(a["dh"], a["x"], a["gate"], a["h"], a["dx"], a["dgate"], a["s_in"], a["ds_out"],
                                                  a["ds_in"], a["offsets"], a["S"], a["ws"], 1 << 24, a["B"], a["N"], a["C"],
                                                  leet.LEET_BF16, leet.LEET_BF16, a["mode"], None)


def _step(leet, a):
    return leet.lib.leet_attn_gated_scan_step(a["x"], a["gate"], a["out"], a["s_out"], 9, 100, leet.LEET_BF16, leet.LEET_BF16,
                                              a["mode"], None)


@needs_no_device
def test_rows(leet):
    INVALID, PASSED = leet.LEET_ERR_INVALID_ARG, leet.LEET_ERR_LAUNCH
    packed = dict(offsets=13 * A, B=1, S=7)
    scan = [dict(out=(1,)), dict(out=(1, 2)), dict(out=(1, -2)), dict(out=(2, 200)), dict(out=(8, -200)), dict(out=(9, 400)),
            dict(s_out=3 * A), dict(s_out=A + 4), dict(s_out=8 * A + 4), dict(s_out=8 * A - 4), dict(s_out=2 * A - 4),
            dict(ws=A), dict(ws=2 * A + 256), dict(ws=3 * A), dict(ws=8 * A), dict(ws=9 * A),
            dict(packed, offsets=3 * A + 4), dict(packed, s_out=13 * A), dict(packed, ws=13 * A)]
    back = [dict(dx=(5,)), dict(dx=(5, 2)), dict(dx=(1, 2)), dict(dx=(4, 200)), dict(dx=(2, -2)), dict(dgate=(6, 2)), dict(dgate=(2,)),
            dict(dgate=(4, 2)), dict(ds_in=8 * A), dict(ds_in=8 * A + 4), dict(ds_in=10 * A + 4), dict(ds_in=6 * A), dict(ds_in=7 * A),
            dict(ds_in=5 * A + 8), dict(dx=(10,)), dict(dgate=(10, 2)), dict(dx=(8,)), dict(ws=4 * A), dict(ws=6 * A), dict(ws=7 * A),
            dict(ws=10 * A), dict(ws=11 * A), dict(packed, dx=(13,)), dict(packed, ws=13 * A)]
    step = [dict(out=(1, 2)), dict(out=(1, 0, 0, 1 << 15)), dict(out=(2, -198)), dict(out=(9, 0)), dict(s_out=A + 4), dict(s_out=2 * A),
            dict(s_out=3 * A + 16)]
    # columns of one buffer, rows of 600 elements; states in place; x and dx of one place where x is not read
    wide = dict(x=(1, 0, 600), gate=(1, 200, 600), out=(1, 400, 600), dh=(1, 600, 600), h=(1, 800, 600), dx=(1, 1000, 600), B=1)
    fine = [{}, packed, wide, dict(s_out=8 * A, ds_in=10 * A), dict(s_in=0, s_out=0, ds_out=0, ds_in=0), dict(out=(1, 2 << 17))]
    for call, refused, good in ((_scan, scan, fine), (_scan_back, back, fine + [dict(dx=(1,), mode=1)]),
                                (_step, step, [{}, dict(out=(1,)), dict(out=(2,)), dict(out=(1, 200))])):
        for change in refused:
            assert call(leet, _rows(leet, **change)) == INVALID, (call, change)
        for change in good:
            assert call(leet, _rows(leet, **change)) == PASSED, (call, change)
