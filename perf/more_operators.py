"""What a training step of a decayed linear attention layer needs beside its forward pass, as timed cases: the attention's
gradient, the norm of a residual sum (with an output in 8 bits for serving) and its gradient, and the norm over all
gradients with the clipping.

A case is one call of an operator.  ``own`` false: the operator in elementary torch operations, in 32 bits (decays, and
sums over whole models, in 64), rounded once at the end.  ``own`` true: the call that a user makes of the library.
``exact`` is the definition in 64 bits.  Sizes are those of the repository's configurations (``workloads.py``) and
generic ragged ones.

Fields of a case: ``op`` and

* "attn_backward": ``B`` sequences of ``N`` tokens, ``H`` heads of rank ``r`` and value width ``dv``; ``dtype`` of all
  tensors; ``mask`` "decay" | "causal" (no decay); ``state``: a state entered and left the forward call, so a gradient
  of the one that left comes in and one of the one that entered goes out.
* "norm", "norm_q8", "norm_backward": ``B`` sequences of ``N`` tokens, ``C`` channels; ``dtype`` of x and the output;
  ``stream`` type of the residual stream, or "none": no residual is added (norm, norm_q8) or comes in (norm_backward);
  ``weights`` "in" (the input type) | "f32"; ``group`` channels that share a scale (norm_q8; 0: a whole row).
* "clip": the gradients of ``layers`` layers of ``width`` channels, their matrices in ``dtype``, norms' weights in f32,
  clipped into buffers of their own; ``limit``: the norm they are clipped to.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
CHUNK = 128          # tokens of a chunk in the attention's plain form
E4M3_MAX = 448.0
LEAST = 2.0 ** -100  # a scale is made for no less than this


def _attn(name, B, H, N, r, dv, dtype, mask="decay", state=False):
    return {"name": name, "op": "attn_backward", "B": B, "H": H, "N": N, "r": r, "dv": dv, "dtype": dtype, "mask": mask,
            "state": state}


def _norm(name, op, B, N, C, dtype, stream, weights="in", group=0):
    case = {"name": name, "op": op, "B": B, "N": N, "C": C, "dtype": dtype, "stream": stream, "weights": weights}
    return {**case, "group": group} if op == "norm_q8" else case


def _clip(name, layers, width, dtype, limit=1.0):
    return {"name": name, "op": "clip", "layers": layers, "width": width, "dtype": dtype, "limit": limit}


def listed():
    return [
        # a few heads of one short sequence: latency
        _attn("attn_backward_short", 1, 8, 64, 64, 64, "bf16"),
        # a training step's batch, 16 heads
        _attn("attn_backward_mid", 4, 16, 4096, 128, 128, "bf16"),
        # one piece of a longer document, with the gradient of the state that goes on to the next piece
        _attn("attn_backward_long", 1, 32, 32768, 128, 128, "bf16", state=True),
        # sequences of an odd length, narrow heads
        _attn("attn_backward_ragged", 3, 12, 1777, 64, 64, "f16"),
        # a small job in fp32
        _attn("attn_backward_f32", 2, 8, 2047, 128, 128, "f32", state=True),
        # the next token of one user
        _norm("norm_one_token", "norm", 1, 1, 4096, "bf16", "bf16"),
        # a training step's batch
        _norm("norm_mid", "norm", 4, 4096, 2048, "bf16", "bf16"),
        # prompts of an odd length, the residual stream in fp32, the output in 8 bits with a scale for 128 channels
        _norm("norm_q8_prompts", "norm_q8", 8, 1777, 4096, "bf16", "f32", group=128),
        # the training step's way back
        _norm("norm_backward_mid", "norm_backward", 4, 4096, 2048, "bf16", "bf16"),
        # a small job in fp32, an odd number of channels
        _norm("norm_backward_odd", "norm_backward", 2, 2047, 1001, "f32", "f32"),
        # a small model's gradients
        _clip("clip_small", 4, 256, "f32"),
        # twelve layers' gradients
        _clip("clip_layers", 12, 2048, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: one token to 32768, one head to 32, 64 to 8192 channels, 1 to 12 layers."""
    while True:
        op = rng.choice(("attn_backward",) * 5 + ("norm", "norm", "norm_q8", "norm_backward", "norm_backward", "clip"))
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        N = rng.choice((1, _log_int(rng, 2, 32768), _log_int(rng, 2, 32768), _log_int(rng, 2, 32768)))
        if op == "attn_backward":
            r, dv = rng.choice(((64, 64), (128, 128), (128, 128)) + (((128, 256),) if dtype != "f32" else ()))
            case = _attn("", _log_int(rng, 1, 32), _log_int(rng, 1, 32), N, r, dv, dtype,
                         mask=rng.choice(("decay", "decay", "decay", "causal")), state=rng.random() < 0.4)
        elif op == "clip":
            case = _clip("", rng.randint(1, 12), _log_int(rng, 64, 2048), dtype, limit=rng.choice((0.5, 1.0, 1e9)))
        else:
            C = rng.choice((128 * rng.randint(1, 64), _log_int(rng, 64, 8192)))
            group = rng.choice((0, 0, 32, 64, 128))
            case = _norm("", op, _log_int(rng, 1, 64), N, C, dtype,
                         stream=rng.choice((dtype, dtype, "f32", "none")), weights=rng.choice(("in", "f32")),
                         group=group if group and C % group == 0 else 0)
        del case["name"]
        if work(case)["bytes"] <= 1.2e9:
            return case


def _isz(dtype):
    return 4 if dtype == "f32" else 2


def _shapes(case):
    """Of the gradients: (number of values, type), five tensors a layer."""
    w = case["width"]
    return [(3 * w * w, case["dtype"]), (w * w, case["dtype"]), (w, "f32"), (w + 1, "f32"), (w * (w // 2) + 3, case["dtype"])] * case["layers"]


def work(case):
    op = case["op"]
    if op == "clip":
        values = sum(n for n, _ in _shapes(case))
        return {"bytes": 2 * sum(n * _isz(t) for n, t in _shapes(case)), "flops": 3 * values}
    isz, rows = _isz(case["dtype"]), case["B"] * case["N"]
    if op == "attn_backward":
        B, H, r, dv = case["B"], case["H"], case["r"], case["dv"]
        states = 4 * B * H * r * dv if case["state"] else 0
        # q, k, v, dout -> dq, dk, dv; the two states and both gradients.  By token: its state and the state's gradient are
        # updated (2 r dv each) and each of the three gradients is a product with one of them
        return {"bytes": rows * H * (4 * r + 3 * dv) * isz + 3 * states, "flops": rows * H * r * dv * 10}
    C = case["C"]
    there = case["stream"] != "none"
    ssz = _isz(case["stream"]) if there else isz
    wsz = C * (4 if case["weights"] == "f32" else isz)
    if op == "norm":  # x, residual -> sum, y
        return {"bytes": rows * C * (2 * isz + (2 * ssz if there else 0)) + wsz, "flops": rows * C * 5}
    if op == "norm_q8":
        scales = 4 * rows * (C // case["group"] if case["group"] else 1)
        return {"bytes": rows * C * (isz + 1 + (2 * ssz if there else 0)) + wsz + scales, "flops": rows * C * 7}
    # dy, h, what comes along the stream -> dx (and the stream's own gradient where its type is another), dw
    out = isz + (ssz if there and ssz != isz else 0)
    return {"bytes": rows * C * (isz + ssz + (ssz if there else 0) + out) + 2 * wsz, "flops": rows * C * 11}


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt, op = DTYPES[case["dtype"]], case["op"]

    def normal(shape, dtype, sigma=1.0, mean=0.0):
        return torch.randn(shape, device=dev, generator=gen, dtype=torch.float32).mul_(sigma).add_(mean).to(dtype)

    st = {"case": case}
    if op == "clip":
        sigma = 0.3 / math.sqrt(sum(n for n, _ in _shapes(case)) / case["layers"])
        st["grads"] = [normal((n,), DTYPES[t], sigma * (1 + i % 7)) for i, (n, t) in enumerate(_shapes(case))]
        st["outs"] = [torch.empty_like(g) for g in st["grads"]]
        return st
    if op == "attn_backward":
        B, H, N, r, dv = case["B"], case["H"], case["N"], case["r"], case["dv"]
        st["q"], st["k"] = normal((B, H, N, r), dt, r ** -0.5), normal((B, H, N, r), dt, r ** -0.5)
        st["v"], st["dout"] = normal((B, H, N, dv), dt, dv ** -0.5), normal((B, H, N, dv), dt)
        # memories of 32 to 1024 tokens over the heads
        h = torch.arange(H, dtype=torch.float64, device=dev)
        st["gamma"] = (1 - torch.exp2(-(5 + 5 * h / max(H - 1, 1)))).float()
        if case["state"]:
            st["state_in"], st["dstate_out"] = normal((B, H, r, dv), torch.float32, 0.1), normal((B, H, r, dv), torch.float32, 0.1)
            st["dstate_in"] = torch.empty_like(st["dstate_out"])
        return st
    shape = (case["B"], case["N"], case["C"])
    wdt = dt if case["weights"] == "in" else torch.float32
    st["weight"] = normal((case["C"],), wdt, 0.2, 1.0)
    sdt = dt if case["stream"] == "none" else DTYPES[case["stream"]]
    if op == "norm_backward":
        st["dout"], st["h"] = normal(shape, dt), normal(shape, sdt, 2.0)
        st["dstream"] = normal(shape, sdt) if case["stream"] != "none" else None
        return st
    st["x"] = normal(shape, dt)
    st["residual"] = normal(shape, sdt, 2.0) if case["stream"] != "none" else None
    return st


# ---- the operators in elementary operations -------------------------------------------------------------------------

def _powers(gamma, n):
    """gamma^n [H, ...] for whole numbers n >= 0 (0^0 = 1), formed in 64 bits."""
    return (gamma.double().view((-1,) + (1,) * n.dim()) ** n.double()).float()


def _attn_backward_plain(st):
    """In chunks of L tokens: products within a chunk, states of the chunks, products with them."""
    case = st["case"]
    B, H, N, L = case["B"], case["H"], case["N"], CHUNK
    gamma = st["gamma"] if case["mask"] == "decay" else torch.ones_like(st["gamma"])
    dt, chunks = st["q"].dtype, -(-N // L)

    def cut(x):  # [B, H, N, d] -> [B, H, chunks, L, d], zeros behind the last token
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, chunks * L - N))
        return x.view(B, H, chunks, L, x.shape[-1])

    def join(x):
        return x.reshape(B, H, chunks * L, x.shape[-1])[:, :, :N]

    q, k, v, do = (cut(st[x]) for x in ("q", "k", "v", "dout"))
    i = torch.arange(L, device=q.device)
    far = i[:, None] - i[None, :]
    M = (_powers(gamma, far.clamp(min=0)) * (far >= 0))[None, :, None]      # [1, H, 1, L, L]
    row = _powers(gamma, i)[None, :, None, :, None]                        # gamma^i
    up, down = row * gamma.view(1, H, 1, 1, 1), _powers(gamma, L - 1 - i)[None, :, None, :, None]
    P = q @ k.transpose(-1, -2) * M
    dP = do @ v.transpose(-1, -2) * M
    dq, dk, dv = dP @ k, dP.transpose(-1, -2) @ q, P.transpose(-1, -2) @ do
    # what each chunk adds to the state behind it and to the gradient of the state before it; sums over the others
    T, U = (k * down).transpose(-1, -2) @ v, (q * row).transpose(-1, -2) @ do
    c = torch.arange(chunks, device=q.device)
    apart = c[:, None] - c[None, :] - 1
    W = _powers(gamma, (apart * L).clamp(min=0)) * (apart >= 0)             # [H, chunks, chunks]
    S = (W @ T.flatten(-2)).view_as(T)
    R = (W.transpose(-1, -2) @ U.flatten(-2)).view_as(U)
    dq = join(dq + up * (do @ S.transpose(-1, -2)))
    late = down * gamma.view(1, H, 1, 1, 1)                                # gamma^(L - j)
    dk, dv = join(dk + late * (v @ R.transpose(-1, -2))), join(dv + late * (k @ R))
    if not case["state"]:
        return dq.to(dt), dk.to(dt), dv.to(dt)
    n = torch.arange(N, device=q.device)
    entered, behind = _powers(gamma, n + 1)[None, :, :, None], _powers(gamma, N - 1 - n)[None, :, :, None]
    dS = st["dstate_out"]
    dq = dq + entered * (st["dout"].float() @ st["state_in"].transpose(-1, -2))
    dk = dk + behind * (st["v"].float() @ dS.transpose(-1, -2))
    dv = dv + behind * (st["k"].float() @ dS)
    left = (entered * st["q"].float()).transpose(-1, -2) @ st["dout"].float()
    left = left + _powers(gamma, torch.tensor(N, device=q.device)).view(1, H, 1, 1) * dS
    return dq.to(dt), dk.to(dt), dv.to(dt), left


def _sum_and_norm(st):
    s = st["x"].float()
    if st["residual"] is not None:
        s = s + st["residual"].float()
    return s, s * torch.rsqrt((s * s).mean(-1, keepdim=True) + EPS) * st["weight"].float()


def _run_plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "attn_backward":
        return _attn_backward_plain(st)
    if op == "clip":
        flat = torch.cat([g.float() for g in st["grads"]])
        norm = torch.sqrt((flat * flat).sum(dtype=torch.float64))
        flat = flat * (case["limit"] / norm).clamp(max=1.0).float()
        parts = flat.split([g.numel() for g in st["grads"]])
        return [p.to(g.dtype) for p, g in zip(parts, st["grads"])], norm.float().view(1)
    if op == "norm_backward":
        h, dy, w = st["h"].float(), st["dout"].float(), st["weight"].float()
        r = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
        n = h * r
        dn = dy * w
        dh = r * (dn - n * (dn * n).mean(-1, keepdim=True))
        if st["dstream"] is not None:
            dh = dh + st["dstream"].float()
        dw = (dy * n).sum((0, 1), dtype=torch.float64).to(st["weight"].dtype)
        if st["h"].dtype == st["dout"].dtype:
            return dh.to(st["h"].dtype), dw
        return dh.to(st["dout"].dtype), dh.to(st["h"].dtype), dw
    s, y = _sum_and_norm(st)
    left = [] if st["residual"] is None else [s.to(st["residual"].dtype)]
    if op == "norm":
        return [y.to(st["x"].dtype)] + left
    groups = y.unflatten(-1, (-1, case["group"] or case["C"]))
    scales = groups.abs().amax(-1).clamp(min=LEAST) / E4M3_MAX
    y8 = (groups / scales[..., None]).flatten(-2).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return [y8, scales] + left


# ---- the library's calls --------------------------------------------------------------------------------------------

def _run_own(st):
    from paper_2501_02573_amd import binding as leet

    case, op = st["case"], st["case"]["op"]
    if op == "attn_backward":
        mask = leet.LEET_MASK_DECAY if case["mask"] == "decay" else leet.LEET_MASK_CAUSAL
        got = leet.leet_attn_backward(st["dout"], st["q"], st["k"], st["v"], st["gamma"], mask=mask,
                                      state_in=st.get("state_in"), dstate_out=st.get("dstate_out"),
                                      dstate_in=st.get("dstate_in"))
        return got + (st["dstate_in"],) if case["state"] else got
    if op == "clip":
        return st["outs"], leet.leet_attn_clip_gradients(st["grads"], case["limit"], outs=st["outs"])
    if op == "norm_backward":
        dx, dstream, dw = leet.leet_attn_add_rms_norm_backward(st["dout"], st["h"], st["weight"], eps=EPS,
                                                               dresidual=st["dstream"])
        return (dx, dw) if dstream is dx else (dx, dstream, dw)
    if op == "norm":
        y, left = leet.leet_attn_add_rms_norm(st["x"], st["residual"], st["weight"], eps=EPS)
        return [y] if left is None else [y, left]
    y8, scales, left = leet.leet_attn_add_rms_norm_q8(st["x"], st["residual"], st["weight"], eps=EPS, group=case["group"])
    return [y8, scales] if left is None else [y8, scales, left]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _attn_backward_exact(st):
    """Token by token: S <- g S + k^T v and dq = S do from the first, G <- g G + q^T do, dk = G v and dv = k G from the last."""
    case = st["case"]
    B, H, N, r, w = case["B"], case["H"], case["N"], case["r"], case["dv"]
    q, k, v, do = (st[x].double().view(B * H, N, -1) for x in ("q", "k", "v", "dout"))
    g = st["gamma"].double() if case["mask"] == "decay" else torch.ones(H, dtype=torch.float64, device=q.device)
    g = g.repeat(B).view(B * H, 1, 1)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    S = torch.zeros((B * H, r, w), dtype=torch.float64, device=q.device)
    if case["state"]:
        S += st["state_in"].view_as(S)
    for t in range(N):
        S.mul_(g).baddbmm_(k[:, t, :, None], v[:, t, None, :])
        dq[:, t] = torch.bmm(S, do[:, t, :, None])[:, :, 0]
    G = S.zero_()
    if case["state"]:
        G += st["dstate_out"].view_as(G)
    for t in range(N - 1, -1, -1):
        G.baddbmm_(q[:, t, :, None], do[:, t, None, :])
        dk[:, t] = torch.bmm(G, v[:, t, :, None])[:, :, 0]
        dv[:, t] = torch.bmm(k[:, t, None, :], G)[:, 0]
        G.mul_(g)
    got = dq.view(B, H, N, r), dk.view(B, H, N, r), dv.view(B, H, N, w)
    return got + (G.view(B, H, r, w),) if case["state"] else got


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "attn_backward":
        return _attn_backward_exact(st)
    if op == "clip":
        norm = math.sqrt(sum(float(torch.dot(g.double(), g.double())) for g in st["grads"]))
        by = min(1.0, case["limit"] / norm)
        return [g.double() * by for g in st["grads"]], torch.tensor([norm], dtype=torch.float64)
    w = st["weight"].double()
    if op == "norm_backward":
        leaves = st["h"].double().requires_grad_(), w.clone().requires_grad_()
        with torch.enable_grad():
            y = leaves[0] / ((leaves[0] ** 2).sum(-1, keepdim=True) / case["C"] + EPS).sqrt() * leaves[1]
        dh, dw = torch.autograd.grad(y, leaves, st["dout"].double())
        if st["dstream"] is not None:
            dh = dh + st["dstream"].double()
        return (dh, dw) if st["h"].dtype == st["dout"].dtype else (dh, dh, dw)
    s = st["x"].double()
    if st["residual"] is not None:
        s = s + st["residual"].double()
    y = w * s / (s.square().sum(-1, keepdim=True) / case["C"] + EPS).sqrt()
    left = [] if st["residual"] is None else [s]
    if op == "norm":
        return [y] + left
    parts = y.unflatten(-1, (-1, case["group"] or case["C"]))
    scales = torch.maximum(parts.abs().max(-1).values, torch.tensor(LEAST, dtype=torch.float64, device=y.device)) / E4M3_MAX
    # before its rounding to 8 bits
    return [(parts / scales[..., None]).flatten(-2), scales] + left
