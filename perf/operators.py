"""The operators beside the attention as timed cases: position rotation, norms of queries and keys with the rotation in
the same pass, and the gated linear recurrence.

A case is one call of an operator.  ``own`` false: the operator in elementary torch operations, in 32 bits (angles in
64), rounded once at the end.  ``own`` true: the call that a user makes of the library.  ``exact`` is the definition in
64 bits.  Sizes are those of the repository's configurations (``workloads.py``) and generic ragged ones.

Fields of a case: ``op`` and

* "rope", "norm_rope", "norm_rope_backward": ``B`` sequences of ``N`` tokens, ``Hq`` query and ``Hk`` key heads of
  width ``d`` of which ``rot`` are rotated; ``layout`` "half" | "interleaved"; ``scaling`` of the frequencies "none" |
  "linear" | "base" | "bands"; ``positions`` "given" (one a token, up to ``far``) | "run" (consecutive from ``far`` on);
  ``dtype``; ``weights`` "in" (the input type) | "f32" (norms only); ``transposed`` (rope only: its gradient).
* "scan", "scan_backward": ``B`` sequences of ``N`` tokens and ``C`` channels; ``gate`` "decay" | "log" | "sigmoid";
  ``dtype`` of x and h, ``gate_dtype``; ``sequences`` > 0: that many sequences of different lengths, some of them
  empty, packed into N rows (B = 1); ``state`` whether a state enters and leaves.
* "scan_step": one token of ``B`` sequences.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
BASE = 10000.0


def _heads(name, op, B, N, Hq, Hk, d, rot, dtype, layout="half", scaling="none", positions="run", far=0, weights="in",
           transposed=False):
    case = {"name": name, "op": op, "B": B, "N": N, "Hq": Hq, "Hk": Hk, "d": d, "rot": rot, "dtype": dtype,
            "layout": layout, "scaling": scaling, "positions": positions, "far": far}
    return {**case, "transposed": transposed} if op == "rope" else {**case, "weights": weights}


def _scan(name, op, B, N, C, dtype, gate_dtype, gate, sequences=0, state=True):
    case = {"name": name, "op": op, "B": B, "C": C, "dtype": dtype, "gate_dtype": gate_dtype, "gate": gate}
    return case if op == "scan_step" else {**case, "N": N, "sequences": sequences, "state": state}


def listed():
    return [
        # the next token of one user: 32 heads of queries and keys, far into a long document
        _heads("rope_one_user", "rope", 1, 1, 32, 32, 128, 128, "bf16", positions="given", far=100000),
        # gradient of the rotation over a long document, half of the head rotated, neighbours paired
        _heads("rope_gradient_long", "rope", 1, 32768, 32, 32, 128, 64, "bf16", layout="interleaved", scaling="bands",
               far=5, transposed=True),
        # the next token of a full batch, each user at a position of its own
        _heads("norm_rope_batch64", "norm_rope", 64, 1, 32, 32, 128, 128, "bf16", positions="given", far=32768),
        # a mid-sized batch of prompts: q and k out of a fused projection into the layout that the prefill reads
        _heads("norm_rope_mid", "norm_rope", 4, 4096, 16, 16, 128, 128, "bf16"),
        # ragged prompts, shared key heads, a quarter of the head rotated, positions stretched
        _heads("norm_rope_shared_heads", "norm_rope", 3, 1777, 32, 8, 64, 16, "f16", layout="interleaved",
               scaling="linear", positions="given", far=131072, weights="f32"),
        # a training step's way back through the same batch
        _heads("norm_rope_backward_mid", "norm_rope_backward", 4, 4096, 16, 16, 128, 128, "bf16"),
        # the same for a small job in fp32
        _heads("norm_rope_backward_f32", "norm_rope_backward", 2, 2047, 8, 8, 64, 64, "f32", scaling="base"),
        # the next token of a full batch through a recurrence of 4096 channels
        _scan("scan_step_batch64", "scan_step", 64, 1, 4096, "bf16", "bf16", "log"),
        # a mid-sized batch of prompts, the state kept for decoding
        _scan("scan_mid", "scan", 4, 4096, 2048, "bf16", "bf16", "log"),
        # one long document, decays in fp32
        _scan("scan_long", "scan", 1, 32768, 4096, "bf16", "f32", "decay", state=False),
        # prompts of different lengths behind one another, an odd number of channels
        _scan("scan_packed", "scan", 1, 20011, 1001, "f16", "f16", "sigmoid", sequences=37),
        # a training step's way back through the batch
        _scan("scan_backward_mid", "scan_backward", 4, 4096, 2048, "bf16", "bf16", "sigmoid"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: one token to 32768, one to 32 heads, 64 to 4096 channels."""
    while True:
        op = rng.choice(("rope", "norm_rope", "norm_rope", "norm_rope_backward", "scan", "scan", "scan_backward",
                         "scan_backward", "scan_step"))
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        N = rng.choice((1, _log_int(rng, 2, 32768), _log_int(rng, 2, 32768), _log_int(rng, 2, 32768)))
        if op.startswith("scan"):
            gate_dtype = rng.choice((dtype, dtype, "f32"))
            gate = rng.choice(("decay", "log", "sigmoid")) if gate_dtype == "f32" else rng.choice(("log", "sigmoid"))
            C = rng.choice((64 * rng.randint(1, 64), _log_int(rng, 64, 4096)))
            if op == "scan_step":
                case = _scan("", op, _log_int(rng, 1, 256), 1, C, dtype, gate_dtype, gate)
            elif rng.random() < 0.4:
                case = _scan("", op, 1, max(N, 64), C, dtype, gate_dtype, gate, sequences=_log_int(rng, 1, 256))
            else:
                case = _scan("", op, _log_int(rng, 1, 32), N, C, dtype, gate_dtype, gate, state=rng.random() < 0.7)
        else:
            d = rng.choice((64, 128, 128, 256))
            rot = rng.choice((d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)))
            Hq = rng.choice((1, 2, 3, 4, 8, 12, 16, 24, 32))
            Hk = Hq if rng.random() < 0.6 else rng.choice([h for h in (1, 2, 3, 4, 8) if Hq % h == 0])
            case = _heads("", op, _log_int(rng, 1, 64), N, Hq, Hk, d, rot, dtype,
                          layout=rng.choice(("half", "interleaved")),
                          scaling=rng.choice(("none", "none", "linear", "base", "bands")),
                          positions=rng.choice(("given", "run")), far=_log_int(rng, 1, 1000000),
                          weights=rng.choice(("in", "f32")), transposed=rng.random() < 0.4)
        del case["name"]
        if work(case)["bytes"] <= 1.0e9:
            return case


def _isz(dtype):
    return 4 if dtype == "f32" else 2


def work(case):
    op, isz, B = case["op"], _isz(case["dtype"]), case["B"]
    if op.startswith("scan"):
        C, gsz = case["C"], _isz(case["gate_dtype"])
        if op == "scan_step":
            return {"bytes": B * C * (2 * isz + gsz + 8), "flops": B * C * 4}
        rows = B * case["N"]
        states = (case["sequences"] or B) * C * 4 if case["state"] or case["sequences"] else 0
        if op == "scan":  # x, gate -> h; states in and out
            return {"bytes": rows * C * (2 * isz + gsz) + 2 * states, "flops": rows * C * 4}
        # dh, gate, h (and x where the gate weighs it) -> dx, dgate; entering state, gradients of both states
        reads = 3 if case["gate"] == "sigmoid" else 2
        return {"bytes": rows * C * ((reads + 1) * isz + 2 * gsz) + 3 * states, "flops": rows * C * 7}
    rows = B * case["N"] * (case["Hq"] + case["Hk"])
    d, rot = case["d"], case["rot"]
    positions = 8 * B * case["N"] if case["positions"] == "given" else 0
    if op == "rope":
        return {"bytes": rows * 2 * d * isz + positions + 4 * rot, "flops": rows * 3 * rot}
    wsz = 2 * d * (4 if case["weights"] == "f32" else isz)
    if op == "norm_rope":
        return {"bytes": rows * 2 * d * isz + positions + 4 * rot + wsz, "flops": rows * (4 * d + 3 * rot)}
    return {"bytes": rows * 3 * d * isz + positions + 4 * rot + 2 * wsz, "flops": rows * (11 * d + 3 * rot)}


def _frequencies(case):
    """(radians a position of each pair, in 64 bits; the factor of the rotated part) for contexts stretched 8 times."""
    rot, factor, trained = case["rot"], 8.0, 4096
    i = torch.arange(rot // 2, dtype=torch.float64)
    base = BASE * factor ** (rot / (rot - 2)) if case["scaling"] == "base" and rot > 2 else BASE
    freq = base ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        return freq / factor, 1.0
    if case["scaling"] != "bands":
        return freq, 1.0
    # pairs that turn over 32 times within the trained length keep their frequency, those under once are stretched
    def index(turns):
        return rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(BASE))
    low, high = max(math.floor(index(32.0)), 0), min(math.ceil(index(1.0)), rot - 1)
    stretched = ((i - low) / max(high - low, 1e-3)).clamp(0, 1)
    return freq * (1 - stretched) + freq / factor * stretched, 0.1 * math.log(factor) + 1.0


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt, B, op = DTYPES[case["dtype"]], case["B"], case["op"]

    def normal(shape, dtype, sigma=1.0, mean=0.0):
        return torch.randn(shape, device=dev, generator=gen, dtype=torch.float32).mul_(sigma).add_(mean).to(dtype)

    st = {"case": case}
    if op.startswith("scan"):
        C, gdt = case["C"], DTYPES[case["gate_dtype"]]
        shape = (B, C) if op == "scan_step" else (B, case["N"], C)
        st["x"] = normal(shape, dt)
        if case["gate"] == "sigmoid":
            st["gate"] = normal(shape, gdt, 1.5, 2.0)
        else:  # memories of one to a thousand tokens, over the channels and moving from token to token
            reach = torch.rand(C, device=dev, generator=gen) * -6.9 + normal(shape, torch.float32, 0.3)
            st["gate"] = reach.exp_().neg_().to(gdt) if case["gate"] == "log" else reach.exp_().neg_().exp_().to(gdt)
        if op == "scan_step":
            st["state"] = normal((B, C), torch.float32, 3.0)
            return st
        S = B
        st["offsets"] = None
        if case["sequences"]:
            S = case["sequences"]
            # lengths spread over two orders of magnitude, every ninth sequence empty, some rows behind the last one
            share = torch.exp(4.6 * torch.rand(S, generator=gen, device=dev))
            share[4::9] = 0
            ends = (share.cumsum(0) / (share.sum() * 1.01) * case["N"]).int()
            st["offsets"] = torch.cat((torch.zeros(1, dtype=torch.int32, device=dev), ends))
        if case["state"] or case["sequences"]:
            st["state_in"] = normal((S, C), torch.float32, 3.0)
            st["state_out"] = torch.zeros((S, C), device=dev)
        if op == "scan":
            st["out"] = torch.zeros(shape, dtype=dt, device=dev)
        else:  # the states that the forward pass left, their gradients and the buffers of the gradients to be
            st["h"], st["dh"] = normal(shape, dt, 2.0), normal(shape, dt)
            st["dx"], st["dgate"] = torch.zeros(shape, dtype=dt, device=dev), torch.zeros(shape, dtype=gdt, device=dev)
            if "state_in" in st:
                st["dstate_out"], st["dstate_in"] = normal((S, C), torch.float32), torch.zeros((S, C), device=dev)
        return st
    N, Hq, Hk, d = case["N"], case["Hq"], case["Hk"], case["d"]

    def split(fused):  # [B, N, (Hq + 2 Hk) d] -> q and k as [B, H, N, d]
        at = fused.view(B, N, Hq + 2 * Hk, d).transpose(1, 2)
        return at[:, :Hq], at[:, Hq:Hq + Hk]

    fused = normal((B, N, (Hq + 2 * Hk) * d), dt)
    freq, st["scale"] = _frequencies(case)
    st["freq"] = freq.to(dev)
    st["positions"] = None
    if case["positions"] == "given":
        st["positions"] = torch.randint(0, case["far"] + 1, (B, N), device=dev, generator=gen)
    if op == "rope" and case["transposed"]:  # gradients come in the attention's layout and go into the projection's
        st["q"], st["k"] = normal((B, Hq, N, d), dt), normal((B, Hk, N, d), dt)
        st["out_q"], st["out_k"] = split(fused)
        return st
    st["q"], st["k"] = split(fused)
    if op != "rope":
        wdt = dt if case["weights"] == "in" else torch.float32
        st["wq"], st["wk"] = normal((d,), wdt, 0.2, 1.0), normal((d,), wdt, 0.2, 1.0)
    if op == "norm_rope_backward":
        st["dq"], st["dk"] = normal((B, Hq, N, d), dt), normal((B, Hk, N, d), dt)
        st["out_q"], st["out_k"] = split(torch.zeros_like(fused))
    return st


# ---- the operators in elementary operations -------------------------------------------------------------------------

def _angles(st, dtype):
    """cos and sin, times the factor, [B or 1, 1, N, rot / 2]."""
    case, pos = st["case"], st["positions"]
    if pos is None:
        pos = torch.arange(case["N"], device=st["freq"].device)[None] + case["far"]
    theta = pos.double()[:, None, :, None] * st["freq"]
    return (theta.cos() * st["scale"]).to(dtype), (theta.sin() * st["scale"]).to(dtype)


def _rotate(x, cos, sin, case):
    rot = case["rot"]
    if case["layout"] == "half":
        x1, x2 = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat((x1 * cos - x2 * sin, x2 * cos + x1 * sin, x[..., rot:]), -1)
    x1, x2 = x[..., 0:rot:2], x[..., 1:rot:2]
    pairs = torch.stack((x1 * cos - x2 * sin, x2 * cos + x1 * sin), -1)
    return torch.cat((pairs.flatten(-2), x[..., rot:]), -1)


def _norm_rope_backward(x, w, dy, cos, sin, case):
    x, w = x.float(), w.float()
    du = _rotate(dy.float(), cos, -sin, case)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dn = du * w
    return r * (dn - n * (dn * n).mean(-1, keepdim=True)), (du * n).sum((0, 1, 2))


def _scan_pairs(a, b, reverse):
    """h_t = a_t h_{t-1} + b_t along dimension 1 (or h_t = a_t h_{t+1} + b_t) by doubling: after a step of length s a
    row holds what the 2 s rows up to it give."""
    N, s = a.shape[1], 1
    while s < N:
        if reverse:
            here, there = slice(0, N - s), slice(s, N)
        else:
            here, there = slice(s, N), slice(0, N - s)
        b_new, a_new = b.clone(), a.clone()
        b_new[:, here] += a[:, here] * b[:, there]
        a_new[:, here] *= a[:, there]
        a, b, s = a_new, b_new, 2 * s
    return b


def _decay(st, dtype):
    z = st["gate"].to(dtype)
    return z if st["case"]["gate"] == "decay" else z.exp() if st["case"]["gate"] == "log" else torch.sigmoid(z)


def _places(st):
    """Of packed rows: which are a sequence's, the sequence, whether it begins or ends there; of sequences: the last
    row, and whether there is one."""
    off, rows = st["offsets"].long(), torch.arange(st["case"]["N"], device=st["x"].device)
    at = torch.searchsorted(off, rows, right=True) - 1
    inside = at < off.numel() - 1
    at = at.clamp(max=off.numel() - 2)
    return inside, at, inside & (rows == off[at]), inside & (rows == off[at + 1] - 1), off[1:] - 1, off[1:] > off[:-1]


def _scan_plain(st):
    case = st["case"]
    a, x = _decay(st, torch.float32), st["x"].float()
    b = torch.sigmoid(-st["gate"].float()) * x if case["gate"] == "sigmoid" else x.clone()
    if st["offsets"] is not None:
        inside, at, first, _, last, some = _places(st)
        b = torch.where(first[None, :, None], a * st["state_in"][at] + b, b)
        h = _scan_pairs(torch.where(first[None, :, None], torch.zeros_like(a), a), b, False)
        left = torch.where(some[:, None], h[0, last.clamp(min=0)], st["state_in"])
        return torch.where(inside[None, :, None], h.to(st["x"].dtype), st["out"]), left
    if "state_in" in st:
        b[:, 0] += a[:, 0] * st["state_in"]
    h = _scan_pairs(a, b, False)
    return (h.to(st["x"].dtype), h[:, -1].clone()) if "state_in" in st else h.to(st["x"].dtype)


def _scan_backward_plain(st):
    case = st["case"]
    a, h, dh = _decay(st, torch.float32), st["h"].float(), st["dh"].float()
    before = torch.cat((torch.zeros_like(h[:, :1]), h[:, :-1]), 1)
    carry = torch.zeros_like(dh)  # what comes in from behind a sequence's last row
    link = a
    if st["offsets"] is not None:
        inside, at, first, final, last, some = _places(st)
        before = torch.where(first[None, :, None], st["state_in"][at][None], before)
        carry = torch.where(final[None, :, None], st["dstate_out"][at][None], carry)
        link = torch.where(final[None, :, None], torch.zeros_like(a), a)
    elif "state_in" in st:
        before[:, 0] = st["state_in"]
        carry[:, -1] = st["dstate_out"]
    # g_t = a_t (dh_t + g_{t+1}), the gradient that flows on into the state before row t
    g = _scan_pairs(link, a * (dh + carry), True)
    behind = torch.cat((g[:, 1:], torch.zeros_like(g[:, :1])), 1)
    if st["offsets"] is not None:
        behind = torch.where(final[None, :, None], torch.zeros_like(behind), behind)
    D = dh + carry + behind
    if case["gate"] == "decay":
        dgate, dx = D * before, D
    elif case["gate"] == "log":
        dgate, dx = a * D * before, D
    else:
        rest = torch.sigmoid(-st["gate"].float())
        dgate, dx = D * (before - st["x"].float()) * a * rest, D * rest
    dgate, dx = dgate.to(st["gate"].dtype), dx.to(st["x"].dtype)
    if st["offsets"] is not None:
        dgate = torch.where(inside[None, :, None], dgate, st["dgate"])
        dx = torch.where(inside[None, :, None], dx, st["dx"])
        off = st["offsets"].long()
        entered = torch.where(some[:, None], g[0, off[:-1].clamp(max=case["N"] - 1)], st["dstate_out"])
        return dx, dgate, entered
    return (dx, dgate, g[:, 0].clone()) if "state_in" in st else (dx, dgate)


def _run_plain(st):
    case = st["case"]
    if case["op"] == "scan_step":
        b = st["x"].float()
        if case["gate"] == "sigmoid":
            b = torch.sigmoid(-st["gate"].float()) * b
        st["state"].copy_(_decay(st, torch.float32) * st["state"] + b)
        return st["state"].to(st["x"].dtype), st["state"]
    if case["op"] == "scan":
        return _scan_plain(st)
    if case["op"] == "scan_backward":
        return _scan_backward_plain(st)
    dt = st["q"].dtype
    cos, sin = _angles(st, torch.float32)
    if case["op"] == "rope":
        sin = -sin if case["transposed"] else sin
        return tuple(_rotate(st[x].float(), cos, sin, case).to(dt) for x in ("q", "k"))
    if case["op"] == "norm_rope":
        def one(x, w):
            x = x.float()
            n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
            return _rotate(n, cos, sin, case).to(dt)
        return one(st["q"], st["wq"]), one(st["k"], st["wk"])
    dxq, dwq = _norm_rope_backward(st["q"], st["wq"], st["dq"], cos, sin, case)
    dxk, dwk = _norm_rope_backward(st["k"], st["wk"], st["dk"], cos, sin, case)
    return dxq.to(dt), dxk.to(dt), dwq.to(st["wq"].dtype), dwk.to(st["wk"].dtype)


# ---- the library's calls --------------------------------------------------------------------------------------------

def _run_own(st):
    from paper_2501_02573_amd import binding as leet

    case = st["case"]
    if case["op"].startswith("scan"):
        mode = {"decay": leet.GATE_DECAY, "log": leet.GATE_LOG, "sigmoid": leet.GATE_SIGMOID}[case["gate"]]
        if case["op"] == "scan_step":
            return leet.leet_attn_gated_scan_step(st["x"], st["gate"], st["state"], mode=mode), st["state"]
        if case["op"] == "scan":
            out = leet.leet_attn_gated_scan(st["x"], st["gate"], mode=mode, out=st["out"], state_in=st.get("state_in"),
                                            state_out=st.get("state_out"), offsets=st["offsets"])
            return (out, st["state_out"]) if "state_out" in st else out
        leet.leet_attn_gated_scan_backward(
            st["dh"], st["x"] if case["gate"] == "sigmoid" else None, st["gate"], st["h"], mode=mode, dx=st["dx"],
            dgate=st["dgate"], state_in=st.get("state_in"), dstate_out=st.get("dstate_out"),
            dstate_in=st.get("dstate_in"), offsets=st["offsets"])
        return (st["dx"], st["dgate"], st["dstate_in"]) if "dstate_in" in st else (st["dx"], st["dgate"])
    how = {"positions": st["positions"], "pos0": 0 if st["positions"] is not None else case["far"], "scale": st["scale"],
           "layout": leet.ROPE_HALF if case["layout"] == "half" else leet.ROPE_INTERLEAVED}
    if case["op"] == "rope":
        return leet.leet_attn_rope(st["q"], st["freq"], k=st["k"], transposed=case["transposed"],
                                   out_q=st.get("out_q"), out_k=st.get("out_k"), **how)
    if case["op"] == "norm_rope":
        return leet.leet_attn_qk_norm_rope(st["q"], st["k"], st["wq"], st["wk"], st["freq"], eps=EPS, **how)
    return leet.leet_attn_qk_norm_rope_backward(st["dq"], st["dk"], st["q"], st["k"], st["wq"], st["wk"], st["freq"],
                                                eps=EPS, dx_q=st["out_q"], dx_k=st["out_k"], **how)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _turned(x, st, case):
    """Pairs as complex numbers, turned by exp(i theta) and scaled."""
    B, H, N, d = x.shape
    pos = st["positions"]
    if pos is None:
        pos = (case["far"] + torch.arange(N, device=x.device)).expand(B, N)
    theta = torch.einsum("bn,f->bnf", pos.double(), st["freq"])[:, None]
    unit = torch.polar(torch.full_like(theta, st["scale"]), -theta if case.get("transposed") else theta)
    head, rest = x.split((case["rot"], d - case["rot"]), -1)
    if case["layout"] == "half":
        y = torch.view_as_real(torch.complex(*head.chunk(2, -1)) * unit).transpose(-1, -2)
    else:
        y = torch.view_as_real(torch.view_as_complex(head.reshape(B, H, N, -1, 2).contiguous()) * unit)
    return torch.cat((y.reshape(B, H, N, case["rot"]), rest), -1)


def _normed(x, w):
    return w * x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()


def _rows_exact(st, t, h):
    """The state after row t of all sequences at once, from h, the state before it."""
    z = st["gate"].select(-2, t).double() if t is not None else st["gate"].double()
    x = st["x"].select(-2, t).double() if t is not None else st["x"].double()
    if st["case"]["gate"] == "decay":
        return z * h + x
    if st["case"]["gate"] == "log":
        return torch.exp(z) * h + x
    return (h + x * torch.exp(-z)) / (1 + torch.exp(-z))


def _back_exact(st, t, h, D):
    """(dx, dgate, gradient of h) of row t, whose state came from h and has the gradient D."""
    z = st["gate"].select(-2, t).double()
    if st["case"]["gate"] == "decay":
        return D, D * h, D * z
    if st["case"]["gate"] == "log":
        return D, D * h * torch.exp(z), D * torch.exp(z)
    f = 1 / (1 + torch.exp(-z))
    f1 = 1 / (1 + torch.exp(z))
    return D * f1, D * (h - st["x"].select(-2, t).double()) * f * f1, D * f


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "scan_step":
        h = _rows_exact(st, None, st["state"].double())
        return h, h
    if op.startswith("scan"):
        B, N, C = st["x"].shape
        off = st["offsets"].tolist() if st["offsets"] is not None else None
        spans = list(zip(off[:-1], off[1:])) if off else [(0, N)]
        zero = torch.zeros((len(spans) if off else B, C), dtype=torch.float64, device=st["x"].device)
        if op == "scan":
            out = st["out"].double()
            left = st["state_in"].double() if "state_in" in st else zero.clone()
            for s, (lo, hi) in enumerate(spans):
                h = left[s:s + 1] if off else left
                for t in range(lo, hi):
                    h = _rows_exact(st, t, h)
                    out[:, t] = h
                if off:
                    left[s] = h[0]
                else:
                    left = h
            return (out, left) if "state_in" in st else out
        dx, dgate = st["dx"].double(), st["dgate"].double()
        entered = st["dstate_out"].double() if "dstate_out" in st else zero.clone()
        enters = st["state_in"].double() if "state_in" in st else zero
        for s, (lo, hi) in enumerate(spans):
            G = entered[s:s + 1] if off else entered
            first = enters[s:s + 1] if off else enters
            for t in range(hi - 1, lo - 1, -1):
                h = st["h"][:, t - 1].double() if t > lo else first
                dx[:, t], dgate[:, t], G = _back_exact(st, t, h, st["dh"][:, t].double() + G)
            if off:
                entered[s] = G[0]
            else:
                entered = G
        return (dx, dgate, entered) if "state_in" in st else (dx, dgate)
    q, k = st["q"].double(), st["k"].double()
    if op == "rope":
        return _turned(q, st, case), _turned(k, st, case)
    wq, wk = st["wq"].double(), st["wk"].double()
    if op == "norm_rope":
        return _turned(_normed(q, wq), st, case), _turned(_normed(k, wk), st, case)
    leaves = [t.detach().clone().requires_grad_() for t in (q, k, wq, wk)]
    with torch.enable_grad():
        y = _turned(_normed(leaves[0], leaves[2]), st, case), _turned(_normed(leaves[1], leaves[3]), st, case)
    return torch.autograd.grad(y, leaves, (st["dq"].double(), st["dk"].double()))
