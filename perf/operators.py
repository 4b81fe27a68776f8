"""Performance cases of the operators of an 8-bit, encoder-conditioned block.

Each case is one call that a sampling program makes of one operator, through
`paper_2609_38984_amd.swam`: the residual addition and RMS norm with 8-bit
output, the row quantiser, the 8-bit matrix product, and the cross attention
to an encoder's states.  Sizes are those of the repository's own workloads
(`workload/`, `bench.py`), or drawn around them.

`prepare` makes what such a program holds before the call, `run` is one pass
(in plain torch, or with `own` the framework's call), `exact` the same result
in float64.
"""
import math
import types

import torch

own = False

EPS = 1e-6


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _norm_case(rows, d, dtype="bf16", residual=True, gain=True, mod=True, pad=0, **kw):
    """pad: elements between the rows of x (a view into a wider buffer)."""
    return dict(op="norm", rows=rows, d=d, dtype=dtype, residual=residual, gain=gain, mod=mod, pad=pad, **kw)


def _quant_case(rows, d, dtype="bf16", pad=0, **kw):
    return dict(op="quant", rows=rows, d=d, dtype=dtype, pad=pad, **kw)


def _gemm_case(m, n, k, dtype="bf16", epilogue="bias", **kw):
    """epilogue: "none", "bias", "gelu" (bias, tanh-GELU) or "gated" (residual + gate (product + bias))."""
    return dict(op="gemm", m=m, n=n, k=k, dtype=dtype, epilogue=epilogue, **kw)


def _attn_case(batch, lq, lk, heads, kv_heads, dim, dtype="bf16", ragged=False, masked=False, shared=False, **kw):
    """lq, lk: the longest sequence's queries and keys; ragged: the others are
    shorter; masked: padded key sequences with a mask over the keys; shared:
    every second sequence attends its neighbour's keys."""
    return dict(op="attn", batch=batch, lq=lq, lk=lk, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype,
                ragged=ragged, masked=masked, shared=shared, **kw)


def listed():
    return [
        # the check run of a two-camera policy in float32: all 326 tokens of one step; latency
        _norm_case(326, 1536, "f32", name="norm_view2_f32"),
        # every token of the 10,160-token world-action model, as before its query projection
        _norm_case(10160, 1536, name="norm_wam"),
        # loading a float32 checkpoint: one MLP matrix [out][in] to codes with a scale per output channel
        _quant_case(1536, 6144, "f32", name="quant_weight_f32"),
        # the MLP hidden of the 17,472-token, d = 2048 model, as before its down projection
        _quant_case(17472, 8192, name="quant_hidden_d2048"),
        # one token (a conditioning or action token on its own): the weights' bytes and latency
        _gemm_case(1, 1536, 1536, name="gemm_1row"),
        # projecting 512 encoder states of width 4096 once per prompt, kept in float32
        _gemm_case(512, 1536, 4096, "f32", name="gemm_encoder_f32"),
        # down projection of the packed step (25% + 64 retained) of the world-action model into the residual
        _gemm_case(3472, 1536, 6144, epilogue="gated", name="gemm_wam_down_packed"),
        # the largest: MLP up projection of the d = 2048 model with its GELU
        _gemm_case(17472, 8192, 2048, epilogue="gelu", name="gemm_d2048_up"),
        # one query token for each of 8 sequences against 10,160 cached states: single-token serving
        _attn_case(8, 1, 10160, 24, 24, 64, name="cross_1tok_b8"),
        # a small policy in float32 against a 77-state prompt
        _attn_case(1, 326, 77, 24, 24, 64, "f32", name="cross_view2_f32"),
        # the world-action model against a prompt padded to 512 states
        _attn_case(1, 10160, 512, 24, 24, 64, masked=True, name="cross_wam"),
        # a serving batch of 8 retained sequences of unequal length, 128-wide heads in groups of 4, masked prompts
        _attn_case(8, 3360, 512, 12, 3, 128, ragged=True, masked=True, shared=True, name="cross_ragged_b8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(max(work(c)["flops"] / 300, work(c)["bytes"]) for c in listed())
    while True:
        op = rng.choice(["norm", "quant", "gemm", "gemm", "attn", "attn"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows = _log_int(rng, 1, 17472)
        if op == "norm":
            d = rng.choice([_log_int(rng, 48, 4096), 64 * rng.randint(1, 64)])
            c = _norm_case(rows, d, dtype, *(rng.random() < 0.6 for _ in range(3)), rng.choice([0, 0, 8, 3]))
        elif op == "quant":
            d = rng.choice([_log_int(rng, 48, 12000), 64 * rng.randint(1, 160)])
            c = _quant_case(rows, d, dtype, rng.choice([0, 0, 8, 5]))
        elif op == "gemm":
            n = rng.choice([_log_int(rng, 24, 8192), 64 * rng.randint(1, 128)])
            c = _gemm_case(rows, n, 16 * _log_int(rng, 2, 512), dtype, rng.choice(["none", "bias", "gelu", "gated"]))
        else:
            dim, group = rng.choice([64, 64, 128]), rng.choice([1, 1, 2, 4, 7])
            kv_heads = rng.randint(1, max(1, 2048 // (dim * group)))
            lq = rng.choice([1, _log_int(rng, 1, 10160)])
            c = _attn_case(rng.choice([1, 1, 2, 3, 8, 24]), lq, _log_int(rng, 1, 10160), kv_heads * group, kv_heads,
                           dim, dtype, *(rng.random() < 0.5 for _ in range(3)))
            # the plain form holds every weight of the softmax
            if c["batch"] * c["heads"] * c["lq"] * c["lk"] > 1.5e9:
                continue
        if max(work(c)["flops"] / 300, work(c)["bytes"]) <= most:
            return c


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------
def _lengths(case):
    """Queries and keys of every sequence, the keys of it that its mask shows,
    and the key sequence that each query sequence attends."""
    b, ragged = case["batch"], case["ragged"]
    lq = [case["lq"] if not ragged or i == 0 else max(1, case["lq"] * (4 + 5 * i % 7) // 10) for i in range(b)]
    lk = [case["lk"] if not ragged or i == 0 else max(1, case["lk"] * (3 + 3 * i % 8) // 10) for i in range(b)]
    # (the fifth prompt of a masked batch has no visible state at all)
    part = [0 if i == 4 else 4 + (5 * i + 3) % 7 for i in range(b)]
    seen = [min(n, -(-n * part[i] // 10)) if case["masked"] else n for i, n in enumerate(lk)]
    of = [i - i % 2 if case["shared"] else i for i in range(b)]
    return lq, lk, seen, of


def work(case):
    """One pass: every input read once, every output written once."""
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("norm", "quant"):
        n = float(case["rows"]) * case["d"]
        if case["op"] == "quant":
            return {"bytes": n * (es + 1) + 4.0 * case["rows"], "flops": 3.0 * n}
        each = es + 1 + (2 * es if case["residual"] else 0)
        row = case["d"] * (es * case["gain"] + 8 * case["mod"])
        return {"bytes": n * each + 4.0 * case["rows"] + row, "flops": 8.0 * n}
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        out = float(m) * n * es * (2 if case["epilogue"] == "gated" else 1)
        return {"bytes": float(m) * k + float(n) * k + out + 4.0 * (m + n), "flops": 2.0 * m * n * k}
    lq, lk, seen, of = _lengths(case)
    kv = sum(seen[i] for i in set(of))
    width = case["heads"] * case["dim"]
    pairs = float(sum(q * seen[i] for q, i in zip(lq, of)))
    return {"bytes": 2.0 * es * (sum(lq) * width + kv * case["kv_heads"] * case["dim"])
            + 4.0 * sum(lq) * case["heads"] + (sum(lk) if case["masked"] else 0),
            "flops": 4.0 * pairs * width}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(0x0B5 + int(seed))
    dt = _dtype(case)
    s = types.SimpleNamespace(case=case)

    def normal(shape, std=1.0, dtype=torch.float32):
        return torch.randn(shape, device="cuda", generator=g).mul_(std).to(dtype)

    def codes(rows, d):
        """A quantised normal matrix: codes with a spread of 127 / 4 and the scale of each row."""
        c = normal((rows, d), 127.0 / 4.0).round_().clamp_(-127, 127).to(torch.int8)
        return c, torch.exp(normal((rows,), 0.3)) * (4.0 / 127.0)

    if case["op"] in ("norm", "quant"):
        rows, d = case["rows"], case["d"]
        # activations with a few channels far above the others, as trained models have
        wide = torch.exp(normal((d,), 0.5))
        x = torch.randn((rows, d + case["pad"]), device="cuda", generator=g)
        x[:, :d] *= wide
        s.x = x.to(dt)[:, :d]
        if case["op"] == "norm":
            s.residual = normal((rows, d), 2.0, dt) if case["residual"] else None
            s.gain = (1.0 + normal((d,), 0.2)).to(dt) if case["gain"] else None
            s.shift, s.scale = (normal((d,), 0.3), normal((d,), 0.3)) if case["mod"] else (None, None)
        return s
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        s.a, s.a_scale = codes(m, k)
        s.w, s.w_scale = codes(n, k)
        s.w_scale = s.w_scale * k ** -0.5
        s.bias = normal((n,), 0.5, dt) if case["epilogue"] != "none" else None
        s.residual = normal((m, n), 1.0, dt) if case["epilogue"] == "gated" else None
        s.gate = normal((n,), 0.5) if case["epilogue"] == "gated" else None
        return s
    lq, lk, seen, of = _lengths(case)
    width = case["heads"] * case["dim"]
    s.q = normal((sum(lq), case["heads"], case["dim"]), 1.0, dt)
    # keys and values side by side, as one projection of the encoder's states leaves them
    kv = normal((sum(lk), 2, case["kv_heads"], case["dim"]), 1.0, dt)
    s.k, s.v = kv[:, 0], kv[:, 1]

    def offsets(n):
        return torch.tensor([0] + n, device="cuda").cumsum(0).to(torch.int32)

    s.cu_q, s.cu_k = offsets(lq), offsets(lk)
    s.kv_seq = torch.tensor(of, device="cuda", dtype=torch.int32) if case["shared"] else None
    s.mask = None
    if case["masked"]:
        # the padding of each prompt stands at its end or, every third one, at its start
        s.mask = torch.zeros(sum(lk), dtype=torch.bool, device="cuda")
        at = 0
        for i, (n, c) in enumerate(zip(lk, seen)):
            lo = at + (n - c if i % 3 == 2 else 0)
            s.mask[lo:lo + c] = True
            at += n
        # what padded states hold does not matter
        s.k[~s.mask] = float("nan")
        s.v[~s.mask] = float("inf")
    return s


def _config(case):
    """The context that the calls belong to: a mid-size model of the repository's workloads."""
    return types.SimpleNamespace(
        batch=1, d_model=1024, n_heads=16, head_dim=64, mlp_ratio=4, n_blocks=1, d_temb=128, n_ctx=256,
        n_frames=4, frame_h=16, frame_w=16, n_act=32, k_core=77, k_anchor=16, k_layer=6, cv_penalty=1.0,
        mass_threshold=0.0, reuse_R=2, dtype=case["dtype"])


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        # the context with its workspace, and the buffers that a sampling program reuses from call to call
        from paper_2609_38984_amd import swam
        s.ctx = swam.Context(_config(case))
        dt, dev = _dtype(case), dict(device="cuda")
        if case["op"] in ("norm", "quant"):
            s.codes = torch.empty((case["rows"], case["d"]), dtype=torch.int8, **dev)
            s.code_scale = torch.empty(case["rows"], **dev)
            s.held = torch.empty((case["rows"], case["d"]), dtype=torch.bfloat16, **dev)
            s.total = torch.empty((case["rows"], case["d"]), dtype=dt, **dev)
        elif case["op"] == "gemm":
            s.c = torch.empty((case["m"], case["n"]), dtype=dt, **dev)
        else:
            s.o = torch.empty_like(s.q)
            s.lse = torch.empty(s.q.shape[:2], **dev)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _held(codes, scale, out=None):
    """The values that 8-bit codes stand for.  A code has 8 bits, as a bf16
    value has: they are returned in that type."""
    out = torch.empty(codes.shape, dtype=torch.bfloat16, device="cuda") if out is None else out
    return torch.mul(codes, scale[:, None], out=out)


def _quantize(y):
    """Codes and scale of rows in 64 bits: which code a value near a border
    gets is decided there."""
    top = y.abs().amax(1)
    codes = torch.where(top[:, None] > 0, torch.round(127.0 * y / top[:, None]), torch.zeros_like(y))
    return codes.float(), (top / 127.0).float()


def _plain_norm(s):
    t = s.x.double()
    if s.residual is not None:
        t = t + s.residual.double()
    y = t * torch.rsqrt(t.square().mean(1, keepdim=True) + EPS)
    if s.gain is not None:
        y = y * s.gain.double()
    if s.shift is not None:
        y = y * (1.0 + s.scale.double()) + s.shift.double()
    codes, scale = _quantize(y)
    out = {"y": _held(codes, scale), "scale": scale}
    if s.residual is not None:
        out["sum"] = t.to(s.x.dtype)
    return out


def _plain_gemm(s):
    acc = s.a.float() @ s.w.float().t()
    y = acc * s.a_scale[:, None] * s.w_scale
    if s.bias is not None:
        y = y + s.bias.float()
    if s.case["epilogue"] == "gelu":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if s.residual is not None:
        y = s.residual.float() + s.gate * y
    return {"c": y.to(_dtype(s.case))}


def _plain_attn(s):
    case = s.case
    cu_q, cu_k = s.cu_q.long(), s.cu_k.long()
    of = s.kv_seq.long() if s.kv_seq is not None else torch.arange(case["batch"], device="cuda")
    # every sequence padded to the longest
    row = torch.arange(case["lq"], device="cuda")
    col = torch.arange(case["lk"], device="cuda")
    iq = cu_q[:-1, None] + row
    ik = cu_k[of][:, None] + col
    has_q = iq < cu_q[1:, None]
    see = ik < cu_k[of + 1][:, None]
    iq, ik = torch.where(has_q, iq, 0), torch.where(see, ik, 0)
    if s.mask is not None:
        see = see & s.mask[ik]
    group = case["heads"] // case["kv_heads"]
    live = see[:, :, None, None]
    k = torch.where(live, s.k[ik].float(), 0.0).repeat_interleave(group, 2)
    v = torch.where(live, s.v[ik].float(), 0.0).repeat_interleave(group, 2)
    q = s.q[iq].float().permute(0, 2, 1, 3).contiguous()
    logit = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * case["dim"] ** -0.5
    logit = logit.masked_fill_(~see[:, None, None, :], -math.inf)
    top = logit.amax(-1, keepdim=True).clamp_min(-3e38)
    p = logit.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v.permute(0, 2, 1, 3).contiguous()) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total))[..., 0]
    return {"o": o.permute(0, 2, 1, 3)[has_q].to(s.q.dtype), "lse": lse.permute(0, 2, 1)[has_q]}


def run(s):
    case = s.case
    if not own:
        if case["op"] == "norm":
            return _plain_norm(s)
        if case["op"] == "quant":
            codes, scale = _quantize(s.x.double())
            return {"y": _held(codes, scale), "scale": scale}
        return _plain_gemm(s) if case["op"] == "gemm" else _plain_attn(s)
    if case["op"] == "norm":
        total = s.total if s.residual is not None else None
        s.ctx.rms_norm_i8(s.x, s.codes, s.code_scale, residual=s.residual, sum_out=total, gain=s.gain,
                          shift=s.shift, scale=s.scale, eps=EPS)
        out = {"y": _held(s.codes, s.code_scale, s.held), "scale": s.code_scale}
        return out if total is None else dict(out, sum=total)
    if case["op"] == "quant":
        s.ctx.quantize_i8(s.x, s.codes, s.code_scale)
        return {"y": _held(s.codes, s.code_scale, s.held), "scale": s.code_scale}
    if case["op"] == "gemm":
        s.ctx.gemm_i8(s.a, s.a_scale, s.w, s.w_scale, s.c, bias=s.bias, residual=s.residual, gate=s.gate,
                      gelu=case["epilogue"] == "gelu")
        return {"c": s.c}
    s.ctx.cross_attention(s.q, s.k, s.v, s.o, cu_q=s.cu_q, cu_k=s.cu_k, kv_seq=s.kv_seq, key_mask=s.mask,
                          lse=s.lse)
    return {"o": s.o, "lse": s.lse}


# ---------------------------------------------------------------------------
# the same in float64, from the definitions
# ---------------------------------------------------------------------------
def _exact_rows(y):
    """The row's values on its grid of 255 levels."""
    top = y.abs().max(1, keepdim=True).values
    level = torch.round(127.0 * y / top.clamp_min(1e-300))
    return level * (top / 127.0), top[:, 0] / 127.0


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "quant":
        y, scale = _exact_rows(s.x.double())
        return {"y": y, "scale": scale}
    if case["op"] == "norm":
        t = s.x.double() if s.residual is None else s.residual.double() + s.x.double()
        length = torch.linalg.vector_norm(t, dim=1, keepdim=True) / math.sqrt(case["d"])
        y = t / torch.sqrt(length * length + EPS)
        y = y * s.gain.double() if s.gain is not None else y
        y = y + y * s.scale.double() + s.shift.double() if s.shift is not None else y
        y, scale = _exact_rows(y)
        out = {"y": y, "scale": scale}
        return out if s.residual is None else dict(out, sum=t)
    if case["op"] == "gemm":
        out = torch.empty((case["m"], case["n"]), dtype=torch.float64, device="cuda")
        w = (s.w.double() * s.w_scale.double()[:, None]).t().contiguous()
        for r in range(0, case["m"], 4096):
            y = (s.a[r:r + 4096].double() * s.a_scale[r:r + 4096, None].double()) @ w
            y = y if s.bias is None else y + s.bias.double()
            if case["epilogue"] == "gelu":
                y = y / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
            out[r:r + 4096] = y if s.residual is None else s.residual[r:r + 4096].double() + s.gate.double() * y
        return {"c": out}
    lq, lk, _, of = _lengths(case)
    group = case["heads"] // case["kv_heads"]
    o = torch.empty(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s.q.shape[:2], dtype=torch.float64, device="cuda")
    start = [sum(lk[:i]) for i in range(case["batch"])]
    at = 0
    for i, n in enumerate(lq):
        keys = slice(start[of[i]], start[of[i]] + lk[of[i]])
        k, v = s.k[keys], s.v[keys]
        if s.mask is not None:
            k, v = k[s.mask[keys]], v[s.mask[keys]]
        for h in range(case["heads"]):
            kt, vh = k[:, h // group].double().t().contiguous(), v[:, h // group].double()
            for r in range(at, at + n, 4096):
                e = min(at + n, r + 4096)
                logit = s.q[r:e, h].double() @ kt / math.sqrt(case["dim"])
                lse[r:e, h] = torch.logsumexp(logit, 1)
                o[r:e, h] = torch.exp(logit - lse[r:e, h, None]) @ vh
        at += n
    return {"o": o, "lse": lse}
