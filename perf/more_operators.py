"""What the operators around a layer's base projections are measured on.

Three operators of a serving step: `norm` (root-mean-square norm with the residual's addition, 16-bit output for the adapters
and 8-bit output with a scale per 128 columns for the base weights), `act` (the FFN's gated activation with the same outputs;
without a gate the quantisation of what the output projection reads) and `gemm` (product of 8-bit activations with 8-bit
weights, scaled per 128 columns of a row and per 128 x 128 of a weight; up to three weights that share their input).
`run` computes them in elementary torch operations, or, with `own`, by the framework's calls.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_DEV = "cuda"
_TOP = 448.0                   # largest e4m3 value
_LEAST = 2.0 ** -126           # a scale is at least this


def _ceil(a, b):
    return -(-a // b)


# ---- cases ---------------------------------------------------------------------------------------
def listed():
    return [
        # one request generates a token, 7B-shaped: the fp32 sum of projection and delta goes into the next norm; latency
        dict(name="norm_one", op="norm", n=1, d=4096, src="fp32", dt="bf16", res="bf16", y=True, q=True, offset=0.0),
        # a decode step of 512 requests, 13B-shaped
        dict(name="norm_decode_512", op="norm", n=512, d=5120, src="fp32", dt="bf16", res="bf16", y=True, q=True, offset=0.0),
        # the prompt batch (32 x 512 tokens) with the hidden size of the mixed workload, 16-bit projections
        dict(name="norm_prompt_16384", op="norm", n=16384, d=8192, src="bf16", dt="bf16", res="bf16", y=True, q=True, offset=0.0),
        # a ragged step: rows whose last block of 128 is not full, IEEE half, fp32 residual stream, weights stored less one
        dict(name="norm_ragged_777", op="norm", n=777, d=4168, src="fp16", dt="fp16", res="fp32", y=True, q=True, offset=1.0),
        # the FFN of a decode step of 512 requests, 13B-shaped: fp32 gate and up (base + delta)
        dict(name="act_decode_512", op="act", n=512, d=13824, src="fp32", dt="bf16", act="silu", gated=True, fused=False, y=True, q=True),
        # the FFN of the prompt batch, gate and up as halves of one 16-bit row
        dict(name="act_prompt_16384", op="act", n=16384, d=13824, src="bf16", dt="bf16", act="silu", gated=True, fused=True, y=True, q=True),
        # what attention gives, to 8 bits for the output projection: a chunk of 2048 tokens, 64 heads of 128
        dict(name="act_quant_2048", op="act", n=2048, d=8192, src="bf16", dt="bf16", act="none", gated=False, fused=False, y=False, q=True),
        # q, k, v of one token, 7B-shaped: the weights' bytes and latency
        dict(name="gemm_one", op="gemm", m=1, k=4096, ns="4096 4096 4096", out="fp32"),
        # up and gate of a decode step of 64 requests, 13B-shaped
        dict(name="gemm_decode_64", op="gemm", m=64, k=5120, ns="13824 13824", out="fp32"),
        # down projection of a decode step of 512 requests, 13B-shaped
        dict(name="gemm_decode_512", op="gemm", m=512, k=13824, ns="5120", out="fp32"),
        # the prompt batch through q, k, v with 64 query and 8 KV heads of 128: the largest product
        dict(name="gemm_prompt_16384", op="gemm", m=16384, k=8192, ns="8192 1024 1024", out="fp32"),
        # a chunk of a prompt, sizes off every tile: the last block of K not full, the last rows and columns neither
        dict(name="gemm_ragged_1111", op="gemm", m=1111, k=4176, ns="2056", out="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "act", "gemm", "gemm"])
    dt = rng.choice(["bf16", "bf16", "fp16"])
    y, q = rng.choice([(True, True), (True, True), (False, True), (True, False)])
    if op == "norm":
        d = 8 * _log(rng, 16, 1024)
        n = _log(rng, 1, 16384)
        return dict(op=op, n=n, d=d, src=rng.choice(["fp32", dt]), dt=dt, res=rng.choice(["none", dt, dt, "fp32"]), y=y, q=q,
                    offset=rng.choice([0.0, 0.0, 1.0]))
    if op == "act":
        d = 8 * _log(rng, 16, 1728)
        n = _log(rng, 1, 8192)
        act = rng.choice(["silu", "silu", "gelu", "none"])
        return dict(op=op, n=n, d=d, src=rng.choice(["fp32", dt]), dt=dt, act=act, gated=act != "none" and rng.random() < 0.8,
                    fused=rng.random() < 0.5, y=y, q=q)
    m = _log(rng, 1, 16384)
    k = 16 * _log(rng, 8, 864)
    ns = [8 * _log(rng, 8, 1728) for _ in range(rng.choice([1, 1, 2, 3]))]
    case = dict(op=op, m=m, k=k, ns=" ".join(map(str, ns)), out=rng.choice(["fp32", "fp32", "bf16", "fp16"]))
    while work(case)["flops"] > 2.7e12:
        case["m"] = max(1, case["m"] * 2 // 3)
    return case


def _ns(case):
    return [int(n) for n in case["ns"].split()]


# ---- inputs ----------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=_DEV)
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype, mul=1.0):
    return (torch.randn(shape, generator=g, device=_DEV) * mul).to(dtype)


def _loud(g, d):
    """Per-channel sizes: most near one, a few channels far louder, as in trained models' activations."""
    size = torch.exp(0.5 * torch.randn(d, generator=g, device=_DEV))
    return size * torch.where(torch.rand(d, generator=g, device=_DEV) < 0.004, 20.0, 1.0)


def _blocks(v, rows):
    """v [r, c] padded to whole blocks and seen as [r / rows, rows, c / 128, 128]."""
    r, c = v.shape
    v = torch.nn.functional.pad(v, (0, -c % 128, 0, -r % rows))
    return v.view(-1, rows, v.shape[1] // 128, 128)


def _quant(v, rows):
    """fp32 v as e4m3 values and a scale for each block of rows x 128."""
    b = _blocks(v, rows)
    scale = (b.abs().amax((1, 3)) / _TOP).clamp(min=_LEAST)
    q = (b / scale[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(-1, b.shape[2] * 128)[:v.shape[0], :v.shape[1]].contiguous(), scale.contiguous()


def _norm_inputs(case, seed):
    g = _gen(seed)
    n, d = case["n"], case["d"]
    loud = _loud(g, d)
    s = dict(x=(torch.randn((n, d), generator=g, device=_DEV) * loud).to(_DT[case["src"]]),
             weight=(_randn(g, (d,), torch.float32, 0.2) + 1.0 - case["offset"]).to(_DT[case["dt"]]), res=None)
    if case["res"] != "none":
        s["res"] = (torch.randn((n, d), generator=g, device=_DEV) * (4.0 * loud)).to(_DT[case["res"]])
    return s


def _act_inputs(case, seed):
    g = _gen(seed)
    n, d, dt = case["n"], case["d"], _DT[case["src"]]
    if not case["gated"]:
        return dict(gate=_randn(g, (n, 2 * d), dt, 1.5)[:, :d] if case["fused"] else _randn(g, (n, d), dt, 1.5), up=None)
    if case["fused"]:
        row = _randn(g, (n, 2 * d), dt, 1.5)
        return dict(gate=row[:, :d], up=row[:, d:])
    return dict(gate=_randn(g, (n, d), dt, 1.5), up=_randn(g, (n, d), dt, 1.5))


def _gemm_inputs(case, seed):
    g = _gen(seed)
    m, k = case["m"], case["k"]
    x, xs = _quant(torch.randn((m, k), generator=g, device=_DEV) * _loud(g, k), 1)
    ws = [_quant(torch.randn((n, k), generator=g, device=_DEV) * k ** -0.5, 128) for n in _ns(case)]
    return dict(x=x, xs=xs, w=[w for w, _ in ws], wscale=[s for _, s in ws])


_INPUTS = {"norm": _norm_inputs, "act": _act_inputs, "gemm": _gemm_inputs}


def prepare(case, seed):
    """Inputs, and the buffers that a server keeps from step to step."""
    s = _INPUTS[case["op"]](case, seed)
    s["case"] = case
    if case["op"] == "gemm":
        s["out"] = [torch.empty((case["m"], n), dtype=_DT[case["out"]], device=_DEV) for n in _ns(case)]
        return s
    n, d = case["n"], case["d"]
    s["y"] = torch.empty((n, d), dtype=_DT[case["dt"]], device=_DEV) if case["y"] else None
    s["q"] = torch.empty((n, _ceil(d, 16) * 16), dtype=torch.float8_e4m3fn, device=_DEV)[:, :d] if case["q"] else None
    s["scale"] = torch.empty((n, _ceil(d, 128)), dtype=torch.float32, device=_DEV) if case["q"] else None
    if case["op"] == "norm":
        s["res_out"] = torch.empty_like(s["res"]) if s["res"] is not None else None
    return s


# ---- the plain forms -------------------------------------------------------------------------------
def _plain_outputs(s, v):
    out = {}
    if s["y"] is not None:
        out["y"] = v.to(s["y"].dtype)
    if s["q"] is not None:
        out["q"], out["scale"] = _quant(v, 1)
    return out


def _plain_norm(s):
    h = s["x"].float()
    if s["res"] is not None:
        h = h + s["res"].float()
    inv = 1.0 / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-5)
    out = _plain_outputs(s, h * inv * (s["weight"].float() + s["case"]["offset"]))
    if s["res"] is not None:
        out["res"] = h.to(s["res"].dtype)
    return out


def _plain_act(s):
    v = s["gate"].float()
    if s["case"]["act"] == "silu":
        v = v / (1.0 + torch.exp(-v))
    elif s["case"]["act"] == "gelu":
        v = 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    if s["up"] is not None:
        v = v * s["up"].float()
    return _plain_outputs(s, v)


def _plain_values(q, scale, rows):
    b = _blocks(q.float(), rows) * scale[:, None, :, None]
    return b.view(-1, b.shape[2] * 128)[:q.shape[0], :q.shape[1]]


def _plain_gemm(s):
    x = _plain_values(s["x"], s["xs"], 1)
    return [(x @ _plain_values(w, ws, 128).T).to(o.dtype) for w, ws, o in zip(s["w"], s["wscale"], s["out"])]


_PLAIN = {"norm": _plain_norm, "act": _plain_act, "gemm": _plain_gemm}


def run(state):
    s, case = state, state["case"]
    if not own:
        return _PLAIN[case["op"]](s)
    import paper_2608_05483_b200 as P
    if case["op"] == "gemm":
        return P.gemm_fp8(s["x"], s["xs"], s["w"], s["wscale"], out=s["out"])
    if case["op"] == "norm":
        P.rms_norm(s["x"], s["weight"], 1e-5, residual=s["res"], residual_out=s["res_out"], offset=case["offset"], y=s["y"], q=s["q"],
                   scale=s["scale"])
    else:
        P.gated_act(s["gate"], s["up"], act=case["act"], y=s["y"], q=s["q"], scale=s["scale"])
    out = {}
    if case["y"]:
        out["y"] = s["y"]
    if case["q"]:
        out["q"], out["scale"] = s["q"], s["scale"]
    if case["op"] == "norm" and s["res"] is not None:
        out["res"] = s["res_out"]
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------
_SIZE = {"none": 0, "fp32": 4, "bf16": 2, "fp16": 2}


def work(case):
    if case["op"] == "gemm":
        m, k, ns = case["m"], case["k"], _ns(case)
        kb = _ceil(k, 128)
        return {"bytes": m * k + 4 * m * kb + sum(n * k + 4 * _ceil(n, 128) * kb + m * n * _SIZE[case["out"]] for n in ns),
                "flops": 2 * m * k * sum(ns)}
    n, d = case["n"], case["d"]
    outs = 2 * n * d * case["y"] + (n * d + 4 * n * _ceil(d, 128)) * case["q"]
    if case["op"] == "norm":
        return {"bytes": n * d * (_SIZE[case["src"]] + 2 * _SIZE[case["res"]]) + 2 * d + outs, "flops": 6 * n * d}
    return {"bytes": n * d * _SIZE[case["src"]] * (1 + case["gated"]) + outs, "flops": 8 * n * d}


# ---- the definitions in 64 bits ---------------------------------------------------------------------
def _exact_outputs(case, v):
    """The values themselves where an output rounds them; q is what the 8 bits stand for before they are rounded."""
    out = {}
    if case["y"]:
        out["y"] = v
    if case["q"]:
        d = v.shape[1]
        top = torch.stack([v[:, a:a + 128].abs().amax(1) for a in range(0, d, 128)], 1)
        out["scale"] = torch.maximum(top / _TOP, torch.full_like(top, _LEAST))
        out["q"] = v / out["scale"].repeat_interleave(128, 1)[:, :d]
    return out


def _exact_norm(case, s):
    h = s["x"].double() if s["res"] is None else s["x"].double() + s["res"].double()
    length = torch.linalg.vector_norm(h, dim=1, keepdim=True)
    gain = s["weight"].double() + case["offset"]
    out = _exact_outputs(case, h / torch.sqrt(length ** 2 / case["d"] + 1e-5) * gain)
    if s["res"] is not None:
        out["res"] = h
    return out


def _exact_act(case, s):
    g = s["gate"].double()
    if case["act"] == "silu":
        g = g * torch.sigmoid(g)
    elif case["act"] == "gelu":
        g = g * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3))
    return _exact_outputs(case, g if s["up"] is None else g * s["up"].double())


def _exact_gemm(case, s):
    """Block of K by block of K: the products of the 8-bit values, then their scales."""
    outs = []
    for w, ws in zip(s["w"], s["wscale"]):
        acc = torch.zeros((case["m"], w.shape[0]), dtype=torch.float64, device=_DEV)
        cols = ws.double().repeat_interleave(128, 0)[:w.shape[0]]
        for b, a in enumerate(range(0, case["k"], 128)):
            part = s["x"][:, a:a + 128].double() @ w[:, a:a + 128].double().T
            acc += part * s["xs"][:, b:b + 1].double() * cols[:, b]
        outs.append(acc)
    return outs


def exact(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    return {"norm": _exact_norm, "act": _exact_act, "gemm": _exact_gemm}[case["op"]](case, s)
