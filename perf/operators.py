"""Performance cases of the 8-bit operators: rows and weights in e4m3 with a power-of-two scale for each block of 128 (a run
of 128 values of a row, a 128 x 128 block of a weight), the products that read them, and what a backward pass makes of them.

Operators ("op"):
  store     rows of bf16 or fp32 -> 8-bit rows and their scales (mb_fp8_quant)
  weights   a weight matrix -> 8 bits, as it is stored and transposed (mb_fp8_quant_weight)
  restore   8-bit rows -> bf16 or fp32 (mb_fp8_dequant)
  linear    8-bit rows times an 8-bit weight; a data gradient is the same call on the transposed weight (mb_linear_fp8_fwd)
  wgrad     weight gradient of such a product from its stored 8-bit rows; dy in bf16 or in 8 bits (mb_linear_fp8_wgrad)
  act       both input projections of the GeGLU feed-forward, its gate, and the result in 8 bits (mb_geglu_fp8_act)
  gate_bwd  backward of the gate, h | g from an 8-bit store or in bf16, the result in 8 bits (mb_gelu_gate_fp8_bwd)

With `own` false a pass is elementary torch operations in fp32, rounded once at the end; with `own` true it is the library's call.
"""
import math

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCK = 128


def listed():
    return [
        # what eight short sequences keep of a layer's input: one small launch
        {"name": "store_small", "op": "store", "T": 945, "W": 768, "dtype": "bf16"},
        # the feed-forward's activation of the base model's microbatch, the largest thing a layer keeps
        {"name": "store_base", "op": "store", "T": 26963, "W": 3072, "dtype": "bf16"},
        # the fp32 master weight of the fused input projections, once per optimizer step
        {"name": "weights_base", "op": "weights", "n_out": 6144, "n_in": 768, "dtype": "f32"},
        # the microbatch's rows back in bf16, for an operator that reads no 8-bit rows
        {"name": "restore_base", "op": "restore", "T": 26963, "W": 768, "dtype": "bf16"},
        # serving, one token: the weight's way through memory and the launch
        {"name": "linear_one", "op": "linear", "T": 1, "n_in": 1024, "n_out": 4096, "dtype": "bf16"},
        # the masked-token head on 30 % of a microbatch: a vocabulary that ends inside a block
        {"name": "linear_vocab", "op": "linear", "T": 8089, "n_in": 768, "n_out": 30528, "dtype": "bf16"},
        # a wide layer on long documents, bound by the matrix cores
        {"name": "linear_large", "op": "linear", "T": 32768, "n_in": 4096, "n_out": 4096, "dtype": "bf16"},
        # query, key and value weights of a small fine-tuning batch
        {"name": "wgrad_small", "op": "wgrad", "T": 945, "n_in": 768, "n_out": 2304, "dy": "bf16"},
        # the input projections' weights, base microbatch, from dh | dg as the gate's backward leaves them
        {"name": "wgrad_base", "op": "wgrad", "T": 26963, "n_in": 768, "n_out": 6144, "dy": "fp8"},
        # feed-forward of a small batch
        {"name": "act_small", "op": "act", "T": 945, "hidden": 768, "inter": 3072},
        # feed-forward of the base microbatch
        {"name": "act_base", "op": "act", "T": 26963, "hidden": 768, "inter": 3072},
        # its gate backwards, h | g kept in 8 bits
        {"name": "gate_bwd_base", "op": "gate_bwd", "T": 26963, "inter": 3072, "hg": "fp8"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row's width: a multiple of 16 values, odd ones and ones that end inside a block among them."""
    if rng.random() < 0.4:
        return rng.choice([w for w in (256, 512, 768, 1024, 2304, 4096) if lo <= w <= hi])
    return 16 * _log_int(rng, lo // 16, hi // 16)


def draw(rng):
    op = rng.choice(["store", "weights", "restore", "linear", "linear", "linear", "wgrad", "wgrad", "act", "gate_bwd"])
    T = _log_int(rng, 1, 32768)
    if op in ("store", "restore"):
        W = _width(rng, 64, 4096)
        return {"op": op, "T": min(T, 26963 * 3072 // W), "W": W, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if op == "weights":
        return {"op": op, "n_out": _width(rng, 64, 4096), "n_in": _width(rng, 64, 4096), "dtype": rng.choice(["bf16", "f32"])}
    if op == "linear":
        return {"op": op, "T": T, "n_in": _width(rng, 64, 4096), "n_out": _width(rng, 64, 4096),
                "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"])}
    if op == "wgrad":
        return {"op": op, "T": T, "n_in": _width(rng, 64, 2304), "n_out": _width(rng, 64, 4096), "dy": rng.choice(["bf16", "fp8"])}
    inter = BLOCK * _log_int(rng, 1, 32)
    if op == "act":
        return {"op": op, "T": T, "hidden": _width(rng, 64, 1024), "inter": inter}
    return {"op": op, "T": min(T, 26963 * 3072 // inter), "inter": inter, "hg": rng.choice(["bf16", "fp8"])}


# ---------------------------------------------------------------------------------------------------- plain forms
def _largest(x, rows):
    """Largest finite magnitude of each block of `rows` rows and 128 columns."""
    a = x.float().abs()
    a = torch.where(a < math.inf, a, 0.0)
    a = torch.nn.functional.pad(a, (0, -a.shape[1] % BLOCK, 0, -a.shape[0] % rows))
    return a.view(a.shape[0] // rows, rows, a.shape[1] // BLOCK, BLOCK).amax((1, 3))


def _spread(e, x, rows):
    """One value for each element of x from one for each block."""
    return e.repeat_interleave(rows, 0).repeat_interleave(BLOCK, 1)[:x.shape[0], :x.shape[1]]


def _store(x, rows=1):
    """x in e4m3 and the scales' bytes: the smallest power of two 2^e, e >= -126, that holds a block's values within 448."""
    m, k = torch.frexp(_largest(x, rows))           # 448 = 0.875 * 2^9
    e = (k - 9 + (m > 0.875).int()).clamp(min=-126)
    e = torch.where(m > 0, e, -126)
    factor = torch.exp2(-e.float())                 # (a power of two: exact)
    y = x.float() * _spread(factor, x, rows)
    y = torch.where(y.abs() <= 448.0, y, math.nan)
    return y.to(E4M3), (e + 127).to(torch.uint8).view(E8M0)


def _values(q, s, rows=1):
    """What 8-bit rows or weights stand for, fp32."""
    return q.float() * _spread(torch.exp2(s.view(torch.uint8).float() - 127.0), q, rows)


def _gelu(h):
    return 0.5 * h * torch.erfc(h * -math.sqrt(0.5))


def _gelu_slope(h):
    return 0.5 * torch.erfc(h * -math.sqrt(0.5)) + h * torch.exp(-0.5 * h * h) * (1.0 / math.sqrt(2.0 * math.pi))


# ---------------------------------------------------------------------------------------------------- inputs
def _normal(gen, shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=F32) * std


def _activations(gen, T, W):
    """Rows as a LayerNorm hands them over: unit variance, and one channel in a hundred a good deal larger."""
    large = torch.where(torch.rand(W, generator=gen, device="cuda") < 0.01, 12.0, 1.0)
    return _normal(gen, (T, W)) * large


def _gradients(gen, T, W):
    """Gradient rows: small, and of very different size from token to token."""
    return _normal(gen, (T, W), 1e-3) * torch.exp(_normal(gen, (T, 1)))


def _dtype(case):
    return F32 if case["dtype"] == "f32" else BF16


def prepare(case, seed):
    gen, op = torch.Generator(device="cuda").manual_seed(seed), case["op"]
    s = {"op": op}
    if op == "store":
        s["x"] = _activations(gen, case["T"], case["W"]).to(_dtype(case))
    elif op == "weights":
        s["w"] = _normal(gen, (case["n_out"], case["n_in"]), 0.02).to(_dtype(case))
    elif op == "restore":
        s["q"], s["s"] = _store(_activations(gen, case["T"], case["W"]))
        s["dtype"] = _dtype(case)
    elif op == "linear":
        s["xq"], s["xs"] = _store(_activations(gen, case["T"], case["n_in"]))
        s["wq"], s["ws"] = _store(_normal(gen, (case["n_out"], case["n_in"]), 0.02), BLOCK)
        s["dtype"] = _dtype(case)
    elif op == "wgrad":
        s["xq"], s["xs"] = _store(_activations(gen, case["T"], case["n_in"]))
        dy = _gradients(gen, case["T"], case["n_out"])
        s["dy"], s["dys"] = _store(dy) if case["dy"] == "fp8" else (dy.to(BF16), None)
    elif op == "act":
        s["xq"], s["xs"] = _store(_activations(gen, case["T"], case["hidden"]))
        s["wq"], s["ws"] = _store(_normal(gen, (2 * case["inter"], case["hidden"]), 0.02), BLOCK)
    else:
        s["da"] = _gradients(gen, case["T"], case["inter"]).to(BF16)
        hg = _normal(gen, (case["T"], 2 * case["inter"]), 0.8)
        s["hg"], s["hgs"] = _store(hg) if case["hg"] == "fp8" else (hg.to(BF16), None)
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def _mb():
    from paper_2312_17482_amd import binding
    return binding


def _run_store(s):
    q, sc = _mb().mb_fp8_quant(s["x"]) if own else _store(s["x"])
    return {"q": q, "s": sc}


def _run_weights(s):
    if own:
        q, sc, qt, st = _mb().mb_fp8_quant_weight(s["w"])
    else:
        q, sc = _store(s["w"], BLOCK)
        qt, st = q.t().contiguous(), sc.view(torch.uint8).t().contiguous().view(E8M0)
    return {"q": q, "s": sc, "qt": qt, "st": st}


def _run_restore(s):
    if own:
        return _mb().mb_fp8_dequant(s["q"], s["s"], s["dtype"])
    return _values(s["q"], s["s"]).to(s["dtype"])


def _run_linear(s):
    if own:
        return _mb().mb_linear_fp8_fwd(s["xq"], s["xs"], s["wq"], s["ws"], dtype=s["dtype"])
    return (_values(s["xq"], s["xs"]) @ _values(s["wq"], s["ws"], BLOCK).t()).to(s["dtype"])


def _run_wgrad(s):
    if own:
        return _mb().mb_linear_fp8_wgrad(s["dy"], s["xq"], s["xs"], dys=s["dys"])
    dy = s["dy"].float() if s["dys"] is None else _values(s["dy"], s["dys"])
    return dy.t() @ _values(s["xq"], s["xs"])


def _run_act(s):
    if own:
        q, sc = _mb().mb_geglu_fp8_act(s["xq"], s["xs"], s["wq"], s["ws"])
    else:
        hg = _values(s["xq"], s["xs"]) @ _values(s["wq"], s["ws"], BLOCK).t()
        inter = hg.shape[1] // 2
        q, sc = _store(_gelu(hg[:, :inter]) * hg[:, inter:])
    return {"q": q, "s": sc}


def _run_gate_bwd(s):
    if own:
        q, sc = _mb().mb_gelu_gate_fp8_bwd(s["da"], s["hg"], hgs=s["hgs"])
    else:
        da = s["da"].float()
        hg = s["hg"].float() if s["hgs"] is None else _values(s["hg"], s["hgs"])
        h, g = hg[:, :da.shape[1]], hg[:, da.shape[1]:]
        q, sc = _store(torch.cat((da * g * _gelu_slope(h), da * _gelu(h)), 1))
    return {"q": q, "s": sc}


_RUN = {"store": _run_store, "weights": _run_weights, "restore": _run_restore, "linear": _run_linear, "wgrad": _run_wgrad,
        "act": _run_act, "gate_bwd": _run_gate_bwd}


def run(s):
    return _RUN[s["op"]](s)


# ---------------------------------------------------------------------------------------------------- work
def _eight(rows, W):
    """Bytes of 8-bit rows and their scales."""
    return rows * (W + -(-W // BLOCK))


def work(case):
    """Each input read once and each output written once; a product's multiplications and additions."""
    op, T = case["op"], case.get("T", 0)
    e = 4 if case.get("dtype") == "f32" else 2
    if op in ("store", "restore"):
        W = case["W"]
        return {"bytes": e * T * W + _eight(T, W), "flops": 0}
    if op == "weights":
        n, k = case["n_out"], case["n_in"]
        return {"bytes": (e + 2) * n * k, "flops": 0}
    if op == "linear":
        n, k = case["n_out"], case["n_in"]
        return {"bytes": _eight(T, k) + n * k + e * T * n, "flops": 2 * T * n * k}
    if op == "wgrad":
        n, k = case["n_out"], case["n_in"]
        return {"bytes": _eight(T, k) + (2 * T * n if case["dy"] == "bf16" else _eight(T, n)) + 4 * n * k, "flops": 2 * T * n * k}
    if op == "act":
        hidden, inter = case["hidden"], case["inter"]
        return {"bytes": _eight(T, hidden) + 2 * inter * hidden + _eight(T, inter), "flops": 4 * T * inter * hidden}
    inter = case["inter"]
    hg = 4 * T * inter if case["hg"] == "bf16" else _eight(T, 2 * inter)
    return {"bytes": 2 * T * inter + hg + _eight(T, 2 * inter), "flops": 0}


# ---------------------------------------------------------------------------------------------------- 64 bits
def _exact_values(q, s, rows=1):
    n, k = q.shape
    scale = torch.pow(2.0, s.view(torch.uint8).double() - 127.0)
    out = torch.empty((n, k), dtype=F64, device=q.device)
    for j in range(scale.shape[1]):
        part = slice(j * BLOCK, min((j + 1) * BLOCK, k))
        column = scale[:, j] if rows == 1 else scale[torch.arange(n, device=q.device) // rows, j]
        out[:, part] = q[:, part].double() * column[:, None]
    return out


def _exact_store(y, rows=1):
    """The quotients before they are rounded to e4m3, and the scales."""
    n, k = y.shape
    nr, nc = -(-n // rows), -(-k // BLOCK)
    scale, q = torch.empty((nr, nc), dtype=F64, device=y.device), torch.empty_like(y)
    for j in range(nc):
        part = slice(j * BLOCK, min((j + 1) * BLOCK, k))
        top = y[:, part].abs().amax(1)
        if rows > 1:
            top = torch.stack([t.max() for t in top.split(rows)])
        scale[:, j] = torch.pow(2.0, torch.ceil(torch.log2(top / 448.0)).clamp(min=-126.0))
        column = scale[:, j] if rows == 1 else scale[torch.arange(n, device=y.device) // rows, j]
        q[:, part] = y[:, part] / column[:, None]
    return q, scale


def _exact_gate(h):
    """GeLU and its derivative."""
    cdf = 0.5 * torch.erfc(-h / math.sqrt(2.0))
    return h * cdf, cdf + h * torch.exp(-h * h / 2.0) / math.sqrt(2.0 * math.pi)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "store":
        q, sc = _exact_store(s["x"].double())
        return {"q": q, "s": sc}
    if op == "weights":
        q, sc = _exact_store(s["w"].double(), BLOCK)
        return {"q": q, "s": sc, "qt": q.t(), "st": sc.t()}
    if op == "restore":
        return _exact_values(s["q"], s["s"])
    x = _exact_values(s["xq"], s["xs"]) if "xq" in s else None
    if op == "wgrad":
        dy = s["dy"].double() if s["dys"] is None else _exact_values(s["dy"], s["dys"])
        return torch.matmul(dy.t().contiguous(), x)
    if op in ("linear", "act"):
        y = torch.matmul(x, _exact_values(s["wq"], s["ws"], BLOCK).t().contiguous())
        if op == "linear":
            return y
        inter = case["inter"]
        q, sc = _exact_store(_exact_gate(y[:, :inter])[0] * y[:, inter:])
        return {"q": q, "s": sc}
    da, inter = s["da"].double(), case["inter"]
    hg = s["hg"].double() if s["hgs"] is None else _exact_values(s["hg"], s["hgs"])
    value, slope = _exact_gate(hg[:, :inter])
    q, sc = _exact_store(torch.cat((da * hg[:, inter:] * slope, da * value), 1))
    return {"q": q, "s": sc}
