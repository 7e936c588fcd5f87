"""The operators between the blocks of a diffusion transformer that this library is timed on, called as a denoising loop calls
them: the root-mean-square norm that takes the residual stream on by a block's output (in bf16, in fp32, and with an 8-bit output
and a scale per row), projections with bias, activation and residual (bf16, fp32, and on 8-bit operands), and the MLP layer that is
made of them.

With `own` false the operators are computed in their plain form (elementary torch operations in 32 bits, 64 where a value next to
a rounding border is decided, one rounding at the end), with `own` true by this library.
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, rows, dim, out=0, dtype="bf16", act="none", bias=True, delta=True):
    """norm, norm_q8: rows x dim, `delta`: with a block's output to add.  linear, linear_q8: rows x dim -> out, `delta`: with a
    residual.  layer: rows x dim, hidden width `out`, `delta`: with a block's output to add first."""
    return dict(name=name, op=op, rows=rows, dim=dim, out=out, dtype=dtype, act=act, bias=bias, delta=delta)


def listed():
    return [
        # the text tokens of a conditional and an unconditional half, 77 each: the smallest norm of a sampler's step
        _case("norm_text", "norm", 154, 1280),
        # the residual stream of 4 images of 128 x 128 tokens: all of it read and written once
        _case("norm_large", "norm", 65536, 640),
        # a high-resolution block's stream on its way into an 8-bit projection
        _case("norm_q8_high", "norm_q8", 8192, 640),
        # the first norm of a model, nothing to add yet, an odd number of rows
        _case("norm_q8_large", "norm_q8", 32767, 1280, delta=False),
        # a modulation vector out of the time embedding, one row for each half of the batch: weights are all there is to read
        _case("linear_embedding", "linear", 2, 1280, 5120, act="silu", delta=False),
        # keys out of the text tokens: few rows, a long contraction
        _case("linear_text", "linear", 154, 2048, 1280, delta=False),
        # a down projection added to the residual stream of 2 x 16384 tokens
        _case("linear_down_large", "linear", 32768, 2560, 640),
        # fp32 mode, a ragged number of rows: what a user checks a bf16 run against
        _case("linear_f32", "linear", 1003, 640, 2560, dtype="f32", act="gelu", delta=False),
        # the 8-bit down projection of two rows
        _case("q8_two_rows", "linear_q8", 2, 5120, 1280),
        # the 8-bit up projection of a large batch
        _case("q8_up_large", "linear_q8", 16384, 1280, 5120, act="gelu_tanh", delta=False),
        # the whole MLP layer of a mid-resolution block on its merged tokens
        _case("layer_mid", "layer", 1024, 1280, 5120, act="gelu"),
        # ... and of a high-resolution block on all of its tokens
        _case("layer_high", "layer", 8192, 640, 2560, act="gelu"),
    ]


def draw(rng):
    """One more call of the same ranges: 1 to 65536 rows, 64 to 4096 channels in steps of 8, every activation, with and without
    bias and residual; no more work than the largest listed call of its operator."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {}
    for c in listed():
        w = work(c)
        best = most.setdefault(c["op"], {"bytes": 0, "flops": 0})
        for key in best:
            best[key] = max(best[key], w[key])
    while True:
        op = rng.choice(["norm", "norm", "norm_q8", "linear", "linear", "linear_q8", "linear_q8", "layer"])
        c = _case("", op, log(1, 65536), 8 * log(8, 512), dtype="bf16", act=rng.choice(["none", "gelu", "gelu_tanh", "silu"]),
                  bias=rng.random() < 0.7, delta=rng.random() < 0.5)
        del c["name"]
        if op in ("norm", "norm_q8"):
            c.update(act="none", bias=False)
        else:
            c["out"] = 8 * log(8, 640)
        if op == "layer":
            c["bias"] = True
        if op in ("norm", "linear", "layer") and rng.random() < 0.2:
            c["dtype"] = "f32"
        w = work(c)
        # fp32 projections run at a twentieth of the tensor cores' rate
        heavy = 16 if c["dtype"] == "f32" and op != "norm" else 1
        if heavy * w["flops"] <= most[op]["flops"] and w["bytes"] <= most[op]["bytes"]:
            return c


def work(case):
    m, k, n = case["rows"], case["dim"], case["out"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        return {"bytes": m * k * e * (4 if case["delta"] else 2) + k * e, "flops": 4 * m * k}
    if case["op"] == "norm_q8":
        return {"bytes": m * k * (7 if case["delta"] else 3) + k * e + 4 * m, "flops": 5 * m * k}
    if case["op"] == "linear":
        return {"bytes": e * (m * k + k * n + m * n * (2 if case["delta"] else 1) + (n if case["bias"] else 0)), "flops": 2 * m * n * k}
    if case["op"] == "linear_q8":
        return {"bytes": m * k + k * n + 2 * m * n * (2 if case["delta"] else 1) + (2 * n if case["bias"] else 0) + 4 * (m + n), "flops": 2 * m * n * k}
    return {"bytes": e * (m * k * (3 if case["delta"] else 2) + 2 * k * n + 2 * k + n), "flops": 4 * m * n * k}


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _stream(gen, rows, dim, dtype):
    """A residual stream: tokens of different lengths, and a few channels that are much larger than the others."""
    length = torch.exp(0.5 * _normal(gen, rows, 1))
    loud = torch.where(torch.rand(dim, generator=gen, device="cuda") < 0.01, 12.0, 1.0)
    return (_normal(gen, rows, dim) * length * loud).to(dtype)


def _to_8_bits(t):
    """Rows of t in e4m3 with a scale for each."""
    scale = t.abs().amax(1).clamp_min(1e-20) / E4M3_MAX
    return (t / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    m, k, n, dt = case["rows"], case["dim"], case["out"], TORCH[case["dtype"]]
    s = {"case": case}

    def empty(rows, cols, dtype=dt):
        return torch.empty(rows, cols, dtype=dtype, device="cuda")

    if case["op"] in ("norm", "norm_q8", "layer"):
        s["x"] = _stream(gen, m, k, dt)
        s["delta"] = _normal(gen, m, k).to(dt) if case["delta"] else None
        s["weight"] = (1 + 0.2 * _normal(gen, k)).to(dt)
    if case["op"] in ("norm", "norm_q8"):
        s["sum"] = empty(m, k) if case["delta"] else None
    if case["op"] == "norm":
        s["y"] = empty(m, k)
    elif case["op"] == "norm_q8":
        # rows of whole 16-byte packets, as the 8-bit projection reads them
        s["q"] = empty(m, (k + 15) // 16 * 16, torch.float8_e4m3fn)[:, :k]
        s["scale"] = torch.empty(m, device="cuda")
    elif case["op"] == "layer":
        s["w1"], s["b1"] = (_normal(gen, k, n) / math.sqrt(k)).to(dt), (0.1 * _normal(gen, n)).to(dt)
        s["w2"], s["b2"] = (_normal(gen, n, k) / math.sqrt(n)).to(dt), (0.1 * _normal(gen, k)).to(dt)
        # room for the normalised rows and the hidden rows, and for each to begin on a line of its own
        s["y"], s["ws"] = empty(m, k), torch.empty(s["x"].element_size() * m * (k + n) + 1024, dtype=torch.uint8, device="cuda")
    else:
        s["bias"] = (0.1 * _normal(gen, n)).to(dt) if case["bias"] else None
        s["residual"] = _stream(gen, m, n, dt) if case["delta"] else None
        s["y"] = empty(m, n)
        a, w = _normal(gen, m, k), _normal(gen, k, n) / math.sqrt(k)
        if case["op"] == "linear":
            s["a"], s["w"] = a.to(dt), w.to(dt)
        else:
            pad = (k + 15) // 16 * 16  # rows of whole 16-byte packets
            for name, t in (("a", a), ("w", w.t())):
                q, s[name + "_scale"] = _to_8_bits(t)
                s[name] = empty(t.shape[0], pad, torch.float8_e4m3fn)[:, :k]
                s[name].copy_(q)
    return s


def _activate(v, act):
    if act == "gelu":
        return v * 0.5 * torch.erfc(-v / math.sqrt(2.0))
    if act == "gelu_tanh":
        return v / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return v


def _norm(s):
    """The stream after the addition, in its type, and 1 / rms of its rows in 32 bits."""
    h = s["x"] if s["delta"] is None else (s["x"].float() + s["delta"].float()).to(s["x"].dtype)
    h32 = h.float()
    return h, h32, torch.rsqrt(h32.square().mean(1, keepdim=True) + EPS)


def _linear(v, s, dtype):
    v = v if s["bias"] is None else v + s["bias"].float()
    v = _activate(v, s["case"]["act"])
    return (v if s["residual"] is None else v + s["residual"].float()).to(dtype)


def run(state):
    s, op, act = state, state["case"]["op"], state["case"]["act"]
    if own:
        import paper_2509_10918_b200 as toma
        if op == "norm":
            toma.toma_rms_norm(s["x"], s["weight"], s["y"], EPS, delta=s["delta"], sum_out=s["sum"])
            return s["y"] if s["sum"] is None else (s["y"], s["sum"])
        if op == "norm_q8":
            toma.toma_rms_norm_q8(s["x"], s["weight"], s["q"], s["scale"], EPS, delta=s["delta"], sum_out=s["sum"])
            return (s["q"], s["scale"]) if s["sum"] is None else (s["q"], s["scale"], s["sum"])
        if op == "linear":
            toma.toma_linear_act(s["a"], s["w"], s["y"], bias=s["bias"], act=act, residual=s["residual"])
        elif op == "linear_q8":
            toma.toma_linear_q8(s["a"], s["a_scale"], s["w"], s["w_scale"], s["y"], bias=s["bias"], act=act, residual=s["residual"])
        else:
            toma.toma_mlp_layer(s["x"], s["weight"], s["w1"], s["b1"], s["w2"], s["b2"], s["y"], s["ws"], act=act, eps=EPS, delta=s["delta"])
        return s["y"]
    if op == "linear":
        return _linear(s["a"].float() @ s["w"].float(), s, s["y"].dtype)
    if op == "linear_q8":
        return _linear((s["a"].float() @ s["w"].float().t()) * s["a_scale"][:, None] * s["w_scale"], s, s["y"].dtype)
    h, h32, r = _norm(s)
    w = s["weight"].float()
    if op == "norm":
        y = (h32 * r * w).to(h.dtype)
        return y if s["sum"] is None else (y, h)
    if op == "norm_q8":
        # 1 / rms is in the scale alone.  The product with 448 is exact in 64 bits and the quotient rounded once, so a value
        # half way between two 8-bit numbers is there exactly and no other looks like one
        p = (h32 * w).double()
        top = p.abs().amax(1)
        q = _round_e4m3(p * E4M3_MAX / top[:, None]).float().to(torch.float8_e4m3fn)
        scale = (top * r[:, 0].double() / E4M3_MAX).float()
        return (q, scale) if s["sum"] is None else (q, scale, h)
    # the layer's normalised and hidden rows are tensors in the stream's type
    y = (h32 * r * w).to(h.dtype)
    t = _activate(y.float() @ s["w1"].float() + s["b1"].float(), act).to(h.dtype)
    return (t.float() @ s["w2"].float() + s["b2"].float() + h32).to(h.dtype)


def _round_e4m3(v):
    """64-bit values to the nearest of 8 bits (1, 4, 3), ties to the even one; values below 2^-6 in steps of 2^-9."""
    exponent = torch.frexp(v)[1] - 1
    step = torch.exp2(torch.clamp(exponent, min=-6).double() - 3)
    return torch.round(v / step) * step


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    op, d = case["op"], {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and k not in ("y", "q", "sum", "scale", "ws")}

    def function(v):
        if act == "gelu":
            return v * torch.special.ndtr(v)
        if act == "gelu_tanh":
            return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
        return v * torch.sigmoid(v) if act == "silu" else v

    def nearest(v):
        """The nearest of the 127 magnitudes that 8 bits stand for; half way between two, the one with the even code."""
        codes = torch.arange(127, device="cuda")
        e, f = codes // 8, (codes % 8).double()
        values = torch.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * torch.exp2(e.double() - 7))
        middles = (values[1:] + values[:-1]) / 2
        low, high = torch.searchsorted(middles, v.abs()), torch.searchsorted(middles, v.abs(), right=True)
        return torch.sign(v) * values[torch.where(low % 2 == 0, low, high)]

    act = case["act"]
    if op in ("linear", "linear_q8"):
        v = d["a"] @ (d["w"] if op == "linear" else d["w"].t())
        if op == "linear_q8":
            v = torch.outer(d["a_scale"], d["w_scale"]) * v
        return function(v + d.get("bias", 0)) + d.get("residual", 0)
    dt = TORCH[case["dtype"]]
    stored = lambda v: v.to(dt).double()  # noqa: E731
    total = d["x"] + d["delta"] if case["delta"] else d["x"]
    h = stored(total)  # the stream is a tensor of its type, and the norm's input
    rms = torch.sqrt((h * h).sum(1) / h.shape[1] + EPS)
    y = h * d["weight"] / rms[:, None]
    if op == "norm":
        return (y, total) if case["delta"] else y
    if op == "norm_q8":
        p = h * d["weight"]
        top = p.abs().max(1).values
        q, scale = nearest(p * E4M3_MAX / top[:, None]), top / rms / E4M3_MAX
        return (q, scale, total) if case["delta"] else (q, scale)
    hidden = function(stored(y) @ d["w1"] + d["b1"])
    return stored(hidden) @ d["w2"] + d["b2"] + h
