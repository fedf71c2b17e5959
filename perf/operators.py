"""Performance cases of the operators around the merged tokens' modules: the norm with the residual's addition, the
linear layer with its epilogue, both in 8 bits as well, and the feed-forward block made of them.

A case is a dict:
    op      "norm"    h = x + r, y = h rsqrt(mean h^2 + eps) g
            "linear"  y = act(x w + b) + r
            "ffn"     h = x + r, y = h + act(norm(h) w1 + b1) w2 + b2
    rows    tokens (or, for a norm of query and key heads, tokens times heads)
    K, N    widths: input and output of a linear layer; a norm's width is K; a block's width is K and its hidden width N
    x       type of the input: "f32", "bf16", or "mx8" (8-bit elements with a power-of-two scale per 32 channels).  A linear layer
            with `pack` gets its input in bf16 and packs it in the call, as after an attention
    y       type of the output: as x, "mx8" behind a norm that an 8-bit product follows, "bf16" behind an 8-bit product (inside
            a block of 8-bit products the first one's output is "mx8" too)
    w       "ffn": type of the weights ("mx8": the whole block runs its products in 8 bits)
    act     "none", "gelu" (by erf), "gelu_tanh", "silu"
    bias, res   whether there is a bias (or a gain), a residual input
"""
import math

import torch

own = False

EPS = 1e-6
ACTS = ("none", "gelu", "gelu_tanh", "silu")


def _case(name, op, rows, K, N=0, x="bf16", y="", w="", act="none", bias=True, res=False, pack=False):
    return dict(name=name, op=op, rows=rows, K=K, N=N, x=x, y=y or x, w=w or x, act=act, bias=bias, res=res, pack=pack)


def listed():
    return [
        # the tiny fp32 layer's merged tokens with text beside them: launches and host path
        _case("norm_tiny_f32", "norm", 205, 64, x="f32", res=True),
        # SDXL's first stage: two samples of 2048 merged tokens, residual stream kept
        _case("norm_sdxl1", "norm", 4096, 640, res=True),
        # queries of ten 64-wide heads, normalised per head before the attention
        _case("norm_heads", "norm", 40960, 64),
        # two 128 x 128 grids, every token, second stage's width: norm in front of an 8-bit product
        _case("norm_mx8_hires", "norm", 32768, 1280, y="mx8", res=True),
        # the timestep embedding of two samples: few rows, bound by reading the weights
        _case("linear_embed", "linear", 2, 1280, 5120, act="silu"),
        # odd token count and widths that fit no tile, fp32
        _case("linear_odd_f32", "linear", 947, 352, 1416, x="f32", act="gelu_tanh", res=True),
        # SDXL's first stage: the MLP's second product with the residual
        _case("linear_down", "linear", 4096, 2560, 640, res=True),
        # merged tokens of two 128 x 128 grids in a wide model: the largest
        _case("linear_up_large", "linear", 16384, 4096, 8192, act="gelu"),
        # projection behind the attention of SDXL's second stage with text tokens, packed in the call
        _case("mx8_proj", "linear", 2 * (512 + 77), 1280, 1280, x="mx8", y="bf16", res=True, pack=True),
        # the same large layer in 8 bits
        _case("mx8_up_large", "linear", 16384, 4096, 8192, x="mx8", y="bf16", act="gelu"),
        # the feed-forward block of SDXL's second stage on merged tokens
        _case("ffn_sdxl2", "ffn", 1024, 1280, 5120, act="gelu", res=True),
        # the same of the first stage of a 128 x 128 grid, products in 8 bits
        _case("ffn_mx8_hires", "ffn", 16384, 640, 2560, w="mx8", act="gelu", res=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["norm", "linear", "linear", "linear", "ffn"])
        act = rng.choice(ACTS)
        bias, res = rng.random() < 0.8, rng.random() < 0.5
        if op == "norm":
            x = rng.choice(["f32", "bf16", "bf16"])
            c = _case("", op, log_int(1, 65536), 32 * log_int(1, 256), x=x, y=rng.choice([x, "mx8"]), bias=bias, res=res)
        elif op == "linear":
            x = rng.choice(["f32", "bf16", "bf16", "mx8", "mx8"])
            if x == "mx8":
                c = _case("", op, log_int(1, 16384), 32 * log_int(2, 256), 8 * log_int(8, 1024), x, "bf16", act=act, bias=bias,
                          res=res, pack=rng.random() < 0.4)
            else:
                c = _case("", op, log_int(1, 16384), 8 * log_int(8, 1024), 8 * log_int(8, 1024), x, act=act, bias=bias, res=res)
        else:
            x, w = rng.choice([("f32", "f32"), ("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "mx8"), ("bf16", "mx8")])
            K = 32 * log_int(2, 64)
            c = _case("", op, log_int(1, 16384), K, 32 * max(2, round(K / 32 * rng.uniform(2, 5))), x, w=w, act=act, bias=bias, res=res)
        w = work(c)
        if w["flops"] > (1.0e11 if c["x"] == "f32" else 1.1e12) or w["bytes"] > 4.7e8:
            continue
        del c["name"]
        return c


def _size(t):
    return {"f32": 4.0, "bf16": 2.0, "mx8": 1.0 + 1.0 / 32}[t]


def work(case):
    rows, K, N, x, y, w = (case[k] for k in ("rows", "K", "N", "x", "y", "w"))
    xin = "bf16" if case["pack"] else x
    b = case["bias"] * (4 if x == "f32" else 2)
    if case["op"] == "norm":
        return {"bytes": rows * K * (_size(x) * (1 + 2 * case["res"]) + _size(y)) + K * b, "flops": 5.0 * rows * K}
    if case["op"] == "linear":
        r = 4 if x == "f32" else 2
        return {"bytes": rows * K * _size(xin) + K * N * _size(x) + rows * N * (_size(y) + case["res"] * r) + N * b,
                "flops": 2.0 * rows * K * N}
    return {"bytes": rows * K * _size(x) * (2 + case["res"]) + 2 * K * N * _size(w) + (2 * K + N) * b, "flops": 4.0 * rows * K * N}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _dtype(t):
    return torch.float32 if t == "f32" else torch.bfloat16


def _pack(x):
    """8-bit elements and scale codes of the rows of x [rows, K]: per 32 channels the smallest power of two by which the largest
    magnitude fits 448; the scales' rows are padded to whole groups of four with code 0."""
    rows, K = x.shape
    b = x.float().reshape(rows, K // 32, 32)
    m, e = torch.frexp(b.abs().amax(-1))
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-127)
    e = torch.where(m == 0, torch.full_like(e, -127), e)
    q = torch.ldexp(b, -e[..., None]).to(torch.float8_e4m3fn).reshape(rows, K).view(torch.uint8)
    s = torch.zeros(rows, 4 * ((K + 127) // 128), dtype=torch.uint8, device=x.device)
    s[:, :K // 32] = (e + 127).to(torch.uint8)
    return q, s


def _value(q, s, dtype=torch.float32):
    """The values that packed rows stand for."""
    rows, K = q.shape
    scale = torch.exp2(s[:, :K // 32].to(dtype) - 127)
    return (q.view(torch.float8_e4m3fn).to(dtype).reshape(rows, K // 32, 32) * scale[..., None]).reshape(rows, K)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def tokens(rows, width):  # hidden states: a few channels stand out, tokens differ in norm
        return normal(rows, width) * (1 + 4 * (normal(width).abs() > 2.5)) * (0.5 + torch.rand(rows, 1, generator=g, device="cuda"))

    rows, K, N = case["rows"], case["K"], case["N"]
    s = {"case": dict(case)}
    dt = _dtype(case["x"])
    x = tokens(rows, K).to(dt)
    if case["op"] == "linear" and case["x"] == "mx8" and not case["pack"]:
        s["x"], s["xs"] = _pack(x)
    else:
        s["x"] = x
    out = K if case["op"] != "linear" else N
    if case["res"]:
        s["r"] = normal(rows, out).to(dt)
    if case["op"] != "linear" and case["bias"]:
        s["g"] = (1 + 0.1 * normal(K)).to(dt)
    for i, (k, n) in enumerate({"norm": [], "linear": [(K, N)], "ffn": [(K, N), (N, K)]}[case["op"]]):
        w = normal(k, n) * k ** -0.5
        if case["w"] == "mx8":
            s["w%d" % i], s["ws%d" % i] = _pack(w.t().contiguous())  # an 8-bit product takes its weights by output channel
        else:
            s["w%d" % i] = w.to(dt)
        if case["bias"]:
            s["b%d" % i] = (0.1 * normal(n)).to(dt)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------

def _act(v, act):
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return v


def _norm(s):
    h = s["x"].float()
    if "r" in s:
        h = h + s["r"].float()
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
    return h, y * s["g"].float() if "g" in s else y


def _product(x, s, i, mx8):
    v = x @ (_value(s["w%d" % i], s["ws%d" % i]).t() if mx8 else s["w%d" % i].float())
    return v + s["b%d" % i].float() if "b%d" % i in s else v


def _plain(s):
    c = s["case"]
    dt = _dtype(c["x"])
    if c["op"] == "norm":
        h, y = _norm(s)
        y = _value(*_pack(y)).to(torch.bfloat16) if c["y"] == "mx8" else y.to(dt)
        return {"h": h.to(dt), "y": y} if c["res"] else {"y": y}
    mx8 = c["w"] == "mx8"
    if c["op"] == "linear":
        x = s["x"].float() if not mx8 else _value(*_pack(s["x"])) if c["pack"] else _value(s["x"], s["xs"])
        v = _act(_product(x, s, 0, mx8), c["act"])
        if "r" in s:
            v = v + s["r"].float()
        return {"y": v.to(dt)}
    h, n = _norm(s)
    u = _act(_product(_value(*_pack(n)) if mx8 else n, s, 0, mx8), c["act"])
    return {"y": (h + _product(_value(*_pack(u)) if mx8 else u, s, 1, mx8)).to(dt)}


def _keep(s):
    """What a program keeps from call to call: descriptor, workspace and output buffers."""
    from paper_2509_10918_amd import binding as tb
    c = s["case"]
    rows, K, N = c["rows"], c["K"], c["N"]
    dt = _dtype(c["x"])
    k = {"tb": tb}
    if c["op"] == "norm":
        k["desc"] = tb.make_norm_desc(rows, K, EPS, c["x"], c["y"])
        k["h"] = torch.empty(rows, K, dtype=dt, device="cuda") if c["res"] else None
        if c["y"] == "mx8":
            k["q"] = tb.alloc_mx(rows, K)
        width = K
    elif c["op"] == "linear":
        k["desc"] = tb.make_linear_desc(rows, K, N, c["x"], c["y"], c["act"])
        k["ws"] = tb.alloc_linear_workspace(k["desc"])
        if c["pack"]:
            k["x"] = tb.alloc_mx(rows, K)
        width = N
    else:
        k["desc"] = tb.make_ffn_desc(rows, K, N, EPS, c["x"], c["w"], c["act"])
        k["ws"] = tb.alloc_ffn_workspace(k["desc"])
        width = K
    k["y"] = torch.empty(rows, width, dtype=torch.bfloat16 if c["y"] == "mx8" else dt, device="cuda")
    return k


def _own(s):
    if "keep" not in s:
        s["keep"] = _keep(s)
    k, c = s["keep"], s["case"]
    tb, desc = k["tb"], k["desc"]
    get = s.get
    if c["op"] == "norm":
        y, ys = k.get("q", (k["y"], None))
        tb.toma_rmsnorm(desc, s["x"], get("r"), get("g"), k["h"], y, ys)
        if ys is not None:
            tb.toma_mx_dequantize(y, ys, k["y"])
    elif c["op"] == "linear":
        x, xs = s["x"], get("xs")
        if c["pack"]:
            tb.toma_mx_quantize(x, *k["x"])
            x, xs = k["x"]
        tb.toma_linear(desc, x, xs, s["w0"], get("ws0"), get("b0"), get("r"), k["y"], None, k["ws"])
    else:
        tb.toma_ffn(desc, s["x"], get("r"), get("g"), s["w0"], get("ws0"), get("b0"), s["w1"], get("ws1"), get("b1"), k["y"], k["ws"])
    return {"h": k["h"], "y": k["y"]} if c["op"] == "norm" and c["res"] else {"y": k["y"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def _grid(v):
    """v [rows, K], 64 bits, on the 8-bit grid: e4m3 has steps of 2^-3 of a value's power of two, 2^-9 at least."""
    b = v.reshape(v.shape[0], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / 448))
    e = torch.where(top > 448 * torch.exp2(e), e + 1, torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e)).clamp(min=-127)
    t = b * torch.exp2(-e)
    p = torch.floor(torch.log2(torch.where(t == 0, torch.full_like(t, 2.0 ** -20), t.abs())))
    p = torch.where(t.abs() < torch.exp2(p), p - 1, torch.where(t.abs() >= torch.exp2(p + 1), p + 1, p)).clamp(min=-6)
    step = torch.exp2(p - 3)
    return (torch.round(t / step) * step * torch.exp2(e)).reshape(v.shape)


def exact(case, seed):
    s = prepare(case, seed)
    mx8 = case["w"] == "mx8"

    def d(name):
        return s[name].double() if name in s else 0.0

    def weight(i):
        return _value(s["w%d" % i], s["ws%d" % i], torch.float64).t().contiguous() if mx8 else d("w%d" % i)

    def act(v):
        if case["act"] == "gelu":
            return v * torch.special.ndtr(v)
        if case["act"] == "gelu_tanh":
            return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
        return v * torch.sigmoid(v) if case["act"] == "silu" else v

    if case["op"] == "linear":
        x = d("x") if not mx8 else _grid(d("x")) if case["pack"] else _value(s["x"], s["xs"], torch.float64)
        return {"y": act(x @ weight(0) + d("b0")) + d("r")}
    h = d("x") + d("r")
    n = h / torch.sqrt((h ** 2).sum(-1, keepdim=True) / case["K"] + EPS) * (d("g") if "g" in s else 1.0)
    if case["op"] == "norm":
        y = _grid(n) if case["y"] == "mx8" else n
        return {"h": h, "y": y} if case["res"] else {"y": y}
    u = act((_grid(n) if mx8 else n) @ weight(0) + d("b0"))
    return {"y": h + (_grid(u) if mx8 else u) @ weight(1) + d("b1")}
