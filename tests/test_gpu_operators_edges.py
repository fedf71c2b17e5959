"""The norm, linear and packing operators on the GPU where values are far out: tails of the activations, infinities and NaN, the ends of
the number ranges, and every kernel of the linear layer by its name.  Tolerances as in test_gpu_operators.py, relative to the
output wherever the inputs of the last step are exact."""
import pytest
import torch

from paper_2509_10918_amd import binding as tb

import operators_ref as ref
from test_gpu_operators import DT, HALF, NAN, check_linear, check_norm, ffn_call, ffn_inputs, gen, linear_case, randn, run_linear, within

pytestmark = pytest.mark.gpu
INF = float("inf")


def act64(v, name):
    """The activations without cancellation: v Phi(v) by the complementary error function, the others by a logistic function."""
    if name == "gelu":
        return 0.5 * v * torch.special.erfc(-v / 2 ** 0.5)   # (torch.special.ndtr is (1 + erf) / 2: off by 2 % at -7.8)
    if name == "gelu_tanh":
        return v * torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (v + 0.044715 * v ** 3))
    return v * torch.sigmoid(v) if name == "silu" else v


# ---- activations where they are small against their argument ----------------------------------------------------------------

def selecting_case(x_type, rows, K, N, lo, hi):
    """x with values from lo to hi, and weights that pick one channel of x for every column: the pre-activations are values of x, exactly
    (sums of one product and zeros)."""
    g = gen(rows + K + N)
    x = lo + (hi - lo) * torch.rand(rows, K, generator=g, device="cuda")
    k = torch.arange(N, device="cuda") % K
    w = torch.zeros(K, N, device="cuda")
    w[k, torch.arange(N, device="cuda")] = 1.0
    if x_type == "mx8":
        x, w = ref.pack(x.to(torch.bfloat16)), ref.pack(w.t().contiguous())
        return x, w, ref.unpack(*x)[:, k]
    x = x.to(DT[x_type])
    return (x, None), (w.to(DT[x_type]), None), x.double()[:, k]


# one size for each kernel, K split and none
SELECTING = [("bf16", 5, 64, 136), ("bf16", 3, 4096, 640), ("bf16", 200, 72, 136), ("bf16", 64, 4096, 256), ("bf16", 2000, 136, 2000), ("bf16", 4096, 640, 2560),
             ("bf16", 40, 24, 72), ("f32", 5, 64, 136), ("f32", 3, 8188, 260), ("f32", 947, 352, 1416), ("f32", 66, 4044, 136), ("f32", 40, 12, 72),
             ("mx8", 5, 64, 136), ("mx8", 77, 8192, 1280), ("mx8", 2000, 128, 2000), ("mx8", 1024, 1280, 5120), ("mx8", 4096, 640, 2560)]
SELECTING += [("bf16", 8190, 64, 4096), ("mx8", 8190, 160, 4096), ("mx8", 2000, 288, 2000)]


@pytest.mark.parametrize("act,lo,hi", [("gelu", -8.0, -3.0), ("gelu", -12.0, 3.0), ("gelu_tanh", -9.0, 3.0), ("silu", -80.0, 3.0)])
@pytest.mark.parametrize("x_type,rows,K,N", [c for c in SELECTING if c[0] != "f32"])
def test_tails_of_the_activations(x_type, rows, K, N, act, lo, hi):
    """Relative to the output: the fitted gelu is off by 2^-14.8 of v Q(|v|), and the exponentials' arguments, up to 116 powers of
    two here, by a few 2^-24 of themselves: 2^-14 in all, then half a step of the output."""
    print(f"[tail] {x_type} {rows} x {K} x {N} {act} {lo} .. {hi}", flush=True)
    x, w, v = selecting_case(x_type, rows, K, N, lo, hi)
    want = act64(v, act)
    for y_type in ("bf16", "mx8") if x_type == "mx8" else (x_type,):
        if y_type == "mx8" and N % 32:
            continue
        y, s = run_linear(x_type, y_type, x, w, None, None, act)
        if y_type == "mx8":
            sc = torch.exp2(s[:, :N // 32].double() - 127).repeat_interleave(32, 1)
            within(ref.unpack(y, s), want, want.abs() * (1 + 2.0 ** -14) * 2.0 ** -4 + want.abs() * 2.0 ** -14 + sc * 2.0 ** -10)
        else:
            within(y, want, want.abs() * (2.0 ** -8 + 2.0 ** -14 * (1 + 2.0 ** -8)))


@pytest.mark.parametrize("lo,hi", [(-8.0, -3.0), (-12.0, 3.0)])
@pytest.mark.parametrize("x_type,rows,K,N", [c for c in SELECTING if c[0] == "f32"])
def test_tail_of_gelu_in_fp32(x_type, rows, K, N, lo, hi):
    """v erfc(-v / sqrt 2) / 2: the argument has two roundings (the factor's and the product's, 2^-24 each at most), and an error of d
    in it changes the result by (v^2 + 1) d at most; erfc has four units in the last place (2^-21), the products less."""
    print(f"[tail] {x_type} {rows} x {K} x {N} {lo} .. {hi}", flush=True)
    x, w, v = selecting_case(x_type, rows, K, N, lo, hi)
    y, _ = run_linear(x_type, x_type, x, w, None, None, "gelu")
    want = act64(v, "gelu")
    within(y, want, want.abs() * (2.0 ** -23 * (v * v + 1) + 2.0 ** -20))


@pytest.mark.parametrize("act,lo,hi", [("silu", -80.0, 3.0), ("silu", -88.5, -80.0), ("gelu_tanh", -9.5, -8.0)])
@pytest.mark.parametrize("x_type,rows,K,N", [c for c in SELECTING if c[0] == "f32"])
def test_logistic_gates_in_fp32(x_type, rows, K, N, act, lo, hi):
    """fp32 to fp32 accuracy: v / (1 + e^-u) has the exponential's one unit in the last place (2^-23), the sum's and the quotient's
    roundings (2^-24 each), to which u's own come (gelu_tanh: a product of three with a constant and an addition: five)."""
    print(f"[gate] {x_type} {rows} x {K} x {N} {act} {lo} .. {hi}", flush=True)
    x, w, v = selecting_case(x_type, rows, K, N, lo, hi)
    want = act64(v, act)
    y, _ = run_linear(x_type, x_type, x, w, None, None, act)
    u = 2 * (2 / torch.pi) ** 0.5 * (v + 0.044715 * v ** 3)
    within(y, want, want.abs() * 2.0 ** -24 * (5 + (5 * u.abs() if act == "gelu_tanh" else 0)) * (1 + 2.0 ** -10))


# ---- every kernel by its name, over the number of its K steps ---------------------------------------------------------------------

# (type, rows, N, kernel): K steps of 128 bytes a row, whole and with a part of the last
STEPS = [("bf16", 2000, 2000, "medium_four_stages", range(1, 9)), ("mx8", 2000, 2000, "medium_four_stages", range(2, 9)), ("bf16", 3900, 2888, "medium", range(1, 6)),
         ("mx8", 3900, 2888, "medium", range(1, 6)), ("bf16", 8190, 4096, "large", range(1, 5)), ("mx8", 8190, 4096, "large", range(1, 6)),
         ("mx8", 300, 648, "small", range(1, 8))]
STEPS = [(x, rows, K, N, kernel) for x, rows, N, kernel, steps in STEPS for n in steps
         for K in ((64 * n, 64 * n + 40) if x == "bf16" else (128 * n, 128 * n + 32 * (1 + n % 3)))]


@pytest.mark.parametrize("x_type,rows,K,N,kernel", STEPS)
def test_every_number_of_K_steps(x_type, rows, K, N, kernel):
    """The loads that a kernel counts on run ahead of its last steps, and its stages are reused in turn: few steps, and every remainder."""
    y_type = "bf16" if x_type == "mx8" else x_type
    assert tb.toma_profile_linear_kernel(tb.make_linear_desc(rows, K, N, x_type, y_type, "silu")) == kernel
    check_linear(x_type, y_type, rows, K, N, "silu", True, False)


# ---- values that are not finite ---------------------------------------------------------------------------------------------

def same_values(got, want):
    """Equal, NaN where NaN."""
    got, want = got.double(), want.double()
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


WHOLE_BLOCKS = [(x, rows, K, (N + 31) // 32 * 32) for x, rows, K, N in SELECTING]


@pytest.mark.parametrize("x_type,rows,K,N", WHOLE_BLOCKS)
def test_activations_of_infinities_and_nan(x_type, rows, K, N):
    """Columns whose bias is infinite, NaN or huge: what the formula gives there, and every other column as without them.  The
    formulas have -inf times zero at -inf (NaN); packed outputs hold no infinity (NaN), and a block's scale goes by its finite values."""
    for act in ref.ACTS:
        print(f"[not finite] {x_type} {rows} x {K} x {N} {act}", flush=True)
        check_columns_that_are_not_finite(x_type, rows, K, N, act)


def check_columns_that_are_not_finite(x_type, rows, K, N, act):
    x, w, b, _, _, _ = linear_case(x_type, "", rows, K, N, act, True, False)
    at = {3: INF, 8: -INF, 21: NAN, N - 1: INF, N // 2: 2.0 ** 120, N // 2 + 1: -2.0 ** 120}
    odd = b.clone()
    for n, v in at.items():
        odd[n] = v
    want = {n: NAN if v == -INF and act != "none" else (0.0 if v < 0 and act != "none" else v) for n, v in at.items()}
    keep = [n for n in range(N) if n not in at]
    for y_type in ("bf16", "mx8") if x_type == "mx8" else (x_type,):
        y, s = run_linear(x_type, y_type, x, w, odd, None, act)
        if y_type == "mx8":
            y = ref.unpack(y, s)
            full, _ = run_linear(x_type, "bf16", x, w, odd, None, act)
            assert not s[:, N // 32:].any()
            # the codes of the finite values; an output beside the rounding to bf16 may lie on the other side of a border
            fin = torch.where(torch.isfinite(full), full.double(), torch.zeros_like(full, dtype=torch.float64))
            code = s[:, :N // 32].long()
            assert ((code >= ref.codes(fin * (1 - 2.0 ** -7))) & (code <= ref.codes(fin * (1 + 2.0 ** -7)))).all()
            for n, v in want.items():
                assert torch.isnan(y[:, n]).all() if v != v or v in (INF, -INF) else (y[:, n] == v).all(), (n, v)
            sc = torch.exp2(code.double() - 127).repeat_interleave(32, 1)
            within(y[:, keep], fin[:, keep], fin[:, keep].abs() * (2.0 ** -4 + 2.0 ** -7) + sc[:, keep] * 2.0 ** -10)
            continue
        plain, _ = run_linear(x_type, y_type, x, w, b, None, act)
        assert torch.equal(y[:, keep], plain[:, keep])
        for n, v in want.items():
            assert same_values(y[:, n], torch.full_like(y[:, n], v)) or (v in (2.0 ** 120, -2.0 ** 120) and (y[:, n].double() / v - 1).abs().max() <= 2.0 ** -20), (n, v)


@pytest.mark.parametrize("x_type,rows,K,N", WHOLE_BLOCKS)
def test_a_row_that_is_not_finite(x_type, rows, K, N):
    """One element of one row: all of that row and nothing else.  (8 bits: packing has made it NaN.)"""
    for act in ref.ACTS:
        for value in (INF, -INF, NAN):
            print(f"[not finite row] {x_type} {rows} x {K} x {N} {act} {value}", flush=True)
            check_row_that_is_not_finite(x_type, rows, K, N, value, act)


def check_row_that_is_not_finite(x_type, rows, K, N, value, act):
    g = gen(rows + K)
    e = DT["f32" if x_type == "f32" else "bf16"]
    xv, wv = randn(g, rows, K), randn(g, K, N) * K ** -0.5
    wv[5] = 0.25 * (1 - 2 * (torch.arange(N, device="cuda") % 2))   # (no zeros in the row of weights that the value meets)
    x0, w = xv.to(e), wv.to(e)
    x1, bad = x0.clone(), rows // 2
    x1[bad, 5] = value
    if x_type == "mx8":
        x0, x1, w = ref.pack(x0), ref.pack(x1), ref.pack(w.t().contiguous())
        assert torch.isnan(ref.unpack(*x1)[bad, 5])
        value = NAN
    else:
        x0, x1, w = (x0, None), (x1, None), (w, None)
    keep = [r for r in range(rows) if r != bad]
    pre = torch.full((N,), value, dtype=torch.float64, device="cuda") * (1 - 2 * (torch.arange(N, device="cuda") % 2))
    want = torch.where(pre < 0, torch.full_like(pre, NAN), pre) if act != "none" else pre
    for y_type in ("bf16", "mx8") if x_type == "mx8" else (x_type,):
        y, s = run_linear(x_type, y_type, x1, w, None, None, act)
        p, t = run_linear(x_type, y_type, x0, w, None, None, act)
        assert torch.equal(y[keep], p[keep])
        if y_type == "mx8":
            assert torch.equal(s[keep], t[keep]) and torch.isnan(ref.unpack(y, s)[bad]).all() and not s[bad].any()
        else:
            assert same_values(y[bad], want)


# ---- norm: accuracy of the row's statistic, and the end of its range ------------------------------------------------------------

@pytest.mark.parametrize("rows,C,res,gain", [(205, 64, True, True), (37, 128, False, True), (130, 640, True, True), (65, 1280, False, False), (17, 4096, True, False),
                                             (5, 8192, False, True), (3, 16384, True, True)])
def test_norm_to_fp32_accuracy(rows, C, res, gain):
    """x + r rounds once (u = 2^-24), which the sum of squares sees as 2 u; eight fused squares in fp32 add at most 8 u, the sums in
    fp64 nothing; the inverse root halves these 10 u, rounds once itself, and two products round: u + 5 u + u + 2 u."""
    print(f"[norm fp32] {rows} x {C} residual={res} gain={gain}", flush=True)
    g = gen(rows * 3 + C)
    x = randn(g, rows, C) * torch.exp2(torch.randint(-20, 21, (rows, 1), generator=g, device="cuda").float())
    r = randn(g, rows, C) if res else None
    gamma = 1 + 0.3 * randn(g, C) if gain else None
    y = torch.empty_like(x)
    tb.toma_rmsnorm(tb.make_norm_desc(rows, C, 1e-6, "f32"), x, r, gamma, None, y)
    _, want = ref.norm(x, r, gamma, float(torch.tensor(1e-6, dtype=torch.float32)))
    within(y, want, want.abs() * 9 * 2.0 ** -24 * (1 + 2.0 ** -10) + 2.0 ** -149)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [64, 1280, 8192])
@pytest.mark.parametrize("value", [2.0 ** 64, -2.0 ** 100])
def test_norm_of_a_row_whose_squares_leave_the_range(dtype, C, value):
    """Zeros in that row, plain and packed (codes 0), h as it is; the other rows as ever.  A row of 2^61 is still in the range."""
    g = gen(C)
    x = randn(g, 5, C).to(DT[dtype])
    x[3] = 2.0 ** 61
    x[1, 7] = value
    r = torch.zeros_like(x)
    d = {out: tb.make_norm_desc(5, C, 1e-6, dtype, out or dtype) for out in ("", "mx8")}
    h, y = torch.empty_like(x), torch.empty_like(x)
    tb.toma_rmsnorm(d[""], x, r, None, h, y)
    assert torch.equal(h, x) and not y[1].any()
    q, s = tb.alloc_mx(5, C)
    tb.toma_rmsnorm(d["mx8"], x, r, None, h, q.fill_(0x55), s.fill_(0x55))
    assert torch.equal(h, x) and not (q[1] & 0x7f).any() and not s[1].any()
    keep = [0, 2, 3, 4]
    check_norm(x[keep], None, None, 1e-6, "")
    check_norm(x[keep], None, None, 1e-6, "mx8")
    want = torch.empty_like(x[keep])
    tb.toma_rmsnorm(tb.make_norm_desc(4, C, 1e-6, dtype), x[keep], r[keep], None, None, want)
    assert torch.equal(y[keep], want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_norm_of_a_row_that_is_not_finite(dtype, value):
    """The formula's result: an infinity makes its own element NaN and the others zero, NaN makes the row NaN."""
    g = gen(4)
    x = randn(g, 6, 96).to(DT[dtype])
    x[2, 50] = value
    y, q, s = torch.empty_like(x), *tb.alloc_mx(6, 96)
    tb.toma_rmsnorm(tb.make_norm_desc(6, 96, 1e-6, dtype), x, None, None, None, y)
    tb.toma_rmsnorm(tb.make_norm_desc(6, 96, 1e-6, dtype, "mx8"), x, None, None, None, q, s)
    nan = torch.zeros(6, 96, dtype=torch.bool, device="cuda")
    nan[2, 50 if value == value else slice(None)] = True
    for v in (y.double(), ref.unpack(q, s)):
        assert torch.equal(torch.isnan(v), nan) and not torch.nan_to_num(v[2]).any()
    check_norm(x[[0, 1, 3, 4, 5]], None, None, 1e-6, "")


# ---- packing at the ends of the range ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_unpacking_the_ends_of_the_range(dtype):
    """Packed values are exact in fp32 and bf16 between 2^-126 and 2^128; a packed 2^128 itself (a magnitude of at
    least 1.9375 x 2^127 rounds to it) is an infinity in either."""
    x = torch.zeros(8, 64, device="cuda")
    x[0, 0] = torch.finfo(DT[dtype]).max
    x[1, 0], x[1, 1] = -torch.finfo(DT[dtype]).max, 1.0
    x[2, 0] = 1.921875 * 2.0 ** 127        # below the border: 1.875 x 2^127
    x[3, 0], x[3, 1] = 2.0 ** 127, -2.0 ** 118
    x[4, 0], x[4, 33] = 2.0 ** -126, 2.0 ** -120
    x[5, 0], x[5, 1] = 448 * 2.0 ** -127, 2.0 ** -126
    x[6, 0] = 2.0 ** -133
    x[7, 0] = 1.0
    x = x.to(DT[dtype])
    q, s = tb.alloc_mx(8, 64)
    tb.toma_mx_quantize(x, q, s)
    want = ref.unpack(q, s)
    assert want[0, 0] == 2.0 ** 128 and want[1, 0] == -2.0 ** 128 and want[2, 0] == 1.875 * 2.0 ** 127
    for out in ("f32", "bf16"):
        y = torch.empty(8, 64, dtype=DT[out], device="cuda")
        tb.toma_mx_dequantize(q, s, y)
        assert y[0, 0] == INF and y[1, 0] == -INF
        y, v = y.double(), want.clone()
        y[0, 0], y[1, 0], v[0, 0], v[1, 0] = 0, 0, 0, 0
        assert torch.equal(y, v)


# ---- 8-bit products at the ends of the scales --------------------------------------------------------------------------------------

@pytest.mark.parametrize("x_type,rows,K,N", [c for c in SELECTING if c[0] == "mx8"])
def test_products_of_extreme_scales(x_type, rows, K, N):
    """Every scale code from 0 to 254 on either side, chosen block by block so that the scales nearly cancel in the products."""
    g = gen(rows + K + 2 * N)

    def elements(*shape):
        return torch.randint(-64, 65, shape, generator=g, device="cuda").float().to(torch.float8_e4m3fn).view(torch.uint8)

    blocks = K // 32
    c = torch.linspace(0, 254, blocks, device="cuda").round().long()[torch.randperm(blocks, generator=g, device="cuda")]
    c[0], c[-1] = 0, 254

    def codes(n, base):
        s = torch.randint(0, 256, (n, ref.stride(K)), generator=g, device="cuda")   # (whatever stands behind the row's blocks)
        s[:, :blocks] = (base + torch.randint(-2, 3, (n, blocks), generator=g, device="cuda")).clamp(0, 254)
        return s.to(torch.uint8)

    x, w = (elements(rows, K), codes(rows, c)), (elements(N, K), codes(N, 254 - c))
    y, _ = run_linear("mx8", "bf16", x, w, None, None, "none")
    x64, w64 = ref.unpack(*x), ref.unpack(*w).t().contiguous()
    want, size = x64 @ w64, x64.abs() @ w64.abs()
    tol = size * (K * 2.0 ** -24 + 2.0 ** -12) + 2.0 ** -20 * want.abs()
    within(y, want, (want.abs() + tol) * HALF[torch.bfloat16] + tol)


# ---- one tensor in two places, and calls that a graph repeats ------------------------------------------------------------------------

@pytest.mark.parametrize("out", ["", "mx8"])
@pytest.mark.parametrize("C", [64, 640, 8192])
def test_norm_of_a_tensor_with_itself(out, C):
    """x as its own residual, and the sum stored over it: as with tensors of their own."""
    x = randn(gen(C), 70, C).to(torch.bfloat16)
    d = tb.make_norm_desc(70, C, 1e-6, "bf16", out or "bf16")
    results = []
    for alias in (False, True):
        a, r = x.clone(), x.clone()
        h = torch.empty_like(x)
        if alias:
            r = h = a
        y = tb.alloc_mx(70, C) if out else (torch.empty_like(x), None)
        tb.toma_rmsnorm(d, a, r, None, h, *y)
        results.append((h, *(y if out else y[:1])))
    assert torch.equal(results[0][0], 2 * x)
    assert all(torch.equal(p, q) for p, q in zip(*results))


@pytest.mark.parametrize("x_type", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 40, 700, 4096])
def test_linear_with_its_input_as_residual(x_type, rows):
    x, w, b, _, _, _ = linear_case(x_type, x_type, rows, 640, 640, "silu", True, False)
    d = tb.make_linear_desc(rows, 640, 640, x_type, None, "silu")
    ws, y, want = tb.alloc_linear_workspace(d), torch.empty_like(x[0]), torch.empty_like(x[0])
    tb.toma_linear(d, x[0], None, w[0], None, b, x[0].clone(), want, None, ws)
    tb.toma_linear(d, x[0], None, w[0], None, b, x[0], y, None, ws)
    assert torch.equal(y, want)


@pytest.mark.parametrize("x_type,w_type", [("bf16", "bf16"), ("bf16", "mx8"), ("f32", "f32")])
@pytest.mark.parametrize("rows", [3, 130, 1500])
def test_ffn_over_either_of_its_inputs(x_type, w_type, rows):
    """Y is X, R, or both of them in one tensor."""
    t = ffn_inputs(rows, 320, 640, x_type, w_type, True, True)
    d = tb.make_ffn_desc(rows, 320, 640, 1e-6, x_type, w_type, "gelu")
    ws = tb.alloc_ffn_workspace(d)
    for same in (False, True):
        base = dict(t, R=t["X"]) if same else t
        want = torch.empty_like(t["X"])
        ffn_call(base, d, want, ws)
        for over in ("X", "R"):
            now = dict(base, X=base["X"].clone(), R=base["R"].clone())
            if same:
                now["R"] = now["X"]
            ffn_call(now, d, now[over], ws)
            assert torch.equal(now[over], want), (same, over)


def test_packing_and_product_replayed_from_a_graph():
    """Packing, an 8-bit product with packed output and its unpacking in one graph, replayed on new inputs between eager calls."""
    rows, K, N = 77, 2080, 640
    x = randn(gen(1), rows, K).to(torch.bfloat16)
    w = tb.alloc_mx(N, K)
    tb.toma_mx_quantize_weight(randn(gen(2), K, N).to(torch.bfloat16), *w)
    d = tb.make_linear_desc(rows, K, N, "mx8", "mx8", "gelu")
    buffers = [(tb.alloc_mx(rows, K), tb.alloc_mx(rows, N), torch.empty(rows, N, device="cuda"), tb.alloc_linear_workspace(d)) for _ in range(2)]

    def call(q, p, y, ws):
        tb.toma_mx_quantize(x, *q)
        tb.toma_linear(d, *q, *w, None, None, *p, ws)
        tb.toma_mx_dequantize(*p, y)

    call(*buffers[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*buffers[0])
    for k in range(4):
        x.copy_(randn(gen(10 + k), rows, K))
        call(*buffers[1])
        buffers[0][2].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(buffers[0][2], buffers[1][2]) and buffers[0][2].any(), k
