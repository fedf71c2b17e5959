"""Host-side behaviour of the norm, linear, packing and feed-forward operators: refusals before any launch, sizes, and the packed
format's definition in the tests.  No GPU."""
import ctypes

import pytest
import torch

from paper_2509_10918_amd import binding as tb

import operators_ref as ref

X = 1 << 20   # aligned address that no refused call reads


def _p(d):
    return ctypes.addressof(d)


def test_scale_stride():
    assert [tb.toma_mx_scale_stride(k) for k in (32, 128, 160, 640, 1280)] == [4, 4, 8, 20, 40]
    assert [tb.toma_mx_scale_stride(k) for k in (0, -32, 33, 48, 1 << 21)] == [0] * 5


def test_packing_refusals():
    L = tb.lib()
    for f in (L.toma_mx_quantize, L.toma_mx_dequantize):
        assert f(1, 4, 64, None, X, X, None) == 1 and f(1, 4, 64, X, None, X, None) == 1 and f(1, 4, 64, X, X, None, None) == 1
        assert f(1, 0, 64, X, X, X, None) == 2 and f(1, 4, 0, X, X, X, None) == 2 and f(1, -1, 64, X, X, X, None) == 2
        assert f(1, 4, 64, X + 8, X, X, None) == 3 and f(1, 4, 64, X, X + 4, X, None) == 3 and f(1, 4, 64, X, X, X + 1, None) == 3
        assert f(2, 4, 64, X, X, X, None) == 5 and f(7, 4, 64, X, X, X, None) == 5
        assert f(1, 4, 48, X, X, X, None) == 5 and f(1, 1 << 27, 32, X, X, X, None) == 5
    w = L.toma_mx_quantize_weight
    assert w(1, 64, 40, None, X, X, None) == 1 and w(1, 64, 0, X, X, X, None) == 2 and w(1, 60, 40, X, X, X, None) == 5
    assert w(0, 64, 40, X, X, X + 2, None) == 3 and w(1, 1 << 16, 1 << 15, X, X, X, None) == 5 and w(1, 32, (1 << 20) + 1, X, X, X, None) == 5


def test_norm_refusals():
    f = tb.lib().toma_rmsnorm
    d = tb.make_norm_desc(10, 64, 1e-6, "bf16")
    m = tb.make_norm_desc(10, 64, 1e-6, "bf16", "mx8")
    assert f(None, X, None, None, None, X, None, None) == 1
    assert f(_p(d), None, None, None, None, X, None, None) == 1 and f(_p(d), X, None, None, None, None, None, None) == 1
    assert f(_p(d), X, None, None, None, X, X, None) == 1 and f(_p(m), X, None, None, None, X, None, None) == 1   # codes exactly with mx8
    for at in range(1, 6):
        args = [_p(d), X, X, X, X, X, None, None]
        args[at] += 8
        assert f(*args) == 3
    assert f(_p(m), X, None, None, None, X, X + 4, None) == 3
    for kw, want in ((dict(rows=0), 2), (dict(C=0), 2), (dict(eps=0.0), 2), (dict(eps=float("nan")), 2), (dict(eps=float("inf")), 2),
                     (dict(C=72), 5), (dict(C=16416), 5), (dict(rows=1 << 28), 5), (dict(x_type="mx8", y_type="mx8"), 5), (dict(y_type="f32"), 5)):
        bad = tb.make_norm_desc(**{**dict(rows=10, C=64, eps=1e-6, x_type="bf16", y_type=None), **kw})
        assert f(_p(bad), X, None, None, None, X, X if bad.y_type == 2 else None, None) == want, kw


def test_linear_refusals():
    L = tb.lib()
    f = L.toma_linear
    d = tb.make_linear_desc(10, 64, 72, "bf16")
    m = tb.make_linear_desc(10, 64, 96, "mx8", "mx8")
    big = 1 << 30
    assert f(None, X, None, X, None, None, None, X, None, X, big, None) == 1
    for at in (1, 3, 7):
        args = [_p(d), X, None, X, None, None, None, X, None, X, big, None]
        args[at] = None
        assert f(*args) == 1
    for at in (2, 4, 8):      # scale codes exactly with mx8
        args = [_p(d), X, None, X, None, None, None, X, None, X, big, None]
        args[at] = X
        assert f(*args) == 1
        args = [_p(m), X, X, X, X, None, None, X, X, X, big, None]
        args[at] = None
        assert f(*args) == 1
    for at in range(1, 9):
        args = [_p(m), X, X, X, X, X, X, X, X, X, big, None]
        args[at] += 4
        assert f(*args) == 3
    for kw, want in ((dict(rows=0), 2), (dict(K=0), 2), (dict(N=-8), 2), (dict(K=68), 5), (dict(N=76), 5), (dict(y_type="f32"), 5),
                     (dict(y_type="mx8"), 5), (dict(x_type="f32", K=66), 5), (dict(x_type="f32", N=73), 5), (dict(x_type="mx8", y_type="bf16", K=72), 5),
                     (dict(x_type="mx8", y_type="f32"), 5), (dict(x_type="mx8", y_type="mx8"), 5), (dict(K=(1 << 20) + 8), 5),
                     (dict(rows=(1 << 28) + 1), 5), (dict(K=1 << 16, N=1 << 15), 5), (dict(rows=1 << 20, K=1 << 14), 5)):
        bad = tb.make_linear_desc(**{**dict(rows=10, K=64, N=72, x_type="bf16", y_type=None), **kw})
        c, y = (X if bad.x_type == 2 else None), (X if bad.y_type == 2 else None)
        assert f(_p(bad), X, c, X, c, None, None, X, y, X, big, None) == want, kw
        assert tb.toma_linear_workspace_bytes(bad) == 0
    bad = tb.make_linear_desc(10, 64, 72, "bf16")
    bad.act = 4
    assert f(_p(bad), X, None, X, None, None, None, X, None, X, big, None) == 5
    # a shape that needs scratch says so
    for shape in ((1, 4096, 640, "bf16"), (3, 8192, 1280, "f32"), (2, 2048, 640, "mx8", "bf16"), (512, 8192, 256, "bf16")):
        d = tb.make_linear_desc(*shape)
        need, c = tb.toma_linear_workspace_bytes(d), X if d.x_type == 2 else None
        if need:
            assert need % 256 == 0
            assert f(_p(d), X, c, X, c, None, None, X, None, None, need, None) == 1
            assert f(_p(d), X, c, X, c, None, None, X, None, X + 16, need, None) == 3
            assert f(_p(d), X, c, X, c, None, None, X, None, X, 128, None) == 4


def test_linear_tile_is_host_arithmetic():
    """Tile and K split come from the descriptor alone; the scratch is what the split's partial sums take."""
    L = tb.lib()
    seen = set()
    for x_type, y_type in (("bf16", None), ("mx8", "bf16"), ("f32", None)):
        for rows, K, N in ((16384, 4096, 8192), (1025, 1376, 4104), (512, 640, 640), (77, 8192, 1280), (1, 8192, 640)):
            d = tb.make_linear_desc(rows, K, N, x_type, y_type)
            bm, bn, split = tb.toma_profile_linear(d)
            assert bm in (16, 32, 64, 128, 256) and bn in (64, 128, 256) and 1 <= split <= (16 if bm <= 32 else 8)
            need = tb.toma_linear_workspace_bytes(d)
            assert need == 0 if split == 1 else need >= 4 * split * rows * N
            seen.add((x_type, bm, bn, split > 1))
    assert {("bf16", 256, 256, False), ("mx8", 256, 256, False), ("mx8", 128, 128, False), ("mx8", 64, 64, False), ("mx8", 64, 64, True),
            ("bf16", 64, 64, True)} <= seen
    d = tb.make_linear_desc(16, 64, 64, "bf16")
    assert L.toma_profile_linear(_p(d), None) == 1 and L.toma_profile_linear(None, None) == 1


def test_ffn_refusals():
    L = tb.lib()
    d = tb.make_ffn_desc(100, 64, 256, 1e-6, "bf16", "mx8")
    need = tb.toma_ffn_workspace_bytes(d)
    assert need > 0 and need % 256 == 0 and tb.toma_ffn_workspace_bytes(None) == 0
    good = [_p(d), X, X, X, X, X, X, X, X, X, X, X, need, None]
    for at in (1, 4, 5, 7, 8, 10, 11):
        args = list(good)
        args[at] = None
        assert L.toma_ffn(*args) == 1
    for at in range(1, 12):
        args = list(good)
        args[at] += 4
        assert L.toma_ffn(*args) == 3
    assert L.toma_ffn(*good[:12], need - 1, None) == 4
    assert L.toma_ffn(None, *good[1:]) == 1
    plain = tb.make_ffn_desc(100, 64, 256, 1e-6, "bf16")
    assert L.toma_ffn(_p(plain), *good[1:]) == 1      # scale codes without mx8 weights
    for kw, want in ((dict(rows=0), 2), (dict(hidden=0), 2), (dict(eps=0.0), 2), (dict(C=72), 5), (dict(hidden=264), 5), (dict(w_type="f32"), 5),
                     (dict(x_type="f32", w_type="mx8"), 5), (dict(C=16416), 5)):
        bad = tb.make_ffn_desc(**{**dict(rows=100, C=64, hidden=256, eps=1e-6, x_type="bf16", w_type="mx8"), **kw})
        assert tb.toma_ffn_workspace_bytes(bad) == 0
        assert L.toma_ffn(_p(bad), *good[1:]) == want, kw


def test_binding_refuses_wrong_tensors():
    """Shapes, types and devices are checked before the library is called (host tensors stand in: every check but the device's)."""
    d = tb.make_linear_desc(2, 32, 40, "bf16")
    x, w, y = torch.zeros(2, 32, dtype=torch.bfloat16), torch.zeros(32, 40, dtype=torch.bfloat16), torch.zeros(2, 40, dtype=torch.bfloat16)
    for args in ((x.float(), None, w, None, None, None, y, None, None), (x[:1], None, w, None, None, None, y, None, None),
                 (x, None, w, None, None, None, y, None, None)):
        with pytest.raises(ValueError):
            tb.toma_linear(d, *args)
    with pytest.raises(ValueError):
        tb.toma_mx_quantize(x.double(), *tb.alloc_mx(2, 32, "cpu"))
    with pytest.raises(tb.TomaError):
        tb.alloc_mx(2, 40, "cpu")
    with pytest.raises(tb.TomaError):
        tb.alloc_ffn_workspace(tb.make_ffn_desc(2, 40, 64, 1e-6, "bf16"), "cpu")
    with pytest.raises(KeyError):
        tb.make_linear_desc(2, 32, 40, torch.float16)


def test_packed_format_of_the_tests():
    """The tests' own packing, on values whose packed form is known."""
    x = torch.zeros(5, 64)
    x[0, 0], x[0, 1], x[0, 2] = 448.0, 1.0, -0.3        # 448 fits 2^0 exactly
    x[1, 0], x[1, 33] = 449.0, 2.0 ** -140              # just over: 2^1; a magnitude that only 2^-127 serves
    x[2, 5], x[2, 6] = float("inf"), 3.0                # not finite: out of the maximum, NaN in the elements
    x[3, :32] = 2.0 ** 127
    q, s = ref.pack(x)
    assert s[0].tolist() == [127, 0, 0, 0] and s[1].tolist() == [128, 0, 0, 0]
    assert s[2, 0] == 127 - 7 and s[3, 0] == 127 + 119 and s[4].tolist() == [0] * 4
    v = ref.unpack(q, s)
    assert v[0, :3].tolist() == [448.0, 1.0, -0.3125] and v[1, 0] == 448.0 and v[1, 33] == 0.0
    assert torch.isnan(v[2, 5]) and v[2, 6] == 3.0 and v[3, 0] == 2.0 ** 127 and not v[4].any()


def test_binding_refuses_transposed_weights():
    """[N, K] where [K, N] is meant holds as many elements; in 8 bits it is the other way round."""
    d, q = tb.make_linear_desc(2, 32, 64, "bf16"), tb.make_linear_desc(2, 32, 64, "mx8", "bf16")
    x, y, w = torch.zeros(2, 32, dtype=torch.bfloat16), torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(64, 32, dtype=torch.bfloat16)
    u8 = lambda *shape: torch.zeros(*shape, dtype=torch.uint8)
    with pytest.raises(ValueError, match="W: last dimension 64"):
        tb.toma_linear(d, _OnDevice(x), None, w, None, None, None, y, None, None)
    with pytest.raises(ValueError, match="W: last dimension 32"):
        tb.toma_linear(q, _OnDevice(u8(2, 32)), None, u8(32, 64), u8(64, 4), None, None, y, None, None)
    f = tb.make_ffn_desc(2, 32, 64, 1e-6, "bf16")
    with pytest.raises(ValueError, match="W1: last dimension 64"):
        tb.toma_ffn(f, _OnDevice(x), None, None, w, None, None, w, None, None, torch.zeros(2, 32, dtype=torch.bfloat16), None)


class _OnDevice:
    """Passes the checks that a tensor on the device would."""

    def __init__(self, t):
        self.dtype, self.t = t.dtype, t

    def numel(self):
        return self.t.numel()

    def get_device(self):
        return torch.cuda.current_device() if torch.cuda.is_initialized() else 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0
