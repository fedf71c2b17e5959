"""Host-side behaviour of the operators around the core modules, beyond their refusals: scratch sizes,
the choice of kernel, and tensors of the right size in the wrong shape.  No GPU."""
import pytest
import torch

from paper_2509_10918_amd import binding as tb


@pytest.mark.parametrize("x_type,rows,K,N", [("bf16", 1, 4096, 640), ("bf16", 7, 8192, 128), ("bf16", 16, 8192, 640), ("bf16", 64, 8192, 256), ("f32", 1, 4096, 256),
                                             ("f32", 3, 8192, 1280), ("f32", 32, 8192, 640), ("f32", 100, 8192, 256), ("mx8", 2, 4096, 640), ("mx8", 77, 8192, 1280)])
def test_shapes_that_split_K_ask_for_the_scratch_of_their_partial_sums(x_type, rows, K, N):
    """fp32 [split][rows][N], rounded up to 256 bytes, and no call without it."""
    d = tb.make_linear_desc(rows, K, N, x_type, "bf16" if x_type == "mx8" else x_type)
    split, need = tb.toma_profile_linear(d)[2], tb.toma_linear_workspace_bytes(d)
    assert split > 1 and need == (4 * split * rows * N + 255) // 256 * 256
    X, c = 1 << 20, (1 << 20 if x_type == "mx8" else None)   # an aligned address that no refused call reads
    call = lambda ws, n: tb.lib().toma_linear(tb._ref(d), X, c, X, c, None, None, X, None, ws, n, None)
    assert call(None, need) == 1 and call(X + 16, need) == 3 and call(X, 4 * split * rows * N - 1) == 4


def test_kernels_by_name():
    """The sizes at which the GPU tests try the activations' tails and values that are not finite reach every kernel, split and not."""
    from test_gpu_operators_edges import SELECTING, STEPS
    taken = set()
    for x, rows, K, N in SELECTING:
        d = tb.make_linear_desc(rows, K, N, x, "bf16" if x == "mx8" else x, "gelu")
        taken.add((x, tb.toma_profile_linear_kernel(d), tb.toma_profile_linear(d)[2] > 1))
    tiles = {(x, kernel, False) for x in ("bf16", "mx8") for kernel in ("medium", "medium_four_stages", "large")}
    plain = {(x, kernel, split) for x in ("bf16", "f32") for kernel in ("few_rows", "planned") for split in (False, True)} | {(x, "short", False) for x in ("bf16", "f32")}
    assert taken == tiles | plain | {("mx8", "small", False), ("mx8", "small", True)}
    for x, rows, K, N, kernel in STEPS:
        assert tb.toma_profile_linear_kernel(tb.make_linear_desc(rows, K, N, x, "bf16" if x == "mx8" else x, "silu")) == kernel, (x, rows, K, N)
    assert tb.toma_profile_linear_kernel(tb.make_linear_desc(4, 12, 64, "bf16")) is None and tb.toma_profile_linear_kernel(None) is None


# ---- tensors that hold as many elements in another order ------------------------------------------------------------------------

class OnDevice:
    """A host tensor that passes the device check: refusals by shape need no GPU."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return torch.cuda.current_device() if torch.cuda.is_initialized() else 0


BF = torch.bfloat16


def dev(*shape, dtype=BF):
    return OnDevice(torch.zeros(*shape, dtype=dtype))


def u8(*shape):
    return dev(*shape, dtype=torch.uint8)


def refused(what, f, *args):
    with pytest.raises(ValueError, match=what):
        f(*args)


def test_transposed_rows_are_refused():
    """Token rows whose dimensions are the other way round: as many elements, another meaning."""
    d = tb.make_linear_desc(6, 32, 40, "bf16")
    x, w, y = dev(6, 32), dev(32, 40), dev(6, 40)
    refused("X", tb.toma_linear, d, dev(32, 6), None, w, None, None, None, y, None, None)
    refused("R", tb.toma_linear, d, x, None, w, None, None, dev(40, 6), y, None, None)
    refused("Y", tb.toma_linear, d, x, None, w, None, None, None, dev(40, 6), None, None)
    refused("Y", tb.toma_linear, d, x, None, w, None, None, None, dev(2, 40, 3), None, None)   # channels in front of the positions
    q = tb.make_linear_desc(6, 64, 96, "mx8", "mx8")
    refused("X:", tb.toma_linear, q, u8(64, 6), u8(6, 4), u8(96, 64), u8(96, 4), None, None, u8(6, 96), u8(6, 4), None)
    refused("Xs", tb.toma_linear, q, u8(6, 64), u8(4, 6), u8(96, 64), u8(96, 4), None, None, u8(6, 96), u8(6, 4), None)
    refused("Ws", tb.toma_linear, q, u8(6, 64), u8(6, 4), u8(96, 64), u8(4, 96), None, None, u8(6, 96), u8(6, 4), None)
    refused("Ys", tb.toma_linear, q, u8(6, 64), u8(6, 4), u8(96, 64), u8(96, 4), None, None, u8(6, 96), u8(4, 6), None)
    n = tb.make_norm_desc(6, 32, 1e-6, "bf16")
    for at, what in ((0, "X"), (1, "R"), (3, "H"), (4, "Y")):
        args = [dev(6, 32), dev(6, 32), dev(32), dev(6, 32), dev(6, 32)]
        args[at] = dev(32, 6)
        refused(what, tb.toma_rmsnorm, n, *args)
    f = tb.make_ffn_desc(6, 32, 64, 1e-6, "bf16")
    for at, what in ((0, "X"), (1, "R"), (9, "Y")):
        args = [dev(6, 32), dev(6, 32), None, dev(32, 64), None, None, dev(64, 32), None, None, dev(6, 32), None]
        args[at] = dev(32, 6)
        refused(what, tb.toma_ffn, f, *args)


def test_transposed_tensors_of_the_packing_calls_are_refused():
    refused("X", tb.toma_mx_quantize, dev(64, 6), u8(6, 64), u8(6, 4))
    refused("S", tb.toma_mx_quantize, dev(6, 64), u8(6, 64), u8(4, 6))
    refused("Q", tb.toma_mx_quantize_weight, dev(64, 6), u8(64, 6), u8(6, 4))
    refused("S", tb.toma_mx_quantize_weight, dev(64, 6), u8(6, 64), u8(4, 6))
    refused("Y", tb.toma_mx_dequantize, u8(6, 64), u8(6, 4), dev(64, 6))


@pytest.mark.parametrize("shape", [(6, 64), (2, 3, 64), (384,), (6, 4, 16), (2, 192), (1, 6, 1, 64), (3, 2, 8, 8), (6, 1, 64)])
def test_any_layout_of_whole_rows_is_taken(shape):
    """Rows one after the other: leading dimensions, heads as a dimension, several rows in one (the norm of single heads), flat."""
    t = dev(*shape)
    assert tb._Call().arg("X", t, BF, (6, 64)) == t.data_ptr()
    assert tb._Call().arg("X", None, BF, (6, 64)) is None
