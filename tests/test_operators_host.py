"""Host-side behaviour of the operators around the core modules, beyond their refusals: scratch sizes.  No GPU."""
import pytest

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
