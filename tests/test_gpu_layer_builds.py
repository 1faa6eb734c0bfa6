"""Every tile shape of the layer products in every mode, in one part and in several, at ragged sizes: the shapes that the library
chooses for large layers are forced on small ones, so that no retuning of that choice leaves a build untested."""
import pytest
import torch

import paper_2009_09271_b200 as sc
from test_gpu_layer import check_input_grad, check_linear, check_weight_grad

pytestmark = pytest.mark.gpu

TYPES = (torch.bfloat16, torch.float16)
TILES = [(256, 256), (128, 256), (128, 128), (128, 64)]
# rows of 16-byte, 8-byte and single-element alignment; whole and ragged tiles; several tiles a CTA, long and short sums
SIZES = [(300, 520, 200), (517, 640, 328), (389, 333, 150), (258, 388, 72), (1025, 128, 513)]


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1)
    yield c
    c.sc_debug_layer_tiles()
    assert c.sc_sync_status() == 0
    c.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("parts", [1, 2, 3])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_every_tile_shape(ctx, dtype, tile, parts, M, N, K):
    ctx.sc_debug_layer_tiles(*tile, parts)
    before = ctx.launch_count
    check_linear(ctx, dtype, "none", M, N, K, False, False, False)
    # the product, its operands' copies where rows are unaligned, and a join where there are several parts
    assert ctx.launch_count - before == 1 + (K % 8 != 0) + (parts > 1)
    check_linear(ctx, dtype, "gelu_tanh", M, N, K, True, True, True)
    check_linear(ctx, dtype, "relu", M, N, K, True, False, True, 8, 8)
    check_linear(ctx, dtype, "silu", M, N, K, False, True, True, 3, 1)
    check_input_grad(ctx, dtype, "none", M, N, K, True)
    check_input_grad(ctx, dtype, "gelu", M, N, K, True)
    check_input_grad(ctx, dtype, "relu", M, N, K, False, 4, 4)
    check_weight_grad(ctx, dtype, M, N, K, "kept")
    check_weight_grad(ctx, dtype, M, N, K, "dense")
    check_weight_grad(ctx, dtype, M, N, K, "dense", 4, 4)
    check_weight_grad(ctx, dtype, M, N, K, "kept", 3, 1)


@pytest.mark.parametrize("tile", TILES)
def test_more_tiles_than_ctas(ctx, tile):
    """Accumulators, stages and output buffers take turns from tile to tile."""
    ctx.sc_debug_layer_tiles(*tile, 1)
    M, N = {(256, 256): (3400, 3600), (128, 256): (2100, 5000), (128, 128): (2100, 2600), (128, 64): (1300, 2100)}[tile]
    check_linear(ctx, torch.bfloat16, "silu", M, N, 136, True, True, True)
    check_linear(ctx, torch.float16, "relu", M, N + 5, 72, True, False, True)
    check_input_grad(ctx, torch.bfloat16, "silu", M, 136, N, True)
    check_weight_grad(ctx, torch.bfloat16, 200, M, N, "kept")
    check_weight_grad(ctx, torch.float16, 900, M, N, "dense", 0, 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1024, 4096, 1024), (1100, 4104, 1000), (1030, 4100, 1016), (2048, 2048, 2048), (900, 3001, 777)])
def test_sizes_of_real_layers(ctx, dtype, M, N, K):
    """In the shapes that the library chooses itself."""
    ctx.sc_debug_layer_tiles()
    check_linear(ctx, dtype, "gelu", M, N, K, True, True, True)
    check_linear(ctx, dtype, "none", M, N, K, False, False, False, 0, 1)
    check_input_grad(ctx, dtype, "silu", M, N, K, True)
    check_weight_grad(ctx, dtype, M, N, K, "kept")
    check_weight_grad(ctx, dtype, M, N, K, "dense", 4, 4)
    check_weight_grad(ctx, dtype, M, N, K, "dense", 1, 3)


def test_forced_tiles_are_checked_and_undone(ctx):
    for bad in ((256, 128, 1), (64, 64, 1), (128, 64, 0), (128, 64, 65), (0, 0, 1), (128, 0, 1), (0, 64, 1)):
        with pytest.raises(sc.SparseCommError):
            ctx.sc_debug_layer_tiles(*bad)
    assert sc.load_library().sc_debug_layer_tiles(None, 0, 0, 0) == -1
    x, w = torch.ones(64, 640, dtype=torch.bfloat16, device="cuda"), torch.ones(64, 640, dtype=torch.bfloat16, device="cuda")
    y = torch.empty(64, 64, dtype=torch.bfloat16, device="cuda")

    def launches():
        before = ctx.launch_count
        ctx.sc_linear(sc.SC_ACT_NONE, x, w, y)
        assert bool((y == 640).all())
        return ctx.launch_count - before

    ctx.sc_debug_layer_tiles()
    own = launches()
    ctx.sc_debug_layer_tiles(128, 64, 1)
    assert launches() == 1
    ctx.sc_debug_layer_tiles(128, 64, 4)
    assert launches() == 2
    ctx.sc_debug_layer_tiles(256, 256, 4)                    # 64 rows: the library's choice
    assert launches() == own
    ctx.sc_debug_layer_tiles()
    assert launches() == own
