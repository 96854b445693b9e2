"""The layer's products on each size of tiles, whichever one a call would take by itself, against the float64 forms of test_gpu_layer
with the bounds of that file: rows, columns and reductions that end inside a tile, shares, many tiles, frames that do not exist."""
import pytest

from paper_2304_13134_amd import binding as lb
import test_gpu_layer as layer
import test_gpu_layer_wide as wide
from gpu_util import announce, library_option

pytestmark = pytest.mark.gpu
# few rows; one tile and a bit of the next in P, Q, both; reductions shorter than a step, in shares, and that end inside one; thirty tiles
SHAPES = [(1, 7, 40, 200), (3, 100, 257, 512), (2, 257, 530, 72), (1, 130, 96, 5000), (2, 128, 256, 256), (4, 610, 530, 72), (5, 300, 515, 1000)]


@pytest.fixture(params=[1, 2, 3], ids=["tiles of 64", "tiles of 128", "tiles of 256"])
def tiles(request):
    announce("tiles", request.param)
    with library_option(lb.OPT_PRODUCT_TILES, request.param):
        yield request.param


@pytest.mark.parametrize("B,T,N,K", SHAPES)
@pytest.mark.parametrize("type_,out,name,bias,res,kind,lens", [
    ("bf16", "bf16", "none", False, False, None, "all"), ("bf16", "bf16", "silu", True, True, None, "some"), ("f16", "f32", "gelu", True, False, "i8", "some"),
    ("bf16", "bf16", "gelu", True, False, "e4m3", "some"), ("bf16", "f32", "tanh", False, True, None, "all"), ("f16", "f16", "relu", True, True, "i8", "some"),
    ("e4m3", "bf16", "none", True, True, None, "some"), ("e4m3", "bf16", "gelu", True, False, "i8", "some"), ("bf16", "i8", "silu", True, True, None, "some"),
    ("bf16", "e4m3", "none", False, False, "i8", "none"), ("f16", "i8", "gelu", True, False, None, "some"), ("e4m3", "e4m3", "gelu", True, False, None, "some")])
def test_product(tiles, B, T, N, K, type_, out, name, bias, res, kind, lens):
    layer.test_product(B, T, N, K, type_, out, name, bias, res, kind, lens)


@pytest.mark.parametrize("B,T,N,K", SHAPES + [(3, 300, 1000, 515)])
@pytest.mark.parametrize("type_,out,kind,name,lens", [("bf16", "bf16", None, "none", "some"), ("bf16", "bf16", "i8", "silu", "some"), ("f16", "f32", "e4m3", "gelu", "all"),
                                                     ("bf16", "f16", "i8", "tanh", "none"), ("f16", "f16", "e4m3", "relu", "some")])
def test_product_input_gradient(tiles, B, T, N, K, type_, out, kind, name, lens):
    layer.test_product_input_gradient(B, T, N, K, type_, out, kind, name, lens)


@pytest.mark.parametrize("B,T,N,K", SHAPES + [(7, 700, 40, 24), (2, 9000, 64, 64), (2, 1100, 300, 290), (1, 200, 2310, 530)])
@pytest.mark.parametrize("type_,out,kind,name,lens", [("bf16", "f32", None, "none", "some"), ("f16", "bf16", None, "none", "all"), ("bf16", "f32", "i8", "none", "some"),
                                                     ("f16", "f16", "e4m3", "gelu", "all"), ("bf16", "f32", "i8", "silu", "some"), ("bf16", "f32", None, "none", "none")])
def test_product_weight_gradient(tiles, B, T, N, K, type_, out, kind, name, lens):
    layer.test_product_weight_gradient(B, T, N, K, type_, out, kind, name, lens)


@pytest.mark.parametrize("B,T,N,K", SHAPES)
@pytest.mark.parametrize("name,bias,res,keep,lens", [("none", False, False, None, "all"), ("silu", True, True, None, "some"), ("gelu", True, False, "i8", "some")])
def test_float32_results_of_eight_bit_operands(tiles, B, T, N, K, name, bias, res, keep, lens):
    wide.test_float32_results_of_eight_bit_operands(B, T, N, K, name, bias, res, keep, lens)


@pytest.mark.parametrize("out", ["bf16", "f32", "i8"])
def test_stretches_without_frames(tiles, out):
    layer.test_stretches_without_frames(833, 512, 2048, out)


def test_operands_as_they_come(tiles):
    layer.test_product_of_strided_and_misaligned_operands()
    layer.test_nan_blocks_and_infinities_stay_in_their_rows()
    wide.test_blocks_that_are_no_numbers(100)
    wide.test_cancelling_terms_of_a_block()


def test_the_same_results_again_and_captured(tiles):
    layer.test_results_do_not_depend_on_timing()
    layer.test_streams_and_graphs()


@pytest.mark.parametrize("rows", [15, 16, 17, 31, 32, 33, 48, 64])
@pytest.mark.parametrize("N,K", [(48, 200), (260, 1000)])
@pytest.mark.parametrize("type_,out,name,bias,res,kind,lens", [("bf16", "bf16", "silu", True, True, None, "some"), ("f16", "f32", "gelu", True, False, "i8", "all"),
                                                              ("e4m3", "bf16", "none", True, True, None, "all"), ("e4m3", "f32", "silu", True, False, "e4m3", "some")])
def test_rows_around_the_kernel_for_few(rows, N, K, type_, out, name, bias, res, kind, lens):
    layer.test_product(1, rows, N, K, type_, out, name, bias, res, kind, lens)
