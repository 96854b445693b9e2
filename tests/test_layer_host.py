"""Host-only checks of the layer between frames and lattice: what the C ABI and the binding refuse, and workspaces."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2304_13134_amd import binding as lb
import layer_oracle as lo

F32, BF16, F16, I8, E4M3 = range(5)
DUMMY = ctypes.c_void_p(0x1000)


@pytest.fixture(scope="module")
def lib():
    return lb.load_library()


def frames(B=2, T=5, lengths=None):
    return lb.LastFrames(B, T, lengths)


def matrix(type_=BF16, pitch=64, data=0x10000, scales=None, scale_pitch=0):
    if type_ in (I8, E4M3) and scales is None:
        scales, scale_pitch = 0x20000, (pitch + 31) // 32
    return lb.LastMatrix(data, type_, pitch, scales, scale_pitch)


def ref(s):
    return None if s is None else ctypes.byref(s)


def norm(lib, fr=None, H=64, x=None, res=None, gain=DUMMY, eps=1e-5, s=None, y=None, kept=None, inv=None):
    return lib.last_residual_norm(ref(fr or frames()), H, ref(x), ref(res), gain, eps, ref(s), ref(y), ref(kept), inv, None)


def test_norm_refuses(lib):
    x, y = matrix(), matrix()
    assert norm(lib, x=None, y=y) == 1
    assert norm(lib, x=x) == 1                                         # no result asked for
    assert norm(lib, x=x, y=y, gain=None) == 1
    assert norm(lib, x=matrix(data=None), y=y) == 1
    assert norm(lib, x=x, y=y, H=0) == 2
    assert norm(lib, x=x, y=y, H=65) == 2                              # pitch below the columns
    assert norm(lib, x=x, y=y, eps=-1.0) == 2 and norm(lib, x=x, y=y, eps=float("nan")) == 2
    assert norm(lib, fr=frames(B=0), x=x, y=y) == 2 and norm(lib, fr=frames(T=-1), x=x, y=y) == 2
    assert norm(lib, fr=frames(B=1 << 20, T=1 << 20), x=x, y=y) == 2
    assert norm(lib, x=matrix(data=0x10001), y=y) == 2                 # not at an element
    assert norm(lib, x=matrix(pitch=1 << 22), y=y) == 2
    assert norm(lib, x=matrix(pitch=20000), y=matrix(pitch=20000), H=20000) == 6
    assert norm(lib, x=matrix(I8), y=y) == 6 and norm(lib, x=x, y=matrix(E4M3)) == 6 and norm(lib, x=x, kept=matrix()) == 6
    assert norm(lib, x=x, res=matrix(F32), y=y) == 6 and norm(lib, x=x, s=matrix(F32)) == 6 and norm(lib, x=matrix(9), y=y) == 6
    assert norm(lib, x=x, kept=lb.LastMatrix(0x10000, I8, 64, None, 2)) == 1
    assert norm(lib, x=x, kept=lb.LastMatrix(0x10000, I8, 64, 0x20000, 1)) == 2
    assert norm(lib, fr=frames(T=0), x=x, y=y) == 0                    # no frames: nothing to do


def test_norm_gradient_refuses(lib):
    def call(dy=matrix(), s=matrix(), gain=DUMMY, inv=DUMMY, ds=None, dx=matrix(), dgain=DUMMY, ws=ctypes.c_void_p(0x10000), n=1 << 20, H=64, fr=frames()):
        return lib.last_residual_norm_grad(ref(fr), H, ref(dy), ref(s), gain, inv, ref(ds), ref(dx), dgain, ws, n, None)
    for missing in ("dy", "s", "gain", "inv", "dx"):
        assert call(**{missing: None}) == 1
    assert call(H=0) == 2 and call(H=16385, dy=matrix(pitch=16385)) == 6
    assert call(ws=None) == 5 and call(n=16) == 5 and call(ws=ctypes.c_void_p(0x10001)) == 5
    assert call(dy=matrix(I8)) == 6 and call(dx=matrix(E4M3)) == 6 and call(ds=matrix(F32)) == 6
    assert call(dy=matrix(BF16), s=matrix(F16)) == 6 and call(dy=matrix(BF16), s=matrix(F32)) == 6
    assert call(s=matrix(pitch=10)) == 2


def test_products_refuse(lib):
    ws, big = ctypes.c_void_p(0x10000), 1 << 30

    def fwd(x=matrix(), w=matrix(), bias=None, act=0, res=None, y=matrix(), kept=None, ws=ws, n=big, N=64, K=64, fr=frames()):
        return lib.last_product(ref(fr), N, K, ref(x), ref(w), bias, act, ref(res), ref(y), ref(kept), ws, n, None)
    assert fwd(x=None) == 1 and fwd(w=None) == 1 and fwd(y=None) == 1
    assert fwd(N=0) == 2 and fwd(K=0) == 2 and fwd(N=1 << 21) == 2 and fwd(K=65) == 2
    assert fwd(act=5) == 6 and fwd(act=-1) == 6
    assert fwd(x=matrix(F32), w=matrix(F32)) == 6 and fwd(w=matrix(F16)) == 6 and fwd(x=matrix(I8), w=matrix(I8)) == 6
    assert fwd(res=matrix(F16)) == 6 and fwd(kept=matrix()) == 6 and fwd(y=matrix(7)) == 6
    assert fwd(ws=None) == 5 and fwd(n=8) == 5
    assert fwd(fr=frames(T=0)) == 0

    def gin(dy=matrix(), w=matrix(), kept=None, act=0, dx=matrix(), ws=ws, n=big, N=64, K=64):
        return lib.last_product_grad_input(ref(frames()), N, K, ref(dy), ref(w), ref(kept), act, ref(dx), ws, n, None)
    assert gin(dy=None) == 1 and gin(w=None) == 1 and gin(dx=None) == 1 and gin(act=2) == 1       # an activation of nothing
    assert gin(N=65) == 2 and gin(dy=matrix(E4M3), w=matrix(E4M3)) == 6 and gin(dx=matrix(I8)) == 6 and gin(kept=matrix(), act=1) == 6
    assert gin(ws=None) == 5

    def gw(dy=matrix(), x=matrix(), act=0, dw=matrix(F32), dbias=DUMMY, ws=ws, n=big, N=64, K=64):
        return lib.last_product_grad_weight(ref(frames()), N, K, ref(dy), ref(x), act, ref(dw), dbias, ws, n, None)
    assert gw(dy=None) == 1 and gw(x=None) == 1 and gw(dw=None) == 1
    assert gw(act=2) == 6 and gw(x=matrix(F16)) == 6 and gw(dy=matrix(F32)) == 6 and gw(dw=matrix(I8)) == 6
    assert gw(K=65) == 2 and gw(n=0) == 5


def test_kept_calls_refuse(lib):
    fr = ref(frames())
    x, k, y = matrix(), matrix(I8), matrix()
    assert lib.last_keep(fr, 64, None, ref(k), None) == 1 and lib.last_keep(fr, 64, ref(x), None, None) == 1
    assert lib.last_keep(fr, 64, ref(k), ref(k), None) == 6 and lib.last_keep(fr, 64, ref(x), ref(x), None) == 6 and lib.last_keep(fr, 0, ref(x), ref(k), None) == 2
    assert lib.last_kept_values(fr, 64, ref(x), 0, ref(y), None) == 6 and lib.last_kept_values(fr, 64, ref(k), 9, ref(y), None) == 6
    assert lib.last_kept_values(fr, 65, ref(k), 0, ref(y), None) == 2 and lib.last_kept_values(None, 64, ref(k), 0, ref(y), None) == 1
    assert lib.last_kept_grad(fr, 64, ref(k), ref(k), 1, ref(y), None) == 6 and lib.last_kept_grad(fr, 64, ref(x), None, 1, ref(y), None) == 1


def test_workspaces(lib):
    def size(op, N, K, a, b, fr=frames(4, 1000)):
        return lib.last_layer_workspace_bytes(op, ref(fr), N, K, ref(a), ref(b))
    m = matrix
    # aligned operands need none to speak of; misaligned ones their size once more
    assert size(lb.OP_PRODUCT, 2048, 512, m(pitch=512), m(pitch=512)) == 256
    assert size(lb.OP_PRODUCT, 2048, 511, m(pitch=511), m(pitch=512)) >= 4000 * 512 * 2
    assert size(lb.OP_PRODUCT, 2048, 512, m(E4M3, 512), m(E4M3, 512)) == 256
    assert size(lb.OP_PRODUCT_GRAD_WEIGHT, 64, 96, m(pitch=64), m(I8, 96)) >= 4000 * 96 * 2
    assert size(lb.OP_RESIDUAL_NORM_GRAD, 1, 512, None, None) >= 512 * 4
    for bad in ((99, 64, 64, m(), m()), (lb.OP_PRODUCT, 0, 64, m(), m()), (lb.OP_PRODUCT, 64, 64, m(), None), (lb.OP_PRODUCT, 64, 64, m(), m(F16)),
                (lb.OP_PRODUCT, 64, 65, m(), m()), (lb.OP_PRODUCT_GRAD_INPUT, 64, 64, m(E4M3), m(E4M3)), (lb.OP_RESIDUAL_NORM_GRAD, 1, 20000, None, None)):
        assert size(*bad) == 0, bad
    assert lb.last_workspace_bytes(lb.LastWeights(lb.WEIGHTS_DENSE, 2, 5, 0x1000, None, None, None, 0), lb.context(3, 1), lb.OP_PRODUCT) == 0


def test_binding_refuses_host_tensors_and_shapes():
    x, w, gain = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(8, 32, dtype=torch.bfloat16), torch.ones(32)
    for call in (lambda: lb.last_residual_norm(x, gain), lambda: lb.last_product(x, w), lambda: lb.last_keep(x), lambda: lb.last_product_grad_input(x, w),
                 lambda: lb.last_kept_values(lb.Kept(x, x)), lambda: lb.last_product(torch.zeros(3), w)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        lb._activation("swish")
    with pytest.raises(ValueError):
        lb._pitch(torch.zeros(4, 8).T, "x")
    with pytest.raises(ValueError):
        lb._pitch(torch.zeros(3, 4, 8)[:, :2], "x")
    assert lb._pitch(torch.zeros(3, 4, 8)[:, :, :5], "x") == 8 and lb._pitch(torch.zeros(1, 8), "x") == 8 and lb._pitch(torch.zeros(3, 1, 8)[:, :, :2], "x") == 8


def test_the_oracle_of_eight_bits():
    """The codes' definition on cases by hand."""
    v = np.zeros((1, 32))
    v[0, :5] = [127.0, 1.5, 2.5, -0.5, 126.5]
    got, scales = lo.encode(v, "i8")
    assert scales[0, 0] == 127 and list(got[0, :5]) == [127, 2, 2, 0, 126]
    v[0, 0] = 127.0001
    got, scales = lo.encode(v, "i8")
    assert scales[0, 0] == 128 and got[0, 0] == 128
    v[0, :4] = [448.0, 17.0, 19.0, 2.0 ** -10]
    got, scales = lo.encode(v, "e4m3")
    assert scales[0, 0] == 127 and list(got[0, :4]) == [448, 16, 20, 0]
    got, scales = lo.encode(np.zeros((1, 33)), "i8")
    assert list(scales[0]) == [0, 0] and not got.any()
    v[0, 7] = np.inf
    got, scales = lo.encode(v, "i8")
    assert scales[0, 0] == 255 and np.isnan(got).all()
    rng = np.random.default_rng(0)
    v = rng.standard_normal((50, 70))
    for kind in ("i8", "e4m3"):
        got, scales = lo.encode(v, kind)
        again, s2 = lo.encode(got, kind)
        assert np.array_equal(again, got) and (s2 <= scales).all()


def test_more_results_than_a_launch_takes_are_refused(lib):
    """2^30 rows of 4096 results: even in tiles of 256 x 256 more than 2^32 threads."""
    fr, x, w, y = ref(frames(1 << 10, 1 << 20)), ref(matrix(pitch=64)), ref(matrix(pitch=64)), ref(matrix(pitch=4096))
    assert lib.last_layer_workspace_bytes(lb.OP_PRODUCT, fr, 4096, 64, x, w) == 0
    assert lib.last_product(fr, 4096, 64, x, w, None, 0, None, y, None, ctypes.c_void_p(0x10000), 1 << 40, None) == 2
    assert lib.last_layer_workspace_bytes(lb.OP_PRODUCT, fr, 64, 64, x, w) > 0
    big = ref(matrix(pitch=1 << 20))
    assert lib.last_layer_workspace_bytes(lb.OP_PRODUCT_GRAD_WEIGHT, ref(frames()), 1 << 20, 1 << 20, big, big) == 0
    assert lib.last_product_grad_weight(ref(frames()), 1 << 20, 1 << 20, big, big, 0, ref(matrix(F32, 1 << 20)), None, ctypes.c_void_p(0x10000), 1 << 50, None) == 2


def test_option_of_tiles(lib):
    """Values outside of 0 .. 3 are refused; the workspace follows the setting: shares of a long reduction go by the tiles."""
    fr, m = ref(frames(1, 20000)), ref(matrix(pitch=640))
    sizes = []
    for v in (0, 1, 2, 3):
        assert lib.last_set_option(lb.OPT_PRODUCT_TILES, v) == 0 and lib.last_get_option(lb.OPT_PRODUCT_TILES) == v
        sizes.append(lib.last_layer_workspace_bytes(lb.OP_PRODUCT_GRAD_WEIGHT, fr, 640, 640, m, m))
    assert lib.last_set_option(lb.OPT_PRODUCT_TILES, 4) == 6 and lib.last_set_option(lb.OPT_PRODUCT_TILES, -1) == 6
    assert lib.last_get_option(lb.OPT_PRODUCT_TILES) == 3
    assert lib.last_set_option(lb.OPT_PRODUCT_TILES, 0) == 0
    assert sizes[0] in sizes[1:] and len(set(sizes[1:])) > 1 and min(sizes) >= 256, sizes
