"""The norm's gradient on more rows than there are wavefronts for: each goes over several, the next one sent for ahead."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from layer_oracle import EIGHT, TYPES, U32, assert_within, decode, exists, f64, rounding
from gpu_util import announce
from test_gpu_layer import dev_lengths, draw, spoil, zeros_where

pytestmark = pytest.mark.gpu
# (items, frames, columns): 4096 rows a turn up to 1024 columns, 1024 up to 4096, 512 beyond; two turns and a bit or more, and row
# counts that no number of workgroups divides
TURNS = [(3, 3001, 96), (2, 4700, 700), (5, 501, 1500), (3, 777, 2100), (3, 401, 4100), (2, 601, 8200)]


def case(B, T, H, dyt, st, dxt, ds, seed=0):
    rng = np.random.default_rng(H + T + seed)
    dy, d = draw(rng, (B, T, H), dyt), draw(rng, (B, T, H), dxt) if ds else None
    s = lb.last_keep(draw(rng, (B, T, H), "f32", 2.0), EIGHT[st]) if st in EIGHT else draw(rng, (B, T, H), st, 2.0)
    sv = decode(s) if st in EIGHT else f64(s)
    gain = 1 + 0.2 * draw(rng, (H,), "f32")
    inv = torch.from_numpy((1 / np.sqrt((sv * sv).mean(-1) + 1e-5)).astype(np.float32)).cuda()
    # ends in the middle, an item without frames, one without an end: every kind of neighbour in a turn
    n = rng.integers(T // 3, T, B).astype(np.int32)
    n[0], n[-1] = (T, n[-1]) if B < 3 else (T, 0)
    return dy, s, sv, d, gain, inv, n


def formula(dy, sv, d, gain, inv, there):
    """(dx, its bound but for the result's rounding, dgain, its bound): see test_gpu_layer.test_norm_gradient."""
    g, i = f64(dy), f64(inv)[..., None]
    u = g * f64(gain)
    dot, mag = (u * sv).mean(-1, keepdims=True), np.abs(u * sv).mean(-1, keepdims=True)
    dd = f64(d) if d is not None else 0 * g
    dx = zeros_where(i * (u - sv * i * i * dot) + dd, there)
    err = zeros_where(i * (8 * U32 * np.abs(u) + np.abs(sv) * i * i * (g.shape[-1] + 16) * U32 * mag) + 4 * U32 * np.abs(dd), there)
    terms = zeros_where(g * sv * i, there)
    return dx, err, terms.sum((0, 1)), (there.size + 8) * U32 * np.abs(terms).sum((0, 1))


@pytest.mark.parametrize("B,T,H", TURNS)
@pytest.mark.parametrize("dyt,st,dxt,ds", [("bf16", "bf16", "bf16", True), ("f32", "f32", "f32", False), ("f32", "f16", "f16", True), ("bf16", "i8", "bf16", True),
                                          ("f32", "e4m3", "f32", True)])
def test_several_rows_each(B, T, H, dyt, st, dxt, ds):
    announce("several rows each", B, T, H, dyt, st, dxt, ds)
    dy, s, sv, d, gain, inv, n = case(B, T, H, dyt, st, dxt, ds)
    there = exists(B, T, n)
    dx, err, dgain, err_gain = formula(dy, sv, d, gain, inv, there)
    spoil(dy, there), spoil(s, there)
    got, got_gain = lb.last_residual_norm_grad(dy, s, gain, inv, ds=d, lengths=dev_lengths(n), dtype=TYPES[dxt])
    assert_within(got, dx, err + rounding(dx, dxt), "dx")
    assert_within(got_gain, dgain, err_gain, "dgain")


@pytest.mark.parametrize("B,T,H", TURNS)
@pytest.mark.parametrize("over", ["dy", "ds"])
def test_written_over_an_operand(B, T, H, over):
    """dx over dy or over ds, which later rows are read from while earlier ones are written: the bits of a call with its own dx."""
    announce("dx over", over, B, T, H)
    dy, s, _, d, gain, inv, n = case(B, T, H, "bf16", "bf16", "bf16", True, seed=1)
    lengths = dev_lengths(n)
    want, want_gain = lb.last_residual_norm_grad(dy, s, gain, inv, ds=d, lengths=lengths)
    lib = lb.load_library()
    fr = lb.LastFrames(B, T, lengths.data_ptr())
    m = {k: lb.LastMatrix(t.data_ptr(), 1, H, None, 0) for k, t in (("dy", dy), ("s", s), ("ds", d))}
    ref = ctypes.byref
    ws = torch.empty(lib.last_layer_workspace_bytes(lb.OP_RESIDUAL_NORM_GRAD, ref(fr), 1, H, None, None), dtype=torch.uint8, device="cuda")
    dgain = torch.empty(H, device="cuda")
    code = lib.last_residual_norm_grad(ref(fr), H, ref(m["dy"]), ref(m["s"]), gain.data_ptr(), inv.data_ptr(), ref(m["ds"]), ref(m[over]), dgain.data_ptr(),
                                       ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert code == 0
    assert torch.equal(dy if over == "dy" else d, want) and torch.equal(dgain, want_gain)


@pytest.mark.parametrize("H", [33, 512, 2048, 4100, 9000])
@pytest.mark.parametrize("over", ["x", "residual"])
def test_sum_written_over_an_operand(H, over):
    """s over x or over the residual, dx of an activation over dy: the bits of calls with results of their own."""
    announce("s over", over, H)
    rng = np.random.default_rng(H)
    B, T = 3, 17
    x, r, gain = draw(rng, (B, T, H), "bf16"), draw(rng, (B, T, H), "bf16"), 1 + 0.2 * draw(rng, (H,), "f32")
    kept = lb.last_keep(draw(rng, (B, T, H), "f32"), EIGHT["i8"])
    lengths = torch.tensor([T, 0, 5], dtype=torch.int32, device="cuda")
    for keep in (None, torch.int8):
        want = lb.last_residual_norm(x, gain, residual=r, lengths=lengths, dtype=torch.bfloat16, keep=keep)
        want_dx = lb.last_kept_grad(r, kept, "silu", lengths=lengths)
        lib, ref, stream = lb.load_library(), ctypes.byref, torch.cuda.current_stream().cuda_stream
        fr, xs, rs, y = lb.LastFrames(B, T, lengths.data_ptr()), x.clone(), r.clone(), torch.empty_like(x)
        m = {k: lb.LastMatrix(t.data_ptr(), 1, H, None, 0) for k, t in (("x", xs), ("residual", rs), ("y", y))}
        blocks = (H + 31) // 32
        codes, scales = torch.empty(B, T, H, dtype=torch.int8, device="cuda"), torch.empty(B, T, blocks, dtype=torch.uint8, device="cuda")
        k8 = lb.LastMatrix(codes.data_ptr(), 3, H, scales.data_ptr(), blocks)
        assert lib.last_residual_norm(ref(fr), H, ref(m["x"]), ref(m["residual"]), gain.data_ptr(), 1e-5, ref(m[over]), ref(m["y"]),
                                      ref(k8) if keep else None, None, stream) == 0
        assert torch.equal(xs if over == "x" else rs, want.s) and torch.equal(y, want.y)
        if keep:
            assert torch.equal(codes, want.kept[0]) and torch.equal(scales, want.kept[1])
        dy = r.clone()
        mdy, mk = lb.LastMatrix(dy.data_ptr(), 1, H, None, 0), lb.LastMatrix(kept[0].data_ptr(), 3, H, kept[1].data_ptr(), blocks)
        assert lib.last_kept_grad(ref(fr), H, ref(mdy), ref(mk), 2, ref(mdy), stream) == 0
        assert torch.equal(dy, want_dx)
