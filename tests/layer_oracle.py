"""Plain float64 forms of the layer between frames and lattice, on the CPU, and the bounds that its results are held to.

Bounds.  u = 2^-24.  A float32 sum of n terms in any order is within n u sum|terms| of the exact one (products of 16-bit and
8-bit operands are exact in float32).  Activations and their derivatives are good to 4e-6 of their magnitude plus 2e-7, and
pass an error of their argument on at most 1.13 times (the largest slope of the four).  A result is rounded once, to half a
unit in its last place: with 8, 11 and 24 significant bits at most 2^-8 of it in bfloat16, 2^-11 in float16 (2^-25 where it is
subnormal), 2^-24 in float32."""
import numpy as np
import torch
from scipy.special import erf, expit

U32 = 2.0 ** -24
EIGHT = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MOST = {"i8": 127.0, "e4m3": 448.0}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def rounding(want, kind):
    w = np.abs(want)
    return {"f32": w * U32 + 1e-44, "bf16": w * 2.0 ** -8 + 1e-39, "f16": w * 2.0 ** -11 + 2.0 ** -25}[kind]


def act(v, kind):
    if kind == "relu":
        return np.where(v < 0, 0.0, v)
    if kind == "silu":
        return v * expit(v)
    if kind == "gelu":
        return 0.5 * v * (1 + erf(v / np.sqrt(2)))
    return np.tanh(v) if kind == "tanh" else v


def slope(v, kind):
    if kind == "relu":
        return (v > 0).astype(float)
    if kind == "silu":
        return expit(v) * (1 + v * expit(-v))
    if kind == "gelu":
        return 0.5 * (1 + erf(v / np.sqrt(2))) + v * np.exp(-v * v / 2) / np.sqrt(2 * np.pi)
    return 1 / np.cosh(np.clip(v, -300, 300)) ** 2 if kind == "tanh" else np.ones_like(v)


def eight_bit_sums(x, w):
    """What the matrix instruction for 8-bit operands leaves out at most: of the products of a block of 32 it keeps multiples of
    2^-13 of the largest one's power of two (1 + 2^-13 comes out as it is, 1 + 2^-14 as 1); blocks are added in float32."""
    out = 0.0
    for k in range(0, x.shape[-1], 32):
        top = np.abs(x[..., k, None] * w[:, k])
        for j in range(k + 1, min(k + 32, x.shape[-1])):
            np.maximum(top, np.abs(x[..., j, None] * w[:, j]), out=top)
        out = out + 32 * 2.0 ** -13 * top
    return out


def exists(B, T, lengths):
    """[B, T] which frames exist"""
    t = np.arange(T)[None, :]
    return np.ones((B, T), bool) if lengths is None else t < np.clip(np.asarray(lengths), 0, T)[:, None]


def blocks(v):
    H = v.shape[-1]
    return np.pad(v, [(0, 0)] * (v.ndim - 1) + [(0, -H % 32)]).reshape(*v.shape[:-1], -1, 32)


def encode(v, kind):
    """(values that the codes stand for, scale bytes): the smallest power of two from 2^-127 at which the block's largest
    magnitude does not pass the largest code; codes to nearest even; byte 255 and NaN for a block that is not finite."""
    H = v.shape[-1]
    b = blocks(np.asarray(v, np.float64))
    bad = ~np.isfinite(b).all(-1)
    top = np.abs(np.where(np.isfinite(b), b, 0)).max(-1)
    m, e = np.frexp(top / MOST[kind])             # top / MOST = m 2^e, 1/2 <= m < 1: exact powers want e - 1
    e = np.where(m == 0.5, e - 1, e)
    e = np.maximum(np.where(top == 0, -127, e), -127)
    # (the division rounds; put right against the exact comparison)
    e = np.where((top > MOST[kind] * np.exp2(e)), e + 1, e)
    e = np.where((e > -127) & (top <= MOST[kind] * np.exp2(e - 1.0)), e - 1, e)
    q = np.where(bad[..., None], 0, b) * np.exp2(-e.astype(float))[..., None]
    if kind == "i8":
        q = np.rint(q)
    else:
        step = np.exp2(np.maximum(np.frexp(np.abs(q))[1] - 1, -6) - 3.0)
        q = np.rint(q / step) * step
    out = q * np.exp2(e.astype(float))[..., None]
    out[bad] = np.nan
    return out.reshape(*v.shape[:-1], -1)[..., :H], np.where(bad, 255, e + 127).astype(np.uint8)


def decode(kept):
    codes, scales = kept[0].cpu(), kept[1].cpu().numpy().astype(int)
    q = codes.to(torch.float32).numpy().astype(np.float64)
    two = np.where(scales == 255, np.nan, np.exp2(scales - 127.0))
    return q * np.repeat(two, 32, -1)[..., :q.shape[-1]]


def assert_within(got, want, bound, what=""):
    got = f64(got) if isinstance(got, torch.Tensor) else np.asarray(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(got - want)) - bound
    bad = ~(off <= 0)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], np.broadcast_to(bound, want.shape)[bad][:3])


def assert_kept(kept, want, error, kind, what=""):
    """Codes of values known to within `error`: each within half a step of it, at the scale of its block."""
    got, scales = decode(kept), kept[1].cpu().numpy().astype(int)
    H = want.shape[-1]
    top, slack = np.abs(blocks(want)).max(-1), blocks(np.broadcast_to(error, want.shape)).max(-1)
    e = scales - 127.0
    assert (top - slack <= MOST[kind] * np.exp2(e)).all(), (what, "a value passes the largest code")
    assert ((scales == 0) | (top + slack > MOST[kind] * np.exp2(e - 1))).all(), (what, "the scale is not the smallest")
    two = np.repeat(np.exp2(e), 32, -1)[..., :H]
    step = two if kind == "i8" else two * np.exp2(np.maximum(np.frexp((np.abs(want) + error) / two)[1] - 1, -6) - 3.0)
    assert_within(got, want, step / 2 * (1 + 1e-6) + error, what)
