"""Rows of attention that infinities and NaN have reached: formed again over what they see alone, at a cost that stays near an ordinary call's."""
import numpy as np
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from attention_oracle import rounded, seen, whole_attention, whole_cached
from layer_oracle import assert_within, f64
from gpu_util import announce
from test_gpu_cached import a_cache
from test_gpu_heads import dev, draw

pytestmark = pytest.mark.gpu

CASES = [  # B, T, heads, kv_heads, width, left, right, sinks, kind, bad frame
    (1, 400, 2, 1, 64, None, 0, 0, "bf16", 300),
    (1, 400, 2, 1, 8, None, 0, 0, "f16", 0),
    (2, 500, 2, 2, 128, 150, 30, 40, "f16", 450),
    (70, 300, 8, 8, 40, 190, 5, 64, "bf16", 290),
    (1, 700, 1, 1, 72, 63, 0, 1, "bf16", 640),
    (1, 500, 2, 1, 32, 200, None, 33, "f16", 20),
]


def columns(x, heads, D, c):
    """all columns of each head but c"""
    return np.delete(x.reshape(*x.shape[:-1], heads, D), c, -1)


@pytest.mark.parametrize("bad", ["nan", "inf"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_a_bad_value(case, bad):
    """One element of one frame's values: the frames that do not see it have the result that they have without it, and so have the other columns
    of those that do."""
    B, T, H, G, D, left, right, sinks, kind, s = case
    announce("bad value", case, bad)
    rng = np.random.default_rng(T + D)
    q, k, v = (draw(rng, (B, T, c * D), kind, 1.2) for c in (H, G, G))
    c = min(5, D - 1)
    want, e, L, eL = whole_attention(f64(q[:1]), f64(k[:1]), f64(v[:1]), D, None, left, right, sinks, D ** -0.5, kind)
    e = rounded(e, want, kind)
    v[0, s, c] = float(bad)
    y, lse = lb.last_attention(q, k, v, D, left=left, right=right, sinks=sinks)
    # (the head that the element is in: the first of keys and values)
    y, lse, first = f64(y[:1]), f64(lse[:1]), H // G
    m = seen(np.arange(T), T, T, left, right, sinks)[:, s]
    assert m.any()
    assert_within(lse, L, eL, "lse")
    assert_within(columns(y, H, D, c), columns(want, H, D, c), columns(e, H, D, c), "other columns")
    assert_within(y[:, ~m], want[:, ~m], e[:, ~m], "rows that do not see it")
    hit = y.reshape(T, H, D)[m][:, :first, c]
    assert np.isnan(hit).all() if bad == "nan" else not np.isfinite(hit).any()


@pytest.mark.parametrize("bad", ["nan", "inf"])
@pytest.mark.parametrize("T,H,G,D,used,left,sinks,kind,s", [(1, 4, 1, 64, 3000, None, 0, "bf16", 1700), (5, 2, 2, 128, 900, 600, 50, "f16", 20),
                                                            (40, 2, 1, 40, 150, 100, 3, "bf16", 189), (3, 1, 1, 8, 70, None, 0, "f16", 70)])
def test_a_bad_value_in_a_cache(T, H, G, D, used, left, sinks, kind, s, bad):
    announce("bad value in a cache", T, H, D, used, bad)
    rng = np.random.default_rng(used)
    page = 48
    cache, table = a_cache(rng, 2, G, D, kind, page, used + T, np.full(2, used + T))
    cache.used.fill_(used)
    q, c = draw(rng, (2, T, H * D), kind), min(5, D - 1)
    want, e = whole_cached(f64(q), np.nan_to_num(f64(cache.k)), np.nan_to_num(f64(cache.v)), table, np.full(2, used), None, left, 0, sinks, D ** -0.5, kind)
    e = rounded(e, want, kind)
    cache.v[table[0, s // page], 0, s % page, c] = float(bad)
    y = lb.last_cached_attention(q, cache, left=left, sinks=sinks)
    lb.check_item_status()
    y = f64(y)
    assert_within(columns(y, H, D, c), columns(want, H, D, c), columns(e, H, D, c), "other columns")
    m = seen(used + np.arange(T), used + T, used + T, left, 0, sinks)[:, s]
    assert m.any()
    assert_within(y[0][~m], want[0][~m], e[0][~m], "rows that do not see it")
    assert_within(y[1], want[1], e[1], "the other stream")
    assert not np.isfinite(y[0].reshape(T, H, D)[m][:, :H // G, c]).any()


def milliseconds(call):
    """the least of three"""
    call()
    times = []
    for _ in range(3):
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        call()
        end.record()
        torch.cuda.synchronize()
        times.append(start.elapsed_time(end))
    return min(times)


@pytest.mark.parametrize("T,D,left,s", [(16384, 64, None, 0), (16384, 64, None, 16000), (16384, 128, 5000, 16300), (1 << 20, 8, 20, (1 << 20) - 30)])
def test_a_bad_key_on_a_long_item(T, D, left, s):
    """All that see the key are NaN, the others have the bits that they have without it, and it takes no longer: a walk through all earlier frames for each row
    would take tens of milliseconds, an ordinary call takes 0.05 to 0.2."""
    announce("bad key, long", T, D, left)
    rng = np.random.default_rng(1)
    q, k, v = (draw(rng, (1, T, D), "bf16") for _ in range(3))
    y0, l0 = lb.last_attention(q, k, v, D, left=left)
    k[0, s, 3] = float("nan")
    y, lse = lb.last_attention(q, k, v, D, left=left)
    t = torch.arange(T, device="cuda")
    sees = (t >= s) & (t <= s + (T if left is None else left))
    assert torch.isnan(y[0, sees]).all() and torch.isnan(lse[0, sees]).all()
    assert torch.equal(y[0, ~sees], y0[0, ~sees]) and torch.equal(lse[0, ~sees], l0[0, ~sees])
    ms = milliseconds(lambda: lb.last_attention(q, k, v, D, left=left))
    print("milliseconds", ms, flush=True)
    assert ms < 2


def test_a_bad_key_in_a_long_cache():
    """A window at the end of a million frames, with first ones, of 32 heads that share keys."""
    announce("bad key in a long cache")
    rng = np.random.default_rng(2)
    D, page, entries = 8, 64, 1 << 14
    k, v = (torch.from_numpy(rng.standard_normal((entries, 1, page, D))).bfloat16().cuda() for _ in range(2))
    used = page * entries - 1
    cache = lb.Cache(k, v, dev(np.arange(entries)[None]), dev([used]))
    q = draw(rng, (1, 1, 32 * D), "bf16")
    k[-1, 0, -2, 3] = float("nan")

    def call():
        return lb.last_cached_attention(q, cache, left=50, sinks=2)
    assert torch.isnan(call()).all()
    lb.check_item_status()
    ms = milliseconds(call)
    print("milliseconds", ms, flush=True)
    assert ms < 2
