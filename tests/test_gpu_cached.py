"""Paged caches: what is appended, and attention to it, against plain float64 forms (attention_oracle.py, which derives the bounds)."""
import numpy as np
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from attention_oracle import frames_there, head_norm, rounded, split, whole_cached
from layer_oracle import TYPES, assert_within, f64
from gpu_util import announce
from test_gpu_heads import dev, draw, much_memory, spoil  # noqa: F401

pytestmark = pytest.mark.gpu
NAN = float("nan")


def a_cache(rng, B, G, D, kind, page, most, used, spare=3, fill=NAN):
    """A Cache whose pages are shuffled; what no item uses holds `fill`, as do places past an item's frames."""
    entries = max(1, -(-most // page))
    pages = B * entries + spare
    k, v = (torch.full((pages, G, page, D), fill, dtype=TYPES[kind], device="cuda") for _ in range(2))
    table = rng.permutation(pages)[:B * entries].reshape(B, entries).astype(np.int32)
    for t in (k, v):
        for b in range(B):
            for j in range(-(-int(used[b]) // page)):
                n = min(page, int(used[b]) - j * page)
                t[table[b, j], :, :n] = torch.from_numpy(rng.standard_normal((G, n, D)) * 1.2).to(TYPES[kind]).cuda()
    return lb.Cache(k, v, dev(table), dev(used)), table


CASES = [  # B, T, heads, kv_heads, width, left, right, sinks, kind, page, used up to, ragged
    (1, 1, 1, 1, 8, None, 0, 0, "bf16", 1, 0, False),
    (3, 1, 8, 8, 64, None, 0, 0, "bf16", 16, 90, False),
    (4, 1, 8, 2, 128, 40, 0, 4, "f16", 48, 300, False),
    (3, 5, 4, 1, 64, None, None, 0, "bf16", 7, 100, True),
    (2, 16, 6, 2, 40, 33, 2, 3, "f16", 33, 200, True),
    (2, 40, 16, 2, 128, 100, None, 64, "bf16", 64, 260, True),
    (1, 1, 1, 1, 64, None, 0, 0, "f16", 128, 3000, False),
    (2, 3, 32, 1, 32, 500, 0, 33, "bf16", 100, 2500, True),
    (5, 1, 5, 5, 72, 0, 0, 0, "bf16", 10, 64, True),
    (1, 70, 2, 1, 64, 1000, 0, 1, "bf16", 200, 1500, False),
    (2, 1, 64, 1, 16, 31, 0, 64, "f16", 5, 40, False),
]


def setting(case):
    B, T, H, G, D, left, right, sinks, kind, page, most, ragged = case
    rng = np.random.default_rng(D * 13 + T + most)
    used = rng.integers(0, most + 1, B)
    used[0] = most
    n = None
    if ragged:
        n = rng.integers(0, T + 1, B)
        n[0], n[-1] = T, 0 if B > 1 else T
    cache, table = a_cache(rng, B, G, D, kind, page, most + T, used)
    return rng, n, used, cache, table, {"left": left, "right": right, "sinks": sinks}


@pytest.mark.parametrize("case", CASES, ids=str)
def test_append_then_attend(case):
    """New frames go to their places and to no other; their queries then see them and the older ones.  What is not seen or does not exist is
    NaN throughout."""
    announce("cache", case)
    B, T, H, G, D, left, right, sinks, kind, page, most, ragged = case
    rng, n, used, cache, table, band = setting(case)
    count, there = frames_there(B, T, n)
    q, k, v = (draw(rng, (B, T, c * D), kind, 1.5) for c in (H, G, G))
    R = D // 16 * 8
    f = (100.0 ** (-np.arange(R // 2) / max(1, R // 2))).astype(np.float32)
    gq, gk = (1 + 0.3 * rng.standard_normal(D).astype(np.float32) for _ in range(2))
    at = used[:, None] + np.arange(T)
    want_q, eq = head_norm(f64(q), D, gq, at, f, there)
    want_k, ek = head_norm(f64(k), D, gk, at, f, there)
    for t in (q, k, v):
        spoil(t, there)
    before = cache.k.clone(), cache.v.clone()
    yq = lb.last_cache_append(k, v, cache, q=q, gain_q=dev(gq, torch.float32), gain_k=dev(gk, torch.float32),
                              frequencies=dev(f, torch.float32) if R else None, lengths=dev(n))
    lb.check_item_status()
    assert_within(yq, want_q.reshape(B, T, -1), rounded(eq, want_q, kind).reshape(B, T, -1), "queries")
    touched = np.zeros(cache.k.shape[:3], bool)
    vs = split(f64(v), D)
    for b in range(B):
        for t in range(count[b]):
            p, row = table[b, at[b, t] // page], at[b, t] % page
            touched[p, :, row] = True
            assert_within(cache.k[p, :, row], want_k[b, t], rounded(ek[b, t], want_k[b, t], kind), "keys")
            assert np.array_equal(f64(cache.v[p, :, row]), vs[b, t])
    keep = torch.from_numpy(~touched).cuda()
    for now, was in zip((cache.k, cache.v), before):
        assert torch.equal(now.view(torch.int16)[keep], was.view(torch.int16)[keep])
    # attention, with the frames that no window reaches taken out
    gone = []
    for b in range(B):
        if left is not None and count[b]:
            for s in range(sinks, max(0, used[b] - left)):
                if s < used[b] + count[b]:
                    cache.k[table[b, s // page], :, s % page] = NAN
                    cache.v[table[b, s // page], :, s % page] = NAN
                    gone.append((b, s))
    pages = f64(cache.k), f64(cache.v)
    want, e = whole_cached(np.nan_to_num(f64(yq)), np.nan_to_num(pages[0]), np.nan_to_num(pages[1]), table, used, n, left, right, sinks, D ** -0.5, kind)
    spoil(yq, there)
    y = lb.last_cached_attention(yq, cache, lengths=dev(n), **band)
    lb.check_item_status()
    assert_within(y, want, rounded(e, want, kind), "y")
    # pages on which nothing is seen may have any entry
    if left is not None:
        loose = table.copy()
        for b in range(B):
            for j in range(table.shape[1]):
                frames = [s for s in range(j * page, (j + 1) * page) if s < used[b] + count[b] and (s >= used[b] - left or s < sinks)]
                if not frames or count[b] == 0:
                    loose[b, j] = rng.choice([-1, cache.k.shape[0], 2 ** 31 - 1, -2 ** 31])
        again = lb.last_cached_attention(yq, lb.Cache(cache.k, cache.v, dev(loose), cache.used), lengths=dev(n), **band)
        lb.check_item_status()
        assert torch.equal(again, y)


@pytest.mark.parametrize("splits", ["few rows", "many rows"])
def test_bad_pages_are_reported(splits):
    """A page that does not exist among those seen or written: item_status 8, NaN for the frames that see it, nothing written to it."""
    announce("bad pages", splits)
    rng = np.random.default_rng(6)
    B, T, G, D, page = (3, 2, 2, 64, 16) if splits == "few rows" else (3, 40, 8, 64, 16)
    used = np.array([1000, 60, 0])
    cache, table = a_cache(rng, B, G, D, "bf16", page, 1000 + T, used, fill=0.0)
    q = draw(rng, (B, T, 4 * G * D), "bf16")
    want = lb.last_cached_attention(q, cache, left=50, sinks=2)
    lb.check_item_status()
    for item, entry, bad in ((0, 60, -1), (1, 0, cache.k.shape[0]), (0, 0, -5), (1, 3, 2 ** 30)):
        broken = table.copy()
        broken[item, entry] = bad
        status = torch.full((B,), 9, dtype=torch.int32, device="cuda")
        c = lb.Cache(cache.k, cache.v, dev(broken), cache.used)
        y = lb.last_cached_attention(q, c, left=50, sinks=2, item_status=status)
        assert status.tolist() == [8 if b == item else 0 for b in range(B)]
        with pytest.raises(lb.LastError):
            lb.check_item_status(status)
        s = np.arange(entry * page, (entry + 1) * page)
        for t in range(T):
            p = used[item] + t
            sees = ((s <= p) & ((s >= p - 50) | (s < 2))).any()
            row = f64(y)[item, t]
            assert np.isnan(row).all() if sees else torch.equal(y[item, t], want[item, t]), (item, entry, t)
        others = [b for b in range(B) if b != item]
        assert torch.equal(y[others], want[others])
    # frames past the table, and an entry that names no page
    k, v = draw(rng, (B, T, G * D), "bf16"), draw(rng, (B, T, G * D), "bf16")
    small = lb.Cache(cache.k, cache.v, cache.table[:, :62].contiguous(), dev([62 * page - 1, 5, 2 ** 31 - 1]))
    before = cache.k.clone()
    status = torch.full((B,), 9, dtype=torch.int32, device="cuda")
    lb.last_cache_append(k, v, small, item_status=status)
    assert status.tolist() == [8, 0, 8]
    changed = (cache.k != before).any(-1).any(1).nonzero().tolist()
    assert sorted(map(tuple, changed)) == sorted([(table[0, 61], page - 1)] + [(table[1, (5 + t) // page], (5 + t) % page) for t in range(T)])
    lb.last_cached_attention(q, small, left=50, item_status=status)
    assert status.tolist() == [8, 0, 8]
    negative = lb.Cache(cache.k, cache.v, cache.table, dev([-3, 0, 0]))         # clamped to 0
    zero = lb.Cache(cache.k, cache.v, cache.table, dev([0, 0, 0]))
    assert torch.equal(lb.last_cached_attention(q, negative), lb.last_cached_attention(q, zero))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_streaming_is_attention(kind):
    """Frames given one chunk after the other, of several sizes, come out as from one call on all of them."""
    announce("streaming", kind)
    rng = np.random.default_rng(9)
    B, T, H, G, D, page = 2, 150, 4, 2, 64, 24
    q, k, v = (draw(rng, (B, T, c * D), kind) for c in (H, G, G))
    g, f = dev(1 + 0.1 * rng.standard_normal(D), torch.float32), dev(0.8 ** np.arange(32), torch.float32)
    band = {"left": 37, "sinks": 3}
    nq, nk = lb.last_head_norm(q, k, D, g, g, f)
    want, _ = lb.last_attention(nq, nk, v, D, **band)
    cache, _ = a_cache(rng, B, G, D, kind, page, T, np.zeros(B, int))
    at = 0
    for n in (1, 1, 30, 1, 64, 5, 48):
        w = slice(at, at + n)
        cq = lb.last_cache_append(k[:, w].contiguous(), v[:, w].contiguous(), cache, q=q[:, w].contiguous(), gain_q=g, gain_k=g, frequencies=f)
        lb.check_item_status()
        assert torch.equal(cq, nq[:, w])
        y = lb.last_cached_attention(cq, cache, **band)
        lb.check_item_status()
        # both are within their bound of the exact result: P's rounding and the result's own, of 38 values near 1 with probabilities that sum to 1
        off = (y.double() - want[:, w].double()).abs().max()
        assert off <= 2 * (torch.finfo(TYPES[kind]).eps / 2) * 2 * float(v.abs().max()), (n, float(off))
        cache.used.add_(n)
        at += n
    assert at == T


@pytest.mark.parametrize("T", [1, 6])
def test_nan_that_is_not_seen(T):
    """A later frame's NaN has no part in what earlier frames of the chunk see, on one workgroup and on several."""
    announce("cached NaN", T)
    rng = np.random.default_rng(11)
    for B, G, used in ((1, 1, 3000), (16, 8, 100)):
        D, page = 64, 64
        cache, table = a_cache(rng, B, G, D, "bf16", page, used + T, np.full(B, used))
        k, v = draw(rng, (B, T, G * D), "bf16"), draw(rng, (B, T, G * D), "bf16")
        lb.last_cache_append(k, v, cache)
        q = draw(rng, (B, T, 2 * G * D), "bf16")
        want = lb.last_cached_attention(q, cache)
        last = used + T - 1
        cache.v[table[0, last // page], :, last % page, 7] = NAN
        y = lb.last_cached_attention(q, cache)
        assert torch.isnan(y[0, -1].reshape(2 * G, D)[:, 7]).all()
        off = (y[0, :-1].double() - want[0, :-1].double()).abs()
        # (formed again without the matrix cores: without P's rounding)
        assert T == 1 or float(off.max()) <= 2 * 2.0 ** -8 * float(v.abs().max() + 6)
        assert torch.equal(y[1:], want[1:])


def test_shared_pages_and_far_pages(much_memory):  # noqa: F811
    """Items that share pages, and a pool of more than 2^32 bytes whose last pages are used."""
    announce("far pages")
    rng = np.random.default_rng(12)
    G, page, D = 2, 64, 128
    pages = (9 << 30) // (2 * G * page * D * 2)
    k, v = (torch.empty(pages, G, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    used = np.array([300, 300, 256])
    table = (pages - 1 - np.arange(15).reshape(3, 5)).astype(np.int32)
    table[1, :4] = table[0, :4]
    small, _ = a_cache(rng, 3, G, D, "bf16", page, 320, np.array([320, 320, 320]), spare=0)
    own = lb.Cache(small.k, small.v, small.table.clone(), dev(used))
    own.table[1, :4] = own.table[0, :4]
    for b in range(3):
        for j in range(5):
            for big, t in ((k, small.k), (v, small.v)):
                big[int(table[b, j])] = t[int(own.table[b, j])]
    far = lb.Cache(k, v, dev(table), dev(used))
    q = draw(rng, (3, 4, 8 * D), "bf16")
    assert torch.equal(lb.last_cached_attention(q, far), lb.last_cached_attention(q, own))
    x = draw(rng, (3, 4, G * D), "bf16")
    for c in (far, own):
        lb.last_cache_append(x, x, lb.Cache(c.k, c.v, c.table, dev([310, 316, 256])))
        lb.check_item_status()
    for b in range(3):
        assert torch.equal(k[int(table[b, 4])], own.k[int(own.table[b, 4])])


def test_no_new_frames():
    announce("no new frames")
    rng = np.random.default_rng(13)
    cache, _ = a_cache(rng, 2, 1, 64, "bf16", 16, 40, np.array([20, 30]))
    before = cache.k.clone(), cache.v.clone()
    x = torch.empty(2, 0, 64, dtype=torch.bfloat16, device="cuda")
    status = torch.full((2,), 9, dtype=torch.int32, device="cuda")
    assert lb.last_cache_append(x, x, cache, q=x, item_status=status).shape == x.shape
    assert status.tolist() == [0, 0]
    status.fill_(9)
    assert lb.last_cached_attention(x, cache, item_status=status).shape == x.shape
    assert status.tolist() == [0, 0]
    none = lb.Cache(cache.k, cache.v, cache.table[:0], cache.used[:0])
    x = torch.empty(0, 3, 64, dtype=torch.bfloat16, device="cuda")
    lb.last_cache_append(x, x, none)
    assert lb.last_cached_attention(x, none).shape == x.shape
    x = draw(rng, (2, 3, 64), "bf16")
    lb.last_cache_append(x, x, cache, lengths=dev([0, 0]))
    y = lb.last_cached_attention(x, cache, lengths=dev([0, -4]))
    lb.check_item_status()
    assert not y.any()
    for now, was in zip((cache.k, cache.v), before):
        assert torch.equal(now.view(torch.int16), was.view(torch.int16))


def test_captured_steps():
    """A captured step of a stream, replayed while `used` counts on, beside eager steps of another cache, and two graphs in turn."""
    announce("captured steps")
    rng = np.random.default_rng(14)
    B, H, G, D, page, most = 2, 4, 2, 64, 32, 700
    f = dev(0.9 ** np.arange(32), torch.float32)
    start = np.array([600, 300])
    first, _ = a_cache(rng, B, G, D, "bf16", page, most, start)
    caches = [first] + [lb.Cache(first.k.clone(), first.v.clone(), first.table, first.used.clone()) for _ in range(2)]
    x = torch.zeros(B, 1, (H + 2 * G) * D, dtype=torch.bfloat16, device="cuda")

    def step(c):
        q, k, v = x.split([H * D, G * D, G * D], -1)
        y = lb.last_cached_attention(lb.last_cache_append(k, v, c, q=q, frequencies=f), c)
        c.used.add_(1)
        return y
    x.copy_(draw(rng, tuple(x.shape), "bf16"))
    step(lb.Cache(first.k.clone(), first.v.clone(), first.table, first.used.clone()))
    torch.cuda.synchronize()
    graphs = []
    for c in caches[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = step(c)
        graphs.append((graph, y))
    for i in range(6):
        x.copy_(draw(rng, tuple(x.shape), "bf16"))
        for graph, _ in graphs:
            graph.replay()
        want = step(caches[2])
        torch.cuda.synchronize()
        for _, y in graphs:
            assert torch.equal(y, want), i
    assert all(torch.equal(c.used, caches[2].used) for c in caches[:2])
    # (as words: places that hold no frame are NaN)
    assert torch.equal(caches[0].k.view(torch.int16), caches[2].k.view(torch.int16))
