"""Operators that let frames see each other, measured: norms of the heads' queries and keys with their rotation, attention over
a band of frames, and its streaming form on a paged cache, through the calls of ``paper_2304_13134_amd.binding``.

A case is a dict of plain values:

    op       "heads"        last_head_norm: queries and keys normed by head and rotated by their frame's position
             "heads_grad"   last_head_norm_grad: the gradients of both and of the two gains
             "attention"    last_attention: the result and the logarithms of the softmax sums
             "attention_grad"  last_attention_grad: the gradients of queries, keys and values
             "append"       last_cache_append: keys (normed, rotated) and values of new frames to their pages, queries beside them
             "cached"       last_cached_attention: new frames' queries on the cache
    B, T     items and (new) frames; `ragged`: an item has [T / 2, T] of them (heads ... attention_grad), or [0, T] (append, cached)
    heads, kv_heads, width    of queries; of keys and values; columns of a head.  `rotated`: of these, how many are rotated
    type     "bf16", "f16" or "f32"
    left, right, sinks        frame t sees the frames from t - left to t + right, and those before `sinks`; -1: no limit
    far      positions begin at up to 100000 instead of at 0 (heads, heads_grad)
    used     frames in the cache, drawn from [used / 2, used]; `page`: frames of a page

Queries, keys and values are columns of one matrix, as one product makes them.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_EPS = 1e-5


def _case(name, op, B, T, heads, kv_heads, width, type="bf16", rotated=None, left=-1, right=0, sinks=0, ragged=False, far=False,
          used=0, page=0):
    return {"name": name, "op": op, "B": B, "T": T, "heads": heads, "kv_heads": kv_heads, "width": width, "type": type,
            "rotated": width if rotated is None else rotated, "left": left, "right": right, "sinks": sinks, "ragged": ragged,
            "far": far, "used": used, "page": page}


def listed():
    return [
        # a training batch of the benchmark's hidden size, 512 columns as eight heads
        _case("heads_batch", "heads", B=16, T=1024, heads=8, kv_heads=8, width=64, ragged=True),
        # pieces of long recordings in 32 bits, a head size that no power of two is, part of it rotated
        _case("heads_far_odd", "heads", B=7, T=333, heads=6, kv_heads=2, width=40, type="f32", rotated=24, far=True),
        # the backward pass of a wide layer whose keys are shared by four heads
        _case("heads_grad_wide", "heads_grad", B=16, T=1024, heads=16, kv_heads=4, width=128, ragged=True),
        # an encoder that sees whole utterances, batch recognition of unequal ones
        _case("attention_whole", "attention", B=16, T=1000, heads=8, kv_heads=8, width=64, right=-1, ragged=True),
        # a long recording in one piece: a causal window, the first frames stay visible
        _case("attention_long", "attention", B=1, T=8192, heads=16, kv_heads=4, width=128, type="f16", left=1023, sinks=4),
        # training an encoder of limited look-back and look-ahead
        _case("attention_grad_band", "attention_grad", B=16, T=1024, heads=8, kv_heads=8, width=64, left=128, right=32, ragged=True),
        # the largest: training on long pieces, far look-back, the first frames stay visible
        _case("attention_grad_long", "attention_grad", B=2, T=4096, heads=16, kv_heads=4, width=128, left=2047, sinks=4),
        # streaming recognition: one new frame of each of 16 streams
        _case("append_one_frame", "append", B=16, T=1, heads=8, kv_heads=8, width=64, used=2000, page=64),
        # streaming recognition by chunks, streams that have no or few new frames among them; pages that no tile divides
        _case("append_chunk", "append", B=32, T=40, heads=16, kv_heads=4, width=128, used=1000, page=48, ragged=True),
        # one frame of one stream: the shortest call
        _case("cached_one_frame", "cached", B=1, T=1, heads=8, kv_heads=8, width=64, left=255, used=1000, page=64),
        # chunks of streams on a window with first frames
        _case("cached_chunk", "cached", B=8, T=16, heads=8, kv_heads=4, width=64, type="f16", left=1023, right=-1, sinks=4, used=4000,
              page=48, ragged=True),
        # one frame of streams that keep all they heard
        _case("cached_long", "cached", B=16, T=1, heads=16, kv_heads=4, width=128, used=32768, page=128),
    ]


def _about(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; one in three is a multiple of 64."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, max(lo, n // 64 * 64)) if n >= 64 and rng.random() < 1 / 3 else n


def draw(rng):
    op = rng.choice(["heads", "heads_grad", "attention", "attention", "attention_grad", "attention_grad", "append", "cached", "cached"])
    kv = rng.choice([1, 2, 4, 8])
    c = _case("", op, B=_about(rng, 1, 32), T=_about(rng, 1, 4096), heads=kv * rng.choice([1, 1, 2, 4, 8]), kv_heads=kv,
              width=rng.choice([64, 64, 128, 128, 8 * rng.randint(1, 16)]), type=rng.choice(["bf16", "bf16", "f16"]))
    if op in ("heads", "heads_grad"):
        c.update(type=rng.choice([c["type"], c["type"], "f32"]), far=rng.random() < 0.3)
    if op in ("append", "cached"):
        c.update(T=rng.choice([1, 1, _about(rng, 2, 64)]), used=_about(rng, 1, 32768), page=rng.choice([16, 64, 128, rng.randint(1, 200)]))
    if op in ("heads", "heads_grad", "append") and rng.random() < 0.3:
        c["rotated"] = 8 * rng.randint(0, c["width"] // 8)
    if op in ("attention", "attention_grad", "cached"):
        c.update(left=rng.choice([-1, _about(rng, 1, 2048)]), right=rng.choice([-1, 0, 0, _about(rng, 1, 64)]))
        c["sinks"] = rng.choice([0, rng.randint(1, 64)]) if c["left"] >= 0 else 0
    # no more than the listed ones: the score matrices that the plain form lays out, products and bytes
    products, bytes_ = work(listed()[6])["flops"], work(listed()[11])["bytes"]
    while c["B"] * c["heads"] * c["T"] * (c["used"] + c["T"]) > 1 << 29 or work(c)["flops"] > products or work(c)["bytes"] > bytes_:
        if c["B"] > 1:
            c["B"] = (c["B"] + 1) // 2
        else:
            c.update(T=(c["T"] + 1) // 2, used=(c["used"] + 1) // 2)
    c["ragged"] = c["T"] > 1 and rng.random() < 0.5
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    type_ = _TYPES[c["type"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(type_)

    def whole(lo, hi, n):
        return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)

    B, T, H, G, D, op = c["B"], c["T"], c["heads"], c["kv_heads"], c["width"], c["op"]
    s = {"case": c, "lengths": None}
    if c["ragged"]:
        s["lengths"] = whole(0 if c["used"] else max(1, T // 2), T, B)
    # columns of unequal size, as a product makes them
    qkv = normal(B, T, (H + 2 * G) * D) * (0.5 + torch.rand((H + 2 * G) * D, generator=g, device="cuda")).to(type_)
    s["q"], s["k"], s["v"] = qkv.split([H * D, G * D, G * D], dim=-1)
    if op in ("heads", "heads_grad", "append"):
        s["gain_q"], s["gain_k"] = (1 + 0.2 * torch.randn(D, generator=g, device="cuda") for _ in range(2))
        R = c["rotated"]
        s["frequencies"] = 10000.0 ** (-torch.arange(R // 2, device="cuda", dtype=torch.float32) / max(1, R // 2))
        s["first"] = whole(0, 100000, B) if c["far"] else None
    if op == "heads_grad":
        s["dyq"], s["dyk"] = normal(B, T, H * D), normal(B, T, G * D)
    if op in ("attention", "attention_grad", "cached"):          # after their norms
        s["q"], s["k"] = normal(B, T, H * D, scale=1.2), normal(B, T, G * D, scale=1.2)
    if op == "attention_grad":
        s["dy"] = normal(B, T, H * D)
        s["y"], s["lse"] = _attention(s)
    if c["used"]:
        entries = (c["used"] + T + c["page"] - 1) // c["page"]
        s["pages"] = [normal(B * entries, G, c["page"], D, scale=1.2) for _ in range(2)]
        # pages in the order in which streams happened to get them
        s["table"] = torch.randperm(B * entries, generator=g, device="cuda").to(torch.int32).reshape(B, entries)
        s["used"] = whole(max(1, c["used"] // 2), c["used"], B)
    return s


# ---------------------------------------------------------------- plain forms

def _there(s):
    """[B, T] which (new) frames exist"""
    B, T = s["q"].shape[:2]
    t = torch.arange(T, device=s["q"].device)
    return (t < s["lengths"][:, None]) if s["lengths"] is not None else torch.ones(B, T, dtype=torch.bool, device=t.device)


def _zero_past(v, there):
    return torch.where(there.reshape(there.shape + (1,) * (v.dim() - 2)), v, torch.zeros((), dtype=v.dtype, device=v.device))


def _turns(s, first):
    """cosines and sines [B, T, 1, R / 2] of the angles, which are formed in 64 bits"""
    p = first[:, None].double() + torch.arange(s["q"].shape[1], device=s["q"].device)
    a = p[:, :, None, None] * s["frequencies"].double()
    return torch.cos(a).float(), torch.sin(a).float()


def _rotate(n, cos, sin):
    h = cos.shape[-1]
    a, b = n[..., :h], n[..., h:2 * h]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, n[..., 2 * h:]], -1)


def _heads(x, gain, cos, sin, there):
    """[B, T, columns] to [B, T, heads, width], normed and rotated"""
    x = x.float().unflatten(-1, (-1, len(gain)))
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + _EPS) * gain
    return _zero_past(_rotate(n, cos, sin), there)


def _heads_grad(dy, x, gain, cos, sin, there):
    x, dy = (_zero_past(v.float().unflatten(-1, (-1, len(gain))), there) for v in (x, dy))
    inv = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + _EPS)
    dn = _rotate(dy, cos, -sin)
    u = dn * gain
    dx = inv * (u - x * inv * inv * (u * x).mean(-1, keepdim=True))
    return dx.flatten(2), (dn * x * inv).flatten(0, 2).sum(0)


def _seen(c, at, n, total):
    """[B, T, n]: whether the frame at position at[b, t] sees frame s < n, of which total[b] exist"""
    f = torch.arange(n, device=at.device)
    there = f < total[:, None, None]
    p = at[:, :, None]
    if c["right"] >= 0:
        there = there & (f <= p + c["right"])
    if c["left"] >= 0:
        there = there & ((f >= p - c["left"]) | (f < c["sinks"]))
    return there


def _by_kv(v, c):
    """[B, T, heads * width] to [B, kv_heads, heads / kv_heads * T, width] in 32 bits"""
    B, T = v.shape[:2]
    return v.float().reshape(B, T, c["kv_heads"], -1, c["width"]).permute(0, 2, 3, 1, 4).reshape(B, c["kv_heads"], -1, c["width"])


def _back(v, c, B, T):
    return v.reshape(B, c["kv_heads"], -1, T, c["width"]).permute(0, 3, 1, 2, 4).reshape(B, T, -1)


def _scores(q, k, c, seen):
    """[B, kv_heads, heads / kv_heads * T, n], -inf where a frame is not seen"""
    S = torch.matmul(q, k.transpose(-1, -2).contiguous()) * c["width"] ** -0.5
    S = S.unflatten(2, (-1, seen.shape[1]))
    return torch.where(seen[:, None, None], S, torch.full((), -math.inf, device=S.device)).flatten(2, 3)


def _softmax(S):
    """(probabilities, logarithms of the sums) of rows of which some may be empty"""
    m = S.amax(-1, keepdim=True)
    e = torch.exp(S - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total), m + torch.log(total)


def _band(s):
    c, there = s["case"], _there(s)
    B, T = there.shape
    at = torch.arange(T, device=there.device).expand(B, T)
    return there, _seen(c, at, T, there.sum(1)) & there[:, :, None]


def _attention(s):
    c = s["case"]
    there, seen = _band(s)
    B, T = there.shape
    P, L = _softmax(_scores(_by_kv(s["q"], c), _by_kv(s["k"], c), c, seen))
    y = _back(torch.matmul(P, _by_kv(_zero_past(s["v"], there), c)), c, B, T)
    L = L.reshape(B, c["heads"], T).transpose(1, 2)
    return y.to(_TYPES[c["type"]]), _zero_past(L, there).contiguous()


def _attention_grad(s):
    c = s["case"]
    there, seen = _band(s)
    B, T = there.shape
    q, k, v, y, dy = (_by_kv(_zero_past(s[x], there), c) for x in ("q", "k", "v", "y", "dy"))
    P = torch.exp(_scores(q, k, c, seen) - s["lse"].transpose(1, 2).reshape(B, c["kv_heads"], -1, 1))
    dv = torch.matmul(P.transpose(-1, -2).contiguous(), dy)
    dS = torch.matmul(dy, v.transpose(-1, -2).contiguous()) - (dy * y).sum(-1, keepdim=True)
    dS = dS * P * c["width"] ** -0.5
    dq, dk = torch.matmul(dS, k), torch.matmul(dS.transpose(-1, -2).contiguous(), q)
    return tuple(_back(g, c, B, T).to(_TYPES[c["type"]]) for g in (dq, dk, dv))


def _append(s):
    c, there = s["case"], _there(s)
    cos, sin = _turns(s, s["used"])
    q, k = (_heads(s[x], s["gain_" + x], cos, sin, there).to(_TYPES[c["type"]]) for x in ("q", "k"))
    p = s["used"][:, None].long() + torch.arange(c["T"], device=cos.device)
    page, row = torch.gather(s["table"].long(), 1, p // c["page"]), p % c["page"]
    for pages, new in zip(s["pages"], (k, s["v"].unflatten(-1, (-1, c["width"])))):
        # (a frame that does not exist leaves its place as it was)
        pages[page, :, row] = torch.where(there[:, :, None, None], new, pages[page, :, row])
    return {"q": q.flatten(2), "k": s["pages"][0], "v": s["pages"][1]}


def _cached(s):
    c, there = s["case"], _there(s)
    B, T = there.shape
    k, v = (x[s["table"].long()].float().transpose(1, 2).flatten(2, 3) for x in s["pages"])      # [B, kv_heads, n, width]
    at = s["used"][:, None] + torch.arange(T, device=there.device)
    seen = _seen(c, at, k.shape[2], s["used"] + there.sum(1)) & there[:, :, None]
    P, _ = _softmax(_scores(_by_kv(s["q"], c), k, c, seen))
    return _back(torch.matmul(P, v), c, B, T).to(_TYPES[c["type"]])


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op in ("heads", "heads_grad"):
        there, type_ = _there(s), _TYPES[c["type"]]
        first = s["first"] if s["first"] is not None else torch.zeros(c["B"], dtype=torch.int32, device="cuda")
        cos, sin = _turns(s, first)
        if op == "heads":
            return {x: _heads(s[x], s["gain_" + x], cos, sin, there).flatten(2).to(type_) for x in ("q", "k")}
        (dq, dgq), (dk, dgk) = (_heads_grad(s["dy" + x], s[x], s["gain_" + x], cos, sin, there) for x in ("q", "k"))
        return {"dq": dq.to(type_), "dk": dk.to(type_), "dgain_q": dgq, "dgain_k": dgk}
    if op == "attention":
        return dict(zip(("y", "lse"), _attention(s)))
    if op == "attention_grad":
        return dict(zip(("dq", "dk", "dv"), _attention_grad(s)))
    return _append(s) if op == "append" else _cached(s)


# ---------------------------------------------------------------- the library's calls

def run(state):
    if not own:
        return _plain(state)
    from paper_2304_13134_amd import binding as last
    s, c, lengths = state, state["case"], state["lengths"]
    op, D = c["op"], c["width"]
    if op in ("heads", "heads_grad"):
        rotation = last.Rotation(s["frequencies"], s["first"])
        if op == "heads":
            q, k = last.last_head_norm(s["q"], s["k"], D, s["gain_q"], s["gain_k"], rotation, lengths=lengths, eps=_EPS)
            return {"q": q, "k": k}
        dq, dk, dgain_q, dgain_k = last.last_head_norm_grad(s["dyq"], s["dyk"], s["q"], s["k"], D, s["gain_q"], s["gain_k"], rotation,
                                                            lengths=lengths, eps=_EPS)
        return {"dq": dq, "dk": dk, "dgain_q": dgain_q, "dgain_k": dgain_k}
    band = {"left": None if c["left"] < 0 else c["left"], "right": None if c["right"] < 0 else c["right"], "sinks": c["sinks"]}
    if op == "attention":
        y, lse = last.last_attention(s["q"], s["k"], s["v"], D, lengths=lengths, **band)
        return {"y": y, "lse": lse}
    if op == "attention_grad":
        dq, dk, dv = last.last_attention_grad(s["dy"], s["q"], s["k"], s["v"], s["y"], s["lse"], D, lengths=lengths, **band)
        return {"dq": dq, "dk": dk, "dv": dv}
    cache = last.Cache(s["pages"][0], s["pages"][1], s["table"], s["used"])
    if op == "append":
        q = last.last_cache_append(s["k"], s["v"], cache, q=s["q"], gain_q=s["gain_q"], gain_k=s["gain_k"],
                                   frequencies=s["frequencies"], lengths=lengths, eps=_EPS)
        return {"q": q, "k": cache.k, "v": cache.v}
    return last.last_cached_attention(s["q"], cache, lengths=lengths, **band)


# ---------------------------------------------------------------- what a pass cannot do without

def _pairs(c, T, before=0):
    """Pairs of a frame and one that it sees, of an item with T (new) frames."""
    n, end = 0, before + T
    for p in range(before, end):
        last = min(end, p + c["right"] + 1) if c["right"] >= 0 else end
        first = max(0, p - c["left"]) if c["left"] >= 0 else 0
        n += last - first + min(c["sinks"], first)
    return n


def work(case):
    c = case
    size, H, G, D = {"bf16": 2, "f16": 2, "f32": 4}[c["type"]], c["heads"], c["kv_heads"], c["width"]
    share = (0.5 if c["used"] else 0.75) if c["ragged"] else 1.0
    R, op = c["B"] * c["T"], c["op"]
    there = share * R                                   # frames that are read
    q, kv = H * D * size, G * D * size                  # bytes of a frame
    if op == "heads":
        return {"bytes": (there + R) * (q + kv), "flops": 10.0 * there * (H + G) * D}
    if op == "heads_grad":
        return {"bytes": (2 * there + R) * (q + kv) + 16 * D, "flops": 20.0 * there * (H + G) * D}
    if op == "append":
        return {"bytes": there * (q + 4 * kv) + R * q, "flops": 10.0 * there * (H + G) * D}
    before = int(0.75 * c["used"])
    T = max(1, round(share * c["T"]))
    pairs = c["B"] * _pairs(c, T, before) * H
    if op == "cached":
        held = before + T
        if c["left"] >= 0:
            held = min(held, c["left"] + T + c["sinks"])
        return {"bytes": there * q + R * q + c["B"] * held * 2 * kv, "flops": 4.0 * D * pairs}
    if op == "attention":
        return {"bytes": there * (q + 2 * kv) + R * (q + 4 * H), "flops": 4.0 * D * pairs}
    return {"bytes": there * (3 * q + 2 * kv + 4 * H) + R * (q + 2 * kv), "flops": 10.0 * D * pairs}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_turned(x, positions, frequencies, sign=1):
    """rows x [n, heads, D], each pair (i, i + R / 2) a complex number times exp(i angle)"""
    h = len(frequencies)
    z = torch.complex(x[..., :h].contiguous(), x[..., h:2 * h].contiguous())
    z = z * torch.polar(torch.ones((), dtype=x.dtype, device=x.device), sign * positions.double()[:, None, None] * frequencies.double())
    return torch.cat([z.real, z.imag, x[..., 2 * h:]], -1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, T, H, G, D, op = c["B"], c["T"], c["heads"], c["kv_heads"], c["width"], c["op"]
    lengths = [T] * B if s["lengths"] is None else s["lengths"].tolist()
    f64 = torch.float64

    def normed(x, gain):
        r = x.square().sum(-1, keepdim=True).div(D).add(_EPS).pow(-0.5)
        return x * r * gain.to(f64), r

    if op in ("heads", "heads_grad", "append"):
        first = s["used"].tolist() if op == "append" else [0] * B if s["first"] is None else s["first"].tolist()
        out = {x: torch.zeros(B, T, n * D, dtype=f64, device="cuda") for x, n in (("q", H), ("k", G))}
        gains = {x: torch.zeros(D, dtype=f64, device="cuda") for x in ("q", "k")}
        pages = [x.to(f64) for x in s["pages"]] if op == "append" else None
        for b in range(B):
            n = lengths[b]
            p = torch.arange(first[b], first[b] + n, device="cuda")
            for x in ("q", "k"):
                rows, gain = s[x][b, :n].to(f64).reshape(n, -1, D), s["gain_" + x]
                if op == "heads_grad":
                    dn = _exact_turned(s["dy" + x][b, :n].to(f64).reshape(n, -1, D), p, s["frequencies"], -1)
                    unit = normed(rows, torch.ones_like(gain))
                    gains[x] += (dn * unit[0]).sum((0, 1))
                    u = dn * gain.to(f64)
                    out[x][b, :n] = (unit[1] * (u - unit[0] * (u * unit[0]).sum(-1, keepdim=True) / D)).flatten(1)
                else:
                    out[x][b, :n] = _exact_turned(normed(rows, gain)[0], p, s["frequencies"]).flatten(1)
            if op == "append":
                table = s["table"][b].tolist()
                for i in range(n):
                    at, row = table[(first[b] + i) // c["page"]], (first[b] + i) % c["page"]
                    pages[0][at, :, row] = out["k"][b, i].reshape(G, D)
                    pages[1][at, :, row] = s["v"][b, i].to(f64).reshape(G, D)
        if op == "append":
            return {"q": out["q"], "k": pages[0], "v": pages[1]}
        return out if op == "heads" else {"dq": out["q"], "dk": out["k"], "dgain_q": gains["q"], "dgain_k": gains["k"]}

    y, lse = torch.zeros(B, T, H * D, dtype=f64, device="cuda"), torch.zeros(B, T, H, dtype=f64, device="cuda")
    dq, dk, dv = (torch.zeros(B, T, n * D, dtype=f64, device="cuda") for n in (H, G, G))
    for b in range(B):
        n, before = lengths[b], int(s["used"][b]) if op == "cached" else 0
        if n == 0:
            continue
        end = before + n
        if op == "cached":
            k, v = (x[s["table"][b].long()].transpose(1, 2).reshape(-1, G, D)[:end].to(f64) for x in s["pages"])
        else:
            k, v = s["k"][b, :n].to(f64).reshape(n, G, D), s["v"][b, :n].to(f64).reshape(n, G, D)
        ahead = torch.arange(end, device="cuda") - torch.arange(before, end, device="cuda")[:, None]
        hidden = torch.zeros_like(ahead, dtype=torch.bool)
        if c["right"] >= 0:
            hidden |= ahead > c["right"]
        if c["left"] >= 0:
            hidden[:, c["sinks"]:] |= ahead[:, c["sinks"]:] < -c["left"]
        for h in range(H):
            at, kv = slice(h * D, (h + 1) * D), h * G // H
            q, kh, vh = s["q"][b, :n, at].to(f64), k[:, kv], v[:, kv]
            S = (q @ kh.t()).div(math.sqrt(D)).masked_fill(hidden, -math.inf)
            L = S.logsumexp(1)
            P = (S - L[:, None]).exp()
            if op != "attention_grad":
                y[b, :n, at], lse[b, :n, h] = P @ vh, L
                continue
            dy, to = s["dy"][b, :n, at].to(f64), slice(kv * D, (kv + 1) * D)
            dP = dy @ vh.t()
            dS = P * (dP - (P * dP).sum(1, keepdim=True)) / math.sqrt(D)
            dq[b, :n, at] = dS @ kh
            dk[b, :n, to] += dS.t() @ q
            dv[b, :n, to] += P.t() @ dy
    return {"y": y, "lse": lse} if op == "attention" else {"dq": dq, "dk": dk, "dv": dv} if op == "attention_grad" else y
