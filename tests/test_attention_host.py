"""Host-only checks of the calls in which frames see each other: what the C ABI and the binding refuse, workspaces, devices."""
import ctypes

import pytest
import torch

from paper_2304_13134_amd import binding as lb
from test_layer_devices_host import devices  # noqa: F401  (a fixture)

F32, BF16, F16, I8 = range(4)
DUMMY, WS = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x10000)


class Heads(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("width", ctypes.c_int32)]


class Band(ctypes.Structure):
    _fields_ = [("left", ctypes.c_int32), ("right", ctypes.c_int32), ("sinks", ctypes.c_int32), ("scale", ctypes.c_float)]


class Rotated(ctypes.Structure):
    _fields_ = [("columns", ctypes.c_int32), ("frequencies", ctypes.c_void_p), ("first", ctypes.c_void_p)]


class Paged(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("type", ctypes.c_int32), ("pages", ctypes.c_int32), ("page", ctypes.c_int32),
                ("entries", ctypes.c_int32), ("table", ctypes.c_void_p), ("used", ctypes.c_void_p)]


@pytest.fixture(scope="module")
def lib():
    return lb.load_library()


def ref(s):
    return None if s is None else ctypes.byref(s)


def frames(B=2, T=5):
    return lb.LastFrames(B, T, None)


def matrix(type_=BF16, pitch=256, data=0x10000):
    return lb.LastMatrix(data, type_, pitch, None, 0)


def cache(**more):
    return Paged(**{**dict(k=0x10000, v=0x20000, type=BF16, pages=10, page=16, entries=4, table=0x3000, used=0x4000), **more})


HEADS = Heads(4, 2, 64)
BAD_HEADS = [(Heads(0, 1, 64), 2), (Heads(4, 0, 64), 2), (Heads(4, 3, 64), 2), (Heads(4, 2, 0), 2), (Heads(2, 4, 64), 2), (Heads(4, 2, 60), 6),
             (Heads(4, 2, 136), 6), (Heads(1 << 17, 1, 8), 2), (None, 1)]
BAD_BANDS = [(None, 1), (Band(-2, 0, 0, 1), 2), (Band(0, -2, 0, 1), 2), (Band(0, 0, -1, 1), 2), (Band(0, 0, 65, 1), 6), (Band(0, 0, 0, 0), 2),
             (Band(0, 0, 0, float("nan")), 2), (Band(0, 0, 0, float("inf")), 2), (Band(0, 0, 0, -1), 2)]
BAD_FRAMES = [(None, 1), (frames(B=0), 2), (frames(T=-1), 2), (frames(1 << 20, 1 << 20), 2)]
BAD_MATRICES = [(matrix(pitch=100), 2), (matrix(data=0x10001), 2), (matrix(data=None), 1), (matrix(I8), 6), (matrix(F16), 6)]


def test_head_norm_refuses(lib):
    def call(fr=frames(), h=HEADS, q=matrix(), k=matrix(), gq=DUMMY, gk=DUMMY, eps=1e-5, r=Rotated(64, 0x1000, None), yq=matrix(), yk=matrix()):
        return lib.last_head_norm(ref(fr), ref(h), ref(q), ref(k), gq, gk, eps, ref(r), ref(yq), ref(yk), None)
    for fr, code in BAD_FRAMES:
        assert call(fr=fr) == code
    for h, code in BAD_HEADS:
        assert call(h=h) == code
    assert call(q=None, k=None) == 1 and call(yq=None) == 1 and call(yk=None) == 1
    assert call(eps=-1.0) == 2 and call(eps=float("nan")) == 2
    for r, code in ((Rotated(-8, 0x1000, None), 2), (Rotated(72, 0x1000, None), 2), (Rotated(12, 0x1000, None), 6), (Rotated(8, None, None), 1)):
        assert call(r=r) == code
    for m, code in BAD_MATRICES:
        assert call(k=m) == code and call(yq=m) == code
    assert call(fr=frames(T=0)) == 0 and call(fr=frames(T=0), q=None, yq=None, r=None, gk=None) == 0
    assert call(fr=frames(1, (1 << 28) + 1)) == 2


def test_head_norm_gradient_refuses(lib):
    def call(fr=frames(), h=HEADS, dyq=matrix(), dyk=matrix(), q=matrix(), k=matrix(), gq=DUMMY, gk=DUMMY, eps=1e-5, r=None, dq=matrix(), dk=matrix(),
             dgq=DUMMY, dgk=DUMMY, ws=WS, n=1 << 20):
        return lib.last_head_norm_grad(ref(fr), ref(h), ref(dyq), ref(dyk), ref(q), ref(k), gq, gk, eps, ref(r), ref(dq), ref(dk), dgq, dgk, ws, n, None)
    for fr, code in BAD_FRAMES:
        assert call(fr=fr) == code
    for h, code in BAD_HEADS:
        assert call(h=h) == code
    assert call(dyq=None, dyk=None) == 1
    for missing in ("q", "k", "dq", "dk"):
        assert call(**{missing: None}) == 1
    assert call(gq=None) == 1 and call(gk=None) == 1 and call(dyq=None) == 1        # a gradient of a gain that is not there
    assert call(ws=None) == 5 and call(n=16) == 5 and call(ws=ctypes.c_void_p(0x10001)) == 5
    for m, code in BAD_MATRICES:
        assert call(k=m) == code and call(dq=m) == code and call(dyk=m) == code


def test_attention_refuses(lib):
    def call(fr=frames(), h=HEADS, b=Band(-1, 0, 0, 1), q=matrix(), k=matrix(), v=matrix(), y=matrix(), lse=None):
        return lib.last_attention(ref(fr), ref(h), ref(b), ref(q), ref(k), ref(v), ref(y), lse, None)

    def grad(fr=frames(), h=HEADS, b=Band(-1, 0, 0, 1), dy=matrix(), q=matrix(), k=matrix(), v=matrix(), y=matrix(), lse=DUMMY, dq=matrix(), dk=matrix(),
             dv=matrix(), ws=WS, n=1 << 20):
        return lib.last_attention_grad(ref(fr), ref(h), ref(b), ref(dy), ref(q), ref(k), ref(v), ref(y), lse, ref(dq), ref(dk), ref(dv), ws, n, None)
    for f in (call, grad):
        for fr, code in BAD_FRAMES:
            assert f(fr=fr) == code
        for h, code in BAD_HEADS:
            assert f(h=h) == code
        for b, code in BAD_BANDS:
            assert f(b=b) == code
        for m, code in BAD_MATRICES:
            assert f(k=m) == code and f(v=m) == code and f(y=m) == code
        assert f(q=matrix(F32), k=matrix(F32), v=matrix(F32), y=matrix(F32)) == 6
        assert f(fr=frames(T=0)) == 0 and f(fr=frames(1, (1 << 28) + 1)) == 2
        # workgroups are numbered in 32 bits
        assert f(fr=frames(1 << 19, 1 << 6), h=Heads(64, 64, 8), q=matrix(pitch=512), k=matrix(pitch=512), v=matrix(pitch=512), y=matrix(pitch=512)) == 2
        for missing in ("q", "k", "v", "y"):
            assert f(**{missing: None}) == 1
    for missing in ("dy", "lse", "dq", "dk", "dv"):
        assert grad(**{missing: None}) == 1
    assert grad(ws=None) == 5 and grad(n=16) == 5 and grad(dk=matrix(F16)) == 6


BAD_CACHES = [(None, 1), (cache(k=None), 1), (cache(v=None), 1), (cache(table=None), 1), (cache(used=None), 1), (cache(pages=0), 2), (cache(page=0), 2),
              (cache(entries=0), 2), (cache(page=1 << 20, entries=1 << 11), 2), (cache(page=(1 << 20) + 1), 2), (cache(k=0x10001), 2), (cache(v=0x20008), 2), (cache(type=F16), 6),
              (cache(type=F32), 6), (cache(type=I8), 6)]


def test_cache_calls_refuse(lib):
    def append(fr=frames(T=0), h=HEADS, q=matrix(), k=matrix(), v=matrix(), gq=DUMMY, gk=DUMMY, eps=1e-5, r=None, c=cache(), yq=matrix(), status=None):
        return lib.last_cache_append(ref(fr), ref(h), ref(q), ref(k), ref(v), gq, gk, eps, ref(r), ref(c), ref(yq), status, None)

    def attend(fr=frames(T=0), h=HEADS, b=Band(-1, 0, 0, 1), q=matrix(), c=cache(), y=matrix(), status=None, ws=WS, n=1 << 20):
        return lib.last_cached_attention(ref(fr), ref(h), ref(b), ref(q), ref(c), ref(y), status, ws, n, None)
    for f in (append, attend):
        assert f() == 0
        for fr, code in BAD_FRAMES:
            assert f(fr=fr) == code
        for h, code in BAD_HEADS:
            assert f(h=h) == code
        for c, code in BAD_CACHES:
            assert f(c=c) == code
        for m, code in BAD_MATRICES:
            assert f(q=m) == code
    for b, code in BAD_BANDS:
        assert attend(b=b) == code
    for m, code in BAD_MATRICES:
        assert append(k=m) == code and append(v=m) == code and append(yq=m) == code and attend(y=m) == code
    assert append(k=None) == 1 and append(v=None) == 1 and append(yq=None) == 1 and append(q=None, yq=None) == 0 and append(eps=-1.0) == 2
    assert append(r=Rotated(8, None, None), fr=frames()) == 1 and append(r=Rotated(100, 0x1000, None)) == 2
    assert attend(fr=frames(1 << 19, 1 << 6), h=Heads(64, 64, 8)) == 2
    assert attend(q=None) == 1 and attend(y=None) == 1 and attend(ws=None) == 5 and attend(n=16) == 5


def test_workspaces(lib):
    def size(op, fr=frames(), h=HEADS, b=Band(-1, 0, 0, 1), c=cache()):
        return lib.last_attention_workspace_bytes(op, ref(fr), ref(h), ref(b), ref(c))
    ops = (lb.OP_HEAD_NORM_GRAD, lb.OP_ATTENTION_GRAD, lb.OP_CACHED_ATTENTION)
    for op in ops:
        assert size(op) >= 256 and size(op) % 256 == 0 and size(op, fr=frames(T=0)) >= 256
        for h, _ in BAD_HEADS:
            assert size(op, h=h) == 0
        for fr, _ in BAD_FRAMES:
            assert size(op, fr=fr) == 0
    for b, _ in BAD_BANDS:
        assert size(ops[1], b=b) == 0 and size(ops[2], b=b) == 0
    for c, code in BAD_CACHES:
        assert code == 6 or size(ops[2], c=c) == 0
    assert size(ops[0], b=None, c=None) >= 256 and size(ops[1], c=None) >= 256
    many = {"fr": frames(1 << 19, 1 << 6), "h": Heads(64, 64, 8)}
    assert size(ops[0], **many) > 0 and size(ops[1], **many) == 0 and size(ops[2], **many) == 0
    assert size(ops[1], fr=frames((1 << 19) - 1, 1 << 6), h=Heads(64, 64, 8)) > 0
    assert size(0) == 0 and size(lb.OP_PRODUCT) == 0 and size(13) == 0
    assert size(ops[1], fr=frames(1, 4096), b=Band(100, 0, 4, 1)) > size(ops[1], fr=frames(1, 4096), b=Band(100, 0, 0, 1))


def calls(dev):
    bf, kind = torch.bfloat16, {"device": "cuda:%d" % dev}
    q, k, v, dy = (torch.empty(2, 6, n * 64, dtype=bf, **kind) for n in (4, 2, 2, 4))
    lengths, gain, f = torch.empty(2, dtype=torch.int32, **kind), torch.empty(64, **kind), torch.empty(32, **kind)
    lse = torch.empty(2, 6, 4, **kind)
    rotation = lb.Rotation(f, torch.empty(2, dtype=torch.int32, **kind))
    pages = [torch.empty(9, 2, 16, 64, dtype=bf, **kind) for _ in range(2)]
    c = lb.Cache(*pages, torch.empty(2, 4, dtype=torch.int32, **kind), torch.empty(2, dtype=torch.int32, **kind))
    status = torch.empty(2, dtype=torch.int32, **kind)
    return {
        "last_head_norm": (lb.last_head_norm, dict(q=q, k=k, width=64, gain_q=gain, gain_k=gain, rotation=rotation, lengths=lengths)),
        "last_head_norm_grad": (lb.last_head_norm_grad, dict(dyq=dy, dyk=k, q=q, k=k, width=64, gain_q=gain, gain_k=gain, rotation=rotation,
                                                             lengths=lengths)),
        "last_attention": (lb.last_attention, dict(q=q, k=k, v=v, width=64, lengths=lengths)),
        "last_attention_grad": (lb.last_attention_grad, dict(dy=dy, q=q, k=k, v=v, y=dy, lse=lse, width=64, lengths=lengths)),
        "last_cache_append": (lb.last_cache_append, dict(k=k, v=v, cache=c, q=q, gain_q=gain, gain_k=gain, frequencies=f, lengths=lengths,
                                                         item_status=status)),
        "last_cached_attention": (lb.last_cached_attention, dict(q=q, cache=c, lengths=lengths, item_status=status)),
    }


NAMES = ["last_head_norm", "last_head_norm_grad", "last_attention", "last_attention_grad", "last_cache_append", "last_cached_attention"]


@pytest.mark.parametrize("name", NAMES)
def test_a_call_runs_on_its_tensors_device(devices, name):  # noqa: F811
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        for dev in (0, 2):
            devices.launched.clear()
            f, arguments = calls(dev)[name]
            f(**arguments)
            assert (name, dev) in devices.launched and all(d == dev for _, d in devices.launched)


@pytest.mark.parametrize("name", NAMES)
def test_operands_of_two_devices_are_refused(devices, name):  # noqa: F811
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        f, arguments = calls(0)[name]
        other = calls(1)[name][1]
        first = {"last_head_norm": "q", "last_head_norm_grad": "dyq", "last_cache_append": "k"}.get(name, "q")
        for key, value in arguments.items():
            if key in ("width", first):
                continue
            parts = [other[key]]
            if isinstance(value, tuple):              # each tensor of a cache or a rotation
                parts = [type(value)(*(o if i == j else s for j, (s, o) in enumerate(zip(value, other[key])))) for i in range(len(value))]
            for part in parts:
                with pytest.raises(ValueError):
                    f(**{**arguments, key: part})
    assert not devices.launched


def test_binding_refuses_shapes(devices):  # noqa: F811
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        def bad(name, error=ValueError, **change):
            f, arguments = calls(0)[name]
            with pytest.raises(error):
                f(**{**arguments, **change})
        kind = {"device": "cuda:0"}
        bf = torch.bfloat16
        wrong = torch.empty(2, 6, 100, dtype=bf, **kind)
        for name, keys in (("last_head_norm", ("q", "k")), ("last_attention", ("q", "k", "v")), ("last_attention_grad", ("dy", "y", "q", "v")),
                           ("last_cache_append", ("k", "v", "q")), ("last_cached_attention", ("q",))):
            for key in keys:
                bad(name, **{key: wrong})
                bad(name, **{key: torch.empty(2, 5, 128, dtype=bf, **kind)} if name != "last_cached_attention" else {key: wrong})
        three = torch.empty(2, 6, 3 * 64, dtype=bf, **kind)
        bad("last_attention", k=three, v=three)
        bad("last_attention", width=0)
        for key in ("left", "right", "sinks"):
            bad("last_attention", **{key: -1})
            bad("last_cached_attention", **{key: -1})
        bad("last_attention", lengths=torch.empty(3, dtype=torch.int32, **kind))
        bad("last_attention", TypeError, lengths=torch.empty(2, dtype=torch.int64, **kind))
        bad("last_head_norm", rotation=lb.Rotation(torch.empty(36, **kind)))
        bad("last_head_norm", rotation=lb.Rotation(torch.empty(3, **kind)))
        bad("last_head_norm", rotation=lb.Rotation(torch.empty(8, **kind), torch.empty(3, dtype=torch.int32, **kind)))
        bad("last_head_norm", gain_q=torch.empty(63, **kind))
        c = calls(0)["last_cached_attention"][1]["cache"]
        for other, error in ((lb.Cache(c.k, c.v[:, :, :8], c.table, c.used), TypeError), (lb.Cache(c.k, c.v[:8], c.table, c.used), ValueError),
                             (lb.Cache(c.k, c.v.half(), c.table, c.used), ValueError), (lb.Cache(c.k.float(), c.v.float(), c.table, c.used), TypeError),
                             (lb.Cache(c.k, c.v, c.table[:1], c.used), ValueError), (lb.Cache(c.k, c.v, c.table, c.used[:1]), ValueError),
                             (lb.Cache(c.k, c.v, c.table.long(), c.used), TypeError)):
            bad("last_cached_attention", error, cache=other)
            bad("last_cache_append", error, cache=other)
        bad("last_cached_attention", item_status=torch.empty(1, dtype=torch.int32, **kind))
        bad("last_cache_append", item_status=torch.empty(1, dtype=torch.int32, **kind))
    assert not devices.launched
