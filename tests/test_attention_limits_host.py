"""The largest sizes that include/last.h allows calls in which frames see each other, and the next ones."""
import pytest

from paper_2304_13134_amd import binding as lb
from test_attention_host import Band, Heads, cache, frames, lib, matrix, ref, DUMMY, WS  # noqa: F401

OPS = (lb.OP_HEAD_NORM_GRAD, lb.OP_ATTENTION_GRAD, lb.OP_CACHED_ATTENTION)
BAND = Band(-1, 0, 0, 1)


def size(lib, op, B, T, heads, c=None):  # noqa: F811
    return lib.last_attention_workspace_bytes(op, ref(frames(B, T)), ref(Heads(heads, heads, 8)), ref(BAND), ref(c or cache()))


def codes(lib, B, T, heads):  # noqa: F811
    """what the calls return that have nothing to refuse but their sizes (asked for refused ones alone: they launch what they take)"""
    f, h, m = ref(frames(B, T)), ref(Heads(heads, heads, 8)), ref(matrix(pitch=8 * heads))
    return [lib.last_head_norm(f, h, m, m, None, None, 1e-5, None, m, m, None),
            lib.last_head_norm_grad(f, h, m, m, m, m, None, None, 1e-5, None, m, m, None, None, WS, 1 << 40, None),
            lib.last_cache_append(f, h, m, m, m, None, None, 1e-5, None, ref(cache()), m, None, None),
            lib.last_attention(f, h, ref(BAND), m, m, m, m, None, None),
            lib.last_attention_grad(f, h, ref(BAND), m, m, m, m, m, DUMMY, m, m, m, WS, 1 << 40, None),
            lib.last_cached_attention(f, h, ref(BAND), m, ref(cache()), m, None, WS, 1 << 40, None)]


@pytest.mark.parametrize("inside,outside", [((1, 1 << 24, 64), (1, 1 << 24, 65)), ((1, 1 << 28, 4), (1, (1 << 28) + 1, 4)), ((1, 1 << 28, 4), (1, 1 << 28, 5)),
                                            ((1, 1 << 14, 1 << 16), (1, 1 << 14, (1 << 16) + 1)), ((1, 1 << 14, 1 << 16), (1, (1 << 14) + 1, 1 << 16))])
def test_frames_and_heads_of_an_item(lib, inside, outside):  # noqa: F811
    assert all(size(lib, op, *inside) > 0 for op in OPS)
    assert all(size(lib, op, *outside) == 0 for op in OPS)
    assert codes(lib, *outside) == [2] * 6


def test_heads_of_a_call(lib):  # noqa: F811
    """2^36 of norms, 2^31 - 1 where there is a band"""
    assert size(lib, OPS[0], 64, 1 << 14, 1 << 16) > 0 and size(lib, OPS[0], 65, 1 << 14, 1 << 16) == 0
    assert codes(lib, 65, 1 << 14, 1 << 16) == [2] * 6
    for op in OPS[1:]:
        assert size(lib, op, 2, (1 << 14) - 1, 1 << 16) > 0 and size(lib, op, 2, 1 << 14, 1 << 16) == 0
    assert codes(lib, 2, 1 << 14, 1 << 16)[3:] == [2] * 3


def test_pages(lib):  # noqa: F811
    for page, entries, taken in ((1 << 20, 1 << 10, True), ((1 << 20) + 1, 1, False), (1 << 20, (1 << 10) + 1, False), (1, 1 << 30, True), (1, (1 << 30) + 1, False)):
        assert (size(lib, OPS[2], 2, 5, 4, cache(page=page, entries=entries)) > 0) == taken
