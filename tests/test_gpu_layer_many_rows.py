"""More rows than a launch has threads for: 2^32 threads are one too many, so such calls go out in pieces."""
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from gpu_util import announce

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    lb.release_workspaces()
    torch.cuda.empty_cache()
    yield
    lb.release_workspaces()
    torch.cuda.empty_cache()


def by_column(rows, columns, period=1009):
    """[rows, columns] bfloat16 whose row r repeats every `period` rows; a prime, so that no piece of a call begins at one."""
    g = torch.Generator(device="cuda").manual_seed(3)
    some = torch.randn(period, columns, generator=g, device="cuda").bfloat16()
    x = torch.empty(rows, columns, dtype=torch.bfloat16, device="cuda")
    whole = rows // period
    x[:whole * period].view(whole, period, columns).copy_(some.expand(whole, period, columns))
    x[whole * period:].copy_(some[:rows - whole * period])
    return x, some


def assert_repeats(y, some, missing=0):
    """Every row of y [rows, columns] is that of `some` (its period's), bit for bit; the last `missing` are zeros."""
    period, rows = some.shape[0], y.shape[0] - missing
    step = max(1, (1 << 30) // some.numel())
    for first in range(0, rows, step * period):
        part = y[first:min(rows, first + step * period)]
        whole = part.shape[0] // period
        assert bool((part[:whole * period].view(whole, period, y.shape[1]) == some).all()), first
        assert torch.equal(part[whole * period:], some[:part.shape[0] - whole * period]), first
    assert not y[rows:].any()


@pytest.mark.parametrize("rows,H,keep", [((1 << 26) + 78, 16, None), ((1 << 26) + 78, 16, torch.int8), ((1 << 24) + 6, 2056, torch.int8)])
def test_norm_of_many_rows(rows, H, keep):
    """One wavefront a row, and four; two items, of which the last two frames do not exist."""
    announce("norm of many rows", rows, H, keep)
    x, some = by_column(rows, H)
    gain = torch.ones(H, device="cuda")
    lengths = torch.tensor([rows // 2, rows // 2 - 2], dtype=torch.int32, device="cuda")
    want = lb.last_residual_norm(some, gain, keep=keep)
    got = lb.last_residual_norm(x.view(2, rows // 2, H), gain, lengths=lengths, keep=keep)
    for y, z in ((got.y, want.y),) if keep is None else zip(got.kept, want.kept):
        assert_repeats(y.view(rows, -1), z, 2)
    assert_repeats(got.inv.view(rows, 1), want.inv[:, None], 2)


def test_product_of_many_rows():
    """Tiles of 64 have a workgroup for 64 rows, and are what a product of one column would take."""
    rows, K = 1 << 30, 8
    announce("product of many rows", rows)
    x, some = by_column(rows, K)
    w = torch.randn(1, K, device="cuda").bfloat16()
    want = lb.last_product(some, w)[0]
    got = lb.last_product(x, w)[0]
    assert_repeats(got, want)


def test_operand_laid_out_in_many_pieces():
    """50 bytes a row, laid out at 64: four threads a row."""
    rows, K = 1 << 30, 25
    announce("operand laid out in many pieces", rows)
    if torch.cuda.get_device_properties(0).total_memory < 200 << 30:
        pytest.skip("needs 130 GB")
    x, some = by_column(rows, K)
    w = torch.randn(1, K, device="cuda").bfloat16()
    want = lb.last_product(some, w)[0]
    got = lb.last_product(x, w)[0]
    assert_repeats(got, want)
