"""Sizes of the paged cache's calls at and behind their limits (host side, no GPU)."""
import pytest

from paper_2605_31105_gb300 import binding as b
from tests.test_abi import lib  # noqa: F401  (builds the library if it is stale)


def size(units=8, group=4, pages=100, page=64, max_pages=32, **kw):
    return b.grkv_cache_workspace_size(b.cache_params(units, group, pages, page, max_pages, **kw))


# U g t of 2^64, 2^63 and 2^58 (the first two are 0 and negative in 64 bits), and just behind 2^28
@pytest.mark.parametrize("units,group,tokens", [
    (1 << 30, 64, 1 << 28), (1 << 29, 64, 1 << 28), (1 << 30, 1, 1 << 28), ((1 << 28) + 1, 1, 1),
    (1 << 23, 64, 1), (1, 64, (1 << 22) + 1)])
def test_rows_of_a_call_are_bounded(lib, units, group, tokens):  # noqa: F811
    with pytest.raises(b.GrkvError) as e:
        size(units=units, group=group, max_pages=1, tokens=tokens)
    assert e.value.code == -2


def test_the_largest_sizes_are_taken(lib):  # noqa: F811
    assert size(units=1 << 22, group=64, max_pages=1, tokens=1) > 0
    assert size(units=1, group=64, tokens=1 << 22) > 0
    assert size(units=1 << 28, group=1, max_pages=4, tokens=1) > 0


@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("f32", 0), ("bf16", b.GRKV_FORCE_SIMT)])
def test_a_workspace_serves_calls_of_fewer_tokens(lib, dtype, flags):  # noqa: F811
    """One sized for the longest draft or chunk is large enough for every shorter one."""
    for group in (1, 2, 3, 4, 5, 7, 8, 11, 16, 21, 32, 33, 64):
        sizes = [size(group=group, tokens=t, dtype=dtype, flags=flags) for t in range(1, 301)]
        assert sizes == sorted(sizes), group
