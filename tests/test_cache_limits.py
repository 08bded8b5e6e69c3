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


class _OnDevice:
    """What the binding asks of a tensor, on a device of a machine that has two."""

    def __init__(self, device, dtype, n=1 << 20):
        import torch
        self.at, self.dtype, self.n = device, dtype, n
        self.device = torch.device("cuda", device)

    get_device = lambda self: self.at
    numel = lambda self: self.n
    is_contiguous = lambda self: True
    data_ptr = lambda self: 1 << 20
    element_size = lambda self: 1


@pytest.mark.parametrize("ws_is_tensor", [True, False])
def test_tensors_of_another_device_are_refused(lib, monkeypatch, ws_is_tensor):  # noqa: F811
    """With the workspace given as a tensor, and as an address."""
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    p = b.cache_params(2, 4, 8, 64, 4)
    ws = _OnDevice(0, torch.uint8, 1 << 30) if ws_is_tensor else 1 << 20
    x, i = (lambda d: _OnDevice(d, torch.bfloat16)), (lambda d: _OnDevice(d, torch.int32))
    # a workspace that is too small ends the calls that the binding lets through, on the host
    kw = dict(ws_bytes=1, stream=0)
    with pytest.raises(b.GrkvError):
        b.grkv_attend(p, x(0), x(0), x(0), i(0), i(0), x(0), ws, **kw)
    for at in range(6):
        d = [0] * 6
        d[at] = 1
        with pytest.raises(ValueError, match="on cuda:1, the call runs on device 0"):
            b.grkv_attend(p, x(d[0]), x(d[1]), x(d[2]), i(d[3]), i(d[4]), x(d[5]), ws, **kw)
    with pytest.raises(ValueError, match="refs is on cuda:1"):
        b.grkv_cache_trim(p, i(0), i(0), i(1), ws, **kw)


def test_packed_rows_at_an_address_need_their_number(lib, monkeypatch):  # noqa: F811
    """The library bounds first_row by new_rows: a number that is not known is not made up."""
    import ctypes

    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    seen = []

    class Lib:
        def grkv_cache_append(self, *a):
            seen.append(ctypes.c_int64(a[4]).value)
            return b.GRKV_OK

    p = b.cache_params(2, 4, 8, 64, 4, tokens=100)
    monkeypatch.setattr(b, "load", lambda: Lib())
    f, kw = 1 << 20, dict(ws_bytes=1, stream=0, first_row=1 << 20)
    rows = lambda n: _OnDevice(0, torch.bfloat16, n * 128)
    for k, v in ((f, f), (rows(70), f), (f, rows(70))):
        with pytest.raises(ValueError, match="new_rows"):
            b.grkv_cache_append(p, k, v, f, f, f, f, f, **kw)
        b.grkv_cache_append(p, k, v, f, f, f, f, f, new_rows=64, **kw)
    b.grkv_cache_append(p, rows(70), rows(71), f, f, f, f, f, **kw)
    with pytest.raises(ValueError, match="v_new holds"):
        b.grkv_cache_append(p, rows(70), rows(50), f, f, f, f, f, new_rows=64, **kw)
    assert seen == [64, 64, 64, 70]
