"""Host-side refusals of the paged cache's entry points (no GPU: they run before any CUDA call)."""
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests.test_abi import lib  # noqa: F401  (builds the library if it is stale)

FAKE = 1 << 20   # never dereferenced: every check below fails on the host


def params(**kw):
    return b.cache_params(8, 4, 100, 64, 32, **kw)


def test_defaults(lib):  # noqa: F811
    p = params()
    assert (p.units, p.group, p.d, p.pages, p.page, p.max_pages) == (8, 4, 128, 100, 64, 32)
    assert (p.tokens, p.window, p.n_sink, p.scale, p.dtype, p.flags) == (1, 0, 4, 0, b.GRKV_BF16, 0)
    assert params(dtype="f32").dtype == b.GRKV_F32


@pytest.mark.parametrize("kw,code", [
    (dict(units=-1), -1), (dict(group=0), -1), (dict(d=0), -1), (dict(pages=0), -1),
    (dict(page=0), -1), (dict(max_pages=0), -1), (dict(tokens=0), -1), (dict(window=-1), -1),
    (dict(n_sink=-1), -1), (dict(scale=-1.0), -1), (dict(scale=float("inf")), -1),
    (dict(scale=float("nan")), -1), (dict(dtype=5), -1), (dict(flags=b.GRKV_DETERMINISTIC), -1),
    (dict(d=64), -2), (dict(group=65), -2), (dict(page=48), -2), (dict(page=256), -2),
    (dict(max_pages=1 << 27), -2), (dict(pages=(1 << 30) + 1), -2), (dict(tokens=(1 << 28) + 1), -2),
    (dict(units=1 << 20, tokens=1 << 10), -2), (dict(units=1 << 26, max_pages=17), -2)])
def test_parameters(lib, kw, code):  # noqa: F811
    p = params()
    for key, val in kw.items():
        setattr(p, key, val)
    with pytest.raises(b.GrkvError) as e:
        b.grkv_cache_workspace_size(p)
    assert e.value.code == code


def calls(p, ws_bytes, at=None, over=FAKE, ws=FAKE):
    """Every entry point that has a pointer argument number `at`, with `over` there."""
    def f(n, distinct=()):
        args = [FAKE * 2 if i in distinct else FAKE for i in range(n)]
        if at is not None and at < n:
            args[at] = over
        return args
    kw = dict(ws_bytes=ws_bytes, stream=0, check=False)
    at = -1 if at is None else at
    return [fn(p, *f(n, distinct), ws, **kw, **extra) for fn, n, distinct, extra in (
        (b.grkv_attend, 6, (), {}), (b.grkv_attend_tree, 7, (), {}),
        (b.grkv_cache_reserve, 6, (), {}), (b.grkv_cache_trim, 3, (), {}),
        (b.grkv_cache_append, 6, (), {}), (b.grkv_cache_compact, 6, (), {}),
        (b.grkv_cache_fork, 6, (3, 4), dict(units_in=8))) if at < n]


def test_workspace_and_pointers(lib):  # noqa: F811
    p = params()
    need = b.grkv_cache_workspace_size(p)
    assert calls(p, need - 1) == [b.GRKV_ERR_WORKSPACE_TOO_SMALL] * 7
    assert calls(p, need, ws=0) == [b.GRKV_ERR_INVALID_ARG] * 7
    assert calls(p, need, ws=FAKE + 8) == [b.GRKV_ERR_MISALIGNED] * 7
    for at in range(7):
        for over, code in ((0, b.GRKV_ERR_INVALID_ARG), (FAKE + 2, b.GRKV_ERR_MISALIGNED)):
            got = calls(p, need, at, over)
            assert got and got == [code] * len(got), (at, over)


def test_fork_onto_itself_and_sizes(lib):  # noqa: F811
    p = params()
    need = b.grkv_cache_workspace_size(p)
    kw = dict(ws_bytes=need, stream=0, check=False)
    inv = b.GRKV_ERR_INVALID_ARG
    assert b.grkv_cache_fork(p, FAKE, FAKE, FAKE, FAKE, FAKE * 2, FAKE, FAKE, units_in=8, **kw) == inv
    assert b.grkv_cache_fork(p, FAKE, FAKE, FAKE, FAKE * 2, FAKE, FAKE, FAKE, units_in=8, **kw) == inv
    assert b.grkv_cache_fork(p, FAKE, FAKE, FAKE, FAKE * 2, FAKE * 3, FAKE, FAKE, units_in=-1,
                             **kw) == inv
    q = params(tokens=257)
    assert b.grkv_attend_tree(q, *[FAKE] * 7, FAKE, ws_bytes=b.grkv_cache_workspace_size(q),
                              stream=0, check=False) == b.GRKV_ERR_UNSUPPORTED
    q = b.cache_params(1, 1, 100, 128, 1 << 21, tokens=1 << 24)   # 2^16 items x 2^21 slot tiles
    assert b.grkv_attend(q, *[FAKE] * 7, ws_bytes=b.grkv_cache_workspace_size(q), stream=0,
                         check=False) == b.GRKV_ERR_UNSUPPORTED
    assert b.strerror(b.GRKV_ERR_NO_PAGES) == "too few free pages in the pool"


def test_workspace_does_not_depend_on_the_call(lib):  # noqa: F811
    small = b.grkv_cache_workspace_size(params())
    assert small > 0
    assert b.grkv_cache_workspace_size(b.cache_params(1, 1, 1 << 22, 16, 4)) >= 4 << 22
    assert b.grkv_cache_workspace_size(b.cache_params(0, 1, 1, 16, 1)) > 0


def test_tensors_are_checked_by_the_binding(lib):  # noqa: F811
    p = params()
    pool = torch.zeros(100, 64, 128, dtype=torch.bfloat16)
    q, out = torch.zeros(8, 4, 1, 128, dtype=torch.bfloat16), torch.zeros(8, 4, 1, 128, dtype=torch.bfloat16)
    table, lens = torch.zeros(8, 32, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)
    kw = dict(ws_bytes=b.grkv_cache_workspace_size(p), stream=0)

    def refused(word, *a, **k):
        with pytest.raises(ValueError, match=word):
            b.grkv_attend(p, *a, FAKE, **{**kw, **k})

    f = FAKE                       # the tensors that are not looked at
    refused("q is torch.float32", q.float(), f, f, f, f, f)
    refused("lens is torch.int64", f, f, f, f, lens.long(), f)
    refused("k_pages is not contiguous", f, pool.transpose(0, 1), f, f, f, f)
    refused("v_pages holds", f, f, pool[:99], f, f, f)
    refused("table holds", f, f, f, table[:7], f, f)
    refused("lse is torch.bfloat16", f, f, f, f, f, f, lse=out)
    refused("q is on cpu", q, f, f, f, f, f)
    assert b.load().grkv_cache_append(p, FAKE, FAKE, FAKE, -1, None, FAKE, FAKE, FAKE, FAKE, FAKE,
                                      kw["ws_bytes"], None) == b.GRKV_ERR_INVALID_ARG
    with pytest.raises(ValueError, match="not on the current CUDA device"):
        b.grkv_attend(p, q, pool, pool, table, lens, out, torch.zeros(kw["ws_bytes"], dtype=torch.uint8))
