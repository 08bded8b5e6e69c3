"""README.md's example runs as it stands, and leaves each key where its comments say."""
import os
import re

import numpy as np
import pytest

from tests import rope_ref
from tests.conftest import ROOT

pytestmark = pytest.mark.gpu


def test_the_example(grkv_lib):
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    env = {}
    exec("\n".join(blocks[:2]), env)
    first = env["k_new"].clone()                 # appended as it is, behind the compressed keys
    exec("\n".join(blocks[2:]), env)
    U, n, B, page = (env[x] for x in ("U", "n", "B", "page"))
    kw = dict(scaling="bands", theta=500000.0, factor=8.0)
    count = int(env["now"][0])
    assert (env["now"] == count).all() and count == env["kept"].shape[1]
    # Every key lies as a key of its position rotated for its slot: what it was turned by is the slot minus the
    # position.  One rounding each; the last token's key was rounded where it was appended, too: half a step
    # (2^-8) of each of a pair, turned.
    for u in (0, 7, U - 1):
        at = env["table"][u].cpu().numpy()[np.arange(count) // page] * page + np.arange(count) % page
        got = env["k_pages"].view(-1, 128).double().cpu().numpy()[at]
        kept = env["kept"][u].cpu().numpy()
        before = np.concatenate([env["k_out"][u].double().cpu().numpy(), first[u].double().cpu().numpy(),
                                 env["k_new"][u].double().cpu().numpy()])[kept]
        pos = np.concatenate([env["idx"][u].cpu().numpy(), [n, 0]])[kept]
        assert kept[-1] == B + 1
        want, err = rope_ref.rotate(before, np.arange(count) - pos, dtype="bf16", **kw)
        i, j = rope_ref.pairs(128, "half")
        both = np.abs(before[-1, i]) + np.abs(before[-1, j])
        err[-1, i] += 2.0 ** -8 * both + err[-1, i]
        err[-1, j] += 2.0 ** -8 * both + err[-1, j]
        rope_ref.check(got, want, err, "bf16")
