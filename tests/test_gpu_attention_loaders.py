"""Attention of bf16 rows over pages where one of the two warps that copy K and V ends before the other: what is lost is NaN and told, what is not is right, the next call too."""
import numpy as np
import pytest
import torch

from test_gpu_attention_values import _stopped
from test_gpu_paged_attention import Paged, _check
from test_gpu_tree_attention import Trees, _parents, _wider, kb  # noqa: F401

pytestmark = pytest.mark.gpu


def _calls(kb, tree, lens, fresh, KV, hd, page):  # noqa: F811
    if not tree:
        p = Paged(71, lens, fresh, KV, hd, page, "bf16")
        return p, p.q(2 * KV, hd, "bf16")
    rng = np.random.default_rng(len(lens))
    p = Trees(kb, 71, lens, [_parents(rng, min(n, 64), 4) for n in fresh], KV, hd, page, "bf16")
    p.table = _wider(p.table, 5000 // page)                          # room for more than the short way takes
    return p, p.q(2 * KV, hd, "bf16")


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens,fresh,KV", [([700], [3], 1), ([30000, 40], [2, 140], 2), ([200] * 90, [1] * 45 + [90] * 45, 4)])
def test_one_copying_warp_ends_before_the_other(kb, tree, page, hd, lens, fresh, KV):  # noqa: F811
    p, q = _calls(kb, tree, lens, fresh, KV, hd, page)
    want, tol = p.want(q)
    kb.knnssd_attention_status()
    for only in (kb.KNNSSD_DEBUG_ONLY_FIRST, kb.KNNSSD_DEBUG_ONLY_SECOND, 0):
        for tiles in (0, 1, 2, 3, 4, 7):
            if only == 0 and tiles > 1:
                continue
            kb.knnssd_debug_attention_timeout(0)
            try:
                got = _stopped(kb, lambda: p.run(kb, q), tiles | only)
            except pytest.fail.Exception:
                assert tiles > 3                                     # no block has that many tiles: nothing was lost
                _check(p.run(kb, q), want, tol, "nothing lost")
                continue
            lost = got.isnan().any(2)
            assert got[lost].isnan().all() and (tiles > 0 or lost.all()) and lost.any()
            _check(got[~lost], want[~lost], tol[~lost], f"rows that were not lost, {tiles} tiles")
            _check(p.run(kb, q), want, tol, "the call behind it")
            kb.knnssd_attention_status()
