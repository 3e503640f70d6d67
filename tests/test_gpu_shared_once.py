"""The halves of a call behind a shared prefix that load their keys as data that is read once, against the definition: eight waves and four, lengths that end
inside a tile and well before their bound, slots behind them that hold NaN, sizes on both sides of the rule."""
import ctypes

import pytest

import paper_2509_15235_amd as vs
from shared_util import Shared

pytestmark = pytest.mark.gpu


@pytest.fixture
def equal_splits():
    vs.lib().vs_internal_set_shared_way(3)
    yield
    vs.lib().vs_internal_set_shared_way(0)


@pytest.mark.parametrize("B,T,Hq,Hkv,P,own,kw,halves,which", [
    (2, 1, 32, 32, 8197, [4099, 3], dict(max_own=4100), 3, None),                            # eight waves
    (2, 1, 32, 32, 5777, [3905, 3800], dict(max_len=5860, max_own=3906), 3, None),           # the smallest of both
    (2, 1, 32, 32, 5777, [3905, 3800], dict(max_len=5859, max_own=3905), 0, None),           # one key less
    (9, 1, 32, 32, 5777, [870, 0, 3, 64, 31, 33, 500, 7, 899], dict(max_len=5900, max_own=900), 3, [0, 1, 4, 8]),  # 288 workgroups: four waves
    (3, 5, 32, 16, 11700, [5204, 1, 2047], dict(max_len=11720, mask=0), 3, [1, 2]),          # thirty rows, trees
    (4, 5, 32, 16, 64, [4100, 5, 2050, 0], {}, 2, [1, 2]),                                   # the own keys only
    (1, 1, 8, 8, 1, [32000], dict(max_own=32001), 2, None),
    (1, 1, 64, 32, 5901, [40], dict(token_major=1), 1, None),                                # heads of a token side by side
])
def test_read_once(B, T, Hq, Hkv, P, own, kw, halves, which, equal_splits):
    s = Shared(B, T, Hq, Hkv, 128, P, own, paged=0, **kw)
    assert vs.lib().vs_internal_shared_way(ctypes.byref(s.desc), ctypes.byref(s.pre)) == 3
    assert vs.lib().vs_internal_shared_reads_once(ctypes.byref(s.desc), ctypes.byref(s.pre)) == halves
    s.run()
    s.check(which)
