"""vs_shared_prefix_attention on values near the smallest that bf16 holds as a normal number: the parts that calls keep between their two halves are as accurate
there as anywhere."""
import ctypes

import pytest
import torch

import paper_2509_15235_amd as vs
from shared_util import Shared

pytestmark = pytest.mark.gpu


@pytest.fixture
def ask():
    yield vs.lib().vs_internal_set_shared_way
    vs.lib().vs_internal_set_shared_way(0)


@pytest.mark.parametrize("exp2", [-110, -116, -118, -120])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", [1, 2, 3, 4, 5])
def test_tiny_values(way, d, exp2, ask):
    ask(way)
    s = Shared(24, 4, 8, 4, d, 500, [(13 * i) % 70 for i in range(24)], v_scale=2.0 ** exp2, q_scale=0.5)
    if vs.lib().vs_internal_shared_way(ctypes.byref(s.desc), ctypes.byref(s.pre)) != way:
        pytest.skip("no way for this call")
    s.run()
    s.check()


@pytest.mark.parametrize("way", [3, 4, 5])
def test_tiny_and_ordinary_channels(way, ask):
    """A channel of ordinary size beside tiny ones: the piece is kept as bf16, one more rounding."""
    ask(way)
    factor = torch.full((128,), 2.0 ** -118)
    factor[37] = 1.0
    s = Shared(24, 4, 8, 4, 128, 500, [(13 * i) % 70 for i in range(24)], v_scale=factor, q_scale=0.5)
    if vs.lib().vs_internal_shared_way(ctypes.byref(s.desc), ctypes.byref(s.pre)) != way:
        pytest.skip("no way for this call")
    s.run()
    s.check(wide=1)
