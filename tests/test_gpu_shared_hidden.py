"""vs_shared_prefix_attention where a mask word shows a node nothing (what vs_tree_mask_build leaves for an invalid tree) and the sequence has no
keys of its own in front of it: the row is what the shared keys make it, and zeros where there are none either. Every way of a call, both types."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2509_15235_amd as vs
from shared_util import Shared

pytestmark = pytest.mark.gpu


@pytest.fixture
def ask():
    yield vs.lib().vs_internal_set_shared_way
    vs.lib().vs_internal_set_shared_way(0)


def _hide(s, rows):
    """Mask words of (sequence, node)s become zero."""
    for b, i in rows:
        s.mask_host[b, i] = 0
    s.mask_dev.copy_(torch.from_numpy(s.mask_host.view(np.int64)))


def _check(s, rows, which):
    """Against the definition; without shared keys, rows that see nothing are zeros."""
    blank = [(b, i) for b, i in rows if s.P == 0 and s.own[b] == 0]
    s.run()
    torch.cuda.synchronize()
    assert (s.status.cpu() == 0).all()
    for b, i in blank:
        assert (s.out[b, i] == 0).all(), (b, i, s.out[b, i].flatten()[:4].tolist())
    for b, i in blank:  # the others: as if the word showed the node itself, whose row is not looked at
        s.mask_host[b, i] = np.uint64(1) << np.uint64(i)
        s.out[b, i] = torch.from_numpy(s.want(b)[0][i]).to(s.dt)
    s.check(which)


WAYS = [(1, 1), (1, 2), (1, 3), (1, 4), (1, 5), (0, 3)]  # bf16 or fp32, way


@pytest.mark.parametrize("P", [0, 1, 500])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bf16,way", WAYS)
def test_rows_that_see_none_of_their_own_keys(bf16, way, d, P, ask):
    ask(way)
    s = Shared(7, 3, 8, 2, d, P, [0, 10, 0, 0, 33, 0, 0], bf16=bf16, max_len=500)
    assert vs.lib().vs_internal_shared_way(ctypes.byref(s.desc), ctypes.byref(s.pre)) == way
    rows = [(0, 0), (0, 1), (0, 2), (1, 1), (2, 1), (4, 0), (4, 1), (4, 2), (6, 2)]  # whole sequences, single nodes, with own keys and without
    _hide(s, rows)
    _check(s, rows, range(7))


@pytest.mark.parametrize("P", [0, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_the_same_behind_the_pipelined_own_keys(d, P):
    """Many sequences of many rows: 48 * 8 * 3 row blocks of own keys."""
    s = Shared(48, 24, 32, 8, d, P, [13 * i % 70 if i % 3 else 0 for i in range(48)], max_len=300)
    rows = [(0, i) for i in range(24)] + [(1, 0), (3, 5), (3, 23), (47, 11)]
    _hide(s, rows)
    _check(s, rows, [0, 1, 3, 47])


def test_an_invalid_tree_of_a_batch():
    """Masks as vs_tree_mask_build makes them: of a tree that it reports, every word is zero."""
    for bf16 in (1, 0):
        s = Shared(3, 4, 8, 2, 64, 100, [0, 0, 20], bf16=bf16)
        s.parent_dev[0, 2] = 3
        depth = torch.empty((3, 4), device="cuda", dtype=torch.int32)
        status = torch.empty((3,), device="cuda", dtype=torch.int32)
        assert vs.vs_tree_mask_build(s.parent_dev, 3, 4, s.mask_dev, depth, status, torch.cuda.current_stream().cuda_stream) == 0
        assert status.cpu().tolist() == [2, 0, 0]
        s.mask_host[0] = 0
        assert torch.equal(s.mask_dev.cpu(), torch.from_numpy(s.mask_host.view(np.int64)))
        s.run()
        s.check(range(3))
