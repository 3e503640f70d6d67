"""A sequence's own keys behind a shared prefix in the pipelined kernel, which large batches of trees take: asked for by name, so that small calls reach it
too - both cache layouts and head sizes, masks given and derived, few and many parts of the shared keys, none at all, sequences that are reported."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2509_15235_amd as vs
from shared_util import Shared

pytestmark = pytest.mark.gpu


@pytest.fixture
def ask():
    lib = vs.lib()
    lib.vs_internal_set_shared_own(2)
    yield lib.vs_internal_set_shared_way
    lib.vs_internal_set_shared_own(0)
    lib.vs_internal_set_shared_way(0)


def _is(s, way):
    args = ctypes.byref(s.desc), ctypes.byref(s.pre)
    return vs.lib().vs_internal_shared_way(*args) == way and vs.lib().vs_internal_shared_own(*args) == 2


CALLS = [
    dict(B=3, T=60, Hq=14, Hkv=2, P=2500, own=[700, 0, 33]),                       # 420 rows: the last of four row groups is a ragged one
    dict(B=5, T=17, Hq=8, Hkv=2, P=449, own=[0, 1, 64, 200, 31], max_own=230),     # 68 rows
    dict(B=2, T=64, Hq=8, Hkv=8, P=64, own=[1000, 2], max_len=4000),               # 64 rows, one tile of a long bound
    dict(B=9, T=3, Hq=12, Hkv=4, P=1030, own=[0, 1, 70, 3, 200, 31, 32, 33, 90], max_len=1500),  # nine rows: three of four waves have none
    dict(B=2, T=33, Hq=4, Hkv=1, P=9000, own=[300, 17]),                           # many parts of a row
    dict(B=4, T=1, Hq=40, Hkv=1, P=700, own=[5000, 0, 63, 65]),                    # single tokens
]


@pytest.mark.parametrize("mask", [0, 1])
@pytest.mark.parametrize("paged", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", [3, 4, 5])
@pytest.mark.parametrize("call", range(len(CALLS)))
def test_against_definition(call, way, d, paged, mask, ask):
    ask(way)
    s = Shared(d=d, paged=paged, mask=mask, **CALLS[call])
    if not _is(s, way):
        pytest.skip("no way for this call")
    s.run()
    s.check()
    first = s.out.clone()
    s.ws.random_(0, 256)
    s.out.fill_(float("nan"))
    s.run()
    torch.cuda.synchronize()
    assert torch.equal(s.out, first)


@pytest.mark.parametrize("paged", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", [3, 4])
def test_reported_sequences_and_no_shared_keys(way, d, paged, ask):
    ask(way)
    s = Shared(6, 20, 8, 2, d, 500, [10, 20, 30, 40, 50, 60], max_own=64, paged=paged, mask=0)
    assert _is(s, way)
    s.lens[1], s.lens[4] = -3, 65
    s.parent_dev[2, 1], s.parent_dev[3, 0] = 7, 0
    for _ in range(2):
        s.out.fill_(float("nan"))
        s.run()
        s.check([0, 5])
        assert s.status.cpu().tolist() == [0, 3, 2, 1, 3, 0]
        assert torch.isnan(s.out[1:5].float()).all()  # nothing is written for them
    s.lens.copy_(torch.from_numpy(s.own))
    s.parent_dev.copy_(torch.from_numpy(s.parent))
    if paged:
        s.table[3, 1] = -1
        s.run()
        s.check([0, 1, 2, 4, 5])
        assert s.status.cpu().tolist() == [0, 0, 0, 4, 0, 0]
        s.table.copy_(torch.from_numpy(s.table_host))
        s.stable[2] = s.pre.num_blocks
        s.run()
        torch.cuda.synchronize()
        assert s.status.cpu().tolist() == [4] * 6
        s.stable.copy_(torch.from_numpy(s.stable_host))
    s.run()
    s.check()
    for bad in (-1, 501):
        s.shared_len.fill_(bad)
        s.run()
        torch.cuda.synchronize()
        assert s.status.cpu().tolist() == [3] * 6
    s.shared_len.fill_(0)
    s.P, s.ks, s.vs = 0, s.ks[:0], s.vs[:0]
    s.run()
    s.check()


@pytest.mark.parametrize("d", [64, 128])
def test_captured_with_other_lengths_between_replays(d, ask):
    ask(4)
    s = Shared(4, 30, 8, 2, d, 640, [100, 3, 0, 64])
    assert _is(s, 4)
    s.run()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        s.run(stream.cuda_stream)
    for P in (640, 65, 300):
        s.P, s.shared_len[0] = P, P
        keep = s.ks, s.vs
        s.ks, s.vs = s.ks[:P], s.vs[:P]
        s.ws.random_(0, 256)
        s.out.fill_(float("nan"))
        graph.replay()
        s.check()
        s.ks, s.vs = keep
        s.run()  # an eager call on the same workspace between the replays


def test_large_trees_take_it_without_being_asked():
    """Both layouts of a call that the rule gives it to, masks derived: some of its sequences."""
    for paged in (0, 1):
        for d in (64, 128):
            s = Shared(40, 33, 16, 4, d, 200, [(17 * i) % 120 for i in range(40)], paged=paged, mask=0)
            assert vs.lib().vs_internal_shared_own(ctypes.byref(s.desc), ctypes.byref(s.pre)) == (2 if 40 * 4 * 5 > 1024 else 1)
            t = Shared(60, 33, 16, 4, d, 200, [(17 * i) % 120 for i in range(60)], paged=paged, mask=0)
            assert vs.lib().vs_internal_shared_own(ctypes.byref(t.desc), ctypes.byref(t.pre)) == 2
            for x in (s, t):
                x.run()
                x.check([0, 7, x.B - 1])
                assert (x.status.cpu().numpy() == np.int32(0)).all()
