"""Which halves of a call behind a shared prefix load their keys as data that is read once: large contiguous caches, one row block of queries. No GPU."""
import ctypes

import pytest

import paper_2509_15235_amd as vs

G = 1 << 20


@pytest.fixture(autouse=True)
def equal_splits():
    vs.lib().vs_internal_set_shared_way(3)
    yield
    vs.lib().vs_internal_set_shared_way(0)


def _halves(P, own, B=2, T=1, Hq=32, Hkv=32, d=128, **kw):
    desc = vs.AttnDesc(B=B, T=T, Hq=Hq, Hkv=Hkv, d=d, dtype=vs.VS_BF16, softmax_scale=0.1, max_prefix_len=own, capacity=own + T,
                       stride_seq=Hkv * (own + T) * d, stride_head=(own + T) * d, stride_tok=d)
    pre = vs.PrefixDesc(max_len=P, capacity=P, stride_head=P * d, stride_tok=d)
    for k, v in kw.items():
        setattr(pre if k.startswith("x_") else desc, k.removeprefix("x_"), v)
    return vs.lib().vs_internal_shared_reads_once(ctypes.byref(desc), ctypes.byref(pre))


@pytest.mark.parametrize("P,own,kw,want", [
    (5860, 10, {}, 1), (5859, 10, {}, 0), (10, 3906, {}, 2), (10, 3905, {}, 0), (5860, 3906, {}, 3),   # 32 heads, K and V: 96 and 128 MB
    (5860, 868, dict(B=9), 3), (5860, 867, dict(B=9), 1),
    (5860, 3906, dict(dtype=vs.VS_F32, stride_tok=128), 0), (5860, 3906, dict(d=64), 0), (11719, 5206, dict(d=64, B=3), 0),
    (11720, 5204, dict(B=3, T=5, Hq=32, Hkv=16), 3), (11720, 5203, dict(B=3, T=5, Hq=32, Hkv=16), 1), (11720, 5203, dict(B=4, T=5, Hq=32, Hkv=16), 2),  # forty rows of a head: two row blocks
    (5860, 3906, dict(x_stride_head=0), 2), (5860, 3906, dict(stride_seq=0), 1),                       # rows of two heads, of two sequences in one place
    (5860, 3906, dict(x_max_len=0), -2),
])
def test_halves(P, own, kw, want):
    assert _halves(P, own, **kw) == want


def test_other_ways_and_paged_caches_never_do():
    paged = dict(paged=1, block_size=16, max_blocks=400, num_blocks=9, stride_block=32 * 16 * 128, stride_head=16 * 128, block_table=G)
    assert _halves(5860, 3906, **paged) == 1
    assert _halves(5860, 3906, **{"x_" + k: v for k, v in paged.items()}) == 2
    for way in (1, 2, 4, 5):
        vs.lib().vs_internal_set_shared_way(way)
        assert _halves(5860, 3906, B=4, T=3, Hq=96) == 0
