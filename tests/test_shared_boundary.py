"""Refusals of vs_shared_prefix_attention and its workspace: found on the host, without a GPU."""
import pytest

import paper_2509_15235_amd as vs

G = 1 << 20


def _descs(**kw):
    d = vs.AttnDesc(B=8, T=4, Hq=28, Hkv=4, d=128, dtype=vs.VS_BF16, softmax_scale=0.1, max_prefix_len=100, capacity=200, stride_seq=4 * 200 * 128,
                    stride_head=200 * 128, stride_tok=128)
    x = vs.PrefixDesc(max_len=1696, capacity=1700, stride_head=1700 * 128, stride_tok=128)
    for k, v in kw.items():
        setattr(x if k.startswith("x_") else d, k.removeprefix("x_"), v)
    return d, x


def _call(d, x, q=G, ks=G, vs_=G, n=G, k=G, v=G, lens=G, parent=G, mask=None, out=G, status=None, ws=G, nbytes=1 << 40):
    return vs.vs_shared_prefix_attention(d, x, q, ks, vs_, n, k, v, lens, parent, mask, out, status, ws, nbytes, None)


PAGED = dict(x_paged=1, x_block_size=16, x_max_blocks=106, x_num_blocks=300, x_stride_block=4 * 16 * 128, x_stride_head=16 * 128, x_block_table=G)


@pytest.mark.parametrize("kw,code", [
    ({"B": 0}, -2), ({"T": 65}, -2), ({"T": 0}, -2), ({"Hq": 30}, -2), ({"d": 96}, -2), ({"dtype": 5}, -3), ({"softmax_scale": 0.0}, -2),
    ({"impl": vs.VS_IMPL_MFMA}, -2), ({"num_splits": 2}, -2), ({"rows_per_wave": 1}, -2), ({"waves_per_group": 8}, -2), ({"schedule": vs.VS_SCHED_LOOP}, -2),
    ({"capacity": 103}, -6), ({"stride_tok": 132}, -6), ({"x_max_len": 0}, -2), ({"x_max_len": -5}, -2), ({"x_capacity": 1695}, -6), ({"x_capacity": 0}, -6),
    ({"x_stride_tok": 120}, -6), ({"x_stride_tok": 132}, -6), ({"x_stride_head": -8}, -6), ({"x_stride_tok": 1 << 30}, -6),
    (dict(PAGED, x_max_len=(1 << 30) + 1, x_max_blocks=1 << 27), -2),
    (dict(paged=1, block_size=16, max_blocks=1 << 27, num_blocks=9, stride_block=8192, stride_head=2048, block_table=G, max_prefix_len=(1 << 30) + 1), -2),
    (dict(PAGED, x_block_size=24), -6), (dict(PAGED, x_max_blocks=105), -6), (dict(PAGED, x_block_table=None), -1), (dict(PAGED, x_num_blocks=0), -6),
    (dict(PAGED, x_stride_block=4 * 16 * 128 + 4), -6), ({"B": 16384, "T": 64, "Hq": 8, "Hkv": 2, "stride_seq": 0}, -2),
])
def test_descriptors(kw, code):
    d, x = _descs(**kw)
    assert vs.vs_shared_prefix_workspace_bytes(d, x) == 0
    assert _call(d, x) == code


@pytest.mark.parametrize("kw,code", [
    ({"q": None}, -1), ({"ks": None}, -1), ({"vs_": None}, -1), ({"n": None}, -1), ({"k": None}, -1), ({"v": None}, -1), ({"lens": None}, -1),
    ({"parent": None}, -1), ({"out": None}, -1), ({"q": G + 8}, -6), ({"ks": G + 2}, -6), ({"vs_": G + 8}, -6), ({"k": G + 8}, -6), ({"v": G + 8}, -6),
    ({"out": G + 8}, -6), ({"ws": None}, -4), ({"ws": G + 128}, -4), ({"nbytes": 100}, -4),
])
def test_arguments(kw, code):
    assert _call(*_descs(), **kw) == code


def test_workspace_covers_the_rows_and_grows_with_them():
    d, x = _descs()
    one = vs.vs_shared_prefix_workspace_bytes(d, x)
    assert one % 256 == 0 and one >= 8 * 4 * 28 * 130 * 4  # a row's sums and its pair, at least once
    d, x = _descs(B=64)
    assert vs.vs_shared_prefix_workspace_bytes(d, x) >= one
    both = dict(paged=1, block_size=16, max_blocks=13, num_blocks=300, stride_block=4 * 16 * 128, block_table=G)
    d, x = _descs(**dict(PAGED, stride_head=16 * 128, **both))
    assert vs.vs_shared_prefix_workspace_bytes(d, x) == one  # both caches paged, or neither: the same way
    d, x = _descs()
    assert _call(d, x, nbytes=one - 1) == -4
    import torch
    if not torch.cuda.is_available():
        assert _call(d, x, nbytes=one) == -7


def _way(**kw):
    import ctypes
    return vs.lib().vs_internal_shared_way(*[ctypes.byref(x) for x in _descs(**kw)])


def test_sizes_from_the_smallest_to_the_largest_have_a_plan_and_a_workspace():
    big = dict(capacity=1 << 20, stride_tok=1024, stride_head=128, stride_seq=1 << 30, x_capacity=1 << 19, x_stride_tok=1024, x_stride_head=128)
    seen = set()
    for dtype in (vs.VS_BF16, vs.VS_F32):
        for B in (1, 2, 16, 64, 300, 8192):
            for T in (1, 4, 17, 64):
                for Hq, Hkv in ((28, 4), (32, 32), (8, 1), (64, 1)):
                    for d in (64, 128):
                        for P in (1, 63, 700, 9000, 1 << 19):
                            if B * T * Hq // Hkv > 1 << 20 or B * Hkv > 65535:
                                continue
                            kw = dict(B=B, T=T, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, x_max_len=P, max_prefix_len=min(P, 4000), **big)
                            way = _way(**kw)
                            assert 1 <= way <= 5 and (dtype == vs.VS_BF16 or way == 3), (kw, way)
                            seen.add(way)
                            need = vs.vs_shared_prefix_workspace_bytes(*_descs(**kw))
                            rows = B * T * (Hq // Hkv)
                            # a place for every row at least, and no more than one for every CU and one more, and the words
                            assert rows * Hkv * d * 2 <= need <= (rows + 31) * Hkv * 257 * (d * 4 + 16) + B * Hkv * 128 + 1024, (kw, need)
    assert seen == {1, 2, 3, 4, 5}


def test_a_way_that_is_asked_for():
    lib = vs.lib()
    try:
        for way in (1, 2, 3, 4, 5):
            lib.vs_internal_set_shared_way(way)
            assert _way() == way
        lib.vs_internal_set_shared_way(1)
        assert _way(T=20) != 1 and _way(dtype=vs.VS_F32) == 3 and _way(**PAGED) != 1  # too many rows of a sequence; not for the type; caches of two kinds
    finally:
        lib.vs_internal_set_shared_way(0)
