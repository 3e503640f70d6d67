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
    d, x = _descs(**PAGED)
    assert vs.vs_shared_prefix_workspace_bytes(d, x) == one
    assert _call(d, x, nbytes=one - 1) == -4
    import torch
    if not torch.cuda.is_available():
        assert _call(d, x, nbytes=one) == -7
