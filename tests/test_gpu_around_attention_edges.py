"""Calls around the attention that the documentation allows and that are far from the usual ones: the most rows behind a shared prefix, a very long prefix,
keys and values side by side in one pool, one row rotated for all rows and heads."""
import ctypes

import numpy as np
import pytest
import torch

import gpu_util as gu
import paper_2509_15235_amd as vs
import rope_util as ru
from shared_util import Shared
from test_gpu_append import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [1, 0])
def test_the_most_rows_behind_a_shared_prefix(bf16):
    """2^20 rows of one KV head: 16384 sequences of four nodes and sixteen heads."""
    B = 16384
    s = Shared(B, 4, 16, 1, 64, 70, np.arange(B) % 5, bf16=bf16, max_len=100, mask=0)
    s.desc.B = B + 1
    assert vs.vs_shared_prefix_workspace_bytes(s.desc, s.pre) == 0  # one sequence more is refused
    s.desc.B = B
    s.run()
    s.check([0, 1, 2, 3, 4, 8191, 8192, 12345, B - 2, B - 1])
    assert (s.status == 0).all() and torch.isfinite(s.out).all()


@pytest.mark.parametrize("way", [1, 2, 3, 4, 5])
def test_a_very_long_prefix(way):
    """Three hundred thousand shared tokens, a bound of a million."""
    try:
        vs.lib().vs_internal_set_shared_way(way)
        s = Shared(3, 1, 11, 1, 64, 300003, [5, 0, 700], max_len=1 << 20, q_scale=1.0)
        assert vs.lib().vs_internal_shared_way(ctypes.byref(s.desc), ctypes.byref(s.pre)) == way
        s.run()
        s.check()
    finally:
        vs.lib().vs_internal_set_shared_way(0)


@pytest.mark.parametrize("bf16", [1, 0])
def test_keys_and_values_side_by_side_in_one_pool(bf16):
    """A pool of blocks that hold keys and values: the append fills it, the attention behind a shared prefix reads it."""
    s = Setup([7, 30, 0, 64], [20, 0, 9, 3], Hq=8, Hkv=2, d=64, bf16=bf16, axes=[16, 8, 8], explicit=1)
    n, Hkv, bs, d = s.k.shape
    pool = torch.empty((n, 2, Hkv, bs, d), device="cuda", dtype=s.dt)
    pool[:, 0], pool[:, 1] = s.k, s.v
    s.k, s.v = pool[:, 0], pool[:, 1]
    s.desc.stride_block = s.k.stride(0)
    s.run()
    s.check()
    x = Shared(3, 4, 8, 2, 64, 200, [20, 3, 41], bf16=bf16)
    both = torch.stack([x.k, x.v], dim=1).contiguous()
    x.k, x.v = both[:, 0], both[:, 1]
    x.k_sh, x.v_sh = x.k, x.v
    x.desc.stride_block = x.pre.stride_block = x.k.stride(0)
    x.run()
    x.check()


@pytest.mark.parametrize("bf16", [1, 0])
def test_one_row_for_all_rows_and_heads(bf16):
    """Strides of zero read one row everywhere; its gradient is the sum of the rotations back, which the caller takes."""
    rows, H, d = 50, 4, 64
    dt = torch.bfloat16 if bf16 else torch.float32
    x = torch.randn((1, 1, d), generator=torch.Generator().manual_seed(2)).to(dt).cuda()
    pos = np.arange(rows, dtype=np.int32)[None] * 3
    freq = gu.dev(ru.frequencies(d))
    out, p = torch.empty((rows, H, d), device="cuda", dtype=dt), gu.dev(pos)
    rc = vs.vs_rope_apply(ru.rope_desc(d, inv_freq=freq.data_ptr()), x, 0, 0, p, rows, H, d, vs.VS_BF16 if bf16 else vs.VS_F32, out, H * d, d, gu.stream_ptr())
    assert rc == 0
    torch.cuda.synchronize()
    host = np.broadcast_to(x.float().cpu().numpy(), (rows, H, d))
    cos, sin = ru.cos_sin(pos, ru.frequencies(d), ru.axis_of_pair(d // 2, [d // 2], False))
    want = ru.rotate(host, cos, sin, d, True)
    assert (np.abs(out.float().cpu().numpy() - want) <= ru.bound(host, want, d, True, bf16)).all()
