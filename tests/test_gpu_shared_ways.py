"""Every way in which vs_shared_prefix_attention works on the shared keys, asked for by name, on calls that are edges for it: sequences whose rows lie in
several row blocks, more sequences than lanes, parts of one tile, prefixes shorter than their bound, one workspace for different ways."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2509_15235_amd as vs
from shared_util import Shared

pytestmark = pytest.mark.gpu
WAYS = {1: "both, eight waves", 2: "both, four waves", 3: "equal splits", 4: "one line of shares", 5: "shares of every row group"}


@pytest.fixture
def ask():
    yield vs.lib().vs_internal_set_shared_way
    vs.lib().vs_internal_set_shared_way(0)


def _is(s, way):
    return vs.lib().vs_internal_shared_way(ctypes.byref(s.desc), ctypes.byref(s.pre)) == way


CALLS = [
    dict(B=1, T=1, Hq=1, Hkv=1, d=64, P=1, own=[0]),
    dict(B=11, T=3, Hq=12, Hkv=4, d=128, P=1030, own=[0, 1, 70, 3, 200, 31, 32, 33, 64, 5, 90], max_len=1500),     # nine rows a sequence: across row blocks
    dict(B=5, T=4, Hq=16, Hkv=2, d=64, P=777, own=[10, 0, 257, 64, 63], paged=0),                                   # 32 rows a sequence
    dict(B=70, T=1, Hq=2, Hkv=2, d=128, P=449, own=[(7 * i) % 50 for i in range(70)], block=64),
    dict(B=40, T=1, Hq=5, Hkv=1, d=64, P=3000, own=[(11 * i) % 90 for i in range(40)], token_major=1, mask=0),
    dict(B=3, T=7, Hq=28, Hkv=4, d=128, P=64, own=[300, 2, 0], max_len=4000),                                       # one tile of a long bound
    dict(B=2, T=1, Hq=8, Hkv=8, d=128, P=5000, own=[1000, 17]),
    dict(B=6, T=11, Hq=14, Hkv=2, d=128, P=2500, own=[0, 40, 333, 16, 15, 100]),                                    # 77 rows a sequence
    dict(B=9, T=30, Hq=8, Hkv=1, d=64, P=1111, own=[3 * i for i in range(9)], block=32),
]


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("call", range(len(CALLS)))
def test_every_way(call, way, ask):
    ask(way)
    s = Shared(**CALLS[call])
    if not _is(s, way):
        pytest.skip("no way for this call")
    s.run()
    s.check()
    first = s.out.clone()
    for _ in range(3):  # whoever comes last: the same result, from a workspace in which anything lies
        s.ws.random_(0, 256)
        s.out.fill_(float("nan"))
        s.run()
        s.run()
    torch.cuda.synchronize()
    assert torch.equal(s.out, first)


@pytest.mark.parametrize("way", [1, 2])
def test_no_shared_keys_and_bad_sequences_in_one_launch(way, ask):
    """Workgroups of sequences that are reported still let the others finish; without shared keys the own rows are all there is."""
    ask(way)
    s = Shared(6, 3, 8, 2, 64, 500, [10, 20, 30, 40, 50, 60], max_own=64)
    assert _is(s, way)
    s.mask_dev = None
    s.lens[1], s.lens[4] = -3, 65
    s.parent_dev[2, 1] = 7
    for _ in range(2):
        s.out.fill_(float("nan"))
        s.run()
        s.check([0, 3, 5])
        assert s.status.cpu().tolist() == [0, 3, 2, 0, 3, 0]
    s.lens.copy_(torch.from_numpy(s.own))
    s.parent_dev.copy_(torch.from_numpy(s.parent))
    s.run()  # the words are at rest
    s.check()
    s.shared_len.fill_(0)
    s.P, s.ks, s.vs = 0, s.ks[:0], s.vs[:0]
    s.run()
    s.check()
    s.shared_len.fill_(-1)
    s.run()
    torch.cuda.synchronize()
    assert s.status.cpu().tolist() == [3] * 6


def test_ways_take_turns_on_one_workspace_and_in_one_graph(ask):
    calls = []
    for way in (1, 4, 2, 3, 5, 1):
        ask(way)
        s = Shared(5, 4, 8, 2, 128, 600, [5, 0, 70, 33, 16], seed=way, max_len=640)
        assert _is(s, way)
        calls.append((way, s))
    ws = torch.randint(0, 256, (max(s.ws_bytes for _, s in calls),), device="cuda", dtype=torch.uint8)
    for _, s in calls:
        s.ws = ws
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def all_of_them(stream=None):
        for way, s in calls:
            ask(way)
            s.run(stream)
    all_of_them()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        all_of_them(stream.cuda_stream)
    for _ in range(3):
        ws.random_(0, 256)
        for _, s in calls:
            s.out.fill_(float("nan"))
            s.status.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        for _, s in calls:
            s.check()
        all_of_them()


def test_two_streams_at_once():
    """Two calls with workspaces of their own on two streams, several times."""
    a, b = Shared(8, 1, 28, 4, 128, 2000, [9 * i for i in range(8)]), Shared(12, 2, 8, 8, 64, 900, [5 * i for i in range(12)], seed=1)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        a.run(streams[0].cuda_stream)
        b.run(streams[1].cuda_stream)
    a.check()
    b.check()


def test_blocks_beyond_32_bits_of_a_pool():
    """A pool of blocks a gigabyte apart: offsets of the last ones pass 2^32 elements."""
    n, Hkv, d, bs = 5, 2, 64, 16
    gap = (1 << 30) + 2048
    pool = [torch.empty(gap * (n - 1) + Hkv * bs * d, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    s = Shared(2, 3, 4, Hkv, d, 20, [9, 5])
    old = s.table_host.reshape(-1).tolist() + s.stable_host.tolist()
    assert len(old) == 4
    names = {o: n - 1 - i for i, o in enumerate(old)}  # the shared blocks' ids 2 and 1, the own ones' 4 and 3
    for src, dst, name in ((s.k, pool[0], "k"), (s.v, pool[1], "v")):
        for o, i in names.items():
            dst[i * gap:i * gap + Hkv * bs * d] = src[o].reshape(-1)
        view = dst.as_strided((n, Hkv, bs, d), (gap, bs * d, d, 1))
        setattr(s, name, view)
        setattr(s, name + "_sh", view)
    s.table.copy_(torch.tensor([[names[int(x)] for x in row] for row in s.table_host], dtype=torch.int32))
    s.stable.copy_(torch.tensor([names[int(x)] for x in s.stable_host], dtype=torch.int32))
    s.desc.num_blocks = s.pre.num_blocks = n
    s.desc.stride_block = s.pre.stride_block = gap
    assert gap * 4 > 1 << 32
    s.run()
    s.check()


def test_large_contiguous_caches_of_one_row_block():
    """Over 128 MB of shared keys and of own ones, read past the caches: two sequences of 32 heads, a length that ends inside a tile."""
    s = Shared(2, 1, 32, 32, 128, 8197, [4099, 3], paged=0, max_own=4100)
    s.run()
    s.check()
    assert s.k.numel() * 4 > 128e6 and s.k_sh.numel() * 4 > 96e6


@pytest.mark.parametrize("way", [1, 2, 3, 4, 5])
def test_infinite_values_stay_in_their_channel(way, ask):
    """A shared and an own value that is infinite: that channel of whoever sees it is, and its neighbours are what they are otherwise."""
    ask(way)
    s = Shared(12, 4, 8, 2, 128, 500, [40] * 12, q_scale=0.5, mask=1)
    assert _is(s, way) or way < 3
    if not _is(s, way):
        pytest.skip("no way for this call")
    inf = float("inf")
    slot = 130  # a shared one; channel 21 of KV head 0
    s.vs[slot, 0, 21] = inf
    s.v_sh[int(s.stable_host[slot // 16]), 0, slot % 16, 21] = inf
    s.vo[3][5, 1, 77] = -inf  # the third sequence's sixth own token
    s.v[int(s.table_host[3, 0]), 1, 5, 77] = -inf
    s.run()
    torch.cuda.synchronize()
    assert (s.status.cpu() == 0).all()
    out = s.out.clone()
    assert (out[:, :, :4, 21] == inf).all() and (out[3, :, 4:, 77] == -inf).all()
    out[:, :, :4, 21] = 0
    out[3, :, 4:, 77] = 0
    assert torch.isfinite(out).all()
    s.vs[slot, 0, 21] = s.vo[3][5, 1, 77] = 0  # the other channels against the definition
    s.v_sh[int(s.stable_host[slot // 16]), 0, slot % 16, 21] = 0
    s.v[int(s.table_host[3, 0]), 1, 5, 77] = 0
    keep = [(slice(None), slice(None), slice(0, 4), 21), (3, slice(None), slice(4, 8), 77)]
    s.run()
    torch.cuda.synchronize()
    s.check()
    for at in keep:
        s.out[at] = 0
    assert torch.equal(s.out, out)


@pytest.mark.parametrize("exp2", [40, -40, 90, 29, 20])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", [1, 2, 3, 4, 5])
def test_channels_of_very_different_size(way, d, exp2, ask):
    """Every sixteenth channel of V is a power of two larger (or smaller) than its neighbours; one is zero throughout. All are as accurate as their own size asks."""
    ask(way)
    factor = torch.ones(d)
    factor[5::16] = 2.0 ** exp2
    factor[9] = 0
    s = Shared(24, 4, 8, 4, d, 500, [(13 * i) % 70 for i in range(24)], v_scale=factor, q_scale=0.5)
    if not _is(s, way):
        pytest.skip("no way for this call")
    s.run()
    s.check(wide=exp2 not in (20,))
    assert (s.out[..., 9] == 0).all()


def test_wide_parts_behind_the_pipelined_own_keys():
    """The same where rows of a sequence's own keys take the pipelined kernel: many sequences of many rows."""
    for d in (64, 128):
        factor = torch.ones(d)
        factor[5::16] = 2.0 ** 40
        s = Shared(48, 24, 32, 8, d, 300, [(13 * i) % 70 for i in range(48)], v_scale=factor, q_scale=0.5)
        s.run()
        s.check(wide=1)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("call", [4, 8, 1, 2])
def test_rows_of_a_table_that_name_the_shared_blocks_first(call, way, ask):
    """One table row per sequence, shared blocks and own ones: the own rows begin inside, their distance is the whole row's length, and behind the last one's
    entries the table ends (nothing there is a block)."""
    ask(way)
    kw = dict(CALLS[call], P=640)  # (whole blocks)
    kw.update(paged=1, max_len=640)
    s = Shared(**kw)
    if not _is(s, way):
        pytest.skip("no way for this call")
    off, row = len(s.stable_host), s.table_host.shape[1]
    big = torch.full((s.B * (off + row) + 5000,), 1 << 30, device="cuda", dtype=torch.int32)
    rows = big[:s.B * (off + row)].view(s.B, off + row)
    rows[:, :off] = s.stable
    rows[:, off:] = s.table
    s.desc.block_table, s.desc.max_blocks = big.data_ptr() + 4 * off, off + row
    s.pre.block_table = big.data_ptr()
    assert vs.vs_shared_prefix_workspace_bytes(s.desc, s.pre) == s.ws_bytes
    s.run()
    s.check()
