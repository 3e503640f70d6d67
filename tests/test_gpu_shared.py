"""vs_shared_prefix_attention against its definition in 64 bits: head layouts, types, lengths, cache layouts, masks, what the device reports, graphs,
and a run of the calls of a decoding step behind a shared prompt."""
import numpy as np
import pytest
import torch

import gpu_util as gu
import paper_2509_15235_amd as vs
from shared_util import Shared

pytestmark = pytest.mark.gpu


def _own(n, hi, seed=0):
    g = np.random.default_rng(seed + n)
    x = g.integers(0, hi + 1, size=n)
    x[0] = hi
    if n > 1:
        x[1] = 0
    return x


HEADS = [(28, 4, 128), (32, 32, 128), (8, 2, 128), (8, 1, 128), (32, 8, 64), (16, 16, 64), (4, 4, 128), (40, 2, 64)]


@pytest.mark.parametrize("bf16", [1, 0])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("B,T,P,hi", [(1, 1, 1, 0), (3, 1, 700, 90), (2, 5, 64, 33), (5, 9, 130, 17)])
def test_head_layouts(heads, B, T, P, hi, bf16):
    s = Shared(B, T, *heads, P, _own(B, hi), bf16=bf16)
    s.run()
    s.check()


@pytest.mark.parametrize("bf16", [1, 0])
@pytest.mark.parametrize("P", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 1000, 2111])
def test_lengths_of_the_prefix(P, bf16):
    s = Shared(4, 3, 8, 2, 128, P, [0, 1, 40, 70], bf16=bf16, max_len=P + 77, max_own=90, block=32, mask=P % 2)
    s.run()
    s.check()


@pytest.mark.parametrize("bf16", [1, 0])
@pytest.mark.parametrize("B,T,heads,P,hi,kw", [
    (70, 1, (8, 2, 128), 300, 30, {}), (33, 2, (14, 2, 64), 77, 50, {}), (2, 64, (8, 2, 128), 500, 300, {}), (3, 60, (7, 1, 128), 333, 700, {}),
    (2, 33, (4, 4, 64), 1500, 10, {}), (9, 7, (8, 8, 128), 200, 1, {}), (4, 1, (8, 2, 128), 5000, 3000, {}), (130, 1, (4, 1, 64), 64, 5, {}),
    (5, 3, (8, 2, 128), 411, 60, dict(paged=0)), (5, 3, (8, 2, 64), 411, 60, dict(paged=0, shared_paged=1)), (5, 3, (8, 2, 64), 411, 60, dict(shared_paged=0)),
    (5, 3, (8, 2, 128), 411, 60, dict(token_major=1)), (5, 3, (8, 2, 128), 411, 60, dict(token_major=1, paged=0)), (6, 17, (28, 4, 128), 257, 100, dict(mask=0)),
    (4, 6, (8, 2, 128), 300, 40, dict(q_scale=60.0)), (4, 6, (8, 2, 64), 300, 40, dict(v_scale=1e30)), (4, 6, (8, 2, 128), 300, 40, dict(scale=1e-6, block=64)),
])
def test_sizes_layouts_and_values(B, T, heads, P, hi, kw, bf16):
    s = Shared(B, T, *heads, P, _own(B, hi), bf16=bf16, **kw)
    s.run()
    s.check()


@pytest.mark.parametrize("bf16", [1, 0])
def test_one_key_holds_everything(bf16):
    """A row whose weight lies on one key only - in the shared prefix, in its own, in the tree - is that key's value, whatever the parts' references are."""
    for where in ("shared", "own", "tree"):
        s = Shared(3, 4, 4, 2, 64, 900, [200, 60, 3], bf16=bf16, q_scale=1.0, paged=0, mask=0)
        s.q.fill_(1.0)
        x = s.k_sh[0, :, 517] if where == "shared" else s.k[:, :, 1] if where == "own" else None
        if where == "tree":  # the root's slot
            for b in range(3):
                s.k[b, :, int(s.own[b])] = 20.0
                s.ko[b][int(s.own[b])] = 20.0
        elif where == "own":
            x.fill_(20.0)
            for b in range(3):
                s.ko[b][1] = 20.0
        else:
            x.fill_(20.0)
            s.ks[517] = 20.0
        s.run()
        s.check()


def test_same_as_the_verification_call_on_whole_caches():
    """The same context as one cache per sequence through vs_tree_verify_attention."""
    s = Shared(4, 11, 28, 4, 128, 640, [16, 0, 130, 77], block=16)
    s.run()
    d = vs.AttnDesc()
    for name, _ in vs.AttnDesc._fields_:
        setattr(d, name, getattr(s.desc, name))
    d.max_prefix_len += 640
    table = np.concatenate([np.repeat(s.stable_host[None], 4, 0), s.table_host], axis=1)
    dev = gu.dev(table)
    d.max_blocks, d.block_table = table.shape[1], dev.data_ptr()
    ws = torch.empty(max(256, vs.vs_attention_workspace_bytes(d)), device="cuda", dtype=torch.uint8)
    out = torch.empty_like(s.out)
    rc = vs.vs_tree_verify_attention(d, s.q, s.k, s.v, s.lens + 640, s.parent_dev, s.mask_dev, out, None, ws, ws.numel(), gu.stream_ptr())
    assert rc == 0
    torch.cuda.synchronize()
    s.check()
    # one more rounding of a row's parts, half a step each, and the two results' own
    assert float((out.float() - s.out.float()).abs().max()) <= 4 * 2.0 ** -8 * float(s.out.float().abs().max())
    # the table's rows with the shared blocks in front, as the documentation has it
    e = vs.AttnDesc()
    for name, _ in vs.AttnDesc._fields_:
        setattr(e, name, getattr(s.desc, name))
    e.max_blocks, e.block_table = table.shape[1], dev.data_ptr() + 4 * 40
    again = torch.empty_like(s.out)
    assert vs.vs_shared_prefix_workspace_bytes(e, s.pre) <= s.ws_bytes
    rc = vs.vs_shared_prefix_attention(e, s.pre, s.q, s.k_sh, s.v_sh, s.shared_len, s.k, s.v, s.lens, s.parent_dev, s.mask_dev, again, None, s.ws, s.ws_bytes,
                                       gu.stream_ptr())
    assert rc == 0
    torch.cuda.synchronize()
    assert torch.equal(again, s.out)


@pytest.mark.parametrize("bf16", [1, 0])
def test_status(bf16):
    def status(change, want, good=()):
        s = Shared(4, 3, 8, 2, 64, 100, [10, 0, 30, 7], bf16=bf16, max_own=40)
        change(s)
        s.run()
        torch.cuda.synchronize()
        assert s.status.cpu().tolist() == want
        s.check(good)
    status(lambda s: None, [0] * 4, range(4))
    status(lambda s: s.shared_len.fill_(-1), [3] * 4)
    status(lambda s: s.shared_len.fill_(101), [3] * 4)
    status(lambda s: s.shared_len.fill_(1 << 30), [3] * 4)
    status(lambda s: s.stable[3:4].fill_(s.pre.num_blocks), [4] * 4)
    status(lambda s: s.stable[6:7].fill_(-1), [4] * 4)
    status(lambda s: s.lens[1:2].fill_(-1), [0, 3, 0, 0], [0, 2, 3])
    status(lambda s: s.lens[2:3].fill_(41), [0, 0, 3, 0], [0, 1, 3])
    status(lambda s: s.table[0, 0:1].fill_(1 << 29), [4, 0, 0, 0], [1, 2, 3])

    def bad_trees(s):
        s.mask_dev = None
        s.parent_dev[0, 0], s.parent_dev[3, 2] = 0, 2
    status(bad_trees, [1, 0, 0, 2], [1, 2])


@pytest.mark.parametrize("bf16", [1, 0])
def test_captured_twice_on_one_workspace_with_other_lengths_between_replays(bf16):
    """Two calls in one graph share their workspace; lengths and inputs change between the replays, an eager call of another size uses the workspace, too."""
    a, b = (Shared(3, 4, 8, 2, 128, 333, own, bf16=bf16, max_len=400, max_own=80, seed=i) for i, own in enumerate(([5, 80, 0], [33, 1, 64])))
    b.ws, b.ws_bytes = a.ws, a.ws_bytes
    a.run()
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.run(stream.cuda_stream)
        b.run(stream.cuda_stream)
    for k in range(3):
        a.out.fill_(float("nan")), b.out.fill_(float("nan"))
        a.ws.random_(0, 256)
        if k == 1:
            a.own = b.own = np.array([7, 0, 31], dtype=np.int32)
            for x in (a, b):
                x.lens.copy_(torch.from_numpy(x.own))
                x.P = 200
                x.shared_len.fill_(200)
                x.ks, x.vs = x.ks[:200], x.vs[:200]
                # what lies behind the new lengths as tree slots
                for c, rows in ((x.k, x.ko), (x.v, x.vo)):
                    for i in range(3):
                        n = int(x.own[i]) + 4
                        if n > len(rows[i]):
                            rows[i] = torch.cat([rows[i], torch.randn((n - len(rows[i]),) + rows[i].shape[1:]).to(rows[i].dtype)])
                        rows[i] = rows[i][:n]
                        t = torch.arange(n)
                        c[torch.from_numpy(x.table_host[i].astype(np.int64))[t // 16].cuda(), :, (t % 16).cuda()] = rows[i].cuda()
        graph.replay()
        torch.cuda.synchronize()
        a.check()
        b.check()


def test_on_another_stream():
    s = Shared(5, 2, 28, 4, 128, 900, [3, 50, 0, 9, 100])
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    s.run(stream.cuda_stream)
    stream.synchronize()
    s.check()
