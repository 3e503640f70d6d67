"""vs_kv_append against its definition: padded trees and packed prompts, both cache layouts, positions of every kind, what stays as it was,
what is refused on the device, and a run of append, attention and commit."""
import numpy as np
import pytest
import torch

import gen
import gpu_util as gu
import paper_2509_15235_amd as vs
import rope_util as ru

pytestmark = pytest.mark.gpu


class Setup:
    """Inputs of one call, and what it has to leave behind."""

    def __init__(self, counts, lens, Hq=4, Hkv=2, d=64, rot=64, bf16=1, halves=1, axes=None, cyclic=0, paged=1, block=16, packed=1, depth=0, offset=0,
                 explicit=0, tail=0, T=None, token_major=0, seed=0):
        g = np.random.default_rng(seed)
        self.__dict__.update(locals())
        B = self.B = len(counts)
        T = self.T = T or max(1, max(counts))
        self.start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32) if packed else (np.arange(B + 1) * T).astype(np.int32)
        rows = self.rows = int(self.start[-1]) + tail
        dt = self.dt = torch.bfloat16 if bf16 else torch.float32
        self.fused = torch.from_numpy(g.standard_normal((rows, Hq + 2 * Hkv, d)).astype(np.float32)).to(dt).cuda()
        self.q, self.kn, self.vn = self.fused[:, :Hq], self.fused[:, Hq:Hq + Hkv], self.fused[:, Hq + Hkv:]
        self.q_out = torch.full((rows, Hq, d), 9.0, device="cuda", dtype=dt)
        most = max(n + l for n, l in zip(counts, lens)) + 3
        self.table = None
        if paged:
            row = (most + block - 1) // block
            self.table_host = g.permutation(B * row + 3)[:B * row].astype(np.int32).reshape(B, row)
            self.table = gu.dev(self.table_host)
            shape = (B * row + 3, block, Hkv, d) if token_major else (B * row + 3, Hkv, block, d)
        else:
            shape = (B, most, Hkv, d) if token_major else (B, Hkv, most, d)
        self.k = torch.full(shape, 3.0, device="cuda", dtype=dt)
        self.v = torch.full(shape, 5.0, device="cuda", dtype=dt)
        kh = self.k.transpose(1, 2) if token_major else self.k  # [., Hkv, slots, d]
        axes = axes or [rot // 2]
        pos = np.zeros((len(axes), rows), dtype=np.int32)
        self.depth_dev = self.offset_dev = self.pos_dev = None
        dep = g.integers(0, 7, size=(B, T)).astype(np.int32)
        off = g.integers(-3, 4, size=B).astype(np.int32)
        self.seq = np.full(rows, -1)
        for b in range(B):
            for i in range(int(self.start[b + 1] - self.start[b])):
                r = int(self.start[b]) + i
                self.seq[r] = b
                pos[:, r] = lens[b] + (off[b] if offset else 0) + (dep[b, i] if depth else i)
        if explicit:
            pos = g.integers(0, 3000, size=pos.shape).astype(np.int32)
            self.pos_dev = gu.dev(pos)
        if depth:
            self.depth_dev = gu.dev(dep)
        if offset:
            self.offset_dev = gu.dev(off)
        freq = ru.frequencies(rot)
        self.freq = gu.dev(freq)
        self.rope = ru.rope_desc(rot, halves, axes, cyclic, stride_axis=rows, inv_freq=self.freq.data_ptr())
        self.prefix = gu.dev(np.array(lens, dtype=np.int32))
        self.start_dev = gu.dev(self.start) if packed else None
        self.status = torch.full((B,), -99, device="cuda", dtype=torch.int32)
        D = self.desc = vs.AppendDesc(B=B, T=T, Hq=Hq, Hkv=Hkv, d=d, dtype=vs.VS_BF16 if bf16 else vs.VS_F32, rows=rows, q_stride=self.q.stride(0),
                                      k_stride=self.kn.stride(0), v_stride=self.vn.stride(0), q_out_stride=Hq * d)
        D.stride_head, D.stride_tok = kh.stride(1), kh.stride(2)
        if paged:
            D.paged, D.block_size, D.max_blocks, D.num_blocks, D.stride_block = 1, block, self.table.shape[1], shape[0], kh.stride(0)
            D.block_table = self.table.data_ptr()
        else:
            D.capacity, D.stride_seq = most, kh.stride(0)
        cos, sin = ru.cos_sin(pos, freq, ru.axis_of_pair(rot // 2, axes, cyclic))
        host = self.fused.float().cpu().numpy()
        self.want = ru.rotate(host, cos, sin, rot, halves)
        self.want[:, Hq + Hkv:] = host[:, Hq + Hkv:]
        self.most_off = ru.bound(host, self.want, rot, halves, bf16)
        self.most_off[:, Hq + Hkv:] = 0

    def run(self, stream=None):
        rc = vs.vs_kv_append(self.desc, self.rope, self.q, self.kn, self.vn, self.pos_dev, self.depth_dev, self.offset_dev, self.prefix, self.start_dev,
                             self.q_out, self.k, self.v, self.status, gu.stream_ptr() if stream is None else stream)
        assert rc == 0, vs.vs_strerror(rc)

    def caches(self):
        f = (lambda x: x.transpose(1, 2)) if self.token_major else (lambda x: x)
        return [f(x).float().cpu().numpy() for x in (self.k, self.v)]

    def check(self, good=None):
        """Rows of the sequences `good` (default: all) are where they belong, everything else is as it was."""
        torch.cuda.synchronize()
        good = range(self.B) if good is None else good
        q = self.q_out.float().cpu().numpy()
        Hq, Hkv = self.Hq, self.Hkv
        k, v = self.caches()
        touched = np.zeros(k.shape[:1] + k.shape[2:3], dtype=bool)
        for r in range(self.rows):
            b = int(self.seq[r])
            if b < 0:
                assert (q[r] == 9.0).all()
                continue
            if b not in good:
                continue
            assert (np.abs(q[r] - self.want[r, :Hq]) <= self.most_off[r, :Hq]).all()
            t = self.lens[b] + r - int(self.start[b])
            at = (self.table_host[b, t // self.block], t % self.block) if self.paged else (b, t)
            touched[at] = True
            assert (np.abs(k[at[0], :, at[1]] - self.want[r, Hq:Hq + Hkv]) <= self.most_off[r, Hq:Hq + Hkv]).all(), (r, b)
            assert (v[at[0], :, at[1]] == self.want[r, Hq + Hkv:]).all(), (r, b)
        for x, was in ((k, 3.0), (v, 5.0)):
            assert (np.moveaxis(x, 2, 1)[~touched] == was).all()


@pytest.mark.parametrize("kw", [
    dict(counts=[1], lens=[0]), dict(counts=[1], lens=[1696], Hq=28, Hkv=4, d=128, rot=128, paged=0, packed=0),
    dict(counts=[60] * 3, lens=[5, 300, 17], Hq=28, Hkv=4, d=128, rot=128, packed=0, depth=1, offset=1),
    dict(counts=[31] * 4, lens=[100, 0, 15, 16], bf16=0, rot=32, halves=0, paged=0, packed=0, depth=1),
    dict(counts=[0, 3, 0, 0, 47, 1, 200, 0], lens=[4, 15, 0, 9, 16, 31, 3, 7], axes=[8, 12, 12], explicit=1, block=32),
    dict(counts=[3, 0, 65, 2], lens=[4, 15, 0, 9], axes=[12, 10, 10], cyclic=1, explicit=1, paged=0, bf16=0, offset=1, tail=9),
    dict(counts=[5, 9, 2], lens=[1, 2, 3], tail=4, offset=1, token_major=1), dict(counts=[7] * 2, lens=[8, 30], packed=0, token_major=1, paged=0),
    dict(counts=[1] * 130, lens=list(range(130)), packed=1), dict(counts=[(5 * i) % 7 for i in range(200)], lens=[i % 40 for i in range(200)], packed=1, tail=2),
    dict(counts=[1100], lens=[13], Hq=3, Hkv=1, d=80, rot=32, packed=0, block=64), dict(counts=[2, 2], lens=[3, 14], rot=16, Hq=1, Hkv=1),
    dict(counts=[9, 1], lens=[0, 0], bf16=0, d=256, rot=256, Hq=2, Hkv=2), dict(counts=[20, 30], lens=[1, 1], Hq=5, Hkv=5, d=96, rot=48, halves=0),
    dict(counts=[4, 4], lens=[12, 28], packed=0, explicit=1, axes=[10, 11, 11], offset=1),
    dict(counts=[300, 1, 280], lens=[7, 0, 40], Hq=28, Hkv=4, d=128, rot=128, axes=[16, 24, 24], explicit=1, tail=3), dict(counts=[700], lens=[3], Hq=8, Hkv=2, d=128, rot=128, bf16=0, packed=0),
])
def test_against_definition(kw):
    s = Setup(**kw)
    s.run()
    s.check()
    assert (s.status.cpu().numpy() == 0).all()


def test_keys_and_values_only_and_queries_in_place():
    s = Setup([30, 2], [3, 40], tail=3)
    s.desc.Hq, s.desc.q_stride, s.desc.q_out_stride = 0, 0, 0
    rc = vs.vs_kv_append(s.desc, s.rope, None, s.kn, s.vn, None, None, None, s.prefix, s.start_dev, None, s.k, s.v, None, gu.stream_ptr())
    assert rc == 0
    k, v = s.k.clone(), s.v.clone()
    t = Setup([30, 2], [3, 40], tail=3)
    t.run()
    torch.cuda.synchronize()
    assert torch.equal(k, t.k) and torch.equal(v, t.v)
    u = Setup([30, 2], [3, 40], tail=3)
    u.q_out, u.desc.q_out_stride = u.q, u.q.stride(0)
    u.run()
    torch.cuda.synchronize()
    assert torch.equal(u.q[:32], t.q_out[:32]) and torch.equal(u.q[32:], t.q[32:]) and torch.equal(u.k, t.k)


@pytest.mark.parametrize("paged", [0, 1])
def test_bad_lengths_and_blocks_are_reported_and_leave_the_others_right(paged):
    s = Setup([5, 20, 3, 4, 0], [10, 15, 7, 100, 3], paged=paged)
    host = s.prefix.cpu().numpy()
    host[0] = -1
    host[2] = 1 << 30
    host[4] = -4
    s.prefix.copy_(torch.from_numpy(host))
    want = [3, 0, 3, 0, 3]
    if paged:
        s.table[1, 1] = s.desc.num_blocks  # slots 16 .. 31
        want[1] = 4
    s.run()
    s.check(good=[3] if paged else [1, 3]) if not paged else torch.cuda.synchronize()
    assert s.status.cpu().tolist() == want
    if paged:  # of sequence 1 what lies in its good blocks may be there; nothing lies anywhere else
        k, v = s.caches()
        mine = np.zeros(k.shape[0], dtype=bool)
        mine[s.table_host[3]] = mine[s.table_host[1, [0, 2]]] = True
        assert (k[~mine] == 3.0).all() and (v[~mine] == 5.0).all()


@pytest.mark.parametrize("row_start,want", [
    ([0, 5, 3, 9], [0, 7, 0]), ([-2, 5, 6, 9], [7, 0, 0]), ([0, 5, 6, 10], [0, 0, 7]), ([0, 5, 6, 1 << 30], [0, 0, 7]),
    ([0, 0, 9, 9], [0, 7, 0]), ([3, 2, 1, 0], [7, 7, 7]), ([-(1 << 31), (1 << 31) - 1, 0, 0], [7, 7, 0]),
])
def test_bad_row_starts(row_start, want):
    """Nine rows, at most six of a sequence: a sequence whose rows are no rows of it writes nothing."""
    s = Setup([5, 1, 3], [10, 15, 7], T=6)
    s.start_dev.copy_(torch.tensor(row_start, dtype=torch.int32))
    s.run()
    torch.cuda.synchronize()
    assert s.status.cpu().tolist() == want
    k, v = s.caches()
    for b in range(3):
        if want[b]:
            assert (k[s.table_host[b]] == 3.0).all() and (v[s.table_host[b]] == 5.0).all()


def test_captured_with_other_lengths_between_replays():
    s = Setup([6, 9], [10, 3])
    t = Setup([6, 9], [14, 11])
    stream = torch.cuda.Stream()
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        s.run(stream.cuda_stream)
    for u in (t, Setup([6, 9], [10, 3]), t):
        s.k.fill_(3.0), s.v.fill_(5.0), s.q_out.fill_(9.0)
        s.prefix.copy_(u.prefix)
        s.lens, s.want, s.most_off = u.lens, u.want, u.most_off
        graph.replay()
        torch.cuda.synchronize()
        s.check()


def test_blocks_beyond_32_bits_of_a_pool():
    """Blocks a gigabyte apart: offsets of the last ones pass 2^32 elements."""
    s = Setup([20, 3], [10, 0], packed=1)
    n, gap = s.k.shape[0], (1 << 29) + 1024
    pools = [torch.empty(gap * (n - 1) + s.k[0].numel(), device="cuda", dtype=torch.bfloat16).as_strided(s.k.shape, (gap,) + s.k.stride()[1:]) for _ in range(2)]
    assert n >= 9 and gap * (n - 1) > 1 << 32
    for pool, name in zip(pools, "kv"):
        pool.copy_(getattr(s, name))
        setattr(s, name, pool)
    s.desc.stride_block = gap
    s.run()
    s.check()


def test_more_rows_than_one_launch_takes():
    """2^25 rows and some of one sequence, a key and a value of four channels each; a second sequence behind it."""
    rows = (1 << 25) + 9
    k, v = (torch.randn((rows, 4), device="cuda", generator=torch.Generator("cuda").manual_seed(s)) for s in (0, 1))
    kc, vc = (torch.full((2, rows, 4), 7.0, device="cuda") for _ in range(2))
    freq, status = gu.dev(ru.frequencies(4)), torch.full((2,), -9, device="cuda", dtype=torch.int32)
    d = vs.AppendDesc(B=2, T=rows, Hq=0, Hkv=1, d=4, dtype=vs.VS_F32, rows=rows, k_stride=4, v_stride=4, capacity=rows, stride_seq=rows * 4, stride_head=rows * 4, stride_tok=4)
    rc = vs.vs_kv_append(d, ru.rope_desc(4, False, inv_freq=freq.data_ptr()), None, k, v, None, None, None, gu.dev(np.array([2, 1], dtype=np.int32)),
                         gu.dev(np.array([0, rows - 4, rows], dtype=np.int32)), None, kc, vc, status, gu.stream_ptr())
    torch.cuda.synchronize()
    assert rc == 0 and status.cpu().tolist() == [0, 0]
    n = rows - 4
    assert torch.equal(vc[0, 2:2 + n], v[:n]) and torch.equal(vc[1, 1:5], v[n:])
    assert (vc[0, :2] == 7).all() and (vc[0, n + 2:] == 7).all() and (vc[1, 0] == 7).all() and (vc[1, 5:] == 7).all()
    at = np.arange(n - 20, n)
    host = k[n - 20:].cpu().numpy()[:, None]
    pos = np.concatenate([at + 2, 1 + np.arange(4)])
    cos, sin = ru.cos_sin(pos[None], ru.frequencies(4), ru.axis_of_pair(2, [2], False))
    want = ru.rotate(host, cos, sin, 4, False)
    got = torch.cat([kc[0, n - 18:n + 2], kc[1, 1:5]]).cpu().numpy()[:, None]
    assert (np.abs(got - want) <= ru.bound(host, want, 4, False, False)).all()


def test_slots_end_where_lengths_do():
    """A cache whose blocks hold more tokens than a length counts: rows that would come behind 2^31 - 1 are refused."""
    s = Setup([4, 4], [3, 0], block=16, packed=0)
    s.desc.block_size, s.desc.max_blocks, s.desc.num_blocks = 1 << 30, 4, 2
    s.table = torch.tensor([[0, 9, 9, 9], [1, 9, 9, 9]], device="cuda", dtype=torch.int32)
    s.desc.block_table = s.table.data_ptr()
    s.desc.stride_head, s.desc.stride_tok, s.desc.stride_block = 64 << 30, 64, 128 << 30
    s.prefix.copy_(torch.tensor([(1 << 31) - 4, (1 << 31) - 3], dtype=torch.int32))
    s.run()
    torch.cuda.synchronize()
    assert s.status.cpu().tolist() == [3, 3]
    k, v = s.caches()
    assert (k == 3.0).all() and (v == 5.0).all()
