"""The calls of a decoder behind a shared prompt, as a program makes them: the prompt and the sequences' own beginnings appended with their positions (an
image's three axes), a draft tree appended by its depths, attention behind the shared prefix, the accepted path committed, and a token decoded from there."""
import numpy as np
import pytest
import torch

import gpu_util as gu
import paper_2509_15235_amd as vs
import rope_util as ru

pytestmark = pytest.mark.gpu
HQ, HKV, D, BS, T, B, P = 6, 2, 64, 16, 7, 3, 53
COUNTS = [8, 12, 12]  # time, height, width


class Decoder:
    """One layer's pools and tables, and in numpy what they ought to hold."""

    def __init__(self, dtype):
        self.dt = torch.bfloat16 if dtype == vs.VS_BF16 else torch.float32
        self.dtype = dtype
        g = self.g = np.random.default_rng(11)
        ids = g.permutation(40).astype(np.int32)
        self.shared_table, self.tables = ids[:4], ids[4:4 + 3 * 6].reshape(3, 6)
        self.k, self.v = (torch.full((40, HKV, BS, D), float("nan"), device="cuda", dtype=self.dt) for _ in range(2))
        self.dev = [gu.dev(self.shared_table[None]), gu.dev(self.tables)]
        self.freq = gu.dev(ru.frequencies(D))
        self.keys = {"shared": [], 0: [], 1: [], 2: []}  # rows of (rotated key, value) in 64 bits
        self.ws = torch.empty(1 << 22, device="cuda", dtype=torch.uint8)

    def rope(self, stride):
        return ru.rope_desc(D, True, COUNTS, stride_axis=stride, inv_freq=self.freq.data_ptr())

    def turned(self, x, positions):
        cos, sin = ru.cos_sin(positions, ru.frequencies(D), ru.axis_of_pair(D // 2, COUNTS, False))
        return ru.rotate(x, cos, sin, D, True)

    def append(self, shared, counts, lens, positions=None, depth=None, offset=None, packed=True):
        """New rows of some sequences; returns the rotated queries and, by row, the sequence and position."""
        n = sum(counts)
        fused = torch.from_numpy(self.g.standard_normal((n, HQ + 2 * HKV, D)).astype(np.float32)).to(self.dt).cuda()
        q, k, v = fused[:, :HQ], fused[:, HQ:HQ + HKV], fused[:, HQ + HKV:]
        out = torch.empty((n, HQ, D), device="cuda", dtype=self.dt)
        table = self.dev[0 if shared else 1]
        d = vs.AppendDesc(B=len(counts), T=max(counts), Hq=HQ, Hkv=HKV, d=D, dtype=self.dtype, rows=n, q_stride=fused.stride(0), k_stride=fused.stride(0),
                          v_stride=fused.stride(0), q_out_stride=HQ * D, paged=1, block_size=BS, max_blocks=table.shape[1], num_blocks=40,
                          stride_block=HKV * BS * D, stride_head=BS * D, stride_tok=D, block_table=table.data_ptr())
        start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        status = torch.full((len(counts),), -9, device="cuda", dtype=torch.int32)
        dev = [None if x is None else gu.dev(np.ascontiguousarray(x)) for x in (positions, depth, offset, np.array(lens, dtype=np.int32))]
        rc = vs.vs_kv_append(d, self.rope(n), q, k, v, dev[0], dev[1], dev[2], dev[3], gu.dev(start) if packed else None, out, self.k, self.v, status, gu.stream_ptr())
        assert rc == 0
        torch.cuda.synchronize()
        assert (status.cpu().numpy() == 0).all()
        host = fused.float().cpu().numpy()
        at = np.zeros((3, n), dtype=np.int64)
        for b, c in enumerate(counts):
            for i in range(c):
                r = start[b] + i
                at[:, r] = positions[:, r] if positions is not None else lens[b] + (offset[b] if offset is not None else 0) + (depth[b, i] if depth is not None else i)
        want = self.turned(host, at)
        most = ru.bound(host, want, D, True, self.dtype == vs.VS_BF16)
        assert (np.abs(out.float().cpu().numpy() - want[:, :HQ]) <= most[:, :HQ]).all()
        for b, c in enumerate(counts):
            rows = self.keys["shared" if shared else b]
            del rows[lens[b]:]
            for r in range(start[b], start[b] + c):
                rows.append((want[r, HQ:HQ + HKV], host[r, HQ + HKV:]))
        return out.reshape(len(counts), -1, HQ, D) if not packed else out, want[:, :HQ]

    def attend(self, q, exact_q, lens, parent):
        t = parent.shape[1]
        d = vs.AttnDesc(B=B, T=t, Hq=HQ, Hkv=HKV, d=D, dtype=self.dtype, softmax_scale=0.125, max_prefix_len=80, paged=1, block_size=BS, max_blocks=6, num_blocks=40,
                        stride_block=HKV * BS * D, stride_head=BS * D, stride_tok=D, block_table=self.dev[1].data_ptr())
        pre = vs.PrefixDesc(max_len=64, paged=1, block_size=BS, max_blocks=4, num_blocks=40, stride_block=HKV * BS * D, stride_head=BS * D, stride_tok=D,
                            block_table=self.dev[0].data_ptr())
        out = torch.full((B, t, HQ, D), float("nan"), device="cuda", dtype=self.dt)
        status = torch.full((B,), -9, device="cuda", dtype=torch.int32)
        n = vs.vs_shared_prefix_workspace_bytes(d, pre)
        assert 0 < n <= self.ws.numel()
        rc = vs.vs_shared_prefix_attention(d, pre, q, self.k, self.v, gu.dev(np.array([P], dtype=np.int32)), self.k, self.v, gu.dev(np.array(lens, dtype=np.int32)),
                                           gu.dev(parent), None, out, status, self.ws, n, gu.stream_ptr())
        assert rc == 0
        torch.cuda.synchronize()
        assert (status.cpu().numpy() == 0).all()
        got = out.double().cpu().numpy()
        exact_q = exact_q.reshape(B, t, HQ, D)
        for b in range(B):
            rows = self.keys["shared"] + self.keys[b]
            assert len(rows) == P + lens[b] + t
            k, v = np.stack([r[0] for r in rows]), np.stack([r[1] for r in rows]).astype(np.float64)
            sees = np.ones((t, len(rows)), dtype=bool)
            for i in range(t):
                sees[i, P + lens[b]:] = False
                j = i
                while j >= 0:
                    sees[i, P + lens[b] + j] = True
                    j = parent[b, j]
            for h in range(HQ):
                s = exact_q[b, :, h] @ k[:, h // 3].T * 0.125
                s[~sees] = -np.inf
                w = np.exp(s - s.max(axis=1, keepdims=True))
                w /= w.sum(axis=1, keepdims=True)
                want, size = w @ v[:, h // 3], w @ np.abs(v[:, h // 3])
                # The queries and keys that the kernel has are rounded (bf16: half a step, 2^-8, and 2^-17 from sines; fp32 4.2e-7) once each: a score is off by
                # that twice of the sum of its products' sizes, a weight by twice that relatively (above and below the line); then bf16's 2^-8 of the weights and of the result
                sizes = np.abs(exact_q[b, :, h]) @ np.abs(k[:, h // 3]).T * 0.125
                step = 2.0 ** -8 + 2.0 ** -17 if self.dt == torch.bfloat16 else 1e-6
                room = (np.expm1(2 * 2 * step * sizes.max(axis=1)))[:, None] * size + step * (size + np.abs(want))
                assert (np.abs(got[b, :, h] - want) <= room).all(), (b, h)

    def commit(self, lens, path, alen):
        d = vs.KVDesc(B=B, T=path.shape[1], Hkv=HKV, d=D, dtype=self.dtype, num_layers=1, paged=1, block_size=BS, max_blocks=6, num_blocks=40, stride_block=HKV * BS * D,
                      stride_head=BS * D, stride_tok=D, block_table=self.dev[1].data_ptr())
        new = torch.full((B,), -9, device="cuda", dtype=torch.int32)
        rc = vs.vs_tree_kv_commit(d, self.k, self.v, gu.dev(np.array(lens, dtype=np.int32)), gu.dev(path), gu.dev(alen), new, None, gu.stream_ptr())
        assert rc == 0
        for b in range(B):
            nodes = self.keys[b][lens[b]:]
            self.keys[b] = self.keys[b][:lens[b]] + [nodes[path[b, k]] for k in range(alen[b] + 1)]
        return new.cpu().tolist()


@pytest.mark.parametrize("dtype", [vs.VS_BF16, vs.VS_F32])
def test_prompt_tree_commit_token(dtype):
    m = Decoder(dtype)
    # the shared prompt: text, an image of 6 x 7, text
    pos = np.tile(np.arange(P), (3, 1)).astype(np.int32)
    pos[:, 5:47] = 5
    pos[1, 5:47] += np.arange(42) // 7
    pos[2, 5:47] += np.arange(42) % 7
    pos[:, 47:] = 5 + 7 + np.arange(6)
    m.append(True, [P], [0], positions=pos)
    # each sequence's own question; positions go on behind the prompt's last one
    offset = np.full(B, 18, dtype=np.int32)
    lens = [9, 0, 30]
    m.append(False, lens, [0, 0, 0], offset=offset)
    # a draft tree each
    parent = np.array([[-1, 0, 0, 1, 1, 2, 3], [-1, 0, 1, 2, 3, 4, 5], [-1, 0, 0, 0, 0, 0, 0]], dtype=np.int32)
    depth = np.array([[0, 1, 1, 2, 2, 2, 3], list(range(7)), [0] + [1] * 6], dtype=np.int32)
    q, exact = m.append(False, [T] * B, lens, depth=depth, offset=offset, packed=False)
    m.attend(q, exact, lens, parent)
    path = np.array([[0, 1, 3, 6, -1, -1, -1], [0, 1, 2, -1, -1, -1, -1], [0] + [-1] * 6], dtype=np.int32)
    alen = np.array([3, 2, 0], dtype=np.int32)
    new = m.commit(lens, path, alen)
    assert new == [13, 3, 31]
    # the bonus tokens, one each, from there
    q, exact = m.append(False, [1] * B, new, offset=offset, packed=False)
    m.attend(q, exact, new, np.full((B, 1), -1, dtype=np.int32))
