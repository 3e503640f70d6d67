"""Attention behind a shared prefix from its definition in 64 bits, and the inputs of a call."""
import math

import numpy as np
import torch

import gpu_util as gu
import paper_2509_15235_amd as vs


def trees(g, B, T, wide=3):
    parent = np.full((B, T), -1, dtype=np.int32)
    for i in range(1, T):
        parent[:, i] = [g.integers(max(0, i - wide), i) for _ in range(B)]
    return parent


def masks(parent):
    B, T = parent.shape
    m = np.zeros((B, T), dtype=np.uint64)
    for i in range(T):
        m[:, i] = np.uint64(1) << np.uint64(i)
        if i:
            m[:, i] |= m[np.arange(B), parent[:, i]]
    return m


class Shared:
    """Device tensors and descriptors of one call; unread slots hold NaN."""

    def __init__(self, B, T, Hq, Hkv, d, P, own, bf16=1, paged=1, shared_paged=None, block=16, mask=1, token_major=0, scale=None, q_scale=2.0,
                 max_len=None, max_own=None, seed=0, v_scale=1.0, same_pool=1):
        g = np.random.default_rng(seed)
        self.__dict__.update(locals())
        self.shared_paged = shared_paged = paged if shared_paged is None else shared_paged
        dt = self.dt = torch.bfloat16 if bf16 else torch.float32
        own = self.own = np.array(own, dtype=np.int32)
        max_own = self.max_own = int(own.max()) if max_own is None else max_own
        max_len = self.max_len = max(1, P) if max_len is None else max_len
        rnd = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).to(dt)  # noqa: E731
        self.q = rnd(B, T, Hq, d).mul_(q_scale).cuda()
        self.parent = trees(g, B, T)
        self.mask_host = masks(self.parent)
        self.scale = scale or 1.0 / math.sqrt(d)
        # logical keys and values
        self.ks, self.vs = rnd(P, Hkv, d), rnd(P, Hkv, d).mul_(v_scale)
        self.ko = [rnd(int(n) + T, Hkv, d) for n in own]
        self.vo = [rnd(int(n) + T, Hkv, d).mul_(v_scale) for n in own]
        desc = vs.AttnDesc(B=B, T=T, Hq=Hq, Hkv=Hkv, d=d, dtype=vs.VS_BF16 if bf16 else vs.VS_F32, softmax_scale=self.scale, max_prefix_len=max_own)
        pre = vs.PrefixDesc(max_len=max_len)
        nan = float("nan")
        most = max_own + T
        row, srow = (most + block - 1) // block, (max_len + block - 1) // block
        n_own = B * row if paged else 0
        n_shared = srow if shared_paged else 0
        ids = g.permutation(n_own + n_shared + 2).astype(np.int32)
        pool = len(ids)

        def cache(*shape):
            return [torch.full(shape, nan, dtype=dt) for _ in range(2)]

        def heads_first(x):  # a view [., Hkv, slots, d] of a cache
            return x.transpose(1, 2) if token_major else x

        pool_shape = (pool, block, Hkv, d) if token_major else (pool, Hkv, block, d)
        pools = cache(*pool_shape)
        own_c = pools if paged else cache(*((B, most, Hkv, d) if token_major else (B, Hkv, most, d)))
        sh_c = pools if shared_paged else cache(*((1, max_len, Hkv, d) if token_major else (1, Hkv, max_len, d)))
        self.table_host = ids[:n_own].reshape(B, row) if paged else None
        self.stable_host = ids[n_own:n_own + n_shared] if shared_paged else None
        for x, shared, logical in ((own_c[0], 0, self.ko), (own_c[1], 0, self.vo), (sh_c[0], 1, [self.ks]), (sh_c[1], 1, [self.vs])):
            view = heads_first(x)
            for b, rows in enumerate(logical):
                t = torch.arange(len(rows))
                if (shared_paged if shared else paged):
                    tab = torch.from_numpy((self.stable_host if shared else self.table_host[b]).astype(np.int64))
                    view[tab[t // block], :, t % block] = rows
                else:
                    view[b, :, t] = rows.transpose(0, 1)
        if pools is own_c or pools is sh_c:
            pools = [x.cuda() for x in pools]
        self.k, self.v = pools if paged else [x.cuda() for x in own_c]
        self.k_sh, self.v_sh = pools if shared_paged else [x.cuda() for x in sh_c]
        vk, vks = heads_first(self.k), heads_first(self.k_sh)
        desc.stride_head, desc.stride_tok = vk.stride(1), vk.stride(2)
        pre.stride_head, pre.stride_tok = vks.stride(1), vks.stride(2)
        self.table = self.stable = None
        if paged:
            self.table = gu.dev(self.table_host)
            desc.paged, desc.block_size, desc.max_blocks, desc.num_blocks, desc.stride_block = 1, block, row, pool, vk.stride(0)
            desc.block_table = self.table.data_ptr()
        else:
            desc.capacity, desc.stride_seq = most, vk.stride(0)
        if shared_paged:
            self.stable = gu.dev(self.stable_host)
            pre.paged, pre.block_size, pre.max_blocks, pre.num_blocks, pre.stride_block = 1, block, srow, pool, vks.stride(0)
            pre.block_table = self.stable.data_ptr()
        else:
            pre.capacity = max_len
        self.desc, self.pre = desc, pre
        self.lens, self.shared_len = gu.dev(own), gu.dev(np.array([P], dtype=np.int32))
        self.parent_dev = gu.dev(self.parent)
        self.mask_dev = gu.dev(self.mask_host.view(np.int64)) if mask else None
        self.out = torch.full((B, T, Hq, d), nan, device="cuda", dtype=dt)
        self.status = torch.full((B,), -99, device="cuda", dtype=torch.int32)
        self.ws_bytes = vs.vs_shared_prefix_workspace_bytes(desc, pre)
        self.ws = torch.randint(0, 256, (max(self.ws_bytes, 256),), device="cuda", dtype=torch.uint8)

    def run(self, stream=None):
        rc = vs.vs_shared_prefix_attention(self.desc, self.pre, self.q, self.k_sh, self.v_sh, self.shared_len, self.k, self.v, self.lens, self.parent_dev,
                                           self.mask_dev, self.out, self.status, self.ws, self.ws_bytes, gu.stream_ptr() if stream is None else stream)
        assert rc == 0, vs.vs_strerror(rc)

    def want(self, b):
        """Rows of sequence b [T, Hq, d], and the sum of |weight * value|, the sum over channels of |q k| at its largest."""
        T, Hq, Hkv, d = self.T, self.Hq, self.Hkv, self.d
        n = int(self.own[b])
        k = torch.cat([self.ks, self.ko[b]]).double().numpy()
        v = torch.cat([self.vs, self.vo[b]]).double().numpy()
        q = self.q[b].double().cpu().numpy()
        sees = np.ones((T, self.P + n + T), dtype=bool)
        for j in range(T):
            sees[:, self.P + n + j] = (self.mask_host[b] >> np.uint64(j)) & np.uint64(1) != 0
        out, size = np.empty((T, Hq, d)), np.empty((T, Hq, d))
        most = 0.0
        for h in range(Hq):
            kk, vv = k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)]
            s = q[:, h] @ kk.T * self.scale
            most = max(most, float((np.abs(q[:, h]) @ np.abs(kk).T).max()) * self.scale)
            s[~sees] = -np.inf
            w = np.exp(s - s.max(axis=1, keepdims=True))
            w /= w.sum(axis=1, keepdims=True)
            out[:, h], size[:, h] = w @ vv, w @ np.abs(vv)
        return out, size, most

    def check(self, which=None, wide=0):
        """fp32 arithmetic: a score is off by (d + 4) half units of the sum of its products' sizes, an exponential by 2^-21 beside that, and a sum of n terms
        by n half units; a weight's error counts once above and once below the line. bf16: a weight that meets a value is rounded by half a step, 2^-8, and
        so is the result; a part's mean once more where some channels dwarf their neighbours (wide)."""
        torch.cuda.synchronize()
        got = self.out.double().cpu().numpy()
        for b in range(self.B) if which is None else which:
            want, size, most = self.want(b)
            n = self.P + int(self.own[b]) + self.T
            off = 2 * ((self.d + 4) * 2.0 ** -24 * most + 2.0 ** -21) + 2 * n * 2.0 ** -24
            room = off * size + ((size * (1 + wide) + np.abs(want)) * 2.0 ** -8 if self.bf16 else 2.0 ** -24 * np.abs(want))
            err = np.abs(got[b] - want)
            bad = ~(err <= room)
            assert not bad.any(), (b, int(bad.sum()), float(np.nanmax(err / room)), np.argwhere(bad)[:4].tolist())
        if which is None:
            assert (self.status.cpu().numpy() == 0).all()
