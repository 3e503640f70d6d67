"""Operators around the tree attention, as cases that can be timed and compared: each in a plain form
(elementary torch operations in 32 bits, angles in 64) and as a user of this library calls it.

  rope     positions of one to three axes (time, height, width) applied to rows of heads
  append   new rows of a layer: queries and keys rotated by their positions, keys and values written
           into the sequences' caches behind their prefixes (prompts, draft trees, single tokens)
  shared   attention of a batch of draft trees (or single tokens) whose sequences share one long prefix,
           stored once, and have a cache of their own behind it

Queries and keys are N(0, 1) with queries twice as large where scores are made of them (a score's standard
deviation is then 2: a few keys hold much of a row), values N(0, 1), all rounded once to the storage type.
"""
import math

import numpy as np
import torch

own = False

HEADS = [(28, 4, 128), (28, 4, 128), (32, 32, 128), (8, 2, 128), (8, 1, 128), (32, 8, 64), (16, 16, 64)]
THETA = 1e6


def _case(name, kind, **sizes):
    return dict(name=name, kind=kind, **sizes)


def listed():
    return [
        # one decoded token's queries and keys, rotated in a model that stores fp32
        _case("rope one token fp32", "rope", dtype="f32", rows=1, H=32, d=128, rot=128, axes=1, order="blocks", pairing="halves",
              inverse=0, far=40000),
        # queries and keys of a prompt with a large image, positions of three axes, the heads of a fused projection
        _case("rope image prompt", "rope", dtype="bf16", rows=6684, H=32, d=128, rot=128, axes=3, order="blocks", pairing="halves",
              inverse=0, far=0),
        # a gradient on its way back through the rotation: half of each head, adjacent channels, two axes, an odd number of rows
        _case("rope gradient adjacent", "rope", dtype="f32", rows=2047, H=16, d=64, rot=32, axes=2, order="cyclic", pairing="adjacent",
              inverse=1, far=0),
        # a single sequence decoding one token at a time
        _case("append one token", "append", dtype="bf16", B=1, T=1, Hq=28, Hkv=4, d=128, lo=1696, hi=1696, paged=0, block=16, packed=0,
              rot=128, axes=1, order="blocks", pairing="halves", tree=0),
        # the draft trees of a serving batch over a paged cache: positions from the nodes' depths
        _case("append trees paged", "append", dtype="bf16", B=16, T=60, Hq=28, Hkv=4, d=128, lo=512, hi=2048, paged=1, block=16, packed=0,
              rot=128, axes=1, order="blocks", pairing="halves", tree=1),
        # prompts of very different lengths, packed, with images: positions of three axes
        _case("append prompts packed", "append", dtype="bf16", B=12, T=4096, Hq=28, Hkv=4, d=128, lo=0, hi=512, paged=1, block=64, packed=1,
              rot=128, axes=3, order="blocks", pairing="halves", tree=0),
        # trees of a model kept in fp32, heads of 64 channels, a contiguous cache, half of each head rotated
        _case("append trees fp32", "append", dtype="f32", B=4, T=31, Hq=8, Hkv=2, d=64, lo=100, hi=600, paged=0, block=16, packed=0,
              rot=32, axes=1, order="blocks", pairing="adjacent", tree=1),
        # a few users who ask about the same image, one token at a time
        _case("shared one token", "shared", dtype="bf16", B=4, T=1, Hq=28, Hkv=4, d=128, prefix=1696, lo=16, hi=128, paged=1, block=16, mask=0),
        # a full server behind one long system prompt with images: short trees
        _case("shared batch trees", "shared", dtype="bf16", B=64, T=4, Hq=28, Hkv=4, d=128, prefix=8192, lo=64, hi=512, paged=1, block=16, mask=1),
        # a multi-head model, one token each: the shared keys are read once instead of 32 times
        _case("shared batch multi-head", "shared", dtype="bf16", B=32, T=1, Hq=32, Hkv=32, d=128, prefix=4099, lo=33, hi=300, paged=0, block=16,
              mask=0),
        # whole draft trees of sixteen sequences: as much arithmetic as there is
        _case("shared large trees", "shared", dtype="bf16", B=16, T=60, Hq=28, Hkv=4, d=128, prefix=6684, lo=32, hi=700, paged=1, block=16, mask=1),
        # fp32 storage: checking a bf16 deployment
        _case("shared fp32", "shared", dtype="f32", B=6, T=5, Hq=8, Hkv=2, d=128, prefix=601, lo=0, hi=90, paged=0, block=16, mask=1),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.499)))))))


def _rotation(rng, d, dtype):
    axes = rng.choice([1, 1, 2, 3, 3])
    return dict(rot=rng.choice([d, d, d // 2, 16]), axes=axes, order=rng.choice(["blocks", "cyclic"]), pairing=rng.choice(["halves", "halves", "adjacent"]))


def draw(rng):
    kind = rng.choice(["rope", "append", "append", "shared", "shared", "shared"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "rope":
        H, d = rng.choice([1, 4, 8, 16, 28, 32, 36]), rng.choice([64, 96, 128])
        rows = _log(rng, 1, max(1, min(16384, 32_000_000 // (H * d))))
        return dict(kind=kind, dtype=dtype, rows=rows, H=H, d=d, **_rotation(rng, d, dtype), inverse=rng.choice([0, 0, 1]),
                    far=rng.choice([0, 0, 1000, 100000, 1000000]))
    Hq, Hkv, d = rng.choice(HEADS)
    c = dict(kind=kind, dtype=dtype, Hq=Hq, Hkv=Hkv, d=d, paged=rng.choice([0, 1, 1]), block=rng.choice([16, 16, 32, 64]))
    if kind == "append":
        packed = rng.choice([0, 1])
        tree = 0 if packed else rng.choice([0, 1])
        B = _log(rng, 1, 64)
        most = min(64 if tree else 4096, 12_000_000 // (B * (Hq + 2 * Hkv) * d))
        T = _log(rng, 1, max(1, most))
        hi = _log(rng, 16, max(16, min(4096, 60_000_000 // (B * Hkv * d))))
        c.update(B=B, T=T, lo=rng.choice([0, hi // 4, hi]), hi=hi, packed=packed, tree=tree, **_rotation(rng, d, dtype))
        if tree:
            c["axes"] = 1
        return c
    B, T = _log(rng, 2, 64), rng.choice([1, 1, 1, _log(rng, 2, 64)])
    if dtype == "f32":
        T = min(T, 8)
        B = min(B, 16)
    rows = B * T * Hq
    prefix = _log(rng, 64, max(64, min(16384, (170_000_000 if dtype == "bf16" else 4_000_000) // rows, 120_000_000 // (Hkv * d))))
    hi = _log(rng, 1, max(1, min(1024, prefix, 40_000_000 // (B * Hkv * d))))
    c.update(B=B, T=T, prefix=prefix, lo=rng.choice([0, hi // 8, hi // 2]), hi=hi, mask=rng.choice([0, 1]))
    return c


# ------------------------------------------------------------------------------- inputs


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _axis_pairs(axes, pairs):
    """Pairs of each axis: a quarter for time and the rest for height and width, or halves, or all."""
    if axes == 1:
        return [pairs]
    if axes == 2:
        return [pairs - pairs // 2, pairs // 2]
    w = pairs * 3 // 8
    return [pairs - 2 * w, w, w]


def _axis_of_pair(axes, pairs, order):
    counts = _axis_pairs(axes, pairs)
    if order == "blocks":
        return np.repeat(np.arange(axes), counts)
    a = np.zeros(pairs, dtype=np.int64)  # round robin as long as an axis has pairs left, the rest is the first axis
    for i in range(pairs):
        x = i % axes
        a[i] = x if i // axes < counts[x] else 0
    return a


def _order(c):
    # round robin gives axis x its k-th pair at k * axes + x: short heads have no room for that many
    counts = _axis_pairs(c["axes"], c["rot"] // 2)
    fits = all((n - 1) * c["axes"] + x < c["rot"] // 2 for x, n in enumerate(counts) if x > 0)
    return "cyclic" if c["order"] == "cyclic" and fits else "blocks"


def _grid_positions(r, rows, axes, start):
    """Positions of a prompt: some text, an image (one time step, a grid of height x width), text behind it."""
    p = np.empty((axes, rows), dtype=np.int32)
    p[:] = start + np.arange(rows)
    if axes > 1 and rows >= 16:
        text = int(r.integers(0, rows // 4 + 1))
        w = max(1, int(math.sqrt(rows / 2)))
        h = max(1, min((rows - text) // w, 2 * w))
        at = np.arange(h * w)
        p[:, text:text + h * w] = start + text
        p[axes - 2, text:text + h * w] += (at // w).astype(np.int32)
        p[axes - 1, text:text + h * w] += (at % w).astype(np.int32)
        rest = text + h * w
        p[:, rest:] = start + text + max(h, w) + np.arange(rows - rest)
    return p


def _lengths(B, T):
    """New tokens of a batch of prompts: spread over their logarithm up to T, and one in eight sequences has none."""
    n = np.exp(np.linspace(0, math.log(T), B) if B > 1 else np.array([math.log(T)])) + 1e-9
    n[:B // 8] = 0
    return n.astype(np.int64)


def _tree(r, T):
    """parent[] and depth[] of a random tree in which every node comes behind its parent."""
    parent, depth = np.full(T, -1, dtype=np.int32), np.zeros(T, dtype=np.int32)
    for i in range(1, T):
        parent[i] = int(r.integers(max(0, i - 12), i))
        depth[i] = depth[parent[i]] + 1
    return parent, depth


def _randn(g, shape, dtype, scale=1.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=dtype)
    return x.mul_(scale) if scale != 1.0 else x


def _frequencies(rot):
    return _dev(THETA ** (-np.arange(0, rot, 2, dtype=np.float64) / rot))


def _cache(r, g, c, slots, most, extra_rows=0):
    """K and V caches with room for slots[b] tokens of each sequence; paged: blocks in random order."""
    B, Hkv, d, bs = c["B"], c["Hkv"], c["d"], c["block"]
    s = {}
    if c["paged"]:
        nblk = (slots.astype(np.int64) + bs - 1) // bs
        row = (most + bs - 1) // bs
        shared = (extra_rows + bs - 1) // bs
        pool = B * row + shared + 2
        ids = r.permutation(pool).astype(np.int32)
        table = np.zeros((B, row), dtype=np.int32)
        table[np.arange(row)[None, :] < nblk[:, None]] = ids[shared:shared + int(nblk.sum())]
        s["table"], s["shared_table"] = _dev(table), _dev(ids[:shared])
        shape = (pool, Hkv, bs, d)
    else:
        shape = (B, Hkv, most, d)
    s["k"], s["v"] = _randn(g, shape, _dtype(c)), _randn(g, shape, _dtype(c))
    if extra_rows and not c["paged"]:
        s["k_shared"], s["v_shared"] = _randn(g, (Hkv, extra_rows, d), _dtype(c)), _randn(g, (Hkv, extra_rows, d), _dtype(c))
    return s


def prepare(case, seed):
    c = dict(case)
    r = np.random.default_rng(seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dtype(c)
    s = {"case": c}
    if c["kind"] != "shared":
        c["order"] = _order(c)
        s["inv_freq"] = _frequencies(c["rot"])
        s["axis"] = _dev(_axis_of_pair(c["axes"], c["rot"] // 2, c["order"]))
    if c["kind"] == "rope":
        # the heads lie in the rows of a wider projection, as queries and keys in front of the values
        s["x"] = _randn(g, (c["rows"], c["H"] + 2, c["d"]), dt)[:, :c["H"]]
        start = int(r.integers(0, c["far"] + 1)) + (c["far"] // 2)
        s["positions"] = _dev(_grid_positions(r, c["rows"], c["axes"], start))
        s["out"] = torch.zeros((c["rows"], c["H"], c["d"]), device="cuda", dtype=dt)
    elif c["kind"] == "append":
        B, T, Hq, Hkv, d = c["B"], c["T"], c["Hq"], c["Hkv"], c["d"]
        lens = r.integers(c["lo"], c["hi"] + 1, size=B).astype(np.int32)
        count = np.full(B, T, dtype=np.int64)
        if c["packed"]:
            count = r.permutation(_lengths(B, T))
        start = np.concatenate([[0], np.cumsum(count)]).astype(np.int32)
        rows = int(start[-1])
        total = rows + (5 if c["packed"] else 0)  # a buffer of a fixed size: rows behind the last sequence
        s.update(_cache(r, g, c, lens + count.astype(np.int32), c["hi"] + T))
        fused = _randn(g, (total, Hq + 2 * Hkv, d), dt)
        s["q"], s["knew"], s["vnew"] = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
        s["rows"], s["total"] = rows, total
        s["row_start"] = _dev(start)
        s["prefix"] = _dev(lens)
        s["q_out"] = torch.zeros((total, Hq, d), device="cuda", dtype=dt)
        s["positions"] = s["depth"] = None
        # text behind an image: its positions are not its slots
        s["offset"] = _dev(r.integers(-min(c["lo"], 200), 1, size=B).astype(np.int32))
        if c["tree"]:
            s["depth"] = _dev(np.stack([_tree(r, T)[1] for _ in range(B)]))
        elif c["axes"] > 1:
            p = np.zeros((c["axes"], total), dtype=np.int32)
            for b in range(B):
                p[:, start[b]:start[b + 1]] = _grid_positions(r, int(count[b]), c["axes"], int(lens[b]))
            s["positions"] = _dev(p)
    else:
        B, T, Hq, Hkv, d = c["B"], c["T"], c["Hq"], c["Hkv"], c["d"]
        lens = r.integers(c["lo"], c["hi"] + 1, size=B).astype(np.int32)
        s.update(_cache(r, g, c, lens + T, c["hi"] + T, c["prefix"]))
        s["q"] = _randn(g, (B, T, Hq, d), dt, 2.0)
        s["lens"] = _dev(lens)
        s["shared_len"] = _dev(np.array([c["prefix"]], dtype=np.int32))
        parent = np.stack([_tree(r, T)[0] for _ in range(B)])
        mask = np.zeros((B, T), dtype=np.uint64)
        for i in range(T):
            mask[:, i] = np.uint64(1) << np.uint64(i)
            if i:
                mask[:, i] |= mask[np.arange(B), parent[:, i]]
        s["parent"], s["tree_mask"] = _dev(parent), _dev(mask.view(np.int64))
        s["out"] = torch.zeros((B, T, Hq, d), device="cuda", dtype=dt)
    if own:
        s["call"] = _handles(s)
    return s


# ------------------------------------------------------------------------------- the library's calls


def _check(rc):
    if rc != 0:
        import paper_2509_15235_amd as vs

        raise vs.VSError(rc, "libvispec_verify")


def _rope_desc(vs, s):
    c = s["case"]
    desc = vs.RopeDesc(rot_dim=c["rot"], pairing=vs.VS_PAIR_HALVES if c["pairing"] == "halves" else vs.VS_PAIR_ADJACENT, num_axes=c["axes"],
                       axis_order=vs.VS_AXES_BLOCKS if c["order"] == "blocks" else vs.VS_AXES_CYCLIC, inverse=c.get("inverse", 0),
                       inv_freq=s["inv_freq"].data_ptr())
    for i, n in enumerate(_axis_pairs(c["axes"], c["rot"] // 2)):
        desc.axis_pairs[i] = n
    if s["positions"] is not None:
        desc.stride_axis = s["positions"].shape[1]
    return desc


def _cache_layout(desc, s):
    c, k = s["case"], s["k"]
    if c["paged"]:
        desc.paged, desc.block_size, desc.num_blocks = 1, c["block"], k.shape[0]
        desc.max_blocks, desc.block_table = s["table"].shape[1], s["table"].data_ptr()
        desc.stride_block, desc.stride_head, desc.stride_tok = k.stride(0), k.stride(1), k.stride(2)
    else:
        desc.capacity = k.shape[2]
        desc.stride_seq, desc.stride_head, desc.stride_tok = k.stride(0), k.stride(1), k.stride(2)


def _handles(s):
    """Descriptors, status and workspace: what a program makes once and keeps."""
    import paper_2509_15235_amd as vs

    c = s["case"]
    code = vs.VS_F32 if c["dtype"] == "f32" else vs.VS_BF16
    if c["kind"] == "rope":
        return vs.vs_rope_apply, _rope_desc(vs, s), code
    status = torch.zeros((c["B"],), device="cuda", dtype=torch.int32)
    if c["kind"] == "append":
        desc = vs.AppendDesc(B=c["B"], T=c["T"], Hq=c["Hq"], Hkv=c["Hkv"], d=c["d"], dtype=code, rows=s["total"], q_stride=s["q"].stride(0),
                             k_stride=s["knew"].stride(0), v_stride=s["vnew"].stride(0), q_out_stride=s["q_out"].stride(0))
        _cache_layout(desc, s)
        return vs.vs_kv_append, desc, _rope_desc(vs, s), status
    desc = vs.AttnDesc(B=c["B"], T=c["T"], Hq=c["Hq"], Hkv=c["Hkv"], d=c["d"], dtype=code, softmax_scale=1.0 / math.sqrt(c["d"]), max_prefix_len=c["hi"])
    _cache_layout(desc, s)
    prefix = vs.PrefixDesc(max_len=c["prefix"])
    if c["paged"]:
        prefix.paged, prefix.block_size, prefix.num_blocks = 1, c["block"], s["k"].shape[0]
        prefix.max_blocks, prefix.block_table = s["shared_table"].shape[0], s["shared_table"].data_ptr()
        prefix.stride_block, prefix.stride_head, prefix.stride_tok = s["k"].stride(0), s["k"].stride(1), s["k"].stride(2)
    else:
        prefix.capacity, prefix.stride_head, prefix.stride_tok = c["prefix"], s["k_shared"].stride(0), s["k_shared"].stride(1)
    nbytes = vs.vs_shared_prefix_workspace_bytes(desc, prefix)
    return vs.vs_shared_prefix_attention, desc, prefix, status, torch.empty(max(nbytes, 256), device="cuda", dtype=torch.uint8), nbytes


def _run_own(s):
    c = s["case"]
    stream = torch.cuda.current_stream().cuda_stream
    if c["kind"] == "rope":
        call, rope, code = s["call"]
        x, out = s["x"], s["out"]
        _check(call(rope, x, x.stride(0), x.stride(1), s["positions"], c["rows"], c["H"], c["d"], code, out, out.stride(0), out.stride(1), stream))
        return [out]
    if c["kind"] == "append":
        call, desc, rope, status = s["call"]
        _check(call(desc, rope, s["q"], s["knew"], s["vnew"], s["positions"], s["depth"], s["offset"], s["prefix"],
                    s["row_start"] if c["packed"] else None, s["q_out"], s["k"], s["v"], status, stream))
        return [s["q_out"], s["k"], s["v"]]
    call, desc, prefix, status, ws, nbytes = s["call"]
    ks, vsh = (s["k"], s["v"]) if c["paged"] else (s["k_shared"], s["v_shared"])
    _check(call(desc, prefix, s["q"], ks, vsh, s["shared_len"], s["k"], s["v"], s["lens"], s["parent"], s["tree_mask"] if c["mask"] else None,
                s["out"], status, ws, nbytes, stream))
    return [s["out"]]


# ------------------------------------------------------------------------------- plain forms


def _rotate(x, cos, sin, rot, pairing):
    """x [rows, H, d] in 32 bits, cos and sin [rows, rot / 2]."""
    cos, sin = cos[:, None, :], sin[:, None, :]
    if pairing == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _cos_sin(s, positions):
    """positions [axes, rows]: each pair takes the angle of its axis; in 64 bits, since positions lie far out."""
    angle = positions.double()[s["axis"]].T * s["inv_freq"]
    if s["case"].get("inverse"):
        angle = -angle
    return angle.cos().float(), angle.sin().float()


def _run_rope(s):
    c = s["case"]
    cos, sin = _cos_sin(s, s["positions"])
    s["out"].copy_(_rotate(s["x"].float(), cos, sin, c["rot"], c["pairing"]))
    return [s["out"]]


def _run_append(s):
    c = s["case"]
    rows, T = s["rows"], c["T"]
    at = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(s["row_start"][1:].contiguous(), at.int(), right=True)
    i = at - s["row_start"][seq]
    slot = s["prefix"][seq] + i
    if s["positions"] is not None:
        positions = s["positions"][:, :rows]
    else:
        step = i if s["depth"] is None else s["depth"].reshape(-1)
        positions = (s["prefix"][seq] + s["offset"][seq] + step)[None, :].expand(c["axes"], rows)
    cos, sin = _cos_sin(s, positions)
    s["q_out"][:rows] = _rotate(s["q"][:rows].float(), cos, sin, c["rot"], c["pairing"]).to(s["q_out"].dtype)
    k = _rotate(s["knew"][:rows].float(), cos, sin, c["rot"], c["pairing"]).to(s["k"].dtype)
    if c["paged"]:
        where, within = s["table"][seq, slot // c["block"]].long(), slot % c["block"]
    else:
        where, within = seq, slot
    s["k"][where, :, within] = k
    s["v"][where, :, within] = s["vnew"][:rows]
    return [s["q_out"], s["k"], s["v"]]


def _run_shared(s):
    c = s["case"]
    B, T, Hq, Hkv, d, P = c["B"], c["T"], c["Hq"], c["Hkv"], c["d"], c["prefix"]
    G, scale, most = Hq // Hkv, 1.0 / math.sqrt(d), c["hi"] + T
    if c["paged"]:
        ks, vs_ = (x[s["shared_table"]].transpose(0, 1).reshape(Hkv, -1, d)[:, :P] for x in (s["k"], s["v"]))
        ko, vo = (x[s["table"]].transpose(1, 2).reshape(B, Hkv, -1, d)[:, :, :most] for x in (s["k"], s["v"]))
    else:
        ks, vs_, ko, vo = s["k_shared"], s["v_shared"], s["k"], s["v"]
    ks, vs_, ko, vo = ks.float(), vs_.float(), ko.float(), vo.float()
    # which of a sequence's own slots node i sees: its prefix, and its ancestors and itself behind it
    at = torch.arange(most, device="cuda")[None, :] - s["lens"][:, None]
    node = at.clamp(0, T - 1)
    ancestor = (s["tree_mask"][:, :, None] >> node[:, None, :]) & 1
    sees = ((at < 0)[:, None, :] | ((at < T)[:, None, :] & (ancestor != 0)))  # [B, T, most]
    vo = torch.where((at < T)[:, None, :, None], vo, 0.0)
    q = s["q"].float().reshape(B, T, Hkv, G, d)
    first = torch.matmul(q.permute(2, 0, 1, 3, 4).reshape(Hkv, B * T * G, d), ks.transpose(1, 2).contiguous()) * scale
    second = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, d), ko.transpose(2, 3).contiguous()) * scale
    second = second.reshape(B, Hkv, T, G, most).masked_fill(~sees[:, None, :, None, :], -math.inf)
    top1 = first.amax(-1).reshape(Hkv, B, T, G).permute(1, 0, 2, 3)
    top = torch.maximum(top1, second.amax(-1))  # [B, Hkv, T, G]
    first = torch.exp(first - top.permute(1, 0, 2, 3).reshape(Hkv, B * T * G, 1))
    second = torch.exp(second - top[..., None])
    total = first.sum(-1).reshape(Hkv, B, T, G).permute(1, 0, 2, 3) + second.sum(-1)
    out = torch.matmul(first, vs_.contiguous()).reshape(Hkv, B, T, G, d).permute(1, 0, 2, 3, 4)
    out = out + torch.matmul(second.reshape(B, Hkv, T * G, most), vo.contiguous()).reshape(B, Hkv, T, G, d)
    out = out / total[..., None]
    s["out"].copy_(out.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, d))
    return [s["out"]]


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    return _run_rope(state) if kind == "rope" else _run_append(state) if kind == "append" else _run_shared(state)


# ------------------------------------------------------------------------------- definitions in 64 bits


def _turned(x, positions, freq, axis, c):
    """Each pair of channels as a complex number, times exp(i angle)."""
    rot, x = c["rot"], x.double()
    if c["pairing"] == "halves":
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous())
    else:
        z = torch.complex(x[..., 0:rot:2].contiguous(), x[..., 1:rot:2].contiguous())
    angle = torch.stack([positions[a].double() * f for a, f in zip(axis.tolist(), freq.tolist())], dim=-1)
    if c.get("inverse"):
        angle = -angle
    z = z * torch.polar(torch.ones_like(angle), angle)[:, None, :]
    y = x.clone()
    if c["pairing"] == "halves":
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["kind"] == "rope":
        return [_turned(s["x"], s["positions"], s["inv_freq"], s["axis"], c)]
    if c["kind"] == "append":
        start, lens, offset = s["row_start"].tolist(), s["prefix"].tolist(), s["offset"].tolist()
        q, k, v = s["q_out"].double(), s["k"].double(), s["v"].double()
        for b in range(c["B"]):
            n = start[b + 1] - start[b]
            if n == 0:
                continue
            at = slice(start[b], start[b + 1])
            if s["positions"] is not None:
                p = s["positions"][:, at]
            else:
                step = torch.arange(n, device="cuda") if s["depth"] is None else s["depth"][b]
                p = (lens[b] + offset[b] + step).expand(c["axes"], n)
            q[at] = _turned(s["q"][at], p, s["inv_freq"], s["axis"], c)
            kr = _turned(s["knew"][at], p, s["inv_freq"], s["axis"], c)
            t = lens[b] + torch.arange(n, device="cuda")
            where, within = (s["table"][b].long()[t // c["block"]], t % c["block"]) if c["paged"] else (torch.full_like(t, b), t)
            k[where, :, within] = kr
            v[where, :, within] = s["vnew"][at].double()
        return [q, k, v]
    B, T, Hq, Hkv, d, P = c["B"], c["T"], c["Hq"], c["Hkv"], c["d"], c["prefix"]
    lens, parent = s["lens"].tolist(), s["parent"].cpu().numpy()
    out = torch.empty((B, T, Hq, d), device="cuda", dtype=torch.float64)

    def rows(x, shared, b, n):  # [Hkv, n, d] of a shared prefix or a sequence's own cache
        if not c["paged"]:
            return x[:, :n] if shared else x[b, :, :n]
        t = torch.arange(n, device="cuda")
        table = s["shared_table"] if shared else s["table"][b]
        return x[table.long()[t // c["block"]], :, t % c["block"]].transpose(0, 1)

    ks, vs_ = ((s["k"], s["v"]) if c["paged"] else (s["k_shared"], s["v_shared"]))
    ks, vs_ = rows(ks, True, 0, P).double(), rows(vs_, True, 0, P).double()
    for b in range(B):
        n = lens[b] + T
        k = torch.cat([ks, rows(s["k"], False, b, n).double()], dim=1)
        v = torch.cat([vs_, rows(s["v"], False, b, n).double()], dim=1)
        hidden = np.zeros((T, P + n), dtype=bool)
        for i in range(T):
            hidden[i, P + lens[b]:] = True
            j = i
            while j >= 0:
                hidden[i, P + lens[b] + j] = False
                j = int(parent[b, j])
        q = s["q"][b].double().transpose(0, 1).reshape(Hkv, Hq // Hkv * T, d)  # [Hkv, (head, node), d]
        w = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        w = w.reshape(Hkv, Hq // Hkv, T, P + n).masked_fill(_dev(hidden), -math.inf).softmax(dim=-1)
        o = torch.matmul(w.reshape(Hkv, Hq // Hkv * T, P + n), v.contiguous())
        out[b] = o.reshape(Hq, T, d).transpose(0, 1)
    return [out]


# ------------------------------------------------------------------------------- work


def work(case):
    c = case
    eb = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "rope":
        n = c["rows"] * c["H"]
        return {"bytes": 2.0 * n * c["d"] * eb + 4.0 * c["axes"] * c["rows"], "flops": 3.0 * n * c["rot"]}
    if c["kind"] == "append":
        rows = float(_lengths(c["B"], c["T"]).sum()) if c["packed"] else c["B"] * c["T"]
        return {"bytes": 2.0 * rows * (c["Hq"] + 2 * c["Hkv"]) * c["d"] * eb, "flops": 3.0 * rows * (c["Hq"] + c["Hkv"]) * c["rot"]}
    B, T, own_keys = c["B"], c["T"], (c["lo"] + c["hi"]) / 2
    keys = c["prefix"] + B * (own_keys + T)
    sees = c["prefix"] + own_keys + min(T, 4)
    return {"bytes": (2.0 * c["Hkv"] * keys + 2.0 * B * T * c["Hq"]) * c["d"] * eb, "flops": 4.0 * c["d"] * c["Hq"] * B * T * sees}
