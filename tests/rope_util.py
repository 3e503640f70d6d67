"""Rotation and cache append from their definitions, in numpy (angles in extended precision, the rest in 64 bits), and descriptors."""
import numpy as np

import paper_2509_15235_amd as vs

THETA = 1e4


def frequencies(rot, theta=THETA):
    return theta ** (-np.arange(0, rot, 2, dtype=np.float64) / max(rot, 1))


def axis_of_pair(pairs, counts, cyclic):
    """Pair -> axis, from the definition: blocks one behind the other, or round robin while an axis (not the first) has pairs left."""
    if len(counts) == 1:
        return [0] * pairs
    if not cyclic:
        return [x for x, n in enumerate(counts) for _ in range(n)]
    given, axes = [0] * len(counts), []
    for i in range(pairs):
        x = i % len(counts)
        if x > 0 and given[x] == counts[x]:
            x = 0
        given[x] += 1
        axes.append(x)
    return axes


def cos_sin(positions, freq, axes, inverse=False):
    """positions [axes][rows] -> cos, sin [rows, pairs]"""
    p = np.stack([positions[a] for a in axes], axis=-1) if len(axes) else np.zeros((positions.shape[1], 0))
    angle = p.astype(np.longdouble) * freq.astype(np.longdouble)
    angle = -angle if inverse else angle
    return np.cos(angle).astype(np.float64), np.sin(angle).astype(np.float64)


def pair_index(rot, halves):
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if halves else (2 * i, 2 * i + 1)


def rotate(x, cos, sin, rot, halves):
    """x [rows, H, d] in 64 bits."""
    y = x.astype(np.float64).copy()
    a, b = pair_index(rot, halves)
    u, v = x[..., a].astype(np.float64), x[..., b].astype(np.float64)
    y[..., a] = u * cos[:, None, :] - v * sin[:, None, :]
    y[..., b] = v * cos[:, None, :] + u * sin[:, None, :]
    return y


def bound(x, want, rot, halves, bf16):
    """How far a rotated value may be off. fp32 arithmetic on a pair (u, v): the fraction of a turn is rounded once to 24 bits (at most 2^-25
    turns of half a turn's value, 2^-25 * 2 pi = 1.9e-7 radians), sine and cosine are off by 2 units in the 24th bit, two products and a
    sum by half a unit each: 1.9e-7 + 3.5 * 2^-24 < 4.2e-7 of |u| + |v|. bf16 storage: the hardware's functions of turns instead, 2^-18,
    and the result rounded once, half a step = 2^-8 of the value."""
    a, b = pair_index(rot, halves)
    size = np.zeros(x.shape)
    pair = np.abs(x[..., a].astype(np.float64)) + np.abs(x[..., b].astype(np.float64))
    size[..., a] = size[..., b] = pair
    if not bf16:
        return 4.2e-7 * size
    return (4.2e-7 + 2.0 ** -18) * size + 2.0 ** -8 * np.abs(want)


def rope_desc(rot, halves=True, counts=None, cyclic=False, inverse=0, stride_axis=0, inv_freq=None):
    d = vs.RopeDesc(rot_dim=rot, pairing=vs.VS_PAIR_HALVES if halves else vs.VS_PAIR_ADJACENT, num_axes=len(counts) if counts else 1,
                    axis_order=vs.VS_AXES_CYCLIC if cyclic else vs.VS_AXES_BLOCKS, inverse=inverse, stride_axis=stride_axis, inv_freq=inv_freq)
    for i, n in enumerate(counts or []):
        d.axis_pairs[i] = n
    return d
