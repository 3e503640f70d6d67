"""Refusals of vs_rope_apply and vs_kv_append, and their descriptors: found on the host, without a GPU."""
import ctypes

import numpy as np
import pytest

import paper_2509_15235_amd as vs
import rope_util as ru
from paper_2509_15235_amd import binding

G = 1 << 20  # an address that nothing reads: every call here is refused first, or finds no device


def _ok(rc):
    return rc in (0, -7)


def _rope(**kw):
    d = ru.rope_desc(128, counts=[16, 24, 24], stride_axis=100, inv_freq=G)
    for k, v in kw.items():
        if k == "axis_pairs":
            for i, n in enumerate(v):
                d.axis_pairs[i] = n
        else:
            setattr(d, k, v)
    return d


def _apply(rope=None, x=G, xr=36 * 128, xh=128, pos=G, rows=100, H=32, d=128, dtype=vs.VS_BF16, out=2 * G, orow=32 * 128, oh=128):
    return vs.vs_rope_apply(rope if rope is not None else _rope(), x, xr, xh, pos, rows, H, d, dtype, out, orow, oh, None)


@pytest.mark.parametrize("kw,code", [
    ({"rot_dim": -16}, -2), ({"rot_dim": 144}, -2), ({"rot_dim": 24, "num_axes": 1}, -6), ({"rot_dim": 8, "num_axes": 1}, -6),
    ({"rot_dim": 8, "num_axes": 1, "pairing": 1, "inv_freq": None}, -1), ({"rot_dim": 4, "num_axes": 1, "pairing": 1}, -6),
    ({"pairing": 2}, -2), ({"pairing": -1}, -2), ({"axis_order": 2}, -2), ({"num_axes": 0}, -2), ({"num_axes": 5}, -2),
    ({"axis_pairs": [16, 24, 23]}, -2), ({"axis_pairs": [-8, 48, 24]}, -2), ({"axis_pairs": [65, -1, 0]}, -2),
    ({"axis_pairs": [0, 0, 64], "axis_order": 1}, -2), ({"axis_pairs": [21, 22, 21], "axis_order": 1}, -2),
    ({"stride_axis": -1}, -6), ({"inv_freq": None}, -1),
])
def test_rotation_descriptor(kw, code):
    assert _apply(_rope(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    ({"x": None}, -1), ({"pos": None}, -1), ({"out": None}, -1), ({"rows": 0}, -2), ({"rows": 1 << 31}, -2), ({"H": 0}, -2), ({"H": 65537}, -2),
    ({"d": 0}, -2), ({"d": 264}, -2), ({"d": 132}, -6), ({"dtype": 2}, -3), ({"x": G + 8}, -6), ({"out": G + 2}, -6),
    ({"xr": 36 * 128 + 4}, -6), ({"xh": 132}, -6), ({"xr": -128}, -6), ({"orow": 127 * 32}, -6), ({"oh": 120}, -6), ({"oh": 1 << 62}, -6),
    ({"orow": 0}, -6), ({"out": G}, -6),
])
def test_rotation_arguments(kw, code):
    assert _apply(**kw) == code


def test_rotations_that_are_taken():
    if not _no_device():
        pytest.skip("would run on this device")
    assert _apply() == -7
    assert _apply(_rope(axis_pairs=[22, 21, 21], axis_order=1)) == -7
    assert _apply(_rope(rot_dim=0, num_axes=1, inv_freq=None)) == -7
    assert _apply(out=G, orow=36 * 128) == -7
    assert _apply(xr=0, xh=0) == -7  # one row for all heads


def _no_device():
    import torch
    return not torch.cuda.is_available()


def _append(rope=None, q=G, k=2 * G, v=3 * G, positions=None, depth=None, offset=None, prefix=G, row_start=None, q_out=4 * G, kc=5 * G, vc=6 * G, **kw):
    d = vs.AppendDesc(B=4, T=60, Hq=28, Hkv=4, d=128, dtype=vs.VS_BF16, rows=240, q_stride=36 * 128, k_stride=36 * 128, v_stride=36 * 128,
                      q_out_stride=28 * 128, capacity=2000, stride_seq=4 * 2000 * 128, stride_head=2000 * 128, stride_tok=128)
    for name, x in kw.items():
        setattr(d, name, x)
    return vs.vs_kv_append(d, rope if rope is not None else ru.rope_desc(128, inv_freq=G), q, k, v, positions, depth, offset, prefix, row_start, q_out, kc, vc,
                           None, None)


PAGED = dict(paged=1, block_size=16, max_blocks=130, num_blocks=600, stride_block=4 * 16 * 128, stride_head=16 * 128, block_table=G)


@pytest.mark.parametrize("kw,code", [
    ({"q": None}, -1), ({"k": None}, -1), ({"v": None}, -1), ({"prefix": None}, -1), ({"q_out": None}, -1), ({"kc": None}, -1), ({"vc": None}, -1),
    ({"B": 0}, -2), ({"T": 0}, -2), ({"Hq": -1}, -2), ({"Hkv": 0}, -2), ({"d": 0}, -2), ({"d": 257}, -2), ({"dtype": 3}, -3), ({"rows": 0}, -2),
    ({"rows": 239}, -2), ({"rows": 1 << 31, "row_start": G}, -2), ({"row_start": G, "depth": G}, -2), ({"Hkv": 65537}, -2),
    ({"q_stride": 27 * 128}, -6), ({"q_out_stride": 27 * 128}, -6), ({"k_stride": 3 * 128}, -6), ({"v_stride": 3 * 128}, -6), ({"q_out": G}, -6),
    ({"k_stride": 36 * 128 + 4}, -6), ({"stride_tok": 64}, -6), ({"stride_tok": 132}, -6), ({"stride_head": -8}, -6), ({"stride_seq": -8}, -6),
    ({"stride_head": 0}, -6), ({"stride_seq": 0}, -6), ({"stride_seq": 3 * 2000 * 128}, -6), ({"stride_head": 1999 * 128}, -6),
    ({"capacity": 59}, -6), ({"capacity": 0}, -6), ({"q": G + 2}, -6), ({"k": G + 8}, -6), ({"v": G + 4}, -6), ({"kc": G + 8}, -6), ({"vc": G + 8}, -6),
    (dict(PAGED, block_size=24), -6), (dict(PAGED, block_size=8), -6), (dict(PAGED, max_blocks=3), -6), (dict(PAGED, num_blocks=0), -6),
    (dict(PAGED, stride_block=0), -6), (dict(PAGED, stride_head=15 * 128), -6),
    (dict(PAGED, block_table=None), -1), (dict(PAGED, stride_block=4 * 16 * 128 + 2), -6),
])
def test_append_arguments(kw, code):
    assert _append(**kw) == code


def test_appends_that_are_taken_and_inverse():
    assert _append(ru.rope_desc(128, inverse=1, inv_freq=G)) == -2
    if not _no_device():
        pytest.skip("would run on this device")
    assert _append() == -7 and _append(**PAGED) == -7
    assert _append(Hq=0, q=None, q_out=None) == -7
    assert _append(q_out=G, q_out_stride=36 * 128) == -7
    assert _append(row_start=G, rows=17) == -7
    assert _append(ru.rope_desc(0)) == -7


def test_status_and_definition():
    assert vs.vs_status_string(7).startswith("row_start")
    assert ru.axis_of_pair(8, [2, 3, 3], False) == [0, 0, 1, 1, 1, 2, 2, 2]
    assert ru.axis_of_pair(8, [4, 2, 2], True) == [0, 1, 2, 0, 1, 2, 0, 0]


def test_descriptors_as_in_the_header():
    """Sizes as a C compiler lays the header's structs out."""
    assert ctypes.sizeof(vs.RopeDesc) == 56 and vs.RopeDesc.stride_axis.offset == 40
    assert ctypes.sizeof(vs.AppendDesc) == 128 and vs.AppendDesc.rows.offset == 24 and vs.AppendDesc.capacity.offset == 80


@pytest.mark.parametrize("name", binding._NATIVE_MORE)
def test_python_calls_pass_their_arguments_on(name):
    """Every parameter in its place and width, structures by reference."""
    types = getattr(vs.lib(), name).argtypes
    structs = [t._type_ if hasattr(t, "_type_") and isinstance(t._type_, type) and issubclass(t._type_, ctypes.Structure) else None for t in types]
    seen = []

    def body(*a):
        seen.append([0 if x is None else x for x in a])
        return 41
    cb = ctypes.CFUNCTYPE(ctypes.c_int32, *[ctypes.c_void_p if s else t for s, t in zip(structs, types)])(body)
    binding._native.bind({name: ctypes.cast(cb, ctypes.c_void_p).value})
    try:
        args = [s() if s else np.float32(0.5) if t is ctypes.c_float else 1000 + 16 * i for i, (s, t) in enumerate(zip(structs, types))]
        assert getattr(vs, name)(*args) == 41
        want = [ctypes.addressof(a) if s else float(a) if t is ctypes.c_float else a for s, t, a in zip(structs, types, args)]
        assert seen[-1] == want
        for i, s in enumerate(structs):
            for wrong in (None, 4096, vs.KVDesc()) if s else ():
                with pytest.raises((TypeError, ctypes.ArgumentError)):
                    getattr(vs, name)(*args[:i], wrong, *args[i + 1:])
        with pytest.raises(TypeError):
            getattr(vs, name)(*args, 1)
    finally:
        binding._load_native()


def test_one_cache_for_keys_and_values():
    assert _append(kc=5 * G, vc=5 * G) == -6
