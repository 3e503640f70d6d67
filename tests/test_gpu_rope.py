"""vs_rope_apply against its definition in 64 bits: pairings, axes, types, strides, far positions, the rotation back and gradients."""
import numpy as np
import pytest
import torch

import gpu_util as gu
import paper_2509_15235_amd as vs
import rope_util as ru

pytestmark = pytest.mark.gpu


def _run(x, positions, desc, out, rows, H, d, stream=None):
    code = vs.VS_BF16 if x.dtype == torch.bfloat16 else vs.VS_F32
    rc = vs.vs_rope_apply(desc, x, x.stride(0), x.stride(1), positions, rows, H, d, code, out, out.stride(0), out.stride(1),
                          gu.stream_ptr() if stream is None else stream)
    assert rc == 0, vs.vs_strerror(rc)


def _case(rows, H, d, rot, bf16, halves, counts, cyclic, inverse, far, seed=0, wide=2):
    g = np.random.default_rng(seed)
    dt = torch.bfloat16 if bf16 else torch.float32
    x = torch.from_numpy(g.standard_normal((rows, H + wide, d)).astype(np.float32)).to(dt).cuda()[:, :H]
    axes = len(counts)
    pos = (far + g.integers(-40, 5000, size=(axes, rows))).astype(np.int32)
    freq = ru.frequencies(rot)
    dev = gu.dev(freq) if rot else None
    desc = ru.rope_desc(rot, halves, counts, cyclic, inverse, stride_axis=rows, inv_freq=dev.data_ptr() if rot else None)
    cos, sin = ru.cos_sin(pos, freq, ru.axis_of_pair(rot // 2, counts, cyclic), inverse)
    host = x.float().cpu().numpy()
    want = ru.rotate(host, cos, sin, rot, halves)
    return x, pos, dev, desc, host, want


@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("halves", [0, 1])
@pytest.mark.parametrize("rows,H,d,rot,counts,cyclic,inverse,far", [
    (1, 1, 64, 64, [32], 0, 0, 0), (1, 36, 128, 128, [64], 0, 0, 40000), (3, 5, 128, 128, [16, 24, 24], 0, 0, 0),
    (7, 4, 96, 48, [8, 8, 8], 1, 0, 100), (61, 32, 128, 128, [22, 21, 21], 1, 1, 0), (257, 28, 128, 64, [16, 16], 0, 1, 1 << 20),
    (2047, 9, 64, 16, [5, 3], 1, 0, 0), (1030, 3, 256, 256, [100, 12, 8, 8], 0, 0, 7), (300, 1, 128, 128, [64], 0, 0, (1 << 31) - 5001),
    (300, 2, 128, 128, [64], 0, 0, 41 - (1 << 31)), (5, 3, 64, 0, [0], 0, 0, 0), (4100, 2, 80, 32, [16], 0, 0, 3), (40, 2, 128, 128, [0, 64], 0, 0, 9),
])
def test_against_definition(rows, H, d, rot, counts, cyclic, inverse, far, bf16, halves):
    x, pos, dev, desc, host, want = _case(rows, H, d, rot, bf16, halves, counts, cyclic, inverse, far)
    out = torch.full((rows + 1, H, d), 7.0, device="cuda", dtype=x.dtype)
    p = gu.dev(pos)
    _run(x, p, desc, out[:rows], rows, H, d)
    torch.cuda.synchronize()
    got = out.float().cpu().numpy().astype(np.float64)
    err = np.abs(got[:rows] - want)
    # (the angle in 64 bits: 2^31 positions times 2^-52)
    most = ru.bound(host, want, rot, halves, bf16) + (5e-7 * np.abs(host).max() * 2 if abs(far) > 1 << 24 else 0)
    assert (err <= most).all(), (err - most).max()
    assert (got[rows] == 7.0).all()
    if d > rot:
        assert (got[:rows, :, rot:] == host[:, :, rot:]).all()


@pytest.mark.parametrize("bf16", [0, 1])
def test_in_place_other_order_and_one_position_for_all_axes(bf16):
    rows, H, d = 130, 6, 128
    x, pos, dev, desc, host, want = _case(rows, H, d, d, bf16, 1, [16, 24, 24], 0, 0, 0)
    pos[:] = pos[0]
    cos, sin = ru.cos_sin(pos, ru.frequencies(d), ru.axis_of_pair(d // 2, [16, 24, 24], 0))
    want = ru.rotate(host, cos, sin, d, True)
    desc.stride_axis = 0
    p = gu.dev(pos[0])
    heads_first = torch.full((H, rows + 3, d), 7.0, device="cuda", dtype=x.dtype)
    _run(x, p, desc, heads_first[:, :rows].transpose(0, 1), rows, H, d)
    rest = x._base[:, H:].clone()
    _run(x, p, desc, x, rows, H, d)
    torch.cuda.synchronize()
    assert torch.equal(heads_first[:, :rows].transpose(0, 1), x) and (heads_first[:, rows:] == 7.0).all() and torch.equal(x._base[:, H:], rest)
    assert (np.abs(x.float().cpu().numpy() - want) <= ru.bound(host, want, d, True, bf16)).all()


@pytest.mark.parametrize("halves", [0, 1])
def test_gradient_against_formula_and_differences(halves):
    """The loss sum(g * rotated(x)) is linear in x: its gradient by the formula is the rotation back of g, and a difference of the loss is exact
    up to the rounding of what it is made of."""
    rows, H, d, rot = 33, 3, 64, 32
    x, pos, dev, desc, host, want = _case(rows, H, d, rot, 0, halves, [8, 4, 4], 0, 0, 500)
    p = gu.dev(pos)
    g = torch.randn((rows, H, d), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    back = ru.rope_desc(rot, halves, [8, 4, 4], False, 1, stride_axis=rows, inv_freq=dev.data_ptr())
    grad = torch.empty_like(g)
    _run(g, p, back, grad, rows, H, d)
    cos, sin = ru.cos_sin(pos, ru.frequencies(rot), ru.axis_of_pair(rot // 2, [8, 4, 4], False), True)
    gh = g.cpu().numpy()
    formula = ru.rotate(gh, cos, sin, rot, halves)
    got = grad.cpu().numpy().astype(np.float64)
    assert (np.abs(got - formula) <= ru.bound(gh, formula, rot, halves, False)).all()
    r = np.random.default_rng(5)
    for _ in range(20):
        at = tuple(int(r.integers(n)) for n in (rows, H, d))
        losses = []
        for h in (-1.0, 1.0):
            y = x.clone()
            y[at] += h
            out = torch.empty_like(g)
            _run(y, p, desc, out, rows, H, d)
            losses.append((out[at[0], at[1]].double().cpu().numpy() * gh[at[0], at[1]]).sum())
        # every rotated value is off by at most 4.2e-7 of its pair, once in each loss; x + h rounds by half a unit of at most 8
        room = 2 * 4.2e-7 * (np.abs(gh[at[0], at[1]]) * 12.0).sum() + 2.0 ** -21 * np.abs(gh[at[0], at[1]]).max() * 2
        assert abs((losses[1] - losses[0]) / 2 - got[at]) <= room
    # there and back
    y = torch.empty_like(g)
    _run(grad, p, desc, y, rows, H, d)
    assert float((y - g).abs().max()) <= 2 * 4.2e-7 * float(g.abs().max()) * 3


def test_other_stream_and_captured():
    rows, H, d = 70, 8, 128
    x, pos, dev, desc, host, want = _case(rows, H, d, d, 1, 1, [64], 0, 0, 0)
    p, out, eager = gu.dev(pos), torch.zeros((rows, H, d), device="cuda", dtype=torch.bfloat16), torch.zeros((rows, H, d), device="cuda", dtype=torch.bfloat16)
    _run(x, p, desc, eager, rows, H, d)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        _run(x, p, desc, out, rows, H, d, stream=s.cuda_stream)
    for k in range(3):
        out.zero_()
        x.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager * 0.5 ** (k + 1))  # powers of two go through every rounding


def test_rows_that_go_past_the_caches_and_beyond_32_bits():
    """Results of over 4 MB, and rows that lie 2^26 elements apart: the last one begins beyond 2^32 bytes."""
    rows, H, d = 700, 32, 128
    x, pos, dev, desc, host, want = _case(rows, H, d, d, 1, 1, [16, 24, 24], 0, 0, 0)
    out = torch.full((rows + 1, H, d), 7.0, device="cuda", dtype=torch.bfloat16)
    _run(x, gu.dev(pos), desc, out[:rows], rows, H, d)
    torch.cuda.synchronize()
    assert (np.abs(out[:rows].float().cpu().numpy() - want) <= ru.bound(host, want, d, True, True)).all() and (out[rows] == 7.0).all()
    rows, H, d, apart = 40, 1, 64, 1 << 26
    x, pos, dev, desc, host, want = _case(rows, H, d, d, 1, 0, [32], 0, 0, 0)
    far = torch.empty(apart * (rows - 1) + d, device="cuda", dtype=torch.bfloat16).as_strided((rows, H, d), (apart, d, 1))
    far.copy_(x)
    _run(far, gu.dev(pos), desc, far, rows, H, d)
    torch.cuda.synchronize()
    assert (np.abs(far.float().cpu().numpy() - want) <= ru.bound(host, want, d, False, True)).all()


def test_more_rows_than_one_launch_takes():
    """2^25 rows and some of one head of four channels, on two axes, in place."""
    rows = (1 << 25) + 7
    x = torch.randn((rows, 1, 4), device="cuda", generator=torch.Generator("cuda").manual_seed(0))
    at = torch.cat([torch.arange(5), torch.arange((1 << 25) - 3, rows)])
    host = x[at.cuda()].cpu().numpy()
    pos = (torch.arange(2 * rows, device="cuda") % 1009).to(torch.int32).reshape(2, rows)
    freq = gu.dev(ru.frequencies(4))
    _run(x, pos, ru.rope_desc(4, False, [1, 1], stride_axis=rows, inv_freq=freq.data_ptr()), x, rows, 1, 4)
    torch.cuda.synchronize()
    cos, sin = ru.cos_sin(pos[:, at.cuda()].cpu().numpy(), ru.frequencies(4), ru.axis_of_pair(2, [1, 1], False))
    want = ru.rotate(host, cos, sin, 4, False)
    assert (np.abs(x[at.cuda()].cpu().numpy() - want) <= ru.bound(host, want, 4, False, False)).all()
