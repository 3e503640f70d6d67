"""vs_kv_append where some sequences of a call are reported: the rows of the others, and those of a reported one that lie in good blocks, are where they
belong. Compared row by row, beside the tests that look at what stays untouched."""
import numpy as np
import pytest
import torch

from test_gpu_append import Setup

pytestmark = pytest.mark.gpu


def _rows_right(s, b, rows):
    """Rows `rows` (counted inside sequence b) of queries, keys and values."""
    torch.cuda.synchronize()
    q = s.q_out.float().cpu().numpy()
    k, v = s.caches()
    Hq, Hkv = s.Hq, s.Hkv
    for i in rows:
        r, t = int(s.start[b]) + i, s.lens[b] + i
        at = (s.table_host[b, t // s.block], t % s.block) if s.paged else (b, t)
        assert (np.abs(q[r] - s.want[r, :Hq]) <= s.most_off[r, :Hq]).all(), (b, i)
        assert (np.abs(k[at[0], :, at[1]] - s.want[r, Hq:Hq + Hkv]) <= s.most_off[r, Hq:Hq + Hkv]).all(), (b, i)
        assert (v[at[0], :, at[1]] == s.want[r, Hq + Hkv:]).all(), (b, i)
    return len(rows)


def _touched(s):
    """(block or sequence, slot)s that hold something new."""
    k, v = s.caches()
    new = (k != 3.0).any(axis=(1, 3)) | (v != 5.0).any(axis=(1, 3))
    return {(int(a), int(t)) for a, t in np.argwhere(new)}


def _slots(s, b, rows):
    return {(int(s.table_host[b, (s.lens[b] + i) // s.block]), (s.lens[b] + i) % s.block) if s.paged else (b, s.lens[b] + i) for i in rows}


@pytest.mark.parametrize("bf16", [1, 0])
@pytest.mark.parametrize("paged", [0, 1])
def test_beside_bad_lengths_and_blocks(paged, bf16):
    s = Setup([5, 20, 3, 4, 0], [10, 15, 7, 100, 3], paged=paged, bf16=bf16, offset=1)
    bad = s.prefix.cpu()
    bad[0], bad[2], bad[4] = -1, 1 << 30, -4
    s.prefix.copy_(bad)
    there = list(range(20))
    if paged:
        s.table[1, 1] = s.desc.num_blocks  # slots 16 .. 31: of sequence 1, row 0 lies in front of them and rows 17 .. 19 behind
        there = [0, 17, 18, 19]
    s.run()
    assert _rows_right(s, 3, range(4)) == 4
    assert _rows_right(s, 1, there) == len(there)
    assert s.status.cpu().tolist() == [3, 4 if paged else 0, 3, 0, 3]
    assert _touched(s) == _slots(s, 1, there) | _slots(s, 3, range(4))


@pytest.mark.parametrize("paged", [0, 1])
@pytest.mark.parametrize("row_start,want,good", [
    ([0, 5, 6, 10], [0, 0, 7], {0: 5, 1: 1}),        # the last one's rows leave the call's nine
    ([0, 5, 6, 1 << 30], [0, 0, 7], {0: 5, 1: 1}),
    ([0, 5, 6, (1 << 31) - 1], [0, 0, 7], {0: 5, 1: 1}),
    ([0, 0, 9, 9], [0, 7, 0], {}),                   # more rows than any sequence may have
    ([0, 1, 2, 9], [0, 0, 7], {0: 1, 1: 1}),
    ([0, 5, 6, 6], [0, 0, 0], {0: 5, 1: 1}),         # fewer than there were: rows behind the last one
])
def test_beside_bad_row_starts(row_start, want, good, paged):
    """Nine rows, at most six of a sequence."""
    s = Setup([5, 1, 3], [10, 15, 7], T=6, paged=paged, explicit=1)
    s.start_dev.copy_(torch.tensor(row_start, dtype=torch.int32))
    s.run()
    # the host's view of the same call: positions are explicit, so a row's rotation does not depend on whose it is
    s.start = np.array(row_start, dtype=np.int64)
    done = sum(_rows_right(s, b, range(n)) for b, n in good.items())
    assert done == sum(good.values())
    assert s.status.cpu().tolist() == want
    assert _touched(s) == set().union(*(_slots(s, b, range(n)) for b, n in good.items()))
    q = s.q_out.float().cpu().numpy()
    last = min(int(row_start[-1]), s.rows)
    assert (q[last:] == 9.0).all()  # behind the last sequence
