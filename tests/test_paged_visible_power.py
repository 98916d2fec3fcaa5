"""CPU: with the inputs of tests/paged_visible.py, one wrong tile among the keys or values of a long sequence moves some
output beyond its bound, at the lengths that the GPU tests use."""
import numpy as np
import pytest

from tests import paged_reference as R
from tests import paged_visible as V

LENGTHS = [(name, q, ctx, seg, dt, d) for name, q, ctx, seg in V.lines() for dt, d in (("bf16", 128), ("bf16", 64), ("f32", 64))]
LENGTHS += [(f"runs {dt} {d} {most}", *V.runs(dt, most, waves, stages), dt, d) for dt, d, most, waves, stages in V.KINDS]


def plant(mistake, st, seq, tile, k, v):
    """Copies of keys and values with a mistake in one 32-token tile of a sequence."""
    k, v = k.copy(), v.copy()
    n, page = int(st.seq_len[seq]), st.page
    t = np.arange(32 * tile, min(32 * tile + 32, n))
    other = t - 32 if tile else t + 32
    at = (st.table[seq, t // page], t % page)
    src = (st.table[seq, other // page], other % page)
    vt, kt = v.transpose(0, 2, 4, 1, 3), k.transpose(0, 2, 1, 3)
    where, there = ((x[0], x[1] // 8, x[1] % 8) for x in (at, src))
    if mistake == "values lost":
        vt[where] = 0
    elif mistake == "neighbour's values":
        vt[where] = vt[there]
    elif mistake == "eight tokens' values":                    # a block of 1 KB, stale
        vt[tuple(x[:8] for x in where)] = vt[tuple(x[:8] for x in there)]
    elif mistake == "neighbour's keys":
        kt[at] = kt[src]
    else:                                                      # the two tiles' values change places
        a, b = vt[where], vt[there]
        vt[where], vt[there] = b, a
    return k, v


@pytest.mark.parametrize("mistake", ["values lost", "neighbour's values", "eight tokens' values", "neighbour's keys", "swapped"])
@pytest.mark.parametrize("case", range(len(LENGTHS)), ids=[x[0] + f" {x[4]} {x[5]}" for x in LENGTHS])
def test_one_tile_is_seen(case, mistake):
    _, q_count, ctx, seg, dt, d = LENGTHS[case]
    bf = dt == "bf16"
    st, *_ = V.state(q_count, ctx, seg, 32, case)
    q, k, v, _ = V.data(st, (2, 1), d, bf, 100 + case)
    b = int(np.argmax(ctx))
    active = np.zeros(st.Nt, dtype=int)
    active[st.q_start[b]:st.q_start[b] + 1] = 1                 # one question will do
    out, lse, tol_o, tol_l = V.attend(st, active, q, k, v, d ** -0.5, bf)
    on = active.astype(bool)
    assert (tol_o[on] > 0).all() and np.isfinite(out[on]).all()
    last = int(st.seq_len[b]) // 32 - 1                         # the last whole tile
    for tile in sorted({0, 1, last // 3, last // 2, last - 1, last}):
        k2, v2 = plant(mistake, st, b, tile, k, v)
        o2, l2, _, _ = V.attend(st, active, q, k2, v2, d ** -0.5, bf)
        seen = max((np.abs(o2 - out)[on] / tol_o[on]).max(), (np.abs(l2 - lse)[on] / tol_l[on]).max())
        assert seen > 2, (tile, seen)


def test_agrees_with_the_other_reference():
    """The same outputs as paged_reference.attend, with narrower bounds."""
    st, *_ = V.state([3, 0, 2], [70, 5, 0], [3, 0, 40, 0, 1], 16, 1)
    for bf in (False, True):
        q, k, v, _ = V.data(st, (4, 2), 64, bf, 2)
        active = [1, 1, 0, 1, 1]
        a, b = V.attend(st, active, q, k, v, 0.125, bf), R.attend(st, active, q, k, v, 0.125, bf)
        assert np.allclose(a[0], b[0], rtol=1e-12, atol=1e-14, equal_nan=True)
        assert np.allclose(a[1][np.isfinite(b[1])], b[1][np.isfinite(b[1])], rtol=1e-12)
        assert np.array_equal(np.isneginf(a[1]), np.isneginf(b[1]))
        on = np.asarray(active, dtype=bool)
        # (with one key sum p |v| is the largest |v|, and the two are equal but for 64-bit rounding)
        assert (a[2][on] <= (1 + 2.0 ** -6) * (1 + 1e-12) * b[2][on] + 1e-29).all()
        assert np.allclose(a[3][on], b[3][on], rtol=1e-9, equal_nan=True)
