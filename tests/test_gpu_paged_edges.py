"""GPU: calls of the paged cache at the edges of what its interface promises."""
import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests.test_gpu_paged import BASE, dev32, half_step, make, put, reserve, tables_of

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ reservation
@pytest.mark.parametrize("pages,held", [(8, 5), (1500, 1400)])
@pytest.mark.parametrize("bad", [-1, "past", 2 ** 31 - 1])
def test_shrink_of_a_table_with_a_page_outside_the_pool(bad, pages, held):
    """Few pages and more than threads are moved: the flag is raised, the ids go to the stack as they are, in order, and
    whoever is given the bad one gets no slots in it."""
    db, st = make([1], (4, 2), 64, "bf16", 16, pages, pages, seed=pages, layers=0)
    reserve(db, st, [16 * held, 3], [0, 16 * held, 16 * held + 3], 16 * held + 3)
    col = held - 2
    st.table[0, col] = pages if bad == "past" else bad
    db.block_table[0, col] = int(st.table[0, col])
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    served = torch.full((2,), 9, dtype=torch.int32, device="cuda")
    db.reserve(dev32([-16 * (held - 1), 0]), dev32([0, 0, 0]), 0, none, none, served)
    want = st.reserve(np.array([-16 * (held - 1), 0]), np.zeros(3, dtype=int), 0)
    assert db.err_flag() == R.BAD
    assert np.array_equal(served.cpu().numpy(), want[2])
    ln, _, free, count = tables_of(db)
    assert np.array_equal(ln, st.seq_len) and count == st.count and np.array_equal(free[:count], st.free[:count])
    # the page kept and the second sequence's are in the pool: nothing to flag
    db.err.zero_()
    db.reserve(dev32([-16, -3]), dev32([0, 0, 0]), 0, none, none, served)
    assert db.err_flag() == 0
    st.reserve(np.array([-16, -3]), np.zeros(3, dtype=int), 0)
    # taken again, the id outside the pool is met by its rows
    slots, pos = (torch.full((16 * held,), 9, dtype=torch.int32, device="cuda") for _ in "sp")
    db.reserve(dev32([16 * held, 0]), dev32([0, 16 * held, 16 * held]), 16 * held, slots, pos, served)
    want = st.reserve(np.array([16 * held, 0]), np.array([0, 16 * held, 16 * held]), 16 * held)
    assert db.err_flag() == R.BAD
    inside = (st.table[0, np.arange(16 * held) // 16] >= 0) & (st.table[0, np.arange(16 * held) // 16] < pages)
    assert (~inside).sum() == 16
    assert np.array_equal(slots.cpu().numpy(), np.where(inside, want[0], -1))
    assert np.array_equal(pos.cpu().numpy(), np.where(inside, want[1], -1))


def test_bad_page_in_a_part_that_stays_is_not_met_by_a_shrink():
    """Ids are looked at as they move: what a sequence keeps is checked by who reads it."""
    db, st = make([0], (4, 2), 64, "bf16", 16, 8, 8, layers=0)
    reserve(db, st, [70], [0, 70], 70)
    st.table[0, 1] = 8
    db.block_table[0, 1] = 8
    reserve(db, st, [-30], [0, 0], 0)


# ----------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,with_q", [(37, True), (1030, False), (2061, True)])
def test_append_of_tensors_at_16_bytes(rows, with_q, d, dtype):
    """Views, pages and results that lie at 16 mod 32 bytes, rows an odd multiple of 16 bytes apart."""
    hq, hkv, page = 6, 2, 32
    bf = dtype == "bf16"
    td, unit = (torch.bfloat16, 8) if bf else (torch.float32, 4)        # elements of 16 bytes
    r = np.random.default_rng(rows + d)
    num_pages = -(-(rows + 3) // page) + 1

    def off(*shape, fill=7.0):
        flat = torch.full((int(np.prod(shape)) + unit,), fill, dtype=td, device="cuda")
        t = flat[unit:].view(*shape)
        assert t.data_ptr() % 32 == 16
        return t

    kp, vp = off(num_pages, hkv, page, d), off(num_pages, hkv, page // 8, d, 8)
    db, _ = make([1], (hq, hkv), d, dtype, page, num_pages, num_pages, k_pages=[kp], v_pages=[vp])
    tok = 3 + np.arange(rows)
    order = r.permutation(num_pages)
    slots = order[tok // page] * page + tok % page
    pos = r.integers(0, 100000, size=rows)
    heads = (hq, hkv, hkv)
    x, host = [], []
    for h in heads:
        wide = off(rows, h * d + unit)
        assert wide.stride(0) // unit % 2 == 1
        wide.copy_(torch.from_numpy(r.standard_normal(tuple(wide.shape)).astype(np.float32)))
        x.append(wide[:, :h * d])
        host.append(x[-1].double().cpu().numpy().reshape(rows, h, d))
    q_rot = off(rows, hq, d)
    db.append(0, dev32(slots), dev32(pos), x[1], x[2], x[0] if with_q else None, q_rot if with_q else None)
    assert db.err_flag() == 0
    want_k, want_v = np.full(kp.shape, 7.0), np.full(vp.shape, 7.0)
    put(want_k, want_v, slots, R.rotate(host[1], pos, BASE), host[2], page)
    assert np.array_equal(vp.double().cpu().numpy(), want_v)
    size = max(np.abs(h).max() for h in host)
    err = np.abs(kp.double().cpu().numpy() - want_k)
    assert (err <= half_step(want_k, bf) + 2 * size * (2e-7 + 2 * R.U32)).all()
    want = R.rotate(host[0], pos, BASE) if with_q else np.full((rows, hq, d), 7.0)
    err = np.abs(q_rot.double().cpu().numpy() - want)
    assert (err <= half_step(want, bf) + 2 * size * (2e-7 + 2 * R.U32)).all()
