"""GPU: the paged attention where a wrong tile shows in the outputs (tests/paged_visible.py), at lengths that cut the
lines into many pieces and in pieces that pass the LDS ring more than twice."""
import numpy as np
import pytest
import torch

from paper_2609_05707_amd.paged import PagedBatch
from tests import paged_visible as V
from tests.test_gpu_paged import BASE, dev32, run

pytestmark = pytest.mark.gpu


def filled(q_count, ctx, seg, heads, d, dtype, page, seed, **kw):
    """A batch of these lengths with the visible inputs; NaN and infinities wherever no token is."""
    st, lens, start, order = V.state(q_count, ctx, seg, page, seed)
    db = PagedBatch(q_count, *heads, d, dtype, page, st.num_pages, st.table_pages, rope_base=BASE, **kw)
    db.free_pages.copy_(dev32(order))
    rows = int(start[-1])
    slots, pos = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in "sp")
    db.reserve(dev32(lens), dev32(start), rows, slots, pos, torch.empty(len(lens), dtype=torch.int32, device="cuda"))
    q, k, v, live = V.data(st, heads, d, dtype == "bf16", seed + 100)
    dead = torch.from_numpy(~live).cuda()
    junk = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device="cuda")
    for dst, src, per_token in ((db.k_pages[0], k, (0, 2, 1, 3)), (db.v_pages[0], v, (0, 2, 4, 1, 3))):
        x = torch.from_numpy(src).cuda()
        y = x.permute(per_token)
        y[dead.reshape(y.shape[:len(per_token) - 2])] = junk[torch.arange(d, device="cuda") % 4]
        dst.copy_(x)
    return db, st, q, k, v


def check(db, st, active, q, k, v):
    db.set_active(active)
    out, ls = run(db, q)
    assert db.err_flag() == 0
    want, lse, tol_o, tol_l = V.attend(st, active, q, k, v, q.shape[2] ** -0.5, db.dtype == "bf16")
    o, s = out.double().cpu().numpy(), ls.double().cpu().numpy()
    on = np.asarray(active, dtype=bool)
    assert (o[~on] == 5.0).all() and (s[~on] == 5.0).all()
    assert np.isfinite(o[on]).all()
    err = np.abs(o - want)[on] / tol_o[on]
    assert err.max() <= 1, (err.max(), np.argwhere(err > 1)[:5])
    err = np.abs(s - lse)[on] / tol_l[on]
    assert err.max() <= 1, err.max()


def cut(db):
    """(waves, tiles a workgroup takes of a task of the block line, those of tasks that a piece goes on into), checked
    against the tasks' tiles."""
    w = db.plan_buf.view(torch.int32).cpu().numpy()
    groups, n1, tasks, waves = int(w[3]), int(w[6]), int(w[10]), int(w[11])
    task1 = 64 + 12 * groups * (1 + waves)
    task = w[task1:task1 + 8 * tasks].reshape(-1, 8)
    first, later, seen = [], [], np.zeros(tasks, dtype=int)
    for b in range(n1):
        i, _, n = w[64 + 12 * b:64 + 12 * b + 3]
        first.append(int(n))
        seen[i] += n
        while i + 1 < tasks and task[i + 1, 5] == b:
            i += 1
            later.append(int(task[i, 7]))
            seen[i] += task[i, 7]
    assert np.array_equal(seen, task[:, 6])
    return waves, first, later


LINES = list(V.lines())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 32), (128, 16)])
@pytest.mark.parametrize("case", range(len(LINES)), ids=[x[0] for x in LINES])
def test_every_tile_of_long_lines(case, d, page, dtype):
    _, q_count, ctx, seg = LINES[case]
    db, st, q, k, v = filled(q_count, ctx, seg, (8, 2), d, dtype, page, case)
    check(db, st, np.arange(st.Nt) != 3, q, k, v)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dtype,d,most,waves,stages", V.KINDS)
def test_pieces_longer_than_the_ring(dtype, d, most, waves, stages, page):
    """Odd and even runs of more than twice the ring's stages, and runs of more than the ring in a piece's next task."""
    q_count, ctx, seg = V.runs(dtype, most, waves, stages)
    db, st, q, k, v = filled(q_count, ctx, seg, (64, 32), d, dtype, page, most + d, max_questions=most)
    check(db, st, np.arange(st.Nt) != 7, q, k, v)
    got, first, later = cut(db)
    assert got == waves
    long = [n for n in first if n > 2 * stages]
    assert {n % 2 for n in long} == {0, 1}, first
    assert max(later) > stages, later


@pytest.mark.parametrize("d,dtype,most", [(128, "bf16", 8), (64, "f32", 8), (128, "bf16", 40)])
@pytest.mark.parametrize("page", [256, 16])
def test_both_lines_in_pages_beyond_32_bits(page, d, dtype, most):
    """A context with more than 16 rows (the block line), one with fewer and the segments (the wave line), in a small
    pool and in pages of a large one that lie more than 2^32 elements behind its first, the rest of it NaN: bit for bit."""
    q_count, ctx, seg = [8, 2], [1300, 500], [40, 3, 17, 300, 0, 9, 60, 1, 33, 5]
    heads = (32, 8)
    db, st, q, k, v = filled(q_count, ctx, seg, heads, d, dtype, page, page + d, max_questions=most)
    check(db, st, np.ones(st.Nt), q, k, v)
    out, ls = run(db, q)
    offset = 2 ** 32 // (heads[1] * page * d) + 3
    large = PagedBatch(q_count, *heads, d, dtype, page, offset + st.num_pages, st.table_pages, rope_base=BASE,
                       max_questions=most)
    for big, small in ((large.k_pages[0], db.k_pages[0]), (large.v_pages[0], db.v_pages[0])):
        big.fill_(float("nan"))
        big[offset:] = small
        assert big[offset].data_ptr() - big.data_ptr() > 2 ** 32 * big.element_size()
    large.block_table.copy_(db.block_table + offset)
    large.seq_len.copy_(db.seq_len)
    got, gl = run(large, q)
    assert large.err_flag() == 0
    assert torch.equal(got, out) and torch.equal(gl, ls)
    assert cut(large)[1] and int(large.plan_buf.view(torch.int32)[7]) > 0        # pieces of both lines
