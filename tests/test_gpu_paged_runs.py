"""GPU: the paged attention where a wrong tile shows in the outputs (tests/paged_visible.py), at lengths that cut the
lines into many pieces."""
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


LINES = list(V.lines())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 32), (128, 16)])
@pytest.mark.parametrize("case", range(len(LINES)), ids=[x[0] for x in LINES])
def test_every_tile_of_long_lines(case, d, page, dtype):
    _, q_count, ctx, seg = LINES[case]
    db, st, q, k, v = filled(q_count, ctx, seg, (8, 2), d, dtype, page, case)
    check(db, st, np.arange(st.Nt) != 3, q, k, v)
