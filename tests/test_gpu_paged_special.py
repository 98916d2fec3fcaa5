"""GPU: infinities and NaN among the visible keys and values of the paged attention, on both lines."""
import numpy as np
import pytest
import torch

from tests import paged_visible as V
from tests.test_gpu_paged import run
from tests.test_gpu_paged_runs import filled

pytestmark = pytest.mark.gpu

# a context of 16 rows (wave line) and one of 60 (block line, if the bound allows more than 16 rows), one empty segment
SHAPES = {"wave": ([2, 1], [150, 70], [40, 0, 9]), "block": ([15, 3], [150, 70], [(7 * i) % 45 for i in range(18)])}
HEADS = (8, 2)


def inputs(line, d, dtype, page):
    """A batch whose queries all have 1 in dim 0."""
    q_count, ctx, seg = SHAPES[line]
    db, st, q, k, v = filled(q_count, ctx, seg, HEADS, d, dtype, page, d + page)
    q[:, :, 0] = 1.0
    return db, st, q, k, v


def put_key(db, st, seq, tokens, g, value):
    t = np.asarray(tokens)
    db.k_pages[0][torch.from_numpy(st.table[seq, t // st.page]).cuda(), g, torch.from_numpy(t % st.page).cuda(), 0] = value


def rows_of(st, prompt, g):
    m = np.zeros((st.Nt, HEADS[0]), dtype=bool)
    gr = HEADS[0] // HEADS[1]
    m[int(st.q_start[prompt]):int(st.q_start[prompt + 1]), g * gr:(g + 1) * gr] = True
    return torch.from_numpy(m).cuda()


def without(st, k, v, seq, tokens):
    """The state and pages with these tokens of a sequence taken out: the last ones take their places."""
    st2, k2, v2 = st.copy(), k.copy(), v.copy()
    n = int(st.seq_len[seq])
    keep = [t for t in range(n) if t not in set(tokens)]
    src, dst = np.array(keep, dtype=int), np.arange(len(keep))
    at = lambda t: (st.table[seq, t // st.page], t % st.page)      # noqa: E731
    kt, vt = k2.transpose(0, 2, 1, 3), v2.transpose(0, 2, 4, 1, 3)
    (ps, os_), (pd, od) = at(src), at(dst)
    kt[pd, od] = kt[ps, os_]
    vt[pd, od // 8, od % 8] = vt[ps, os_ // 8, os_ % 8]
    st2.seq_len[seq] = len(keep)
    return st2, k2, v2


KINDS = [(line, d, dtype, page) for line in SHAPES for d in (64, 128) for dtype in ("bf16", "f32") for page in (16, 64)]


@pytest.mark.parametrize("line,d,dtype,page", KINDS)
def test_nan_and_infinite_keys_reach_their_rows_only(line, d, dtype, page):
    """A NaN or a score of +inf makes the rows that see it NaN; the other heads' and prompts' bits stay."""
    db, st, q, k, v = inputs(line, d, dtype, page)
    ref, rl = run(db, q)
    for value in (float("nan"), float("-nan"), float("inf")):
        for token in (0, 37, 149):
            db.k_pages[0].copy_(torch.from_numpy(k))
            put_key(db, st, 0, [token], 1, value)
            out, ls = run(db, q)
            hit = rows_of(st, 0, 1)
            assert db.err_flag() == 0
            assert torch.isnan(out[hit]).all() and torch.isnan(ls[hit]).all(), (value, token)
            assert torch.equal(out[~hit], ref[~hit]) and torch.equal(ls[~hit], rl[~hit])


@pytest.mark.parametrize("line,d,dtype,page", KINDS)
def test_special_values_reach_their_dim_only(line, d, dtype, page):
    """A value of inf, -inf or NaN makes its dim that; the other dims, lse, other heads and prompts keep their bits."""
    db, st, q, k, v = inputs(line, d, dtype, page)
    ref, rl = run(db, q)
    for value in (float("inf"), -float("inf"), float("nan")):
        for token, dim in ((0, 0), (45, 17), (149, d - 1)):
            db.v_pages[0].copy_(torch.from_numpy(v))
            db.v_pages[0][int(st.table[0, token // page]), 0, token % page // 8, dim, token % 8] = value
            out, ls = run(db, q)
            assert db.err_flag() == 0 and torch.equal(ls, rl)
            hit = rows_of(st, 0, 0)
            x = out[hit][:, dim].float()
            assert (torch.isnan(x) if value != value else x == value).all()
            out[:, :, dim][hit] = 0
            want = ref.clone()
            want[:, :, dim][hit] = 0
            assert torch.equal(out, want)


@pytest.mark.parametrize("tokens", [[0], [33], [149], list(range(32)), list(range(30, 70)), list(range(149)), list(range(150))],
                         ids=lambda t: f"{t[0]}..{t[-1]}")
@pytest.mark.parametrize("line,d,dtype,page", KINDS)
def test_scores_of_minus_infinity_weigh_nothing(line, d, dtype, page, tokens):
    """Keys whose every score is -inf, single ones, whole tiles, a context of them, are as if they were not there."""
    db, st, q, k, v = inputs(line, d, dtype, page)
    for g in range(HEADS[1]):
        put_key(db, st, 0, tokens, g, -float("inf"))
    out, ls = run(db, q)
    assert db.err_flag() == 0
    st2, k2, v2 = without(st, k, v, 0, tokens)
    want, lse, tol_o, tol_l = V.attend(st2, np.ones(st.Nt), q, k2, v2, d ** -0.5, dtype == "bf16")
    o, s = out.double().cpu().numpy(), ls.double().cpu().numpy()
    none = np.isneginf(lse)                       # an empty segment behind a context of such keys: no key at all
    assert np.array_equal(np.isneginf(s), none) and (o[none] == 0).all()
    assert (len(tokens) == 150) == none.any()
    assert (np.abs(o - want) <= tol_o).all()
    assert (np.abs(s[~none] - lse[~none]) <= tol_l[~none]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_special_values_and_bad_pages_in_many_states(d, dtype):
    """One request of 12003 tokens: more states than one wave joins.  A NaN reaches the outputs of its kv head, a page
    outside the pool leaves them all unwritten, a first tile without weight changes nothing but by its keys."""
    db, st, q, k, v = filled([1], [12003], [5], HEADS, d, dtype, 64, d)
    q[:, :, 0] = 1.0
    ref, rl = run(db, q)
    states = db.plan_buf.view(torch.int32)[9]
    assert int(states) > 20 * 64 // (d // 4)
    gr = HEADS[0] // HEADS[1]
    for token in (0, 6001, 12002):
        db.k_pages[0].copy_(torch.from_numpy(k))
        put_key(db, st, 0, [token], 1, float("nan"))
        out, ls = run(db, q)
        assert torch.isnan(out[:, gr:]).all() and torch.isnan(ls[:, gr:]).all()
        assert torch.equal(out[:, :gr], ref[:, :gr]) and torch.equal(ls[:, :gr], rl[:, :gr])
    db.k_pages[0].copy_(torch.from_numpy(k))
    tokens = list(range(64))
    for g in range(HEADS[1]):
        put_key(db, st, 0, tokens, g, -float("inf"))
    out, ls = run(db, q)
    st2, k2, v2 = without(st, k, v, 0, tokens)
    want, lse, tol_o, tol_l = V.attend(st2, [1], q, k2, v2, d ** -0.5, dtype == "bf16")
    assert (np.abs(out.double().cpu().numpy() - want) <= tol_o).all()
    assert (np.abs(ls.double().cpu().numpy() - lse) <= tol_l).all()
    assert db.err_flag() == 0
    for col in (0, 90, 12002 // 64):
        was = int(db.block_table[0, col])
        db.block_table[0, col] = st.num_pages
        db.err.zero_()
        out, ls = run(db, q)
        db.block_table[0, col] = was
        assert db.err_flag() == 2 and (out == 5.0).all() and (ls == 5.0).all()
