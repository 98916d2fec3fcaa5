"""GPU: the paged cache (reserve, append, plan, decode attention) against the plain
64-bit forms of tests/paged_reference.py, with tolerances derived there."""
import numpy as np
import pytest
import torch

from paper_2609_05707_amd import _lib as L
from paper_2609_05707_amd.paged import PagedBatch
from paper_2609_05707_amd.session import DecodeBatch
from tests import paged_reference as R

pytestmark = pytest.mark.gpu

BASE = 10000.0


def dev32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def tables_of(db):
    return (db.seq_len.cpu().numpy(), db.block_table.cpu().numpy(), db.free_pages.cpu().numpy(),
            int(db.free_count.cpu()[0]))


def same_state(db, st):
    ln, table, free, count = tables_of(db)
    assert np.array_equal(ln, st.seq_len)
    assert count == st.count
    assert np.array_equal(free[:count], st.free[:count])
    for s in range(st.B + st.Nt):
        n = st.pages(int(st.seq_len[s]))
        assert np.array_equal(table[s, :n], st.table[s, :n]), s


def reserve(db, st, new, start, rows):
    """One call on both; slots, positions, served and the moved state agree.  Returns the device arrays."""
    slots = torch.full((rows,), 99, dtype=torch.int32, device="cuda")
    pos = torch.full((rows,), 99, dtype=torch.int32, device="cuda")
    served = torch.full((st.B + st.Nt,), 99, dtype=torch.int32, device="cuda")
    db.err.zero_()
    db.reserve(dev32(new), dev32(start), rows, slots, pos, served)
    want = st.reserve(np.asarray(new), np.asarray(start), rows)
    assert np.array_equal(slots.cpu().numpy(), want[0])
    assert np.array_equal(pos.cpu().numpy(), want[1])
    assert np.array_equal(served.cpu().numpy(), want[2])
    assert db.err_flag() == want[3]
    db.err.zero_()
    same_state(db, st)
    return slots, pos, served


def make(q_count, heads, d, dtype, page, num_pages, table_pages, seed=0, **kw):
    """A batch and its reference, pages taken in a shuffled order."""
    order = np.random.default_rng(seed).permutation(num_pages)
    st = R.State(q_count, page, num_pages, table_pages, order)
    db = PagedBatch(q_count, heads[0], heads[1], d, dtype, page, num_pages, table_pages, rope_base=BASE, **kw)
    db.free_pages.copy_(dev32(order))
    return db, st


# ------------------------------------------------------------------ reservation
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("q_count", [[1], [3, 0, 5], [0, 0], [70] * 30, [1] * 600])
def test_reserve_sequence_of_calls(q_count, page):
    """Admission, single tokens, rollbacks, growth and release in mixed calls, to and from empty."""
    b, nt = len(q_count), sum(q_count)
    n = b + nt
    r = np.random.default_rng(page + n)
    db, st = make(q_count, (4, 2), 64, "bf16", page, 4 * n + 40, 5, seed=n, layers=0)
    grow = r.integers(0, 2 * page, size=n)
    start = np.concatenate([[0], np.cumsum(grow)])
    reserve(db, st, grow, start, int(start[-1]))
    for step in range(4):
        one = np.where(np.arange(n) >= b, r.integers(0, 2, size=n), 0)
        start = np.concatenate([np.zeros(b, dtype=int), np.arange(nt + 1)])
        reserve(db, st, one, start, nt)
        reserve(db, st, -r.integers(0, 3, size=n), np.zeros(n + 1), 0)
        mixed = r.integers(-page - 1, page + 2, size=n)
        start = np.concatenate([[2], 2 + np.cumsum(np.maximum(mixed, 0) + r.integers(0, 3, size=n))])
        reserve(db, st, mixed, start, int(start[-1]) + 3)
    gone = np.where(r.random(n) < 0.5, -2 ** 31, -10 ** 6)
    reserve(db, st, gone, np.zeros(n + 1), 0)
    assert st.count == st.num_pages


def test_reserve_takes_back_what_it_gave():
    db, st = make([4, 9], (4, 2), 64, "bf16", 32, 200, 20, seed=3, layers=0)
    new = np.array([300, 17] + [5, 33, 64, 1] * 3 + [40])
    start = np.concatenate([[0], np.cumsum(new)])
    before = tables_of(db)
    reserve(db, st, new, start, int(start[-1]))
    reserve(db, st, -new, start, int(start[-1]))
    after = tables_of(db)
    assert np.array_equal(before[2], after[2]) and before[3] == after[3]


@pytest.mark.parametrize("rows", [8192, 8193, 70001])
def test_reserve_many_rows(rows):
    """Both sides of the slot map's own launch."""
    db, st = make([2, 3], (4, 2), 64, "bf16", 64, 1300, 1200, layers=0)
    new = np.array([rows - 60, 7, 0, 13, 1, 20, 19])
    start = np.concatenate([[0], np.cumsum(new)])
    assert start[-1] == rows
    reserve(db, st, new, start, rows)
    reserve(db, st, -new, start, rows)


def test_reserve_many_sequences():
    """More sequences than the fused launch holds, and than one window of the scans."""
    q = [1000, 0, 1024, 500, 1]
    db, st = make(q, (4, 2), 64, "bf16", 16, 6000, 4, layers=0)
    n = st.B + st.Nt
    r = np.random.default_rng(1)
    new = r.integers(0, 33, size=n)
    start = np.concatenate([[0], np.cumsum(new)])
    reserve(db, st, new, start, int(start[-1]))
    mixed = r.integers(-40, 3, size=n)
    start = np.concatenate([[0], np.cumsum(np.maximum(mixed, 0))])
    reserve(db, st, mixed, start, int(start[-1]))


@pytest.mark.parametrize("prompts,pages", [(3, 700), (3, 9001), (70, 9001), (900, 9001)])
def test_reserve_many_pages(prompts, pages):
    """More pages in a call than threads, and than one round of them moves; some prompts get none, some give
    back a part; the last that asks for more than is left gets nothing."""
    r = np.random.default_rng(prompts + pages)
    db, st = make([0] * prompts, (4, 2), 64, "bf16", 16, pages, pages, seed=pages, layers=0)
    share = np.sort(r.integers(0, pages - 1, size=prompts - 1))
    new = 16 * np.diff(np.concatenate([[0], share, [pages]])) - r.integers(0, 16, size=prompts)
    new = np.maximum(new, 0)
    new[r.integers(0, prompts, size=prompts // 4)] = 0
    start = np.concatenate([[0], np.cumsum(new)])
    reserve(db, st, new, start, int(start[-1]))
    reserve(db, st, -r.integers(0, 16 * pages // prompts, size=prompts), np.zeros(prompts + 1), 0)
    new = r.integers(0, 40, size=prompts)
    new[-1] = 16 * pages
    start = np.concatenate([[0], np.cumsum(new)])
    reserve(db, st, new, start, int(start[-1]))
    reserve(db, st, -st.seq_len, np.zeros(prompts + 1), 0)
    assert st.count == pages


def test_reserve_refuses_what_does_not_fit():
    """A full row, an exhausted stack (and later sequences that need no page), all or nothing per sequence."""
    db, st = make([3], (4, 2), 64, "bf16", 16, 6, 4, layers=0)
    reserve(db, st, [33, 10, 16, 1], [0, 33, 43, 59, 60], 60)           # 3 + 1 + 1 + 1 pages: all there are
    reserve(db, st, [16, 6, 1, 15], [0, 16, 22, 23, 38], 38)            # 0 has no page, 1 and 3 fit what they hold
    reserve(db, st, [-33, 60, 0, 0], [0, 0, 60, 60, 60], 60)            # freed pages serve the same call; 1's row full
    reserve(db, st, [64, 48, 1, 0], [0, 64, 112, 113, 113], 113)


@pytest.mark.parametrize("rows", [40, 9000])
@pytest.mark.parametrize("fault", ["start decreases", "start past rows", "negative start", "more than the rows", "length",
                                   "negative length", "count", "negative count", "freed twice"])
def test_reserve_bad_layout_moves_nothing(fault, rows):
    db, st = make([2], (4, 2), 64, "bf16", 16, 8, 4, layers=0)
    new, start = np.array([20, 3, 5]), np.array([0, 20, 23, 28])
    reserve(db, st, new, start, 28)
    new, start = np.array([4, 1, -2]), np.array([0, 4, 5, 5])
    if fault == "start decreases":
        start = np.array([0, 4, 2, 5])
    elif fault == "start past rows":
        start = np.array([0, 4, 5, rows + 1])
    elif fault == "negative start":
        start = np.array([-1, 4, 5, 5])
    elif fault == "more than the rows":
        new = np.array([5, 1, 0])
    elif fault in ("length", "negative length"):
        st.seq_len[1] = 65 if fault == "length" else -1
        db.seq_len.copy_(dev32(st.seq_len))
    elif fault in ("count", "negative count"):
        st.count = 9 if fault == "count" else -1
        db.free_count.copy_(dev32([st.count]))
    else:
        st.count = 8
        db.free_count.copy_(dev32([8]))
        new = np.array([0, 0, -5])
    before = tables_of(db)
    slots, pos, served = (torch.full((m,), 7, dtype=torch.int32, device="cuda") for m in (rows, rows, 3))
    db.reserve(dev32(new), dev32(start), rows, slots, pos, served)
    assert db.err_flag() == R.BAD
    assert (slots == -1).all() and (pos == -1).all() and (served == 0).all()
    after = tables_of(db)
    assert all(np.array_equal(x, y) for x, y in zip(before, after))


@pytest.mark.parametrize("rows", [40, 9000])
def test_reserve_page_on_the_stack_outside_the_pool(rows):
    """Its tokens get no slot; the others theirs."""
    db, st = make([1], (4, 2), 64, "bf16", 16, 8, 8, layers=0)
    db.free_pages[7] = 8                                    # the first page taken
    slots, pos, served = (torch.full((m,), 7, dtype=torch.int32, device="cuda") for m in (rows, rows, 2))
    db.reserve(dev32([20, 3]), dev32([0, 20, 23]), rows, slots, pos, served)
    assert db.err_flag() == R.BAD
    want = st.reserve(np.array([20, 3]), np.array([0, 20, 23]), rows)
    got = slots.cpu().numpy()
    assert (got[:16] == -1).all() and np.array_equal(got[16:], want[0][16:])
    assert (pos.cpu().numpy()[:16] == -1).all() and np.array_equal(pos.cpu().numpy()[16:], want[1][16:])


# ----------------------------------------------------------------------- append
def put(kp, vp, slots, k, v, page):
    for row, s in enumerate(slots):
        if s >= 0:
            kp[s // page, :, s % page] = k[row]
            vp[s // page, :, s % page // 8, :, s % 8] = v[row]


def half_step(x, bf):
    """fp32 rotation: the angle's cos and sin to 2e-7, two products and a sum; then the cache's rounding."""
    return np.abs(x) * (R.U16 if bf else R.U32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,heads,rows,lead,with_q", [
    (16, (4, 2), 1, 0, True), (32, (3, 3), 37, 0, True), (64, (16, 1), 1024, 3, False), (128, (10, 2), 1025, 0, True),
    (256, (8, 8), 1300, 5, False), (16, (5, 5), 2001, 1, True), (64, (8, 1), 1031, 7, True), (32, (6, 3), 2049, 0, True),
    (16, (5, 1), 2051, 6, True), (128, (10, 2), 2103, 3, False)])
def test_append_against_64_bits(dtype, d, page, heads, rows, lead, with_q):
    """Rows whose slots run over pages from an offset of `lead`, with gaps, single rows out of order and rows without a
    slot; q, k, v as views of one projection with rows further apart than they are long."""
    hq, hkv = heads
    bf = dtype == "bf16"
    r = np.random.default_rng(rows + d + page)
    num_pages = -(-(rows + lead + 40) // page) + 2
    db, _ = make([1], heads, d, dtype, page, num_pages, num_pages, layers=1)
    order = r.permutation(num_pages)
    tok = lead + np.arange(rows)
    slots = order[tok // page] * page + tok % page
    if rows > 30:
        slots[9] = -1
        slots[[20, 25]] = slots[[25, 20]]
    pos = r.integers(0, 200000, size=rows)
    wide = (hq + 2 * hkv) * d + 16
    x = torch.from_numpy(r.standard_normal((rows, wide)).astype(np.float32)).to(db.tdtype).cuda()
    q, k, v = x[:, 8:8 + hq * d], x[:, 8 + hq * d:8 + (hq + hkv) * d], x[:, 8 + (hq + hkv) * d:8 + (hq + 2 * hkv) * d]
    db.k_pages[0].fill_(7.0)
    db.v_pages[0].fill_(7.0)
    q_rot = torch.full((rows, hq, d), 7.0, dtype=db.tdtype, device="cuda")
    db.append(0, dev32(slots), dev32(pos), k, v, q if with_q else None, q_rot if with_q else None)
    assert db.err_flag() == 0
    host = lambda t, h: t.double().cpu().numpy().reshape(rows, h, d)   # noqa: E731
    kr, qr = R.rotate(host(k, hkv), pos, BASE), R.rotate(host(q, hq), pos, BASE)
    kp, vp = np.full(db.k_pages[0].shape, 7.0), np.full(db.v_pages[0].shape, 7.0)
    put(kp, vp, slots, kr, host(v, hkv), page)
    assert np.array_equal(db.v_pages[0].double().cpu().numpy(), vp)
    size = np.abs(x.double().cpu().numpy()).max()
    err = np.abs(db.k_pages[0].double().cpu().numpy() - kp)
    assert (err <= half_step(kp, bf) + 2 * size * (2e-7 + 2 * R.U32)).all()
    want = np.where((slots >= 0)[:, None, None], qr, 7.0) if with_q else np.full((rows, hq, d), 7.0)
    err = np.abs(q_rot.double().cpu().numpy() - want)
    assert (err <= half_step(want, bf) + 2 * size * (2e-7 + 2 * R.U32)).all()


@pytest.mark.parametrize("rows", [5, 1040])
def test_append_skips_slots_outside_the_pool(rows):
    db, _ = make([1], (4, 2), 64, "bf16", 16, 70, 70, layers=1)
    slots = np.arange(rows)
    slots[3], slots[1] = 70 * 16, 2 ** 31 - 1
    x = torch.randn(rows, 2, 64, device="cuda").to(torch.bfloat16)
    db.k_pages[0].fill_(7.0)
    db.v_pages[0].fill_(7.0)
    db.append(0, dev32(slots), dev32(np.zeros(rows)), x, x)
    assert db.err_flag() == R.BAD
    kp, vp = np.full(db.k_pages[0].shape, 7.0), np.full(db.v_pages[0].shape, 7.0)
    slots[[1, 3]] = -1
    host = x.double().cpu().numpy()
    put(kp, vp, slots, host, host, 16)
    assert np.array_equal(db.k_pages[0].double().cpu().numpy(), kp)      # position 0 turns nothing
    assert np.array_equal(db.v_pages[0].double().cpu().numpy(), vp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_holds_the_contiguous_cache_s_bits(dtype):
    """A context filled through ippd_load_context and through pages, and a step's token, bit for bit."""
    hq, hkv, d, n = 8, 2, 128, 1207
    r = np.random.default_rng(5)
    k, v = (r.standard_normal((n, hkv, d)).astype(np.float32) for _ in range(2))
    ref = DecodeBatch([n], [1], hq, hkv, d, dtype, 16, rope_base=BASE)
    ref.load_context(0, k, v)
    q1, k1, v1 = (ref.to_dev(r.standard_normal((1, h, d)).astype(np.float32)) for h in (hq, hkv, hkv))
    ref.append(0, q1, k1, v1)
    db, st = make([1], (hq, hkv), d, dtype, 64, 24, 20, layers=1)
    slots, pos, _ = reserve(db, st, [n, 0], [0, n, n], n)
    db.append(0, slots, pos, ref.to_dev(k), ref.to_dev(v))
    slots, pos, _ = reserve(db, st, [0, 1], [0, 0, 1], 1)
    q_rot = torch.empty_like(q1)
    db.append(0, slots, pos, k1, v1, q1, q_rot)
    assert torch.equal(q_rot, ref.q_rot[:1])
    kp, vp = db.k_pages[0].float().cpu().numpy(), db.v_pages[0].float().cpu().numpy()
    kc, vc = R.gather(st, 0, kp, vp)
    assert np.array_equal(kc, ref.ctx_k[0].double().cpu().numpy()[:, :n])
    assert np.array_equal(vc, ref.ctx_values(0).double().cpu().numpy()[:, :, :n].transpose(0, 2, 1))
    ks, vs = R.gather(st, 1, kp, vp)
    assert np.array_equal(ks[:, 0], ref.seg_k[0].double().cpu().numpy()[0, :, 0])
    assert np.array_equal(vs[:, 0], ref.seg_values(0).double().cpu().numpy()[0, :, :, 0])


# -------------------------------------------------------------------- attention
def filled(q_count, ctx, seg, heads, d, dtype, page, seed=0, boost=True, spare=3, **kw):
    """A batch whose sequences have the given lengths, pages of random keys and values (NaN and infinities behind the
    last token of every sequence and in the free pages), queries whose last keys weigh as much as the others together."""
    hq, hkv = heads
    lens = np.concatenate([ctx, seg]).astype(np.int64)
    need = -(-lens // page)
    db, st = make(q_count, heads, d, dtype, page, int(need.sum()) + spare, max(1, int(need.max(initial=0))), seed=seed,
                  layers=1, **kw)
    start = np.concatenate([[0], np.cumsum(lens)])
    reserve(db, st, lens, start, int(start[-1]))
    r = np.random.default_rng(seed + 100)
    rnd = (lambda x: R.bf16(x)) if dtype == "bf16" else (lambda x: x.astype(np.float32))
    k = rnd(r.standard_normal((st.num_pages, hkv, page, d)))
    v = rnd(r.standard_normal((st.num_pages, hkv, page // 8, d, 8)))
    q = rnd(r.standard_normal((max(st.Nt, 1), hq, d)))[:st.Nt]
    if boost:
        for i in range(st.Nt):                              # the last key of each question's keys stands out
            s = st.B + i if st.seq_len[st.B + i] else st.prompt(i)
            t = int(st.seq_len[s]) - 1
            n = int(st.seq_len[st.B + i] + st.seq_len[st.prompt(i)])
            if t >= 0 and n > 1:
                for g in range(hkv):
                    u = q[i, g * (hq // hkv)].astype(np.float64)
                    k[st.table[s, t // page], g, t % page] = rnd(u * np.log(n) * np.sqrt(d) / (u @ u))
    live = np.zeros((st.num_pages, page), dtype=bool)
    for s in range(st.B + st.Nt):
        t = np.arange(int(st.seq_len[s]))
        live[st.table[s, t // page], t % page] = True
    junk = np.array([np.nan, np.inf, -np.inf, 3e38], dtype=np.float32)
    kd, vd = k.copy(), v.copy()
    kd.transpose(0, 2, 1, 3)[~live] = junk[r.integers(0, 4, size=(int((~live).sum()), hkv, d))]
    vv = vd.transpose(0, 2, 4, 1, 3)
    vv[:] = v.transpose(0, 2, 4, 1, 3)
    flat = live.reshape(st.num_pages, page // 8, 8)
    vv[~flat] = junk[r.integers(0, 4, size=(int((~flat).sum()), hkv, d))]
    db.k_pages[0].copy_(torch.from_numpy(kd))
    db.v_pages[0].copy_(torch.from_numpy(vd))
    return db, st, q, k, v


def run(db, q, fill=5.0, lse=True):
    qd = torch.from_numpy(np.ascontiguousarray(q)).to(db.tdtype).cuda()
    out = torch.full(qd.shape, fill, dtype=db.tdtype, device="cuda")
    ls = torch.full(qd.shape[:2], fill, dtype=torch.float32, device="cuda")
    db.ws.fill_(255)
    db.plan_buf.fill_(255)
    db.plan()
    db.decode(0, qd, out, ls if lse else None)
    return out, ls


def check(db, st, active, q, k, v, scale=None):
    db.set_active(active)
    out, ls = run(db, q)
    o, s = out.double().cpu().numpy(), ls.double().cpu().numpy()
    scale = scale or 1.0 / np.sqrt(q.shape[2])
    want, lse, tol_o, tol_l = R.attend(st, active, q, k, v, scale, db.dtype == "bf16")
    off = ~np.asarray(active, dtype=bool)
    assert db.err_flag() == 0
    assert (o[off] == 5.0).all() and (s[off] == 5.0).all()
    on = ~off
    empty = np.isneginf(lse[on])
    assert np.array_equal(np.isneginf(s[on]), empty)
    err = np.abs(o[on] - want[on])
    assert (err <= tol_o[on]).all(), (err.max(), tol_o[on][err > tol_o[on]][:3])
    el = np.abs(s[on][~empty] - lse[on][~empty])
    assert (el <= tol_l[on][~empty]).all(), (el.max(), tol_l[on][~empty].min())
    return out, ls


CASES = [
    # q_count, ctx, seg, heads
    ([1], [1], [0], (1, 1)),
    ([1], [0], [1], (2, 1)),
    ([2], [31], [1, 33], (4, 2)),
    ([3], [32], [0, 32, 31], (6, 2)),
    ([4, 0, 1], [65, 7, 0], [64, 0, 15, 17, 0], (8, 2)),
    ([5], [129], [3, 40, 0, 1, 16], (16, 1)),
    ([9], [257], [1] * 9, (4, 1)),
    ([33], [300], list(range(33)), (3, 1)),
    ([13, 2, 30], [511, 64, 130], [(7 * i) % 70 for i in range(45)], (10, 2)),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_against_64_bits(case, page, d, dtype):
    q_count, ctx, seg, heads = CASES[case]
    db, st, q, k, v = filled(q_count, ctx, seg, heads, d, dtype, page, seed=case)
    check(db, st, np.ones(st.Nt), q, k, v)
    if st.Nt > 1:
        active = np.random.default_rng(case).random(st.Nt) < 0.5
        check(db, st, active, q, k, v)
    check(db, st, np.zeros(st.Nt), q, k, v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [64, 256])
@pytest.mark.parametrize("n", [1, 2, 3, 5, 8])
def test_attention_row_groups(n, page, dtype):
    """G = 16: 16 rows a question, so that 1 to 8 questions cross from the wave line to one, two and more row groups."""
    db, st, q, k, v = filled([n, 1], [777, 95], [i % 3 for i in range(n + 1)], (16, 1), 128, dtype, page, seed=n)
    check(db, st, np.ones(st.Nt), q, k, v)


def test_attention_of_many_questions():
    """1024 questions of one prompt with G = 5 (row groups that end inside 16-row blocks), some stopped; sampled rows."""
    n = 1024
    r = np.random.default_rng(2)
    db, st, q, k, v = filled([n], [150], r.integers(0, 40, size=n), (5, 1), 64, "bf16", 16, seed=8, boost=False)
    active = r.random(n) < 0.8
    check(db, st, active, q, k, v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_long_lines(dtype):
    """Lengths that cut both lines into many pieces: a long shared context, long segments, many short ones."""
    r = np.random.default_rng(4)
    seg = np.concatenate([[2500, 1, 0, 777], r.integers(1, 60, size=30)])
    db, st, q, k, v = filled([10, 24], [6001, 333], seg, (8, 2), 128, dtype, 32, seed=9)
    check(db, st, np.ones(st.Nt), q, k, v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_count", [[1], [1] * 2, [1] * 3, [1] * 5, [6], [6] * 2, [6] * 3, [40, 0, 5, 1], [40] * 3])
def test_attention_of_long_tasks(q_count, dtype):
    """One, two and more tasks of many pieces on either line, prompts of several row groups beside prompts of one."""
    r = np.random.default_rng(sum(q_count))
    ctx = 1400 + 37 * np.arange(len(q_count))
    seg = r.integers(0, 50, size=sum(q_count))
    seg[-1] = 900
    db, st, q, k, v = filled(q_count, ctx, seg, (8, 2), 64, dtype, 32, seed=len(q_count))
    check(db, st, np.arange(st.Nt) != 3, q, k, v)


def test_attention_many_prompts():
    """More prompts than a window of the plan's scans; most contexts on the wave line, some empty."""
    b = 1100
    r = np.random.default_rng(6)
    qc = r.integers(0, 3, size=b)
    qc[::97] = 20
    ctx = r.integers(0, 70, size=b)
    ctx[5] = 900
    db, st, q, k, v = filled(qc.tolist(), ctx, r.integers(0, 20, size=int(qc.sum())), (2, 1), 64, "f32", 16, seed=7)
    check(db, st, r.random(st.Nt) < 0.7, q, k, v)


def test_attention_scale_and_bounds():
    """A scale of the caller's, a bound on the questions above what prompts have, no lse."""
    db, st, q, k, v = filled([3, 6], [100, 40], [5] * 9, (8, 2), 64, "f32", 32, seed=11, scale=0.3, max_questions=500)
    out, _ = check(db, st, np.ones(9), q, k, v, scale=0.3)
    again, ls = run(db, q, lse=False)
    assert torch.equal(out, again) and (ls == 5.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_large_scores(dtype):
    """Scores of thousands: the running maximum carries them; later keys above earlier ones and below."""
    db, st, q, k, v = filled([6], [400], [70] * 6, (8, 2), 64, dtype, 64, seed=12, boost=False)
    q = q * 64
    check(db, st, np.ones(6), q, k, v)


def test_attention_non_finite_values():
    """A NaN among the visible keys reaches the rows that see it and no other; -inf scores weigh nothing."""
    db, st, q, k, v = filled([2, 2], [40, 50], [3, 4, 5, 6], (2, 1), 64, "f32", 16, seed=13, boost=False)
    ref, _ = check(db, st, np.ones(4), q, k, v)
    db.k_pages[0][int(st.table[0, 1]), 0, 3, 5] = float("nan")
    out, ls = run(db, q)
    assert torch.isnan(out[:2]).all() and torch.isnan(ls[:2]).all()
    assert torch.equal(out[2:], ref[2:])


@pytest.mark.parametrize("bad", [-1, "past", 2 ** 31 - 1])
@pytest.mark.parametrize("where", ["context", "segment"])
@pytest.mark.parametrize("page", [16, 64])
def test_attention_page_outside_the_pool(page, where, bad):
    """The questions that meet it get no output, the others theirs."""
    db, st, q, k, v = filled([5, 4], [200, 90], [20] * 9, (8, 2), 64, "bf16", page, seed=14)
    ref, _ = check(db, st, np.ones(9), q, k, v)
    seq, col = (0, 200 // page - 1) if where == "context" else (2 + 3, 0)
    db.block_table[seq, col] = st.num_pages if bad == "past" else bad
    out, ls = run(db, q)
    assert db.err_flag() == R.BAD
    hit = np.arange(9) < 5 if where == "context" else np.arange(9) == 3
    hit = torch.from_numpy(hit).cuda()
    assert (out[hit] == 5.0).all() and (ls[hit] == 5.0).all()
    assert torch.equal(out[~hit], ref[~hit])


def test_attention_refuses_other_plans():
    """No plan, another batch's plan: flagged, nothing written.  A plan keeps its lengths and flags."""
    db, st, q, k, v = filled([2, 1], [40, 20], [3, 4, 5], (4, 2), 64, "bf16", 16, seed=15)
    ref, _ = check(db, st, np.ones(3), q, k, v)
    qd = torch.from_numpy(q).to(db.tdtype).cuda()
    out = torch.full(qd.shape, 5.0, dtype=db.tdtype, device="cuda")
    db.set_active([0, 0, 0])
    db.seq_len.zero_()
    db.decode(0, qd, out)
    assert torch.equal(out, ref) and db.err_flag() == 0
    other, *_ = filled([3], [40], [3, 4, 5], (4, 2), 64, "bf16", 16)
    other.plan()
    for buf in (torch.zeros_like(db.plan_buf), torch.full_like(db.plan_buf, 255), other.plan_buf):
        db.plan_buf[:min(len(buf), len(db.plan_buf))].copy_(buf[:len(db.plan_buf)])
        out.fill_(5.0)
        db.err.zero_()
        db.decode(0, qd, out)
        assert db.err_flag() == R.BAD and (out == 5.0).all()


@pytest.mark.parametrize("most", [1, 20])
def test_attention_refuses_plans_of_other_workgroups(most):
    """With 256 kv heads an fp32 and a bf16 batch agree in everything but the waves of a workgroup, and
    with them in where the plan's arrays lie."""
    kw = dict(hq=1024, hkv=256, head_dim=128, page_tokens=16, num_pages=8, table_pages=4, layers=1)
    f = PagedBatch([most], dtype="f32", **kw)
    b = PagedBatch([most], dtype="bf16", **kw)
    assert f.plan_bytes != b.plan_bytes
    plan = torch.zeros(max(f.plan_bytes, b.plan_bytes), dtype=torch.uint8, device="cuda")
    L.ippd_paged_plan(f.batch, plan.data_ptr(), plan.numel(), torch.cuda.current_stream().cuda_stream)
    q = torch.zeros(most, 1024, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    L.ippd_paged_decode_attention(b.batch, b.pages[0], plan.data_ptr(), plan.numel(), q.data_ptr(), out.data_ptr(), None,
                                  b.ws.data_ptr(), b.ws_bytes, torch.cuda.current_stream().cuda_stream)
    assert b.err_flag() == L.IPPD_FLAG_BAD_LAYOUT and f.err_flag() == 0
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("fault", ["length", "negative", "questions", "csr"])
def test_plan_bad_layout_serves_nothing(fault):
    db, st, q, k, v = filled([3, 1], [40, 20], [3, 4, 5, 6], (4, 2), 64, "bf16", 16, seed=16)
    if fault == "length":
        db.seq_len[1] = db.table_pages * 16 + 1
    elif fault == "negative":
        db.seq_len[3] = -1
    elif fault == "questions":
        db.q_start[1] = 4                                   # four questions, and the bound is three
    else:
        db.q_start[2] = 3
    out, ls = run(db, q)
    assert db.err_flag() == R.BAD
    assert (out == 5.0).all() and (ls == 5.0).all()


# ---------------------------------------------------------------- used together
def steps_of(db, st, layers, steps, active_of, seed, heads, d):
    """Decode steps as a model runs them, on both; yields per step and layer the device out and its reference."""
    hq, hkv = heads
    r = np.random.default_rng(seed)
    n = st.B + st.Nt
    start = np.concatenate([np.zeros(st.B, dtype=int), np.arange(st.Nt + 1)])
    kp = [p.double().cpu().numpy() for p in db.k_pages]
    vp = [p.double().cpu().numpy() for p in db.v_pages]
    for t in range(steps):
        active = active_of(t)
        db.set_active(active)
        slots, pos, _ = reserve(db, st, np.concatenate([np.zeros(st.B, dtype=int), active]), start, st.Nt)
        db.plan()
        for layer in range(layers):
            x = torch.from_numpy(r.standard_normal((st.Nt, hq + 2 * hkv, d)).astype(np.float32)).to(db.tdtype).cuda()
            q, k, v = x.split([hq, hkv, hkv], dim=1)
            q_rot = torch.zeros(st.Nt, hq, d, dtype=db.tdtype, device="cuda")
            out = torch.full((st.Nt, hq, d), 5.0, dtype=db.tdtype, device="cuda")
            db.append(layer, slots, pos, k, v, q, q_rot)
            db.decode(layer, q_rot, out)
            kp[layer], vp[layer] = db.k_pages[layer].double().cpu().numpy(), db.v_pages[layer].double().cpu().numpy()
            want, _, tol, _ = R.attend(st, active, q_rot.double().cpu().numpy(), kp[layer], vp[layer], 1 / np.sqrt(d),
                                       db.dtype == "bf16")
            yield active, out.double().cpu().numpy(), want, tol


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("f32", 32)])
def test_prompts_from_admission_to_release(dtype, page):
    """Admit, fill, decode with stopping questions, roll back, go on, release: tables, slots and outputs at every step."""
    heads, d, layers = (8, 2), 64, 2
    db, st = make([3, 4], heads, d, dtype, page, 60, 12, seed=20, layers=layers)
    lens = np.array([90, 33, 5, 0, 17, 16, 31, 32, 1])
    start = np.concatenate([[0], np.cumsum(lens)])
    rows = int(start[-1])
    slots, pos, _ = reserve(db, st, lens, start, rows)
    r = np.random.default_rng(21)
    for layer in range(layers):
        k, v = (torch.from_numpy(r.standard_normal((rows, 2, d)).astype(np.float32)).to(db.tdtype).cuda() for _ in "kv")
        db.append(layer, slots, pos, k, v)
    stop = np.array([2, 9, 4, 9, 9, 1, 6])

    def go(steps, t0):
        for active, out, want, tol in steps_of(db, st, layers, steps, lambda t: (stop > t + t0).astype(int), 22 + t0, heads, d):
            on = active.astype(bool)
            assert (out[~on] == 5.0).all()
            assert (np.abs(out[on] - want[on]) <= tol[on]).all()

    go(3, 0)
    n = st.B + st.Nt
    reserve(db, st, np.array([0, 0, 0, -2, -1, 0, 0, 0, -3]), np.zeros(n + 1, dtype=int), 0)
    go(2, 3)
    reserve(db, st, np.full(n, -2 ** 31), np.zeros(n + 1, dtype=int), 0)
    assert st.count == st.num_pages


def test_agrees_with_the_contiguous_cache():
    """The same prompts and steps through DecodeBatch: fp32 outputs within the derived bounds of each other."""
    hq, hkv, d = 8, 2, 128
    ctx, qc, seg = [300, 77], [5, 3], np.array([3, 20, 1, 40, 9, 16, 2, 31])
    r = np.random.default_rng(30)
    kc, vc = (r.standard_normal((377, hkv, d)).astype(np.float32) for _ in "kv")
    ks, vs = (r.standard_normal((int(seg.sum()), hkv, d)).astype(np.float32) for _ in "kv")
    ref = DecodeBatch(ctx, qc, hq, hkv, d, "f32", 64, rope_base=BASE)
    ref.load_context(0, kc, vc)
    ref.load_segments(0, ks, vs, seg)
    db, st = make(qc, (hq, hkv), d, "f32", 32, 60, 12, seed=31, layers=1)
    lens = np.concatenate([ctx, seg])
    start = np.concatenate([[0], np.cumsum(lens)])
    slots, pos, _ = reserve(db, st, lens, start, int(start[-1]))
    db.append(0, slots, pos, ref.to_dev(np.concatenate([kc, ks])), ref.to_dev(np.concatenate([vc, vs])))
    for t in range(3):
        q, k, v = (ref.to_dev(r.standard_normal((8, h, d)).astype(np.float32)) for h in (hq, hkv, hkv))
        ref.decode_step(0, q, k, v)
        slots, pos, _ = reserve(db, st, [0, 0] + [1] * 8, [0, 0] + list(range(9)), 8)
        q_rot, out = torch.empty_like(q), torch.empty_like(q)
        lse = torch.empty(8, hq, device="cuda")
        db.append(0, slots, pos, k, v, q, q_rot)
        db.plan()
        db.decode(0, q_rot, out, lse)
        assert torch.equal(q_rot, ref.q_rot)
        _, _, tol_o, tol_l = R.attend(st, np.ones(8), q_rot.cpu().numpy(), db.k_pages[0].cpu().numpy(),
                                      db.v_pages[0].cpu().numpy(), 1 / np.sqrt(d), False)
        assert (np.abs(out.cpu().numpy() - ref.out.cpu().numpy()) <= 2 * tol_o).all()
        assert (np.abs(lse.cpu().numpy() - ref.lse.cpu().numpy()) <= 2 * tol_l).all()


def test_captured_step_replays():
    """Reserve, plan, append and attention in one graph; every replay is one decode step, as the eager ones."""
    heads, d = (8, 2), 128
    hq, hkv = heads
    db, st = make([6, 3], heads, d, "bf16", 16, 120, 16, seed=40, layers=2)
    eager, _ = make([6, 3], heads, d, "bf16", 16, 120, 16, seed=40, layers=2)
    lens = np.array([150, 47] + [7, 15, 16, 1, 30, 2, 8, 9, 4])
    start = np.concatenate([[0], np.cumsum(lens)])
    rows = int(start[-1])
    g = torch.Generator(device="cuda").manual_seed(1)
    fill = [torch.randn(rows, 2 * hkv, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    step = dev32(np.concatenate([np.zeros(2, dtype=int), np.arange(10)]))
    new = dev32([0, 0] + [1] * 9)
    x = torch.zeros(9, hq + 2 * hkv, d, dtype=torch.bfloat16, device="cuda")
    bufs = {}
    for name, b in (("graph", db), ("eager", eager)):
        slots, pos = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in "sp")
        served = torch.empty(11, dtype=torch.int32, device="cuda")
        b.reserve(dev32(lens), dev32(start), rows, slots, pos, served)
        for layer in range(2):
            b.append(layer, slots, pos, fill[layer][:, :hkv], fill[layer][:, hkv:])
        bufs[name] = dict(slots=slots[:9].clone(), pos=pos[:9].clone(), served=served,
                          q=torch.empty(9, hq, d, dtype=torch.bfloat16, device="cuda"),
                          out=[torch.zeros(9, hq, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)],
                          lse=[torch.zeros(9, hq, device="cuda") for _ in range(2)])

    def one(b, o):
        b.reserve(new, step, 9, o["slots"], o["pos"], o["served"])
        b.plan()
        q, k, v = x.split([hq, hkv, hkv], dim=1)
        for layer in range(2):
            b.append(layer, o["slots"], o["pos"], k, v, q, o["q"])
            b.decode(layer, o["q"], o["out"][layer], o["lse"][layer])

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(db, bufs["graph"])
    for t in range(5):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda").to(torch.bfloat16))
        graph.replay()
        one(eager, bufs["eager"])
        torch.cuda.synchronize()
        for layer in range(2):
            assert torch.equal(bufs["graph"]["out"][layer], bufs["eager"]["out"][layer]), t
            assert torch.equal(bufs["graph"]["lse"][layer], bufs["eager"]["lse"][layer]), t
        assert torch.equal(db.seq_len, eager.seq_len) and torch.equal(db.block_table, eager.block_table)
    assert db.err_flag() == 0


def test_two_streams_with_workspaces_of_their_own():
    """Two layers at once on two streams, one plan, two workspaces."""
    db, st, q, k, v = filled([20], [900], [30] * 20, (8, 2), 64, "bf16", 32, seed=50)
    ref, _ = check(db, st, np.ones(20), q, k, v)
    qd = torch.from_numpy(q).to(db.tdtype).cuda()
    ws = torch.empty_like(db.ws)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(qd) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o, w in zip(streams, outs, (db.ws, ws)):
            with torch.cuda.stream(s):
                L.ippd_paged_decode_attention(db.batch, db.pages[0], db.plan_buf.data_ptr(), db.plan_bytes,
                                              qd.data_ptr(), o.data_ptr(), None, w.data_ptr(), db.ws_bytes, s.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], ref) and torch.equal(outs[1], ref)


@pytest.mark.parametrize("page,offset", [(256, 16900), (16, 270000)])
def test_pages_beyond_32_bits(page, offset):
    """The same steps in a small pool and in pages of a large one whose offsets pass 32 bits, bit for bit: both append
    kernels, both lines of the attention."""
    heads, d, need = (32, 8), 128, 4096 // page
    lens = np.array([1300, 500, 40, 3, 17, 300])
    dbs = []
    for pool, base in ((need, 0), (offset + need, offset)):
        st = R.State([2, 2], page, need, need)
        db = PagedBatch([2, 2], heads[0], heads[1], d, "bf16", page, pool, need, rope_base=BASE, layers=1)
        db.free_pages[:need] = dev32(base + np.arange(need - 1, -1, -1))
        db.free_count.fill_(need)
        dbs.append((db, base))
    g = torch.Generator(device="cuda").manual_seed(5)
    start = np.concatenate([[0], np.cumsum(lens)])
    rows = int(start[-1])
    fill = torch.randn(rows, 16, d, generator=g, device="cuda").to(torch.bfloat16)
    x = torch.randn(4, 48, d, generator=g, device="cuda").to(torch.bfloat16)
    got = []
    for db, base in dbs:
        slots, pos = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in "sp")
        served = torch.empty(6, dtype=torch.int32, device="cuda")
        db.reserve(dev32(lens), dev32(start), rows, slots, pos, served)
        db.append(0, slots, pos, fill[:, :8], fill[:, 8:])
        db.reserve(dev32([0, 0, 1, 1, 1, 1]), dev32([0, 0, 0, 1, 2, 3, 4]), 4, slots[:4], pos[:4], served)
        q, k, v = x.split([32, 8, 8], dim=1)
        q_rot, out, lse = torch.empty(4, 32, d, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(q).contiguous(), \
            torch.zeros(4, 32, device="cuda")
        db.append(0, slots[:4], pos[:4], k, v, q, q_rot)
        db.plan()
        db.decode(0, q_rot, out, lse)
        assert db.err_flag() == 0
        held = int(db.free_count)                            # pages base + held .. base + need - 1 are taken
        assert int(slots[:4].max()) >= base * page
        got.append((out, lse, q_rot, slots[:4] - base * page, held))
    for a, b in zip(*got):
        assert torch.equal(a, b) if torch.is_tensor(a) else a == b
    # what of the pages was written agrees too: the tokens of every sequence
    (small, _), (large, _) = dbs
    ids = small.block_table.long()
    for s, n in enumerate(lens + np.array([0, 0, 1, 1, 1, 1])):
        m = -(-int(n) // page)
        ks, kl = small.k_pages[0][ids[s, :m]], large.k_pages[0][ids[s, :m] + offset]
        vs, vl = small.v_pages[0][ids[s, :m]], large.v_pages[0][ids[s, :m] + offset]
        for a, b, order in ((ks, kl, (0, 2, 1, 3)), (vs, vl, (0, 2, 4, 1, 3))):
            assert torch.equal(a.permute(order).reshape(m * page, -1)[:n], b.permute(order).reshape(m * page, -1)[:n])


def test_calls_go_to_the_current_stream():
    """A step queued on another stream behind a long kernel there, its inputs written just before."""
    db, st, q, k, v = filled([6, 2], [120, 40], [9] * 8, (8, 2), 64, "bf16", 16, seed=60)
    ref, _ = check(db, st, np.ones(8), q, k, v)
    qd = torch.from_numpy(q).to(db.tdtype).cuda()
    out, buf = torch.zeros_like(qd), torch.zeros_like(qd)
    big = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    db.plan_buf.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(5):
            big = big @ big * 1e-3
        buf.copy_(qd)
        db.plan()
        db.decode(0, buf, out)
    side.synchronize()
    assert torch.equal(out, ref)


def test_no_questions():
    db, st = make([0, 0], (4, 2), 64, "bf16", 16, 10, 4, layers=1)
    slots, pos, _ = reserve(db, st, [20, 3], [0, 20, 23], 23)
    x = torch.randn(23, 2, 64, device="cuda").to(torch.bfloat16)
    db.append(0, slots, pos, x, x)
    db.plan()
    db.decode(0, x[:0], x[:0])
    assert db.err_flag() == 0
