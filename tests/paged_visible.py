"""Inputs for the paged attention in which every tile of 32 keys is seen in the outputs, bounds narrow enough to see it,
and the lengths they are used at (numpy only).

With random values a lost tile of a long context hides: the values' mean is near zero, and a bound from the largest
value is wider than what a hundred tiles leave of one.  Here each tile of a sequence lights one dim: its tokens hold
values in [1, 2) there and nearly nothing elsewhere.  A dim's output is then a sum of few tiles' positive values, its
bound the rounding of that sum."""
from __future__ import annotations

import numpy as np

from tests import paged_reference as R
from tests.paged_reference import U16, U32


def rounded(bf):
    return R.bf16 if bf else (lambda x: np.asarray(x, dtype=np.float32))


def data(st, heads, d, bf, seed):
    """q [Nt, Hq, D], and keys [pages, Hkv, P, D] and values [pages, Hkv, P / 8, D, 8] of a State's sequences, zero where
    none has a token, as float32; live [pages, P]."""
    hq, hkv = heads
    r = np.random.default_rng(seed)
    rnd = rounded(bf)
    page = st.page
    k = np.zeros((st.num_pages, hkv, page, d), dtype=np.float32)
    v = np.zeros((st.num_pages, hkv, page // 8, d, 8), dtype=np.float32)
    live = np.zeros((st.num_pages, page), dtype=bool)
    vt = v.transpose(0, 2, 4, 1, 3)
    for s in range(st.B + st.Nt):
        n = int(st.seq_len[s])
        t = np.arange(n)
        ids, off = st.table[s, t // page], t % page
        live[ids, off] = True
        k[ids, :, off] = rnd(r.standard_normal((n, hkv, d), dtype=np.float32))
        x = r.standard_normal((n, hkv, d), dtype=np.float32) * 2.0 ** -9
        g = np.arange(hkv)
        lit = (t[:, None] // 32 + 3 * s + 5 * g) % d
        x[t[:, None], g, lit] = (1 + (t % 32) / 32)[:, None]
        vt[ids, off // 8, off % 8] = rnd(x)
    q = rnd(r.standard_normal((st.Nt, hq, d)))
    return q, k, v, live


def attend(st, active, q, k, v, scale, bf):
    """out [Nt, Hq, D], lse [Nt, Hq] and bounds on the kernels' errors, per element; NaN for inactive questions.

    A weight is off by a factor 1 + e (paged_reference.attend derives e), sums of n of them by (n + 64) u more, u = 2^-24,
    and a bf16 cache's weights are rounded to it for the value product, 2^-8 of each.  So with the weights p that sum to
    one, out_d is off by sum_k p_k |v_kd| times 2 e + 2 (n + 64) u + 2^-8, and by its own rounding (2^-8, or 2 u).
    Products of these terms: a factor 1 + 2^-6 on the whole covers them, each being 2^-7 at most together."""
    nt, hq, d = q.shape
    hkv = k.shape[1]
    g = hq // hkv
    out, lse = np.full((nt, hq, d), np.nan), np.full((nt, hq), np.nan)
    tol_o, tol_l = np.zeros((nt, hq, d)), np.zeros((nt, hq))
    q64 = q.astype(np.float64).reshape(nt, hkv, g, d)
    for b in range(st.B):
        todo = [i for i in range(int(st.q_start[b]), int(st.q_start[b + 1])) if active[i]]
        if not todo:
            continue
        kc, vc = R.gather(st, b, k, v)
        for h in range(hkv):
            qs = q64[todo, h].reshape(-1, d)
            xc = scale * (qs @ kc[h].T)                        # [questions x G, context]
            ac = (scale * (np.abs(qs) @ np.abs(kc[h]).T)).max(-1, initial=0.0)
            for j, i in enumerate(todo):
                ks, vs = R.gather(st, st.B + i, k[:, h:h + 1], v[:, h:h + 1])
                rows = slice(j * g, (j + 1) * g)
                x = np.concatenate([xc[rows], scale * (qs[rows] @ ks[0].T)], axis=1)
                n = x.shape[1]
                hs = slice(h * g, (h + 1) * g)
                if n == 0:
                    out[i, hs], lse[i, hs] = 0.0, -np.inf
                    continue
                size = np.maximum(ac[rows], (scale * (np.abs(qs[rows]) @ np.abs(ks[0]).T)).max(-1, initial=0.0))
                m = x.max(-1)
                p = np.exp(x - m[:, None])
                total = p.sum(-1)
                p /= total[:, None]
                c = xc.shape[1]
                o = p[:, :c] @ vc[h] + p[:, c:] @ vs[0]
                a = p[:, :c] @ np.abs(vc[h]) + p[:, c:] @ np.abs(vs[0])
                e = (d + 1) * U32 * size + 8 * U32 * (1 + 2 * np.abs(x).max(-1))
                f = 2 * e + 2 * (n + 64) * U32 + (U16 if bf else 0.0)
                out[i, hs], lse[i, hs] = o, m + np.log(total)
                tol_o[i, hs] = (1 + 2.0 ** -6) * (a * f[:, None] + (U16 if bf else 2 * U32) * np.abs(o)) + 1e-30
                tol_l[i, hs] = e + (n + 64) * U32 + 8 * U32 * np.abs(lse[i, hs])
    return out, lse, tol_o, tol_l


def state(q_count, ctx, seg, page, seed, spare=3):
    """A State whose sequences have these lengths, pages in a shuffled order, and that order."""
    lens = np.concatenate([ctx, seg]).astype(np.int64)
    need = -(-lens // page)
    num_pages, width = int(need.sum()) + spare, max(1, int(need.max(initial=0)))
    order = np.random.default_rng(seed).permutation(num_pages)
    st = R.State(q_count, page, num_pages, width, order)
    start = np.concatenate([[0], np.cumsum(lens)])
    st.reserve(lens, start, int(start[-1]))
    return st, lens, start, order


# ------------------------------------------------------------------ lengths
# Lines that are cut into many pieces (the lengths of test_gpu_paged's tests of that): questions, contexts, segments.
def lines():
    r = np.random.default_rng(4)
    yield "long lines", [10, 24], [6001, 333], np.concatenate([[2500, 1, 0, 777], r.integers(1, 60, size=30)])
    for q_count in ([1], [1] * 3, [6] * 2, [40, 0, 5, 1]):
        r = np.random.default_rng(sum(q_count))
        seg = r.integers(0, 50, size=sum(q_count))
        seg[-1] = 900
        yield f"long tasks {q_count}", q_count, 1400 + 37 * np.arange(len(q_count)), seg


# Pieces of the block line longer than twice the LDS ring's stages: 32 kv heads leave 16 workgroups a head (8 with eight
# waves), and the piece per workgroup grows with the lengths.  (type, head_dim, max_questions, waves, stages); G = 2, so
# max_questions alone chooses the waves and whether one or two 16-row blocks are a wave's.
KINDS = [("bf16", 64, 32, 4, 9), ("bf16", 64, 64, 4, 9), ("bf16", 64, 130, 8, 9),
         ("bf16", 128, 32, 4, 5), ("bf16", 128, 64, 4, 5), ("bf16", 128, 130, 8, 9),
         ("f32", 64, 32, 4, 5), ("f32", 128, 64, 8, 4)]


def runs(dtype, max_questions, waves, stages):
    """Questions, contexts and segments of a kind: an odd number of tokens in each last tile, few segments."""
    q_count = {32: [20, 9, 32], 64: [40, 9, 64], 130: [70, 9, 130]}[max_questions]
    if waves == 4:
        tiles = [int(3 * stages * x) for x in (5.5, 0.3, 8.6)]
    else:                                                      # (130 questions are two row groups, each over all its tiles)
        tiles = [int(4 * stages * x) for x in (1.5, 0.2, 2.5 if dtype == "bf16" else 4.9)]
    ctx = np.array([32 * tiles[0] - 13, 32 * tiles[1] - 31, 32 * tiles[2] - 1])
    seg = np.array([(7 * i) % 70 if i % 12 == 3 else 0 for i in range(sum(q_count))])
    return q_count, ctx, seg
