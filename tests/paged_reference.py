"""Plain 64-bit form of the paged cache's operators (numpy), for the tests.

A State holds lengths, block tables and the stack of free pages; reserve()
moves it by the rules of ippd_paged_reserve, one sequence after another.
attend() is the definition of the attention, one question after another."""
from __future__ import annotations

import copy

import numpy as np

FULL, BAD, EXHAUSTED = 1, 2, 4


def bf16(x):
    """Round to bfloat16, to nearest even, as float32 (finite inputs)."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    r = (u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000)
    return r.view(np.float32)


class State:
    def __init__(self, q_count, page, num_pages, table_pages, order=None):
        self.q_start = np.concatenate([[0], np.cumsum(q_count)]).astype(np.int64)
        self.B, self.Nt = len(q_count), int(np.sum(q_count))
        self.page, self.num_pages, self.table_pages = page, num_pages, table_pages
        n = self.B + self.Nt
        self.seq_len = np.zeros(n, dtype=np.int64)
        self.table = np.zeros((n, table_pages), dtype=np.int64)
        self.free = np.arange(num_pages - 1, -1, -1) if order is None else np.array(order, dtype=np.int64)
        self.count = num_pages

    def copy(self):
        return copy.deepcopy(self)

    def pages(self, tokens):
        return -(-tokens // self.page)

    def prompt(self, i):
        return int(np.searchsorted(self.q_start, i, side="right")) - 1

    def reserve(self, new, start, rows):
        """(slots, positions, served, flags) and the state moved."""
        n = self.B + self.Nt
        slots, pos = np.full(rows, -1), np.full(rows, -1)
        served = np.zeros(n, dtype=np.int64)
        cap = self.page * self.table_pages
        back = [self.pages(int(ln)) - self.pages(max(0, int(ln + c))) if c < 0 else 0
                for ln, c in zip(self.seq_len, new)]
        ok = 0 <= self.count <= self.num_pages and all(0 <= ln <= cap for ln in self.seq_len)
        ok = ok and all(0 <= a <= e <= rows and c <= e - a for a, e, c in zip(start[:-1], start[1:], new))
        if not ok or self.count + sum(back) > self.num_pages:
            return slots, pos, served, BAD
        flags = 0
        given = []
        for s in range(n):
            if new[s] < 0:
                keep = max(0, int(self.seq_len[s] + new[s]))
                given += [self.table[s, j] for j in range(self.pages(keep), self.pages(int(self.seq_len[s])))]
                served[s] = keep - self.seq_len[s]
                self.seq_len[s] = keep
        self.free[self.count:self.count + len(given)] = given[::-1]
        self.count += len(given)
        needed, have = 0, self.count
        for s in range(n):
            if new[s] <= 0:
                continue
            if self.seq_len[s] + new[s] > cap:
                flags |= FULL
                continue
            first = self.pages(int(self.seq_len[s]))
            need = self.pages(int(self.seq_len[s] + new[s])) - first
            needed += need
            if need and needed > have:
                flags |= EXHAUSTED
                continue
            for j in range(need):
                self.count -= 1
                self.table[s, first + j] = self.free[self.count]
            served[s] = new[s]
            self.seq_len[s] += new[s]
        for s in range(n):
            base = self.seq_len[self.prompt(s - self.B)] if s >= self.B else 0
            for j in range(max(0, int(served[s]))):
                t = int(self.seq_len[s] - served[s]) + j
                slots[start[s] + j] = self.table[s, t // self.page] * self.page + t % self.page
                pos[start[s] + j] = base + t
        return slots, pos, served, flags


def rotate(x, pos, base):
    """R(pos) x for x [rows, heads, D] in 64 bits."""
    d = x.shape[-1]
    theta = base ** (-2.0 * np.arange(d // 2) / d)
    a = pos[:, None].astype(np.float64) * theta
    z = (x[..., :d // 2] + 1j * x[..., d // 2:]) * np.exp(1j * a)[:, None, :]
    return np.concatenate([z.real, z.imag], axis=-1)


def gather(st, seq, k_pages, v_pages):
    """Keys and values [Hkv, len, D] of a sequence from [pages, Hkv, P, D] and [pages, Hkv, P/8, D, 8]."""
    n = int(st.seq_len[seq])
    ids = st.table[seq, :st.pages(n)]
    hkv, d = k_pages.shape[1], k_pages.shape[3]
    k = k_pages[ids].transpose(1, 0, 2, 3).reshape(hkv, -1, d)[:, :n]
    v = v_pages[ids].transpose(1, 0, 2, 4, 3).reshape(hkv, -1, d)[:, :n]
    return k.astype(np.float64), v.astype(np.float64)


U32, U16 = 2.0 ** -24, 2.0 ** -8      # half steps of fp32 and bf16, relative to the value


def attend(st, active, q_rot, k_pages, v_pages, scale, bf):
    """out [Nt, Hq, D], lse [Nt, Hq] and bounds on the kernels' errors, NaN for inactive questions.

    The bounds.  A score is a sum of D products held in fp32: off by (D + 1) u sum|q k| at
    most, u = 2^-24; scaling, the offset and exp2's argument add a few u times their sizes,
    exp2 itself 2u.  So a weight is off by a factor 1 + e, e = scale (D + 1) u sum|q k| + 8 u
    (1 + |x| + |m|) at most, and the sums over n keys (and the join's factors) by (n + 64) u.
    out: 2 e + 2 (n + 64) u times the largest |v|, and with a bf16 cache the rounding of each
    weight (2^-8) times it and of the result (2^-8 of itself).  lse: e + (n + 64) u absolute,
    8 u of itself."""
    nt, hq, d = q_rot.shape
    hkv = k_pages.shape[1]
    g = hq // hkv
    out, lse = np.full((nt, hq, d), np.nan), np.full((nt, hq), np.nan)
    tol_o, tol_l = np.zeros((nt, hq, 1)), np.zeros((nt, hq))
    q = q_rot.astype(np.float64)
    for i in range(nt):
        if not active[i]:
            continue
        kc, vc = gather(st, st.prompt(i), k_pages, v_pages)
        ks, vs = gather(st, st.B + i, k_pages, v_pages)
        k, v = np.concatenate([kc, ks], axis=1), np.concatenate([vc, vs], axis=1)
        n = k.shape[1]
        if n == 0:
            out[i], lse[i] = 0.0, -np.inf
            continue
        for h in range(hq):
            x = scale * (k[h // g] @ q[i, h])
            m = x.max()
            w = np.exp(x - m)
            out[i, h] = (w @ v[h // g]) / w.sum()
            lse[i, h] = m + np.log(w.sum())
            size = scale * (np.abs(k[h // g]) @ np.abs(q[i, h])).max()
            e = (d + 1) * U32 * size + 8 * U32 * (1 + 2 * np.abs(x).max())
            top = np.abs(v[h // g]).max()
            tol_o[i, h] = top * (2 * e + 2 * (n + 64) * U32 + (U16 if bf else 0.0))
            tol_l[i, h] = e + (n + 64) * U32 + 8 * U32 * abs(lse[i, h])
    return out, lse, tol_o + (U16 if bf else 2 * U32) * np.abs(np.nan_to_num(out)), tol_l
