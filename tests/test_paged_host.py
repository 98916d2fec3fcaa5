"""CPU: the paged cache's host side: refusals of every entry point, sizes, the C layout against the binding, the
host code under sanitizers, the ISA of the attention's DMAs, and whether the reference and its bounds see mistakes."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2609_05707_amd import _lib as L
from paper_2609_05707_amd import build as B
from paper_2609_05707_amd.paged import PagedBatch
from tests import paged_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, MISALIGNED = 0x10000, 0x10009          # never dereferenced: refused before any launch


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        pytest.fail("libippd.so not built (run __graft_entry__.build())")
    return L.load_library()


def batch(**kw):
    bt = L.IppdPagedBatch()
    bt.num_prompts, bt.num_questions, bt.num_q_heads, bt.num_kv_heads = 2, 6, 8, 2
    bt.head_dim, bt.dtype = 128, L.IPPD_DTYPE_BF16
    bt.page_tokens, bt.num_pages, bt.table_pages, bt.max_questions = 64, 100, 20, 4
    bt.rope_base, bt.scale = 10000.0, 0.0
    for f in ("q_start", "seq_len", "block_table", "free_pages", "free_count", "active", "err_flag"):
        setattr(bt, f, FAKE)
    for k, v in kw.items():
        setattr(bt, k, v)
    return bt


def pages(k=FAKE, v=FAKE):
    p = L.IppdPages()
    p.k, p.v = k, v
    return p


def reserve(lib, bt, new=FAKE, start=FAKE, rows=4, slots=FAKE, pos=FAKE, served=FAKE):
    return lib.ippd_paged_reserve(ctypes.byref(bt), new, start, rows, slots, pos, served, None)


def append(lib, bt, pg=None, rows=4, slots=FAKE, pos=FAKE, q=FAKE, qs=1024, k=FAKE, ks=256, v=FAKE, vs=256, qr=FAKE):
    return lib.ippd_paged_append(ctypes.byref(bt), ctypes.byref(pg or pages()), rows, slots, pos, q, qs, k, ks, v, vs, qr,
                                 None)


def plan(lib, bt, buf=FAKE, size=1 << 30):
    return lib.ippd_paged_plan(ctypes.byref(bt), buf, size, None)


def attend(lib, bt, pg=None, pl=FAKE, pl_bytes=1 << 30, q=FAKE, out=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 40):
    return lib.ippd_paged_decode_attention(ctypes.byref(bt), ctypes.byref(pg or pages()), pl, pl_bytes, q, out, lse, ws,
                                           ws_bytes, None)


@pytest.mark.parametrize("field,value,status", [
    ("num_prompts", 0, L.IPPD_ERR_SHAPE), ("num_questions", -1, L.IPPD_ERR_SHAPE),
    ("num_prompts", L.IPPD_PAGED_MAX_SEQUENCES - 5, L.IPPD_ERR_SHAPE),
    ("num_questions", L.IPPD_PAGED_MAX_SEQUENCES - 1, L.IPPD_ERR_SHAPE), ("num_questions", 2 ** 31 - 1, L.IPPD_ERR_SHAPE),
    ("num_kv_heads", 3, L.IPPD_ERR_SHAPE), ("num_kv_heads", 0, L.IPPD_ERR_SHAPE), ("num_q_heads", 34, L.IPPD_ERR_SHAPE),
    ("num_q_heads", 2048, L.IPPD_ERR_SHAPE), ("head_dim", 96, L.IPPD_ERR_SHAPE), ("dtype", 2, L.IPPD_ERR_DTYPE),
    ("page_tokens", 8, L.IPPD_ERR_SHAPE), ("page_tokens", 48, L.IPPD_ERR_SHAPE), ("page_tokens", 512, L.IPPD_ERR_SHAPE),
    ("num_pages", 0, L.IPPD_ERR_SHAPE), ("num_pages", 2 ** 25, L.IPPD_ERR_SHAPE), ("table_pages", 0, L.IPPD_ERR_SHAPE),
    ("table_pages", 2 ** 25, L.IPPD_ERR_SHAPE), ("max_questions", 0, L.IPPD_ERR_SHAPE),
    ("max_questions", 1025, L.IPPD_ERR_SHAPE), ("rope_base", 0.0, L.IPPD_ERR_SHAPE),
    ("rope_base", float("nan"), L.IPPD_ERR_SHAPE), ("scale", float("inf"), L.IPPD_ERR_SHAPE),
    ("q_start", None, L.IPPD_ERR_NULL), ("seq_len", None, L.IPPD_ERR_NULL), ("block_table", None, L.IPPD_ERR_NULL),
    ("free_pages", None, L.IPPD_ERR_NULL), ("free_count", None, L.IPPD_ERR_NULL), ("active", None, L.IPPD_ERR_NULL),
    ("err_flag", None, L.IPPD_ERR_NULL)])
def test_batch_refusals(lib, field, value, status):
    bt = batch(**{field: value})
    assert reserve(lib, bt) == append(lib, bt) == plan(lib, bt) == attend(lib, bt) == status
    assert lib.ippd_paged_plan_bytes(ctypes.byref(bt)) == 0
    assert lib.ippd_paged_workspace_bytes(ctypes.byref(bt)) == 0


def test_null_batch(lib):
    assert lib.ippd_paged_reserve(None, FAKE, FAKE, 1, FAKE, FAKE, FAKE, None) == L.IPPD_ERR_NULL
    assert lib.ippd_paged_append(None, None, 1, FAKE, FAKE, None, 0, FAKE, 256, FAKE, 256, None, None) == L.IPPD_ERR_NULL
    assert lib.ippd_paged_plan(None, FAKE, 1 << 20, None) == L.IPPD_ERR_NULL
    assert lib.ippd_paged_decode_attention(None, None, FAKE, 1, FAKE, FAKE, None, FAKE, 1, None) == L.IPPD_ERR_NULL
    assert lib.ippd_paged_plan_bytes(None) == lib.ippd_paged_workspace_bytes(None) == 0


def test_reserve_refusals(lib):
    bt = batch()
    for kw in (dict(new=None), dict(start=None), dict(slots=None), dict(pos=None), dict(served=None)):
        assert reserve(lib, bt, **kw) == L.IPPD_ERR_NULL, kw
    assert reserve(lib, bt, rows=-1) == L.IPPD_ERR_SHAPE
    assert reserve(lib, bt, rows=L.IPPD_PAGED_MAX_ROWS + 1) == L.IPPD_ERR_SHAPE


def test_append_refusals(lib):
    bt = batch()
    for kw in (dict(slots=None), dict(pos=None), dict(k=None), dict(v=None), dict(qr=None), dict(pg=pages(k=None)),
               dict(pg=pages(v=None))):
        assert append(lib, bt, **kw) == L.IPPD_ERR_NULL, kw
    for kw in (dict(q=MISALIGNED), dict(k=MISALIGNED), dict(v=MISALIGNED), dict(qr=MISALIGNED),
               dict(pg=pages(k=MISALIGNED)), dict(pg=pages(v=MISALIGNED))):
        assert append(lib, bt, **kw) == L.IPPD_ERR_ALIGN, kw
    for kw in (dict(rows=-1), dict(rows=L.IPPD_PAGED_MAX_ROWS + 1), dict(ks=248), dict(vs=248), dict(qs=1016),
               dict(ks=260), dict(vs=257), dict(qs=1028), dict(ks=-256)):
        assert append(lib, bt, **kw) == L.IPPD_ERR_SHAPE, kw
    assert append(lib, bt, rows=0) == L.IPPD_OK
    assert append(lib, batch(dtype=L.IPPD_DTYPE_F32), rows=0, ks=260, vs=260, qs=1028) == L.IPPD_OK   # 16 bytes are 4 floats


def test_plan_and_attention_refusals(lib):
    bt = batch()
    need, ws = lib.ippd_paged_plan_bytes(ctypes.byref(bt)), lib.ippd_paged_workspace_bytes(ctypes.byref(bt))
    assert need > 0 and ws > 0
    assert plan(lib, bt, buf=None) == plan(lib, bt, size=need - 1) == L.IPPD_ERR_WORKSPACE
    assert plan(lib, bt, buf=FAKE + 16) == L.IPPD_ERR_ALIGN
    for kw in (dict(q=None), dict(out=None), dict(pg=pages(k=None)), dict(pg=pages(v=None))):
        assert attend(lib, bt, **kw) == L.IPPD_ERR_NULL, kw
    for kw in (dict(q=MISALIGNED), dict(out=MISALIGNED), dict(lse=FAKE + 2), dict(pg=pages(v=MISALIGNED)),
               dict(pl=FAKE + 128), dict(ws=FAKE + 128)):
        assert attend(lib, bt, **kw) == L.IPPD_ERR_ALIGN, kw
    for kw in (dict(pl=None), dict(pl_bytes=need - 1), dict(ws=None), dict(ws_bytes=ws - 1)):
        assert attend(lib, bt, **kw) == L.IPPD_ERR_WORKSPACE, kw
    assert attend(lib, batch(num_questions=0), pl=None, ws=None) == L.IPPD_OK


def test_sizes_grow_with_the_batch(lib):
    """States: two per question row, and one for each row of every cut of a line."""
    def sizes(**kw):
        bt = batch(**kw)
        return lib.ippd_paged_plan_bytes(ctypes.byref(bt)), lib.ippd_paged_workspace_bytes(ctypes.byref(bt))
    a, b = sizes(num_questions=6), sizes(num_questions=7)
    g, d, hkv = 4, 128, 2
    assert b[0] > a[0]
    assert abs((b[1] - a[1]) - 2 * g * hkv * (d + 2) * 4) <= 512
    assert sizes(num_pages=1000, table_pages=500) == sizes()          # neither depends on the pool
    assert sizes(num_questions=0)[0] > 0


def test_layout_matches_c(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not available")
    fields = [("ippd_paged_batch_t", L.IppdPagedBatch), ("ippd_pages_t", L.IppdPages)]
    lines = []
    for name, cls in fields:
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    lines += [f'printf("{n} %lld\\n", (long long){n});' for n in ("IPPD_PAGED_MAX_SEQUENCES", "IPPD_PAGED_MAX_ROWS",
                                                                 "IPPD_FLAG_PAGES_EXHAUSTED")]
    src = tmp_path / "layout.c"
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"ippd.h\"\nint main(void) {\n" + "\n".join(lines)
                   + "\nreturn 0;\n}\n")
    exe = tmp_path / "layout"
    r = subprocess.run([gcc, "-std=c11", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__",
                        f"-I{os.path.join(ROOT, 'include')}", "-isystem", "/opt/rocm/include", str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = dict(line.split() for line in subprocess.run([str(exe)], capture_output=True, text=True).stdout.splitlines())
    for name, cls in fields:
        assert int(out[name]) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(out[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)
    for n in ("IPPD_PAGED_MAX_SEQUENCES", "IPPD_PAGED_MAX_ROWS", "IPPD_FLAG_PAGES_EXHAUSTED"):
        assert int(out[n]) == getattr(L, n)


SANITIZED = r"""
#include <stdint.h>
#include <stdio.h>
#include <string.h>
#include "ippd.h"
#define FAKE ((void *)(size_t)0x10000)
int main(void) {
  size_t total = 0;
  int bad = 0;
  ippd_paged_batch_t bt;
  ippd_pages_t pg = {FAKE, FAKE};
  memset(&bt, 0, sizeof bt);
  bt.rope_base = 10000.0;
  bt.q_start = FAKE; bt.seq_len = FAKE; bt.block_table = FAKE; bt.free_pages = FAKE; bt.free_count = FAKE;
  bt.active = FAKE; bt.err_flag = FAKE;
  const int questions[5] = {0, 1, 300, 100000, IPPD_PAGED_MAX_SEQUENCES - 1}, page[5] = {16, 32, 64, 128, 256};
  const int maxq[4] = {1, 5, 64, 1024}, kv[3] = {1, 8, 1024}, group[4] = {1, 3, 8, 16};
  for (int dt = 0; dt < 2; ++dt) for (int d = 64; d <= 128; d *= 2) for (int q = 0; q < 5; ++q) for (int p = 0; p < 5; ++p)
    for (int m = 0; m < 4; ++m) for (int k = 0; k < 3; ++k) for (int g = 0; g < 4; ++g) {
      bt.num_prompts = 1; bt.num_questions = questions[q]; bt.num_kv_heads = kv[k]; bt.num_q_heads = kv[k] * group[g];
      bt.head_dim = d; bt.dtype = dt; bt.page_tokens = page[p]; bt.num_pages = INT32_MAX / page[p];
      bt.table_pages = INT32_MAX / page[p]; bt.max_questions = maxq[m];
      total += ippd_paged_plan_bytes(&bt) / 256 + ippd_paged_workspace_bytes(&bt) / 256;
      if (ippd_paged_plan(&bt, NULL, 0, NULL) == IPPD_OK) bad |= 1;
      if (questions[q] && ippd_paged_decode_attention(&bt, &pg, FAKE, 0, FAKE, FAKE, NULL, FAKE, 0, NULL) == IPPD_OK) bad |= 2;
      if (ippd_paged_append(&bt, &pg, 1, FAKE, FAKE, NULL, 0, FAKE, INT64_MIN, FAKE, INT64_MAX, NULL, NULL) == IPPD_OK) bad |= 4;
      if (ippd_paged_reserve(&bt, FAKE, FAKE, INT32_MIN, FAKE, FAKE, FAKE, NULL) == IPPD_OK) bad |= 8;
    }
  printf("total %zu bad %d\n", total, bad);
  return bad != 0;
}
"""


def test_host_code_under_sanitizers(tmp_path, monkeypatch):
    other = pytest.importorskip("tests.test_host_sanitizers")
    monkeypatch.setattr(other, "C_SOURCE", SANITIZED)
    # the same program with the paged cache's host code built for them, the other objects as they are
    objects = tmp_path / "objects"
    objects.mkdir()
    for o in os.listdir(B.BUILD_DIR):
        if o.endswith(".o") and o != "paged_api.o":
            os.symlink(os.path.join(B.BUILD_DIR, o), objects / o)
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all"]
    r = subprocess.run([B.hipcc(), *B.flags_for("paged_api.hip"), *san, "-c", os.path.join(B.CSRC, "paged_api.hip"), "-o",
                        str(objects / "paged_api.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    monkeypatch.setattr(B, "BUILD_DIR", str(objects))
    other.test_host_code_under_asan_and_ubsan(tmp_path)


@pytest.mark.skipif(not os.path.exists(B.hipcc()), reason="hipcc not available")
def test_dma_bases_in_sgprs_with_wait_states(tmp_path):
    """The block line's DMAs with a scalar base wait out the five states a vector write of the base needs; the others
    take a 64-bit address per lane."""
    out = tmp_path / "paged_attend.s"
    flags = [f for f in B.flags_for("paged_attend.hip") if f != "-fPIC"]
    r = subprocess.run([B.hipcc(), *flags, "--cuda-device-only", "-S", os.path.join(B.CSRC, "paged_attend.hip"), "-o",
                        str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = [line.strip() for line in out.read_text().splitlines()]
    seen = {"s": 0, "off": 0}
    for n, t in enumerate(lines):
        if not t.startswith("global_load_lds_dwordx4"):
            continue
        base = t.split(",")[1].split()[0]
        if base == "off":
            seen["off"] += 1
            continue
        assert base.startswith("s["), t
        assert lines[n - 1] == "s_nop 4", (lines[n - 1], t)
        seen["s"] += 1
    assert seen["s"] and seen["off"]


# ------------------------------------------------------------- the torch-side class
def cpu_batch(**kw):
    args = dict(q_count=[2, 1], hq=4, hkv=2, head_dim=64, dtype="f32", page_tokens=16, num_pages=20, table_pages=6,
                layers=1, device="cpu")
    args.update(kw)
    return PagedBatch(**args)


def test_class_refuses_sizes_and_tensors():
    with pytest.raises(ValueError):
        cpu_batch(page_tokens=24)
    with pytest.raises(ValueError):
        cpu_batch(head_dim=80)
    i32 = torch.int32
    with pytest.raises(ValueError):
        cpu_batch(seq_len=torch.zeros(4, dtype=i32))                    # five sequences
    with pytest.raises(ValueError):
        cpu_batch(block_table=torch.zeros(5, 6, dtype=torch.int64))
    with pytest.raises(ValueError):
        cpu_batch(block_table=torch.zeros(6, 5, dtype=i32).t())
    with pytest.raises(ValueError):
        cpu_batch(k_pages=[torch.zeros(20, 2, 16, 64)])                 # and no values
    with pytest.raises(ValueError):
        cpu_batch(k_pages=[torch.zeros(20, 2, 16, 64)], v_pages=[torch.zeros(20, 2, 16, 64)])


def test_class_refuses_calls():
    db = cpu_batch()
    i32 = torch.int32
    z = lambda *s: torch.zeros(*s, dtype=i32)      # noqa: E731
    good = dict(new=z(5), start=z(6), rows=3, slots=z(3), pos=z(3), served=z(5))
    for kw in (dict(new=z(4)), dict(start=z(5)), dict(slots=z(4)), dict(pos=z(3).long()), dict(served=z(10)[::2])):
        a = dict(good, **kw)
        with pytest.raises(ValueError):
            db.reserve(a["new"], a["start"], a["rows"], a["slots"], a["pos"], a["served"])
    k = torch.zeros(3, 2, 64)
    for kw in (dict(k=torch.zeros(3, 2, 32)), dict(k=k.bfloat16()), dict(v=torch.zeros(2, 2, 64)),
               dict(k=torch.zeros(2, 3, 64).transpose(0, 1)), dict(k=torch.zeros(3, 64, 2).transpose(1, 2)),
               dict(q=torch.zeros(3, 4, 64)), dict(q=torch.zeros(3, 4, 64), q_rot=torch.zeros(3, 256))):
        a = dict(dict(k=k, v=k, q=None, q_rot=None), **kw)
        with pytest.raises(ValueError):
            db.append(0, z(3), z(3), a["k"], a["v"], a["q"], a["q_rot"])
    q = torch.zeros(3, 4, 64)
    for kw in (dict(q=q[:2]), dict(out=q.bfloat16()), dict(lse=torch.zeros(3, 4, 1)), dict(out=torch.zeros(3, 64, 4).transpose(1, 2))):
        a = dict(dict(q=q, out=q, lse=None), **kw)
        with pytest.raises(ValueError):
            db.decode(0, a["q"], a["out"], a["lse"])
    # right arguments, but nothing here is on a GPU
    with pytest.raises(ValueError):
        db.reserve(good["new"], good["start"], 3, good["slots"], good["pos"], good["served"])
    with pytest.raises(ValueError):
        db.append(0, z(3), z(3), k, k)
    with pytest.raises(ValueError):
        db.plan()
    with pytest.raises(ValueError):
        db.decode(0, q, q)


# -------------------------------------------------------------- the reference itself
def small(bf, seed=0):
    r = np.random.default_rng(seed)
    st = R.State([2, 1], 16, 30, 6, r.permutation(30))
    lens = np.array([40, 7, 3, 17, 1])
    st.reserve(lens, np.concatenate([[0], np.cumsum(lens)]), int(lens.sum()))
    rnd = R.bf16 if bf else (lambda x: x.astype(np.float32))
    k, v = rnd(r.standard_normal((30, 2, 16, 64))), rnd(r.standard_normal((30, 2, 2, 64, 8)))
    return st, rnd(r.standard_normal((3, 4, 64))), k, v


def test_reference_against_torch():
    st, q, k, v = small(False)
    out, lse, tol_o, tol_l = R.attend(st, [1, 0, 1], q, k, v, 0.125, False)
    assert np.isnan(out[1]).all() and np.isfinite(tol_o).all()
    for i in (0, 2):
        ks, vs = zip(R.gather(st, st.prompt(i), k, v), R.gather(st, 2 + i, k, v))
        kk = torch.from_numpy(np.concatenate(ks, axis=1)).repeat_interleave(2, 0)
        vv = torch.from_numpy(np.concatenate(vs, axis=1)).repeat_interleave(2, 0)
        x = torch.matmul(kk, torch.from_numpy(q[i]).double()[:, :, None])[..., 0] * 0.125
        assert np.allclose(torch.logsumexp(x, -1), lse[i], atol=1e-12)
        assert np.allclose((torch.softmax(x, -1)[..., None] * vv).sum(1), out[i], atol=1e-12)


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("mistake", ["last key", "first key", "other page", "other head", "scale", "last value"])
def test_bounds_see_mistakes(mistake, bf):
    """A planted mistake moves outputs by more than the bounds allow."""
    st, q, k, v = small(bf)
    out, lse, tol_o, tol_l = R.attend(st, [1, 1, 1], q, k, v, 0.125, bf)
    scale = 0.125
    st2, k2, v2 = st.copy(), k.copy(), v.copy()
    if mistake == "last key":
        st2.seq_len[0] -= 1
    elif mistake == "first key":
        v2[st.table[0, 0], :, 0, :, 0] = 0
        k2[st.table[0, 0], :, 0] = -1e4 * np.sign(q[0, ::2].sum(0))
    elif mistake == "other page":
        st2.table[0, [0, 1]] = st2.table[0, [1, 1]]
    elif mistake == "other head":
        k2 = k2[:, ::-1]
    elif mistake == "scale":
        scale = 0.1251
    else:
        v2[st.table[0, 2], :, 0, :, 7] = 0                   # token 39
    o2, l2, _, _ = R.attend(st2, [1, 1, 1], q, k2, v2, scale, bf)
    assert (np.abs(o2 - out) > tol_o).any() if mistake != "scale" else (np.abs(l2 - lse) > tol_l).any()


def test_reference_pages_are_held_once():
    r = np.random.default_rng(3)
    st = R.State([3, 2], 16, 40, 7, r.permutation(40))
    for _ in range(200):
        new = r.integers(-40, 40, size=7)
        start = np.concatenate([[0], np.cumsum(np.maximum(new, 0))])
        st.reserve(new, start, int(start[-1]))
        held = np.concatenate([st.table[s, :st.pages(int(st.seq_len[s]))] for s in range(7)])
        both = np.concatenate([held, st.free[:st.count]])
        assert sorted(both) == list(range(40))
