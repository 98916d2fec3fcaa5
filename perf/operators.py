"""Performance cases of the paged cache: block tables and slot maps, the append
into pages, and the decode attention that reads them.

Sequences are numbered contexts first (0 .. B-1), then the questions' segments
(B .. B+Nt-1).  A page holds ``page`` tokens of all kv heads: keys
[page][D] per head, values in 8-token column blocks [page/8][D][8].

A case is a dict of plain values:
  op        "tables": reserve rows and pages for new tokens, then take them
            back (a rollback or the end of the requests); "append": rotate new
            tokens and write them through the slot map; "attend": one decode
            step's plan and the attention of every layer
  step      tables, append: one new token per active question (a decode
            step), else every sequence whole (an admission, a prefill)
  dtype, hq, hkv, d, page       element type, head shape, tokens per page
  prompts, ctx_lo, ctx_hi       prompts and their context lengths (uniform)
  q_lo, q_hi                    questions per prompt
  seg_lo, seg_hi                tokens cached per question
  stopped                       share of questions that have finished
  with_q                        append: queries are rotated too
  layers                        layers, each with pages of its own
  lens                          seed of the lengths
"""
import math

import numpy as np
import torch

own = False
ROPE_BASE = 10000.0
DEV = "cuda"


def _case(name, op, dtype, heads, page, prompts, ctx, q, seg, step=True, with_q=True, stopped=0.0, layers=1, lens=1):
    c = dict(op=op, step=step, dtype=dtype, hq=heads[0], hkv=heads[1], d=heads[2], page=page, prompts=prompts,
             ctx_lo=ctx[0], ctx_hi=ctx[1], q_lo=q[0], q_hi=q[1], seg_lo=seg[0], seg_hi=seg[1], stopped=stopped,
             with_q=with_q, layers=layers, lens=lens)
    if name:
        c["name"] = name
    return c


def listed():
    llama = (32, 8, 128)
    return [
        # A decode step's bookkeeping: one slot per active question, taken and rolled back; latency.
        _case("tables-step-n256", "tables", "bf16", llama, 64, 8, (8192, 8192), (32, 32), (32, 96)),
        # A serving batch of documents with their questions admitted at once, and released.
        _case("tables-admit-b32", "tables", "bf16", llama, 32, 32, (1024, 8192), (4, 32), (16, 96), step=False, lens=3),
        # The smallest append: four fp32 tokens, one layer.
        _case("append-step-tiny-f32", "append", "f32", (4, 2, 64), 16, 1, (256, 256), (4, 4), (24, 24)),
        # The append of a decode step with 256 questions, four layers, q/k/v as views of one projection.
        _case("append-step-n256", "append", "bf16", llama, 64, 8, (8192, 8192), (32, 32), (32, 96), layers=4),
        # The fill that a prefill does: whole contexts of 1k to 8k tokens and their questions.
        _case("append-fill-b8", "append", "bf16", llama, 64, 8, (1024, 8192), (8, 24), (9, 43), step=False,
              with_q=False, lens=2),
        # A fill in fp32 with small pages and odd lengths, queries too.
        _case("append-fill-odd-f32", "append", "f32", (6, 2, 64), 16, 5, (1, 1999), (1, 7), (1, 33), step=False, lens=5),
        # The smallest attention: one short fp32 prompt, 4 questions.
        _case("attend-tiny-f32", "attend", "f32", (4, 2, 64), 16, 1, (256, 256), (4, 4), (24, 24)),
        # One user's document with a handful of questions; eight layers of a decode step.
        _case("attend-lc4096-n16", "attend", "bf16", llama, 64, 1, (4096, 4096), (16, 16), (32, 96), layers=8),
        # A serving batch of documents of all lengths with 4 to 32 questions each.
        _case("attend-ragged-b32", "attend", "bf16", llama, 64, 32, (1024, 8192), (4, 32), (16, 96), layers=2, lens=3),
        # A book: one very long context with many questions.
        _case("attend-lc32768-n64", "attend", "bf16", llama, 128, 1, (32768, 32768), (64, 64), (16, 128), layers=3),
        # A uniform batch in the middle of its answers: four in ten questions have stopped.
        _case("attend-b8-lc8192-n32", "attend", "bf16", llama, 64, 8, (8192, 8192), (32, 32), (33, 120), stopped=0.4,
              layers=3),
        # Independent requests, one question each, of one token to 16k: nothing is shared.
        _case("attend-requests-b64", "attend", "bf16", (64, 8, 128), 16, 64, (1, 16384), (1, 1), (1, 200), lens=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "append", "append", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    hkv = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 3, 4, 5, 8, 16])
    d = rng.choice([64, 128])
    page = rng.choice([16, 32, 64, 128, 256])
    step = rng.random() < 0.5
    hi = _log(rng, 1, 32768)
    lo = rng.randint(1, hi)
    prompts = min(_log(rng, 1, 64), max(1, 131072 // hi))
    q_hi = min(_log(rng, 1, 64), max(1, 1024 // prompts))
    if op == "attend":
        while q_hi > 1 and prompts * hi * q_hi * g * hkv > 10 ** 9:
            q_hi = (q_hi + 1) // 2
    seg_hi = _log(rng, 1, 512)
    if op == "append" and not step:
        prompts = min(prompts, max(1, 32768 // hi))
        q_hi = min(q_hi, max(1, 8192 // (prompts * seg_hi)))
    layers = 1 if op == "tables" else rng.choice([1, 2]) if hi * prompts < 65536 else 1
    return _case(None, op, dtype, (hkv * g, hkv, d), page, prompts, (lo, hi), (rng.randint(1, q_hi), q_hi),
                 (rng.randint(1, seg_hi), seg_hi), step=step, with_q=rng.random() < 0.5,
                 stopped=rng.choice([0.0, 0.0, 0.3, 0.8]), layers=layers, lens=rng.randint(1, 10 ** 6))


# ---------------------------------------------------------------------- shapes
def _shape(case):
    """Lengths of the case, on the host: question counts, lengths of the sequences, active flags."""
    r = np.random.default_rng([case["lens"], 11])
    b = case["prompts"]
    ctx = r.integers(case["ctx_lo"], case["ctx_hi"], size=b, endpoint=True)
    qc = r.integers(case["q_lo"], case["q_hi"], size=b, endpoint=True)
    nt = int(qc.sum())
    seg = r.integers(case["seg_lo"], case["seg_hi"], size=nt, endpoint=True)
    active = r.random(nt) >= case["stopped"]
    active[0] = True
    q_start = np.concatenate([[0], np.cumsum(qc)])
    return dict(ctx=ctx, qc=qc, nt=nt, seg=seg, active=active, q_start=q_start, lens=np.concatenate([ctx, seg]),
                prompt=np.repeat(np.arange(b), qc))


def _pages(lens, page):
    return -(-lens // page)


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def _random(g, *shape, dtype):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _new_tokens(case, sh):
    """New tokens per sequence and the rows they sit at."""
    b = case["prompts"]
    if case["step"]:
        new = np.concatenate([np.zeros(b, dtype=np.int64), sh["active"].astype(np.int64)])
        start = np.concatenate([np.zeros(b, dtype=np.int64), np.arange(sh["nt"] + 1)])
    else:
        new = sh["lens"]
        start = np.concatenate([[0], np.cumsum(new)])
    return new, start


def prepare(case, seed):
    sh = _shape(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    b, page, hq, hkv, d = case["prompts"], case["page"], case["hq"], case["hkv"], case["d"]
    new, start = _new_tokens(case, sh)
    op = case["op"]
    have = sh["lens"] if op == "attend" or case["step"] else np.zeros_like(sh["lens"])
    most = sh["lens"] + 1                                       # room for the step's token
    held, room = _pages(have, page), _pages(most, page)
    num_pages = int(room.sum()) + 7
    width = int(room.max()) + 1
    perm = torch.randperm(num_pages, generator=g, device=DEV).to(torch.int32)   # pages in the order of past traffic
    starts = np.concatenate([[0], np.cumsum(held)])
    table = torch.zeros(b + sh["nt"], width, dtype=torch.int32, device=DEV)
    rows = np.repeat(np.arange(b + sh["nt"]), held)
    cols = np.arange(int(held.sum())) - np.repeat(starts[:-1], held)
    used = int(held.sum())
    table[torch.from_numpy(rows).to(DEV), torch.from_numpy(cols).to(DEV)] = perm[:used]
    free = torch.zeros(num_pages, dtype=torch.int32, device=DEV)
    free[:num_pages - used] = perm[used:]
    s = dict(case=case, q_start=_i32(sh["q_start"]), prompt=_i32(sh["prompt"]), active=_i32(sh["active"]).to(torch.uint8),
             seq_len=_i32(have), table=table, free=free, free_count=_i32([num_pages - used]), num_pages=num_pages,
             width=width, nt=sh["nt"], max_q=int(sh["qc"].max()), max_ctx=int(sh["ctx"].max()),
             max_seg=int(sh["seg"].max()))
    inv = ROPE_BASE ** (-2.0 * np.arange(d // 2) / d)
    s["inv_freq"] = torch.from_numpy(inv).to(DEV)
    nrows = int(start[-1])
    s["rows"] = nrows
    td = _dtype(case)
    if op == "tables":
        s["new"], s["back"], s["start"] = _i32(new), _i32(-new), _i32(start)
        s["slots"] = torch.zeros(nrows, dtype=torch.int32, device=DEV)
        s["positions"] = torch.zeros(nrows, dtype=torch.int32, device=DEV)
        s["served"] = torch.zeros(b + sh["nt"], dtype=torch.int32, device=DEV)
        s["slots2"], s["positions2"], s["served2"] = (torch.zeros_like(s[k]) for k in ("slots", "positions", "served"))
    else:
        s["k_pages"] = [_random(g, num_pages, hkv, page, d, dtype=td) for _ in range(case["layers"])]
        s["v_pages"] = [_random(g, num_pages, hkv, page // 8, d, 8, dtype=td) for _ in range(case["layers"])]
    if op == "append":
        # slots and positions as the reservation gives them
        ctx = sh["lens"][:b] if not case["step"] else have[:b]
        seq = np.repeat(np.arange(b + sh["nt"]), np.diff(start))
        j = np.arange(nrows) - start[:-1][seq]
        live = j < new[seq]
        tok = have[seq] + j
        all_pages = perm.cpu().numpy()
        first = np.concatenate([[0], np.cumsum(room)])          # each sequence's pages in this layout
        slot = all_pages[first[seq] + tok // page].astype(np.int64) * page + tok % page
        base = np.where(seq >= b, ctx[sh["prompt"][np.maximum(seq - b, 0)]], 0)
        s["slots"] = _i32(np.where(live, slot, -1))
        s["positions"] = _i32(np.where(live, base + tok, -1))
        s["qkv"] = [_random(g, nrows, (hq + 2 * hkv) * d, dtype=td) for _ in range(case["layers"])]
        s["q_rot"] = [torch.zeros(nrows, hq, d, dtype=td, device=DEV) for _ in range(case["layers"])]
    if op == "attend":
        s["q_rot"] = [_random(g, sh["nt"], hq, d, dtype=td) for _ in range(case["layers"])]
        s["out"] = [torch.zeros(sh["nt"], hq, d, dtype=td, device=DEV) for _ in range(case["layers"])]
        s["lse"] = [torch.zeros(sh["nt"], hq, dtype=torch.float32, device=DEV) for _ in range(case["layers"])]
    if own:
        from paper_2609_05707_amd.paged import PagedBatch
        s["batch"] = PagedBatch(sh["qc"].tolist(), hq, hkv, d, case["dtype"], page, num_pages, width,
                                rope_base=ROPE_BASE, seq_len=s["seq_len"], block_table=table, free_pages=free,
                                free_count=s["free_count"], active=s["active"], k_pages=s.get("k_pages", ()),
                                v_pages=s.get("v_pages", ()))
    return s


# ------------------------------------------------------------------ plain forms
def _plain_reserve(s, new, slots, positions, served):
    """Shrink, then grow: pages pushed to and popped from the stack in sequence order, served while they last."""
    page = s["case"]["page"]
    b, n = s["case"]["prompts"], s["seq_len"].numel()
    width, total = s["width"], s["num_pages"]
    dev = new.device
    ln = s["seq_len"].long()
    new = new.long()
    free0 = s["free_count"].long()
    cut = torch.where(new < 0, (ln + new).clamp(min=0), ln)
    had = (ln + page - 1) // page
    kept = (cut + page - 1) // page
    back = had - kept
    col = torch.arange(width, device=dev)
    gone = (col[None, :] >= kept[:, None]) & (col[None, :] < had[:, None])
    rank = (torch.cumsum(back, 0) - back)[:, None] + (col[None, :] - kept[:, None])
    total_back = back.sum()
    at = torch.where(gone, free0 + total_back - 1 - rank, torch.full_like(rank, total))
    roomy = torch.cat([s["free"], s["free"].new_zeros(1)])
    roomy[at.reshape(-1)] = torch.where(gone, s["table"], torch.zeros_like(s["table"])).reshape(-1)
    free = roomy[:total]
    f1 = free0 + total_back
    want = torch.where(new > 0, new, torch.zeros_like(new))
    need = torch.where(want > 0, (cut + want + page - 1) // page - kept, torch.zeros_like(want))
    cum = torch.cumsum(need, 0)
    ok = (want > 0) & ((need == 0) | (cum <= f1))
    first = cum - need
    got = torch.where(ok, want, torch.zeros_like(want))
    after = cut + got
    owns = (after + page - 1) // page
    fresh = (col[None, :] >= kept[:, None]) & (col[None, :] < owns[:, None])
    idx = (f1 - 1 - first[:, None] - (col[None, :] - kept[:, None])).clamp(0, total - 1)
    s["table"].copy_(torch.where(fresh, free[idx], s["table"]))
    taken = torch.where(ok, need, torch.zeros_like(need)).sum()
    s["free"].copy_(free)
    s["free_count"].copy_((f1 - taken).to(torch.int32))
    s["seq_len"].copy_(after.to(torch.int32))
    row = torch.arange(s["rows"], device=dev)
    seq = torch.searchsorted(s["start"].long(), row, right=True) - 1
    seq = seq.clamp(0, n - 1)
    j = row - s["start"].long()[seq]
    live = j < got[seq]
    tok = torch.where(live, cut[seq] + j, torch.zeros_like(j))
    slot = s["table"].long()[seq, tok // page] * page + tok % page
    base = torch.zeros_like(after)
    base[b:] = after[:b][s["prompt"].long()]
    slots.copy_(torch.where(live, slot, torch.full_like(slot, -1)).to(torch.int32))
    positions.copy_(torch.where(live, base[seq] + tok, torch.full_like(slot, -1)).to(torch.int32))
    served.copy_(torch.where(new < 0, cut - ln, got).to(torch.int32))


def _rotate(x, cos, sin):
    h = x.shape[-1] // 2
    lo, hi = x[..., :h], x[..., h:]
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)


def _plain_append(s, layer):
    c = s["case"]
    hq, hkv, d, page = c["hq"], c["hkv"], c["d"], c["page"]
    qkv = s["qkv"][layer]
    live = s["slots"] >= 0
    angle = s["positions"].double()[:, None] * s["inv_freq"][None, :]
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    k = _rotate(qkv[:, hq * d:(hq + hkv) * d].reshape(-1, hkv, d).float(), cos, sin).to(qkv.dtype)
    v = qkv[:, (hq + hkv) * d:].reshape(-1, hkv, d)
    slot = s["slots"][live].long()
    pg, off = slot // page, slot % page
    s["k_pages"][layer][pg, :, off] = k[live]
    s["v_pages"][layer].permute(0, 2, 4, 1, 3)[pg, off // 8, off % 8] = v[live]
    if c["with_q"]:
        q = _rotate(qkv[:, :hq * d].reshape(-1, hq, d).float(), cos, sin).to(qkv.dtype)
        s["q_rot"][layer].copy_(torch.where(live[:, None, None], q, s["q_rot"][layer]))
    return s["k_pages"][layer], s["v_pages"][layer], s["q_rot"][layer]


def _gather(s, layer, table, tokens):
    """Keys [n, Hkv, L, D] and values the same, in 32 bits, of the first `tokens` tokens of each table row."""
    c = s["case"]
    pages = max(1, _pages(tokens, c["page"]))
    t = table[:, :pages].long()
    n = t.shape[0]
    k = s["k_pages"][layer][t].permute(0, 2, 1, 3, 4).reshape(n, c["hkv"], pages * c["page"], c["d"])
    v = s["v_pages"][layer][t].permute(0, 2, 1, 3, 5, 4).reshape(n, c["hkv"], pages * c["page"], c["d"])
    return k.float(), v.float()


def _plain_attend(s, layer):
    c = s["case"]
    b, hq, hkv, d = c["prompts"], c["hq"], c["hkv"], c["d"]
    nt, gr = s["nt"], hq // hkv
    lens = s["seq_len"].long()
    scale = 1.0 / math.sqrt(d)
    q = s["q_rot"][layer].float().reshape(nt, hkv, gr, d)
    # the prompts' questions, padded to the most of any prompt
    slot = torch.arange(nt, device=q.device) - s["q_start"].long()[s["prompt"].long()]
    qp = q.new_zeros(b, s["max_q"], hkv, gr, d)
    qp[s["prompt"].long(), slot] = q
    qp = qp.permute(0, 2, 1, 3, 4).reshape(b, hkv, s["max_q"] * gr, d)
    k, v = _gather(s, layer, s["table"][:b], s["max_ctx"])
    sc = torch.matmul(qp, k.transpose(-1, -2)) * scale
    del k
    hide = torch.arange(sc.shape[-1], device=q.device)[None, :] >= lens[:b, None]
    sc.masked_fill_(hide[:, None, None, :], -math.inf)
    m0 = sc.amax(-1)
    sc = torch.exp(sc - torch.where(m0 == -math.inf, torch.zeros_like(m0), m0)[..., None])
    l0 = sc.sum(-1)
    o0 = torch.matmul(sc, v)
    del sc, v
    pick = lambda x: x.reshape(b, hkv, s["max_q"], gr, -1)[s["prompt"].long(), :, slot]   # noqa: E731
    m0, l0, o0 = pick(m0)[..., 0], pick(l0)[..., 0], pick(o0)
    k, v = _gather(s, layer, s["table"][b:], s["max_seg"])
    sc = torch.matmul(q, k.transpose(-1, -2)) * scale
    hide = torch.arange(sc.shape[-1], device=q.device)[None, :] >= lens[b:, None]
    sc.masked_fill_(hide[:, None, None, :], -math.inf)
    m1 = sc.amax(-1)
    sc = torch.exp(sc - torch.where(m1 == -math.inf, torch.zeros_like(m1), m1)[..., None])
    l1 = sc.sum(-1)
    o1 = torch.matmul(sc, v)
    m = torch.maximum(m0, m1)
    safe = torch.where(m == -math.inf, torch.zeros_like(m), m)
    a0, a1 = torch.exp(m0 - safe), torch.exp(m1 - safe)
    den = a0 * l0 + a1 * l1
    out = (a0[..., None] * o0 + a1[..., None] * o1) / torch.where(den > 0, den, torch.ones_like(den))[..., None]
    lse = safe + torch.log(den)
    on = s["active"].bool()
    s["out"][layer].copy_(torch.where(on[:, None, None], out.reshape(nt, hq, d).to(s["out"][layer].dtype),
                                      s["out"][layer]))
    s["lse"][layer].copy_(torch.where(on[:, None], lse.reshape(nt, hq), s["lse"][layer]))
    return s["out"][layer], s["lse"][layer]


# -------------------------------------------------------------------------- run
def run(s):
    c = s["case"]
    op, layers = c["op"], range(c["layers"])
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if own:
        db = s["batch"]
        if op == "tables":
            db.reserve(s["new"], s["start"], s["rows"], s["slots"], s["positions"], s["served"])
            db.reserve(s["back"], s["start"], s["rows"], s["slots2"], s["positions2"], s["served2"])
        elif op == "append":
            for i in layers:
                q, k, v = s["qkv"][i].split([hq * d, hkv * d, hkv * d], dim=1)
                db.append(i, s["slots"], s["positions"], k, v, q if c["with_q"] else None,
                          s["q_rot"][i] if c["with_q"] else None)
        else:
            db.plan()
            for i in layers:
                db.decode(i, s["q_rot"][i], s["out"][i], s["lse"][i])
    elif op == "tables":
        _plain_reserve(s, s["new"], s["slots"], s["positions"], s["served"])
        _plain_reserve(s, s["back"], s["slots2"], s["positions2"], s["served2"])
    elif op == "append":
        [_plain_append(s, i) for i in layers]
    else:
        [_plain_attend(s, i) for i in layers]
    if op == "tables":
        return {k: s[k] for k in ("slots", "positions", "served", "slots2", "positions2", "served2", "table", "free",
                                  "free_count", "seq_len")}
    if op == "append":
        return {"k": s["k_pages"], "v": s["v_pages"], "q": s["q_rot"]}
    return {"out": s["out"], "lse": s["lse"]}


def exact(case, seed):
    """In 64 bits, prompt by prompt and question by question, from the definitions."""
    if case["op"] == "tables":
        return None
    s = prepare(case, seed)
    sh = _shape(case)
    b, hq, hkv, d, page = case["prompts"], case["hq"], case["hkv"], case["d"], case["page"]
    gr = hq // hkv
    if case["op"] == "append":
        h = d // 2
        theta = torch.tensor([math.exp(-2.0 * j / d * math.log(ROPE_BASE)) for j in range(h)], dtype=torch.float64,
                             device=DEV)
        turn = torch.polar(torch.ones(s["rows"], h, dtype=torch.float64, device=DEV),
                           s["positions"].double()[:, None] * theta)[:, None, :]

        def rotated(x):
            z = torch.complex(x[..., :h].contiguous(), x[..., h:].contiguous()) * turn
            return torch.cat([z.real, z.imag], dim=-1)

        live = (s["slots"] >= 0).nonzero()[:, 0]
        slot = s["slots"][live].long()
        ks, vs, qs = [], [], []
        for i in range(case["layers"]):
            x = s["qkv"][i].double().reshape(s["rows"], hq + 2 * hkv, d)
            kp, vp, qp = s["k_pages"][i].double(), s["v_pages"][i].double(), s["q_rot"][i].double()
            kr, qr = rotated(x[:, hq:hq + hkv]), rotated(x[:, :hq])
            for g in range(hkv):
                kp[slot // page, g, slot % page] = kr[live, g]
                vp[slot // page, g, slot % page // 8, :, slot % 8] = x[live, hq + hkv + g]
            if case["with_q"]:
                qp[live] = qr[live]
            ks.append(kp), vs.append(vp), qs.append(qp)
        return {"k": ks, "v": vs, "q": qs}
    outs, lses = [], []
    for i in range(case["layers"]):
        out = torch.zeros(sh["nt"], hq, d, dtype=torch.float64, device=DEV)
        lse = torch.zeros(sh["nt"], hq, dtype=torch.float64, device=DEV)

        def keys(seq, n, i=i):
            t = s["table"][seq, :-(-n // page)].long()
            k = s["k_pages"][i][t].double().transpose(0, 1).reshape(hkv, -1, d)[:, :n]
            v = s["v_pages"][i][t].double().permute(1, 0, 2, 4, 3).reshape(hkv, -1, d)[:, :n]
            return k, v

        for p in range(b):
            ck, cv = keys(p, int(sh["ctx"][p]))
            todo = [j for j in range(sh["q_start"][p], sh["q_start"][p + 1]) if sh["active"][j]]
            if not todo:
                continue
            qs = s["q_rot"][i][todo].double().reshape(len(todo), hkv, gr, d).transpose(0, 1)
            shared = torch.matmul(qs.reshape(hkv, len(todo) * gr, d), ck.transpose(1, 2)) / math.sqrt(d)
            shared = shared.reshape(hkv, len(todo), gr, -1)
            tops, sums = shared.amax(-1), None
            weights = torch.exp(shared - tops[..., None])
            sums = weights.sum(-1)
            vals = torch.matmul(weights.reshape(hkv, len(todo) * gr, -1), cv).reshape(hkv, len(todo), gr, d)
            for n, j in enumerate(todo):
                sk, sv = keys(b + j, int(sh["seg"][j]))
                own_sc = torch.matmul(qs[:, n], sk.transpose(1, 2)) / math.sqrt(d)
                lc = tops[:, n] + torch.log(sums[:, n])
                ls = torch.logsumexp(own_sc, -1)
                z = torch.logaddexp(lc, ls)
                o = torch.exp(lc - z)[..., None] * vals[:, n] / sums[:, n][..., None]
                o = o + torch.matmul(torch.exp(own_sc - z[..., None]), sv)
                out[j], lse[j] = o.reshape(hq, d), z.reshape(hq)
        outs.append(out), lses.append(lse)
    return {"out": outs, "lse": lses}


def work(case):
    sh = _shape(case)
    e = 4 if case["dtype"] == "f32" else 2
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    new, start = _new_tokens(case, sh)
    n = len(sh["lens"])
    if case["op"] == "tables":
        have = sh["lens"] if case["step"] else np.zeros_like(sh["lens"])
        pages = int((_pages(have + new, page) - _pages(have, page)).sum())
        grown = int((new > 0).sum())
        # both calls: counts, rows' offsets, lengths read; lengths of grown sequences, slots, positions, served
        # written; pages moved between stack and tables
        one = 4 * (n + n + 1 + n) + 4 * (grown + 2 * int(start[-1]) + n)
        return {"bytes": 2 * one + 4 * 4 * pages + 16, "flops": 0}
    if case["op"] == "append":
        t = int(new.sum())
        heads = 2 * hkv + (hq if case["with_q"] else 0)
        turned = hkv + (hq if case["with_q"] else 0)
        return {"bytes": case["layers"] * (2 * t * heads * d * e + 8 * int(start[-1])),
                "flops": case["layers"] * 3 * t * turned * d}
    act = np.add.reduceat(sh["active"].astype(np.int64), sh["q_start"][:-1])
    na = int(act.sum())
    seg = int(sh["seg"][sh["active"]].sum())
    ctx = int(sh["ctx"][act > 0].sum())
    seen = int((sh["ctx"] * act).sum()) + seg
    return {"bytes": case["layers"] * (2 * (ctx + seg) * hkv * d * e + na * hq * (2 * d * e + 4)),
            "flops": case["layers"] * 4 * d * hq * seen}
