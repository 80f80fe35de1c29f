"""Layers that keep their full cache, as measurable cases: the plain forms and the framework's calls.

A full cache holds every token of a row, in pages of ``page`` tokens that the rows' page tables name:
token p of row b lies in slot p % page of page table[b, p // page] of the pools [pages, kv heads,
page, d].  Row b of the cache holds lengths[b] tokens when a call is made, and gets the call's new
tokens (one for each row, or the tokens cu_seqlens[b] .. cu_seqlens[b + 1] - 1 of packed tensors
[T, heads, d]) at the positions lengths[b], lengths[b] + 1, ...; a negative length marks a row of the
batch that is not in use.  Three operators, in the kinds of pass that a program makes of them:

- ``rotate``: the position rotation of packed queries and keys, and its gradients, as a training
  step has them around causal attention (``DMCRotation.forward``, ``DMCRotation.backward``).
- ``append``: new keys, rotated on the way, and values enter the pages, and the queries come out
  rotated (``DMCFull.append``).
- ``attend``: the new tokens attend to their row's cache, up to themselves (``DMCFull.attend``): a
  decode step, a draft to check, a piece of a prompt.

The rotation takes pair j of a head, elements (j, j + r / 2) ("halves") or (2 j, 2 j + 1)
("adjacent") of its first r, by the angle p f_j at position p.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda"
ROTATE = dict(kind="rotate", hq=32, hkv=32, d=128, dtype="bf16", rotary=128, pairs="halves", rows=1,
              longest=1024, ragged=False, fused=False, start=0)
APPEND = dict(kind="append", hq=32, hkv=32, d=128, dtype="bf16", rotary=128, pairs="halves", page=32,
              rows=1, context=0, chunk=1, ragged=False, fused=False, queries=True, idle=0)
ATTEND = dict(kind="attend", hq=32, hkv=32, d=128, dtype="bf16", page=32, rows=1, context=0, chunk=1,
              ragged=False, fused=False, idle=0)


def listed():
    return [
        # Queries and keys of a training step on packed documents, 7B layer: rotation and gradients.
        dict(ROTATE, name="rotate_7b", rows=6, longest=4096, ragged=True, fused=True),
        # A small model at the size of a gradient check: fp32, half of the elements, far positions.
        dict(ROTATE, name="rotate_small", hq=8, hkv=4, d=64, dtype="fp32", rotary=32, pairs="adjacent",
             rows=4, longest=77, ragged=True, start=1000000),
        # The new tokens of a decode step of a serving batch, 70B grouped-query layer.
        dict(APPEND, name="append_step", hq=64, hkv=8, rows=32, context=2000, ragged=True),
        # Whole ragged prompts, packed, into empty rows (7B layer, views of one projection).
        dict(APPEND, name="append_prompts", rows=6, chunk=4096, ragged=True, fused=True),
        # A small model's short questions, keys and values only, as they are (no rotation).
        dict(APPEND, name="append_small", hq=8, hkv=8, d=64, dtype="fp32", rotary=0, page=16, rows=3,
             context=90, chunk=40, ragged=True, queries=False),
        # One user, a short cache: nothing but latency.
        dict(ATTEND, name="step_one", hq=16, hkv=4, context=900),
        # A serving batch, 7B layer, 4096 tokens of context.
        dict(ATTEND, name="step_7b", rows=48, context=4095),
        # The same on a 70B layer at long, uneven contexts, two rows of the batch not in use.
        dict(ATTEND, name="step_70b", hq=64, hkv=8, rows=18, context=24000, ragged=True, idle=2),
        # fp32 as parity and debugging work runs, odd sizes.
        dict(ATTEND, name="step_fp32_odd", hq=12, hkv=6, d=64, dtype="fp32", page=16, rows=5,
             context=1501, ragged=True),
        # Drafted tokens to check, 70B layer.
        dict(ATTEND, name="draft_70b", hq=64, hkv=8, rows=16, context=8192, chunk=4, ragged=True),
        # Pieces of long prompts behind what is already cached.
        dict(ATTEND, name="piece_70b", hq=64, hkv=8, rows=4, context=12000, chunk=512, fused=True),
        # The next turn of a few conversations, fp32, odd sizes, a row without new tokens.
        dict(ATTEND, name="turn_fp32", hq=12, hkv=6, d=64, dtype="fp32", page=16, rows=5, context=700,
             chunk=77, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case of the listed ones' ranges."""
    kind = rng.choice(["rotate", "append", "append", "attend", "attend", "attend", "attend"])
    fp32 = rng.random() < 0.25
    es = 4 if fp32 else 2
    g = rng.choice([1, 1, 2, 3, 4, 8])
    hkv = rng.choice([2, 4, 6, 8, 16, 32]) if g <= 2 else rng.choice([1, 2, 4, 8])
    d = rng.choice([64, 128, 128])
    shape = dict(hq=hkv * g, hkv=hkv, d=d, dtype="fp32" if fp32 else "bf16", ragged=rng.random() < 0.7,
                 fused=rng.random() < 0.4)
    turn = dict(rotary=rng.choice([d, d, d // 2, 16]), pairs=rng.choice(["halves", "halves", "adjacent"]))
    most = (1 << 31) // (32 * (g + 1) * hkv * d * es)   # tokens of a rotation
    if kind == "rotate":
        longest = _log_int(rng, 1, min(8192, most))
        return dict(ROTATE, **shape, **turn, longest=longest, start=rng.choice([0, 0, 0, _log_int(rng, 10, 1 << 22)]),
                    rows=_log_int(rng, 1, max(1, min(48, most // longest))))
    shape.update(page=rng.choice([8, 16, 32, 32, 32, 64, 256]))
    room = 3 << 30   # bytes of the pools
    if kind == "append":
        if rng.random() < 0.2:
            turn["rotary"] = 0
        chunk = rng.choice([1, _log_int(rng, 1, 4096)])
        context = rng.choice([0, _log_int(rng, 1, 4096)])
        rows = _log_int(rng, 1, max(1, min(64, most // chunk, room // ((context + chunk) * hkv * d * es * 2))))
        return dict(APPEND, **shape, **turn, chunk=chunk, context=context, rows=rows,
                    queries=rng.random() < 0.8, idle=rng.choice([0, 0, 1]) if rows > 2 else 0)
    pairs = (1 << 26) if fp32 else (1 << 30)   # (query, key) pairs that a pass may take, all heads
    chunk = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 2, 256 if fp32 else 1024)])
    context = rng.choice([_log_int(rng, 1, 32768), _log_int(rng, 200, 32768), 0 if chunk > 1 else 1])
    context = min(context, pairs // (2 * chunk * hkv * g), room // (hkv * d * es * 2))
    rows = _log_int(rng, 1, max(1, min(64, pairs // (chunk * (context + chunk) * hkv * g),
                                       room // ((context + chunk + shape["page"]) * hkv * d * es * 2))))
    return dict(ATTEND, **shape, chunk=chunk, context=context, rows=rows,
                idle=rng.choice([0, 0, 1]) if rows > 2 else 0)


# ---------------------------------------------------------------------------
# Lengths and inputs
# ---------------------------------------------------------------------------

def _lens(case):
    """New tokens of every row: one, or the longest, or spread below it (one row as long, one empty)."""
    rows, longest = case["rows"], case["longest"] if case["kind"] == "rotate" else case["chunk"]
    if longest == 1 or not case["ragged"]:
        return [longest] * rows
    rng = random.Random(longest * 131 + rows)
    lens = [max(1, int(longest * (0.15 + 0.85 * rng.random()))) for _ in range(rows)]
    lens[rng.randrange(rows)] = longest
    if rows > 4:
        lens[(lens.index(longest) + 2) % rows] = 0
    return lens


def _contexts(case):
    """Tokens that every row has cached; -1 for the last ``idle`` rows."""
    rows, n = case["rows"], case["context"]
    rng = random.Random(n * 17 + rows)
    held = [int(n * (1.0 - 0.75 * rng.random())) if case["ragged"] and i else n for i in range(rows)]
    return held[:rows - case["idle"]] + [-1] * case["idle"]


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEVICE)


def _freqs(case):
    r = case["rotary"]
    return None if r == 0 else (10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float().to(DEVICE)


def _heads(case, gen, tokens, *heads):
    """Tensors [T, heads, d] ~ N(0, 1): separate ones, or views of one projection."""
    d, dt = case["d"], _dtype(case)

    def make(h):
        return torch.randn((tokens, h, d), generator=gen, device=DEVICE, dtype=dt)

    return make(sum(heads)).split(heads, 1) if case["fused"] else [make(h) for h in heads]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed((seed * 1009 + 7) & 0x7FFFFFFFFFFF)
    hq, hkv, d, dt = case["hq"], case["hkv"], case["d"], _dtype(case)
    lens = _lens(case)
    T = sum(lens)
    st = dict(case=case, lens=lens)
    if own:
        import paper_2403_09636_amd as dmc
    if case["kind"] == "rotate":
        st["q"], st["k"] = _heads(case, gen, T, hq, hkv)
        st["gq"], st["gk"] = _heads(case, gen, T, hq, hkv)
        st["positions"] = _int32([case["start"] + i for n in lens for i in range(n)])
        st["freqs"] = _freqs(case)
        for x, y in (("q_out", "q"), ("k_out", "k"), ("dq", "q"), ("dk", "k")):
            st[x] = torch.empty(st[y].shape, device=DEVICE, dtype=dt)
        if own:
            cfg = dmc.make_rotary_config(hq, hkv, d, case["dtype"], rotary_dim=case["rotary"], pairs=case["pairs"])
            st["rotation"] = dmc.DMCRotation(cfg, st["freqs"], device=DEVICE)
        return st

    held, page = _contexts(case), case["page"]
    need = [-(-(max(n, 0) + m) // page) for n, m in zip(held, lens)]
    width, pages = max(need), sum(need) + 3
    st.update(held=held, freqs=_freqs(case) if case["kind"] == "append" else None)
    if own:
        cfg = dmc.make_full_config(case["rows"], hq, hkv, d, case["dtype"], page_size=page, max_pages=width,
                                   num_pages=pages, rotary_dim=case.get("rotary", 0),
                                   pairs=case.get("pairs", "halves"))
        full = dmc.DMCFull(cfg, max_tokens=T, max_chunk=case["chunk"], inv_freq=st["freqs"], device=DEVICE)
        st.update(full=full, kp=full.k_pages[0], vp=full.v_pages[0], table=full.page_table, lengths=full.lengths)
    else:
        st["kp"], st["vp"] = (torch.empty((pages, hkv, page, d), device=DEVICE, dtype=dt) for _ in range(2))
        st["table"], st["lengths"] = _int32([[0] * width] * case["rows"]), _int32([0] * case["rows"])
    st["lengths"].copy_(_int32(held))
    # the pages of a cache that has been in use for a while lie in no order
    order = torch.randperm(pages, generator=gen, device=DEVICE, dtype=torch.int32)
    st["table"].fill_(-1)
    for b, (at, n) in enumerate(zip(_cu(need), need)):
        st["table"][b, :n] = order[at:at + n]
    st["kp"].normal_(generator=gen)
    st["vp"].normal_(generator=gen)
    st["q"], k, v = _heads(case, gen, T, hq, hkv, hkv)
    st["cu"] = None if case["chunk"] == 1 else _int32(_cu(lens))
    if case["kind"] == "append":
        st.update(k=k, v=v, q_out=torch.empty((T, hq, d), device=DEVICE, dtype=dt))
    else:
        st["q"] *= 2   # scores that tell tokens apart
        st.update(out=torch.empty((T, hq, d), device=DEVICE, dtype=dt), lse=torch.empty((T, hq), device=DEVICE))
    return st


def run(st):
    if own:
        return _run_own(st)
    return _run_plain(st)


def _run_own(st):
    case = st["case"]
    if case["kind"] == "rotate":
        rot = st["rotation"]
        rot.forward(st["q"], st["k"], st["positions"], q_out=st["q_out"], k_out=st["k_out"])
        rot.backward(st["gq"], st["gk"], st["positions"], dq=st["dq"], dk=st["dk"])
        return {x: st[x] for x in ("q_out", "k_out", "dq", "dk")}
    full = st["full"]
    if case["kind"] == "append":
        if not case["queries"]:
            full.append(0, st["k"], st["v"], cu_seqlens=st["cu"])
            return dict(kp=st["kp"], vp=st["vp"])
        full.append(0, st["k"], st["v"], q=st["q"], q_out=st["q_out"], cu_seqlens=st["cu"])
        return dict(kp=st["kp"], vp=st["vp"], q_out=st["q_out"])
    full.attend(0, st["q"], cu_seqlens=st["cu"], max_chunk=case["chunk"], out=st["out"], lse=st["lse"])
    return dict(out=st["out"], lse=st["lse"])


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------

def _run_plain(st):
    case = st["case"]
    if case["kind"] == "rotate":
        c, s = _angles(st["positions"], st["freqs"])
        st["q_out"].copy_(_turn(case, st["q"], c, s))
        st["k_out"].copy_(_turn(case, st["k"], c, s))
        st["dq"].copy_(_turn(case, st["gq"], c, -s))
        st["dk"].copy_(_turn(case, st["gk"], c, -s))
        return {x: st[x] for x in ("q_out", "k_out", "dq", "dk")}
    if case["kind"] == "append":
        return _plain_append(st)
    return _plain_attend(st)


def _angles(positions, freqs):
    a = positions.double()[:, None] * freqs.double()   # (64 bits: far positions)
    return a.cos().float()[:, None], a.sin().float()[:, None]


def _turn(case, x, c, s):
    """x [T, heads, d] rotated by the angles of cos, sin [T, 1, r / 2]."""
    r, y = case["rotary"], x.float().clone()
    if case["pairs"] == "halves":
        a, b = y[..., :r // 2].clone(), y[..., r // 2:r].clone()
        y[..., :r // 2], y[..., r // 2:r] = a * c - b * s, b * c + a * s
    else:
        a, b = y[..., 0:r:2].clone(), y[..., 1:r:2].clone()
        y[..., 0:r:2], y[..., 1:r:2] = a * c - b * s, b * c + a * s
    return y.to(x.dtype)


def _rows_positions(st):
    """Row and position of every new token; a negative position in rows that are not in use."""
    lens = torch.tensor(st["lens"], device=DEVICE)
    row = torch.repeat_interleave(torch.arange(len(st["lens"]), device=DEVICE), lens, output_size=sum(st["lens"]))
    i = torch.arange(len(row), device=DEVICE) - (lens.cumsum(0) - lens)[row]
    n = st["lengths"].long()[row]
    return row, torch.where(n < 0, -1, n + i)


def _plain_append(st):
    case = st["case"]
    row, pos = _rows_positions(st)
    k, q = st["k"], st["q"]
    if case["rotary"]:
        c, s = _angles(pos, st["freqs"])
        k = _turn(case, k, c, s)
        if case["queries"]:
            q = _turn(case, q, c, s)
    if case["queries"]:
        st["q_out"].copy_(torch.where((pos >= 0)[:, None, None], q, 0))
    used = (pos >= 0).nonzero()[:, 0]
    page = st["table"][row, pos // case["page"]].long()[used]
    slot = (pos % case["page"])[used]
    st["kp"][page, :, slot] = k[used]
    st["vp"][page, :, slot] = st["v"][used]
    return dict(kp=st["kp"], vp=st["vp"], **(dict(q_out=st["q_out"]) if case["queries"] else {}))


def _plain_attend(st):
    case = st["case"]
    G, hkv, d, page = case["hq"] // case["hkv"], case["hkv"], case["d"], case["page"]
    lo = 0
    for b, (n, m) in enumerate(zip(st["held"], st["lens"])):
        r = slice(lo, lo + m)
        lo += m
        if m == 0:
            continue
        if n < 0:
            st["out"][r], st["lse"][r] = 0, -math.inf
            continue
        pages = st["table"][b, :-(-(n + m) // page)].long()

        def cached(x):   # [hkv, n + m, d]
            return x[pages].transpose(0, 1).reshape(hkv, -1, d)[:, :n + m].float()

        K, V = cached(st["kp"]), cached(st["vp"])
        q = st["q"][r].view(m, hkv, G, d).permute(1, 2, 0, 3).reshape(hkv, G * m, d).float()
        s = (q @ K.transpose(1, 2)).mul_(1 / math.sqrt(d))
        if m > 1:
            t = torch.arange(n + m, device=DEVICE)
            s.view(hkv, G, m, n + m).masked_fill_(t > n + t[:m, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        s.sub_(top).exp_()
        tot = s.sum(-1, keepdim=True)
        o = (s @ V) / tot
        st["out"][r] = o.view(hkv, G, m, d).permute(2, 0, 1, 3).reshape(m, hkv * G, d).to(st["out"].dtype)
        st["lse"][r] = (top + tot.log()).view(hkv, G, m).permute(2, 0, 1).reshape(m, hkv * G)
    return dict(out=st["out"], lse=st["lse"])


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    es = 4 if case["dtype"] == "fp32" else 2
    hq, hkv, d, lens = case["hq"], case["hkv"], case["d"], _lens(case)
    tok = sum(lens)
    if case["kind"] == "rotate":   # forward and gradients: two tensors read and two written each
        return dict(bytes=4 * tok * (hq + hkv) * d * es + 4 * tok, flops=2 * 3 * tok * (hq + hkv) * case["rotary"])
    held = _contexts(case)
    live = sum(m for n, m in zip(held, lens) if n >= 0)
    if case["kind"] == "append":   # (the rotated queries of rows that are not in use are written, as zeros)
        heads = (hq if case["queries"] else 0) + hkv
        nbytes = (live * 2 * (heads + hkv) + (tok - live) * (heads - hkv)) * d * es
        return dict(bytes=nbytes, flops=3 * live * heads * case["rotary"])
    seen = sum(n + m for n, m in zip(held, lens) if n >= 0 and m)
    pairs = sum(m * n + m * (m + 1) // 2 for n, m in zip(held, lens) if n >= 0)
    return dict(bytes=seen * 2 * hkv * d * es + (live + tok) * hq * d * es + 4 * tok * hq, flops=4 * d * hq * pairs)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "rotate":
        pos = st["positions"].double()
        return dict(q_out=_exact_turn(case, st["q"], pos, 1), k_out=_exact_turn(case, st["k"], pos, 1),
                    dq=_exact_turn(case, st["gq"], pos, -1), dk=_exact_turn(case, st["gk"], pos, -1))
    if case["kind"] == "append":
        return _exact_append(st)
    return _exact_attend(st)


def _exact_turn(case, x, pos, sign):
    """Pairs as complex numbers, times exp(i sign p f_j)."""
    r, y = case["rotary"], x.double()
    if r == 0:
        return y
    f = _freqs(case).double()
    z = torch.exp(torch.complex(torch.zeros_like(pos)[:, None], sign * pos[:, None] * f))[:, None]
    head, rest = y[..., :r], y[..., r:]
    if case["pairs"] == "halves":
        w = torch.complex(*head.unflatten(-1, (2, r // 2)).unbind(-2)) * z
        return torch.cat([w.real, w.imag, rest], -1)
    w = torch.complex(*head.unflatten(-1, (r // 2, 2)).unbind(-1)) * z
    return torch.cat([torch.stack([w.real, w.imag], -1).flatten(-2), rest], -1)


def _exact_append(st):
    case, page = st["case"], st["case"]["page"]
    kp, vp = st["kp"].double(), st["vp"].double()
    pos = [n + i if n >= 0 else -1 for n, m in zip(st["held"], st["lens"]) for i in range(m)]
    row = [b for b, m in enumerate(st["lens"]) for _ in range(m)]
    at = torch.tensor(pos, device=DEVICE, dtype=torch.float64)
    k, q = _exact_turn(case, st["k"], at, 1), _exact_turn(case, st["q"], at, 1)
    table = st["table"].tolist()
    live = [t for t, p in enumerate(pos) if p >= 0]
    pages = [table[row[t]][pos[t] // page] for t in live]
    where = torch.tensor([x * page + pos[t] % page for x, t in zip(pages, live)], device=DEVICE, dtype=torch.long)
    live = torch.tensor(live, device=DEVICE, dtype=torch.long)
    for pool, new in ((kp, k), (vp, st["v"].double())):
        flat = pool.transpose(1, 2).reshape(-1, case["hkv"], case["d"]).clone()
        flat[where] = new[live]
        pool.copy_(flat.view(len(pool), page, case["hkv"], case["d"]).transpose(1, 2))
    res = dict(kp=kp, vp=vp)
    if case["queries"]:
        res["q_out"] = torch.zeros_like(q).index_copy_(0, live, q[live])
    return res


def _exact_attend(st):
    """Head by head; log sum exp and softmax of the scores that each token sees."""
    case = st["case"]
    G, hkv, d = case["hq"] // case["hkv"], case["hkv"], case["d"]
    if case["rows"] * case["hq"] > 4000 or work(case)["flops"] > 2e12:
        return None
    out = torch.zeros_like(st["out"], dtype=torch.float64)
    lse = torch.full_like(st["lse"], -math.inf, dtype=torch.float64)
    cu = _cu(st["lens"])
    for b, n in enumerate(st["held"]):
        m = st["lens"][b]
        if m == 0 or n < 0:
            continue
        p = torch.arange(n + m, device=DEVICE)
        page, slot = st["table"][b].long()[p // case["page"]], p % case["page"]
        unseen = p[None] > n + torch.arange(m, device=DEVICE)[:, None]
        for h in range(case["hq"]):
            K, V = st["kp"][page, h // G, slot].double(), st["vp"][page, h // G, slot].double()
            s = torch.mm(st["q"][cu[b]:cu[b + 1], h].double(), K.t()) * d ** -0.5
            s = torch.where(unseen, -math.inf, s)
            z = torch.logsumexp(s, 1)
            lse[cu[b]:cu[b + 1], h] = z
            out[cu[b]:cu[b + 1], h] = torch.mm(torch.exp(s - z[:, None]), V)
    return dict(out=out, lse=lse)
