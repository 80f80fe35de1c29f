"""Attention on packed sequences, as measurable cases: the plain forms and the framework's calls.

Packed sequences lie one after another in tensors [T, heads, d]; row b holds the tokens
cu_seqlens[b] .. cu_seqlens[b + 1] - 1, and rows of a buffer behind the last sequence stay as they
are.  Four operators, in the kinds of pass that a program makes of them:

- ``attend``: a chunk of new tokens attends over a paged, compressed cache (``DMCChunk.attend``),
  which stays as it is: the check of drafted tokens, or a piece of a prompt.
- ``serve``: prompts enter an emptied cache in pieces, each attended and appended
  (``DMCChunk.attend``, ``DMCChunk.append``); the cache comes out at the end, as a session that is
  parked.  With ``attend`` false the pieces are only appended.
- ``forward``: causal attention of whole sequences without a cache (``DMCCausal.forward``).
- ``train``: that, and its gradients (``DMCCausal.backward``).

The update of the cache is Algorithm 1 of the DMC paper: token t of a unit (one row, one kv head)
merges into the open slot when k_t[0] > c, else opens a new slot; an empty unit opens one.  A slot
is the omega-weighted mean of its tokens (k[0] as 0), omega_t = sigmoid(q_t[0]).  Token t attends to
the closed slots and to its own slot as it stands after the token's update.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda"
ATTEND = dict(kind="attend", hq=32, hkv=32, d=128, dtype="bf16", page=32, rows=1, context=0, chunk=8,
              ragged=False, fused=False, cr="mix", omega="lead", decision="per_head", bias=0.0, tail=0)
SERVE = dict(ATTEND, kind="serve", pieces=1, attend=True)
FORWARD = dict(kind="forward", hq=32, hkv=32, d=128, dtype="bf16", rows=1, longest=1024, ragged=False,
               fused=False, tail=0)
TRAIN = dict(FORWARD, kind="train")


def listed():
    return [
        # One user, four drafted tokens to check, a short cache: nothing but latency.
        dict(ATTEND, name="verify_one", hq=16, hkv=4, context=900, chunk=4),
        # Drafted tokens of a serving batch, 7B layer at 4096 tokens of context, uneven heads.
        dict(ATTEND, name="verify_7b", rows=24, context=4096, chunk=6, ragged=True),
        # The same on a 70B grouped-query layer at long context.
        dict(ATTEND, name="verify_70b", hq=64, hkv=8, rows=16, context=16384, chunk=4, cr="two"),
        # Pieces of long prompts behind what is already cached (prompts fed in pieces of 512).
        dict(ATTEND, name="piece_70b", hq=64, hkv=8, rows=4, context=12000, chunk=512, cr="two",
             fused=True),
        # The next turn of a few conversations: ragged questions over ragged caches, odd sizes,
        # fp32 as parity and debugging work runs.
        dict(ATTEND, name="turn_fp32_odd", hq=12, hkv=6, d=64, dtype="fp32", page=16, rows=5,
             context=1500, chunk=77, ragged=True, omega="group_mean", bias=0.5, tail=9),
        # Whole ragged prompts, packed, into an empty cache with attention (7B layer).
        dict(SERVE, name="prompts_7b", rows=6, chunk=4096, ragged=True, tail=64),
        # Prompts fed in pieces, grouped heads: attend and append, four times.
        dict(SERVE, name="pieces_gqa", hq=32, hkv=8, rows=7, chunk=301, pieces=4, ragged=True),
        # A small model's short questions, only appended (a cache that is filled ahead of use).
        dict(SERVE, name="append_small", hq=8, hkv=8, d=64, dtype="fp32", page=16, rows=3, chunk=40,
             ragged=True, attend=False),
        # A small model's answer checked as a whole (scoring): short packed sequences.
        dict(FORWARD, name="score_small", hq=8, hkv=4, d=64, rows=6, longest=90, ragged=True, tail=7),
        # Long documents and short ones through an uncompressed layer of the 7B shape.
        dict(FORWARD, name="forward_7b", rows=5, longest=8192, ragged=True, fused=True),
        # Training on packed documents, grouped heads.
        dict(TRAIN, name="train_gqa", hq=32, hkv=8, rows=6, longest=4096, ragged=True, tail=100),
        # fp32 training at the size of a gradient check or a small model.
        dict(TRAIN, name="train_fp32", hq=8, hkv=4, d=64, dtype="fp32", rows=4, longest=640, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case of the listed ones' ranges."""
    kind = rng.choice(["attend", "attend", "attend", "serve", "serve", "forward", "train", "train"])
    fp32 = rng.random() < 0.25
    g = rng.choice([1, 1, 2, 4, 8])
    hkv = rng.choice([2, 4, 6, 8, 16, 32]) if g <= 2 else rng.choice([1, 2, 4, 8])
    d = rng.choice([64, 128, 128])
    shape = dict(hq=hkv * g, hkv=hkv, d=d, dtype="fp32" if fp32 else "bf16", ragged=rng.random() < 0.7,
                 fused=rng.random() < 0.4, tail=rng.choice([0, 0, 1, 50]))
    # (query, key) pairs that a pass may take, all heads
    pairs = (1 << 29) if fp32 else (6 << 30)
    if kind in ("forward", "train"):
        longest = _log_int(rng, 1, 1200 if fp32 else 8192)
        most = pairs // (3 if kind == "train" else 1) * 2 // (longest * longest * hkv * g)
        rows = _log_int(rng, 1, max(1, min(48, most, 24576 // longest)))
        return dict(FORWARD if kind == "forward" else TRAIN, **shape, rows=rows, longest=longest)
    shape.update(page=rng.choice([8, 16, 32, 32, 32, 64, 256]), cr=rng.choice(["mix", "two", "skew"]),
                 omega=rng.choice(["lead", "lead", "group_mean", "uniform"]),
                 decision=rng.choice(["per_head", "per_head", "per_head", "shared_layer"]),
                 bias=rng.choice([0.0, 0.0, 1.5]))
    if kind == "attend":
        context = rng.choice([0, _log_int(rng, 1, 16384), _log_int(rng, 200, 16384)])
        chunk = rng.choice([_log_int(rng, 1, 16), _log_int(rng, 1, 512 if fp32 else 2048)])
        most = min(pairs // 2 // (chunk * (context + chunk) * hkv * g),
                   (1 << 31) // (max(context, 64) * hkv * d * (8 if fp32 else 4)))
        return dict(ATTEND, **shape, context=context, chunk=chunk,
                    rows=_log_int(rng, 1, max(1, min(48, most))))
    pieces = rng.choice([1, 2, 3, 5])
    total = _log_int(rng, pieces, 900 if fp32 else 4096)
    chunk = -(-total // pieces)
    most = min(pairs // 2 // (total * total * hkv * g), 16384 // total)
    return dict(SERVE, **shape, chunk=chunk, pieces=pieces, rows=_log_int(rng, 1, max(1, min(24, most))),
                attend=rng.random() < 0.7)


# ---------------------------------------------------------------------------
# Lengths and inputs
# ---------------------------------------------------------------------------

def _crs(case):
    """Compression ratio of every kv head: 1, 2, 4, 8 in turn; 2; or every tenth head 1 and the
    others spread over 16 .. 32."""
    h = case["hkv"]
    if case["cr"] == "two":
        return [2.0] * h
    if case["cr"] == "skew":
        return [1.0 if i % 10 == 3 else 16.0 * 2.0 ** ((i * 7 % 10) / 9) for i in range(h)]
    return [(1.0, 2.0, 4.0, 8.0)[i % 4] for i in range(h)]


def _lens(case, longest):
    """Tokens of every row: the longest, or spread below it (one row as long, one or two empty)."""
    rows = case["rows"]
    if not case["ragged"]:
        return [longest] * rows
    rng = random.Random(longest * 131 + rows)
    lens = [int(longest * (0.15 + 0.85 * rng.random())) for _ in range(rows)]
    lens[rng.randrange(rows)] = longest
    if rows > 4:
        lens[(lens.index(longest) + 2) % rows] = 0
    return lens


def _contexts(case):
    """Tokens that every row has cached."""
    if not case["ragged"]:
        return [case["context"]] * case["rows"]
    rng = random.Random(case["context"] * 17 + case["rows"])
    return [int(case["context"] * (1.0 - 0.75 * rng.random())) for _ in range(case["rows"])]


def _slots(case):
    """Slots cached by every unit, [rows][hkv]."""
    if case["decision"] == "shared_layer":
        return [[math.ceil(n / _crs(case)[0])] * case["hkv"] for n in _contexts(case)]
    return [[math.ceil(n / cr) for cr in _crs(case)] for n in _contexts(case)]


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _generator(seed, stream):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed((seed * 1009 + stream) & 0x7FFFFFFFFFFF)
    return gen


def _qkv(case, gen, tokens):
    """q [T, Hq, d], k, v [T, Hkv, d] ~ N(0, 1): three tensors, or views of one projection."""
    hq, hkv, d, dt = case["hq"], case["hkv"], case["d"], _dtype(case)
    rows = tokens + case["tail"]

    def make(h):
        return torch.randn((rows, h, d), generator=gen, device=DEVICE, dtype=dt)

    if case["fused"]:
        x = make(hq + 2 * hkv)
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    return make(hq), make(hkv), make(hkv)


def _decisions(case, gen, k):
    """k[..., 0] := decision logits that append with probability 1 / CR of the head (the first
    head's decide for all of them with ``shared_layer``)."""
    u = torch.rand(k.shape[:2], generator=gen, device=DEVICE).clamp_(1e-6, 1 - 1e-6)
    noise = torch.log(u) - torch.log1p(-u)
    cr = torch.tensor(_crs(case), device=DEVICE)
    k[..., 0] = torch.where(cr > 1, noise + torch.log((cr - 1).clamp_min(1e-6)), -1 - noise.abs()).to(k.dtype)


def _outputs(case, rows, *heads):
    return [torch.zeros((rows, h, case["d"]), device=DEVICE, dtype=_dtype(case)) for h in heads]


def prepare(case, seed):
    gen = _generator(seed, 1)
    st = dict(case=case)
    if case["kind"] in ("forward", "train"):
        lens = _lens(case, case["longest"])
        q, k, v = _qkv(case, gen, sum(lens))
        st.update(lens=lens, q=q, k=k, v=v, cu=torch.tensor(_cu(lens), dtype=torch.int32, device=DEVICE),
                  out=_outputs(case, len(q), case["hq"])[0],
                  lse=torch.zeros((len(q), case["hq"]), device=DEVICE))
        if case["kind"] == "train":
            st["dout"] = torch.randn(q.shape, generator=gen, device=DEVICE, dtype=q.dtype)
            st["grads"] = _outputs(case, len(q), case["hq"], case["hkv"], case["hkv"])
        if own:
            import paper_2403_09636_amd as dmc
            cfg = dmc.make_causal_config(case["hq"], case["hkv"], case["d"], case["dtype"])
            st["causal"] = dmc.DMCCausal(cfg, len(q), device=DEVICE)
        return st

    pieces = case.get("pieces", 1)
    total = _lens(case, case["chunk"] * pieces)
    st["pieces"] = []
    for i in range(pieces):
        lens = [min(max(n - i * case["chunk"], 0), case["chunk"]) for n in total]
        q, k, v = _qkv(case, gen, sum(lens))
        _decisions(case, gen, k)
        st["pieces"].append(dict(lens=lens, q=q, k=k, v=v, out=_outputs(case, len(q), case["hq"])[0],
                                 slots=torch.full((len(q), case["hkv"]), -1, dtype=torch.int32, device=DEVICE),
                                 cu=torch.tensor(_cu(lens), dtype=torch.int32, device=DEVICE)))
    most = max(len(p["q"]) for p in st["pieces"])
    rows, hkv, d = case["rows"], case["hkv"], case["d"]
    slots = torch.tensor(_slots(case), dtype=torch.int32, device=DEVICE)
    held = max(1, max(max(s) for s in _slots(case)))
    st["dense"] = case["chunk"] * pieces
    if case["kind"] == "attend":
        K, V = (torch.randn((rows, hkv, held, d), generator=gen, device=DEVICE, dtype=_dtype(case))
                for _ in range(2))
        K[..., 0] = 0
        z = torch.rand((rows, hkv), generator=gen, device=DEVICE) * 3 + 0.1
        st.update(K=K, V=V, z=z, slots=slots)
    if own:
        import paper_2403_09636_amd as dmc
        cfg = dmc.make_config(1, rows, case["hq"], hkv, d, case["dtype"], page_size=case["page"],
                              max_slots_per_seq=held + case["chunk"] * pieces, max_prompt_len=1,
                              decision_bias=case["bias"], omega_src=case["omega"],
                              decision_src=case["decision"])
        st["cache"] = dmc.DMCCache(cfg, device=DEVICE)
        if case["kind"] == "attend":
            st["cache"].import_(0, K, V, slots, z)
            del st["K"], st["V"]
        st["chunk"] = dmc.DMCChunk(st["cache"], most, case["chunk"])
    return st


def run(st):
    if own:
        return _run_own(st)
    return _run_plain(st)


def _run_own(st):
    case = st["case"]
    if case["kind"] in ("forward", "train"):
        causal = st["causal"]
        causal.forward(st["q"], st["k"], st["v"], st["cu"], out=st["out"], lse=st["lse"])
        if case["kind"] == "forward":
            return dict(out=st["out"], lse=st["lse"])
        dq, dk, dv = st["grads"]
        causal.backward(st["q"], st["k"], st["v"], st["cu"], st["out"], st["lse"], st["dout"], dq=dq, dk=dk, dv=dv)
        return dict(out=st["out"], lse=st["lse"], dq=dq, dk=dk, dv=dv)
    chunk, cache = st["chunk"], st["cache"]
    if case["kind"] == "attend":
        p = st["pieces"][0]
        return dict(out=chunk.attend(0, p["q"], p["k"], p["v"], p["cu"], out=p["out"]))
    cache.reset()
    res = {}
    for i, p in enumerate(st["pieces"]):
        if case["attend"]:
            res[f"out{i}"] = chunk.attend(0, p["q"], p["k"], p["v"], p["cu"], out=p["out"])
        chunk.append(0, p["k"], p["v"], p["q"], p["cu"], slot_index=p["slots"])
        res[f"slots{i}"] = p["slots"]
    K, V, z = cache.export(0, st["dense"])
    return dict(res, K=K, V=V, z=z, lengths=cache.lengths(0))


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------

def _run_plain(st):
    case = st["case"]
    if case["kind"] in ("forward", "train"):
        return _plain_causal(st)
    if case["kind"] == "attend":
        p = st["pieces"][0]
        _plain_attend(case, p, (st["K"], st["V"], st["slots"], st["z"]))
        return dict(out=p["out"])
    rows, hkv, d, dt = case["rows"], case["hkv"], case["d"], _dtype(case)
    K, V = (torch.zeros((rows, hkv, st["dense"], d), device=DEVICE, dtype=dt) for _ in range(2))
    L = torch.zeros((rows, hkv), device=DEVICE, dtype=torch.int32)
    z = torch.zeros((rows, hkv), device=DEVICE)
    res = {}
    for i, p in enumerate(st["pieces"]):
        if case["attend"]:
            _plain_attend(case, p, (K, V, L, z))
            res[f"out{i}"] = p["out"]
        _plain_append(case, p, (K, V, L, z))
        res[f"slots{i}"] = p["slots"]
    return dict(res, K=K, V=V, z=z, lengths=L)


def _plain_states(case, p, cache, b0, b1):
    """The slot that each token of rows b0 .. b1 - 1 goes to, as it stands after the token: token
    indexes and whether there is such a token [R, M], decisions, slot numbers and omega sums
    [R, Hkv, M], key and value means [R, Hkv, M, d]."""
    K, V, L, z = cache
    lens = p["lens"][b0:b1]
    R, M, G = b1 - b0, max(max(lens), 1), case["hq"] // case["hkv"]
    t = torch.arange(M, device=DEVICE)
    here = t < torch.tensor(lens, device=DEVICE)[:, None]
    at = (p["cu"][b0:b1].long()[:, None] + t).clamp(max=max(len(p["q"]) - 1, 0))
    k, v, q0 = p["k"][at].float(), p["v"][at].float(), p["q"][..., 0][at].float()   # [R, M, H, (d)]
    merge = k[..., 0] > case["bias"]
    if case["omega"] == "uniform":
        w = torch.ones_like(k[..., 0])
    else:
        w = torch.sigmoid(q0).clamp_min(2.0 ** -100).view(R, M, -1, G)
        w = w[..., 0] if case["omega"] == "lead" else w.mean(-1)
    if case["decision"] == "shared_layer":
        merge, w = merge[..., :1].expand_as(merge), w[..., :1].expand_as(w)
    k[..., 0] = 0
    k, v, merge, w = k.transpose(1, 2), v.transpose(1, 2), merge.transpose(1, 2).clone(), w.transpose(1, 2)
    L, z = L[b0:b1].long(), z[b0:b1].double()
    merge[..., 0] &= L > 0
    merge |= ~here[:, None]
    w = torch.where(here[:, None], w, 0.0).double()
    seg = (~merge).long().cumsum(-1)                      # 0: the cached open slot
    start = torch.where(merge, -1, t).cummax(-1).values   # first token of the segment, -1: before the chunk
    first = start.clamp_min(0)

    def since_start(x, held):   # sums of x over the segment's tokens up to each token (64 bits: long sums)
        s = x.cumsum(2)
        at0 = first if x.dim() == 3 else first[..., None].expand_as(x)
        old = start < 0 if x.dim() == 3 else (start < 0)[..., None]
        return s - torch.where(old, -held.unsqueeze(2), (s - x).gather(2, at0))

    j = (L - 1).clamp_min(0)[..., None, None].expand(-1, -1, 1, case["d"])
    zs = since_start(w, z)
    ks = since_start(k * w[..., None], K[b0:b1].gather(2, j)[:, :, 0].double() * z[..., None])
    vs = since_start(v * w[..., None], V[b0:b1].gather(2, j)[:, :, 0].double() * z[..., None])
    d = zs.clamp_min(1e-300)[..., None]
    return at, here, merge, L[..., None] - 1 + seg, zs, (ks / d).float(), (vs / d).float()


def _plain_attend(case, p, cache):
    K, V, L, _ = cache
    G, hkv, d = case["hq"] // case["hkv"], case["hkv"], case["d"]
    most = max(max(p["lens"]), 1)
    S = max(1, int(min(K.shape[2], max(max(s) for s in _slots(case)) if case["kind"] == "attend" else K.shape[2])))
    step = max(1, (1 << 29) // (case["hq"] * most * (S + most)))   # rows at a time
    for b0 in range(0, case["rows"], step):
        b1 = min(b0 + step, case["rows"])
        M = max(max(p["lens"][b0:b1]), 1)
        t = torch.arange(M, device=DEVICE)
        at, here, merge, _, _, ks, vs = _plain_states(case, p, cache, b0, b1)
        q = p["q"][at].float()
        q[..., 0] = 0
        q = q.view(b1 - b0, M, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(b1 - b0, hkv, G * M, d) / math.sqrt(d)
        Kc, Vc = K[b0:b1, :, :S].float(), V[b0:b1, :, :S].float()
        s1 = q @ Kc.transpose(2, 3)
        s2 = q @ ks.transpose(2, 3)
        seen = L[b0:b1].long() - merge[..., 0].long()
        s1.masked_fill_((torch.arange(S, device=DEVICE) >= seen[..., None])[:, :, None], -math.inf)
        closed = torch.zeros_like(merge)
        closed[..., :-1] = ~merge[..., 1:]
        see = (closed[:, :, None] & (t < t[:, None])) | (t == t[:, None])
        s2.view(b1 - b0, hkv, G, M, M).masked_fill_(~see[:, :, None], -math.inf)
        top = torch.maximum(s1.amax(-1, keepdim=True), s2.amax(-1, keepdim=True))
        s1, s2 = (s1 - top).exp_(), (s2 - top).exp_()
        o = (s1 @ Vc + s2 @ vs) / (s1.sum(-1, keepdim=True) + s2.sum(-1, keepdim=True))
        o = o.view(b1 - b0, hkv, G, M, d).permute(0, 3, 1, 2, 4).reshape(b1 - b0, M, hkv * G, d)
        p["out"][at[here]] = o[here].to(p["out"].dtype)


def _plain_append(case, p, cache):
    K, V, L, z = cache
    at, here, merge, slot, zs, ks, vs = _plain_states(case, p, cache, 0, case["rows"])
    p["slots"][at[here]] = slot.transpose(1, 2)[here].int()
    last = torch.tensor(p["lens"], device=DEVICE) - 1
    t = torch.arange(here.shape[1], device=DEVICE)
    keep = torch.zeros_like(merge)
    keep[..., :-1] = ~merge[..., 1:]                    # the last token of a closed segment
    keep |= (t == last[:, None])[:, None]               # and the last of the chunk
    keep &= here[:, None]
    b, h, i = keep.nonzero(as_tuple=True)
    K[b, h, slot[b, h, i]] = ks[b, h, i].to(K.dtype)
    V[b, h, slot[b, h, i]] = vs[b, h, i].to(V.dtype)
    some = (last >= 0)[:, None]
    end = last.clamp_min(0)[:, None, None].expand(-1, case["hkv"], 1)
    L.copy_(torch.where(some, slot.gather(2, end)[..., 0].int() + 1, L))
    z.copy_(torch.where(some, zs.gather(2, end)[..., 0].float(), z))


def _plain_causal(st):
    case = st["case"]
    G, hkv, d = case["hq"] // case["hkv"], case["hkv"], case["d"]
    sc = 1.0 / math.sqrt(d)
    cu = _cu(st["lens"])
    grads = case["kind"] == "train"
    for b, n in enumerate(st["lens"]):
        if n == 0:
            continue
        r = slice(cu[b], cu[b] + n)
        later = torch.ones((n, n), dtype=torch.bool, device=DEVICE).triu_(1)
        step = max(1, (1 << 30) // (n * n * G))   # kv heads at a time
        for h0 in range(0, hkv, step):
            h1 = min(h0 + step, hkv)
            qs = slice(h0 * G, h1 * G)

            def heads(x, h):   # [H, G or 1, n, d]
                return x.float().transpose(0, 1).reshape(h1 - h0, -1, n, d).contiguous()

            q, k, v = heads(st["q"][r, qs], h0), heads(st["k"][r, h0:h1], h0), heads(st["v"][r, h0:h1], h0)
            s = q @ k.transpose(2, 3)
            s.mul_(sc).masked_fill_(later, -math.inf)
            top = s.amax(-1, keepdim=True)
            s.sub_(top).exp_()
            tot = s.sum(-1, keepdim=True)
            s.div_(tot)
            o = s @ v
            st["out"][r, qs] = o.reshape(-1, n, d).transpose(0, 1).to(st["out"].dtype)
            st["lse"][r, qs] = (top + tot.log()).reshape(-1, n).transpose(0, 1)
            if not grads:
                continue
            dq, dk, dv = st["grads"]
            do = heads(st["dout"][r, qs], h0)
            dp = do @ v.transpose(2, 3)
            dp.sub_((do * o).sum(-1, keepdim=True)).mul_(s).mul_(sc)

            def rows(x):
                return x.reshape(-1, n, d).transpose(0, 1).to(st["out"].dtype)

            dv[r, h0:h1] = rows((s.transpose(2, 3) @ do).sum(1))
            dk[r, h0:h1] = rows((dp.transpose(2, 3) @ q).sum(1))
            dq[r, qs] = rows(dp @ k)
    res = dict(out=st["out"], lse=st["lse"])
    if grads:
        res.update(zip(("dq", "dk", "dv"), st["grads"]))
    return res


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def _pairs(n):
    return n * (n + 1) // 2


def work(case):
    es = 4 if case["dtype"] == "fp32" else 2
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["kind"] in ("forward", "train"):
        lens = _lens(case, case["longest"])
        tok, pairs = sum(lens), sum(map(_pairs, lens)) * hq
        rows = tok * d * es
        # q, k, v read, out and the row statistics written; with gradients: out's gradient read, three written
        if case["kind"] == "forward":
            return dict(bytes=rows * (2 * hq + 2 * hkv) + 4 * tok * hq, flops=4 * d * pairs)
        return dict(bytes=rows * (4 * hq + 4 * hkv) + 4 * tok * hq, flops=14 * d * pairs)
    G, crs = hq // hkv, _crs(case)
    if case["decision"] == "shared_layer":
        crs = [crs[0]] * hkv
    if case["kind"] == "attend":
        lens = _lens(case, case["chunk"])
        held = [s if n else [0] * hkv for n, s in zip(lens, _slots(case))]
        pairs = sum(n * s + _pairs(n) / cr for n, row in zip(lens, held) for s, cr in zip(row, crs)) * G
        return dict(bytes=int(sum(map(sum, held)) * 2 * d * es + sum(lens) * (2 * hq + 2 * hkv) * d * es),
                    flops=int(4 * d * pairs))
    lens = _lens(case, case["chunk"] * case["pieces"])
    slots = sum(n / cr for n in lens for cr in crs)
    # k, v read, slots written, and the parked cache (read and written, zeros behind its slots)
    nbytes = (sum(lens) * 2 * hkv + slots * 4 + case["rows"] * hkv * case["chunk"] * case["pieces"] * 2) * d * es
    pairs = 0
    if case["attend"]:
        nbytes += sum(lens) * 2 * hq * d * es
        pairs = sum(_pairs(n) / cr for n in lens for cr in crs) * G
    return dict(bytes=int(nbytes), flops=int(4 * d * pairs + sum(lens) * hkv * d * 4))


# ---------------------------------------------------------------------------
# The definitions in 64 bits, one unit at a time
# ---------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["kind"] in ("forward", "train"):
        return _exact_causal(st)
    return _exact_chunks(st)


def _exact_causal(st):
    """Scores, softmax and the chain rule through it, head by head."""
    case, d = st["case"], st["case"]["d"]
    G = case["hq"] // case["hkv"]
    if sum(n * n for n in st["lens"]) * case["hq"] > 6 << 30:
        return None
    res = {x: st[x].double() for x in ("out", "lse")}
    if case["kind"] == "train":
        res.update(zip(("dq", "dk", "dv"), (x.double() for x in st["grads"])))
    lo = 0
    for n in st["lens"]:
        hi = lo + n
        if n == 0:
            continue
        low = torch.ones((n, n), device=DEVICE, dtype=torch.float64).tril()
        for h in range(case["hq"]):
            q, k, v = st["q"][lo:hi, h].double(), st["k"][lo:hi, h // G].double(), st["v"][lo:hi, h // G].double()
            s = torch.mm(q, k.t()) * d ** -0.5
            lse = torch.logsumexp(torch.where(low > 0, s, -math.inf), 1)
            prob = torch.exp(s.clamp(max=lse.max()) - lse[:, None]) * low
            res["out"][lo:hi, h] = torch.mm(prob, v)
            res["lse"][lo:hi, h] = lse
            if case["kind"] == "train":
                do = st["dout"][lo:hi, h].double()
                g = torch.mm(do, v.t())
                g = prob * (g - (prob * g).sum(1, keepdim=True)) * d ** -0.5
                res["dq"][lo:hi, h] = torch.mm(g, k)
                res["dk"][lo:hi, h // G] += torch.mm(g.t(), q)
                res["dv"][lo:hi, h // G] += torch.mm(prob.t(), do)
        lo = hi
    return res


def _exact_chunks(st):
    """Per unit: the weight of every token (and of the cached open slot) in every state, as a matrix;
    states, scores and outputs as products with it.  Pieces of a prompt are one long chunk."""
    case, d, hkv = st["case"], st["case"]["d"], st["case"]["hkv"]
    G, rows, P = case["hq"] // hkv, case["rows"], st["pieces"]
    lens = [sum(p["lens"][b] for p in P) for b in range(rows)]
    if sum(n * (n + 20000) for n in lens) * hkv * (1 + G / 4) > 8e10 or rows * hkv > 2500:
        return None
    serve = case["kind"] == "serve"
    outs = [torch.zeros_like(p["out"], dtype=torch.float64) for p in P]
    slots = [torch.full_like(p["slots"], -1) for p in P]
    if serve:
        K, V = (torch.zeros((rows, hkv, st["dense"], d), device=DEVICE, dtype=torch.float64) for _ in range(2))
        L = torch.zeros((rows, hkv), device=DEVICE, dtype=torch.int32)
        z = torch.zeros((rows, hkv), device=DEVICE, dtype=torch.float64)
    cus = [_cu(p["lens"]) for p in P]
    for b in range(rows):
        n = lens[b]
        if n == 0:
            continue
        parts = [slice(c[b], c[b + 1]) for c in cus]
        q = torch.cat([p["q"][r] for p, r in zip(P, parts)]).double()
        k = torch.cat([p["k"][r] for p, r in zip(P, parts)]).double()
        v = torch.cat([p["v"][r] for p, r in zip(P, parts)]).double()
        lower = torch.ones((n, n), device=DEVICE, dtype=torch.bool).tril()
        for h in range(hkv):
            src = 0 if case["decision"] == "shared_layer" else h
            new = k[:, src, 0] <= case["bias"]
            w = torch.sigmoid(q[:, src * G:(src + 1) * G, 0])
            w = torch.ones(n, device=DEVICE, dtype=torch.float64) if case["omega"] == "uniform" else (
                w[:, 0] if case["omega"] == "lead" else w.mean(1))
            held = 0 if serve else int(_slots(case)[b][h])
            if held == 0:
                new[0] = True
            seg = new.long().cumsum(0)
            W = (seg[:, None] == seg) & lower
            W = W * w
            zs, kk = W.sum(1), k[:, h].clone()
            kk[:, 0] = 0
            ks, vs = W @ kk, W @ v[:, h]
            if held:
                z0 = (seg == 0) * st["z"][b, h].double()
                Kc, Vc = st["K"][b, h, :held].double(), st["V"][b, h, :held].double()
                zs, ks, vs = zs + z0, ks + z0[:, None] * Kc[-1], vs + z0[:, None] * Vc[-1]
            ks, vs = ks / zs[:, None], vs / zs[:, None]
            ends = torch.cat([new[1:], new.new_ones(1)])
            if case.get("attend", True):
                qq = q[:, h * G:(h + 1) * G].transpose(0, 1).clone()   # [G, n, d]
                qq[..., 0] = 0
                see = (lower & ends) | torch.eye(n, device=DEVICE, dtype=torch.bool)
                s = torch.matmul(qq, ks.t().contiguous()) * d ** -0.5
                s = torch.where(see, s, -math.inf)
                vals = vs
                if held:
                    keep = held if bool(new[0]) else held - 1
                    old = torch.matmul(qq, Kc[:keep].t().contiguous()) * d ** -0.5
                    s, vals = torch.cat([s, old], 2), torch.cat([vs, Vc[:keep]])
                o = torch.matmul(torch.softmax(s, 2), vals).transpose(0, 1)
                for x, r, y in zip(outs, parts, o.split([r.stop - r.start for r in parts])):
                    x[r, h * G:(h + 1) * G] = y
            if serve:
                for x, r, y in zip(slots, parts, (seg - 1).split([r.stop - r.start for r in parts])):
                    x[r, h] = y.int()
                m = int(seg[-1])
                K[b, h, :m], V[b, h, :m] = ks[ends], vs[ends]
                L[b, h], z[b, h] = m, zs[-1]
    if not serve:
        return dict(out=outs[0])
    res = {}
    for i in range(len(P)):
        if case["attend"]:
            res[f"out{i}"] = outs[i]
        res[f"slots{i}"] = slots[i]
    return dict(res, K=K, V=V, z=z, lengths=L)
