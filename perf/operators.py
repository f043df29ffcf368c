"""The operators of serving with drafted tokens over per-head caches, as measurable cases.

A speculative step drafts a tree of tokens, writes their keys and values behind every head's entries (rotated by their
positions on the way), attends with all drafted rows at once to the cache and to their ancestors, and keeps the
accepted path.  Per-head caches have lengths of their own after compression, so they live either head-major
([B, Hkv, Lmax, hd], "page" 0) or in pages that heads draw from one pool ([n_pages, page, hd] and a table
[B, Hkv, max_pages]).

  append   keys and values of `rows` tokens per sequence into the cache, keys and queries rotated (kv_append)
  pack     compressed head-major lists, every head of its own length, into pages (kv_append without rotation)
  attn     attention of `rows` drafted rows over the cache (tree_attn)
  commit   the accepted path of the drafted rows moves together behind the committed entries (tree_commit)

Where `own` is false each operator is computed from elementary tensor operations in 32 bits (angles in 64).
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}

# (query heads, KV heads, head dimension, type) of the decoder layers in use, and a 64-channel layer in bf16
_LAYERS = {"tiny": (4, 4, 64, "f32"), "64ch": (16, 4, 64, "bf16"), "7b": (28, 4, 128, "bf16"), "8b": (32, 8, 128, "bf16"),
           "26b": (48, 8, 128, "bf16"), "38b": (40, 8, 128, "bf16")}
_THETA = 1e6


def listed():
    return [
        # the smallest call there is: one token of the tiny fp32 layer behind 256 entries
        {"name": "append_one_token_f32", "op": "append", "layer": "tiny", "batch": 1, "rows": 1, "len": 256, "page": 0,
         "ragged": False, "rotate": "half", "pos": 640},
        # a drafting step of 16 image conversations: trees of up to 32 tokens, positions of three axes, pages of 64
        {"name": "append_tree_batch16_pages", "op": "append", "layer": "7b", "batch": 16, "rows": 32, "len": 1024, "page": 64,
         "ragged": True, "rotate": "sections", "pos": 2113},
        # the prefill of the 16384-token image sequence straight into pages, far positions and all query heads
        {"name": "append_prefill_16512_pages", "op": "append", "layer": "26b", "batch": 1, "rows": 16512, "len": 0, "page": 256,
         "ragged": False, "rotate": "half", "pos": 0},
        # after compression: the lists of eight layers of the batch of eight leave their reserved slots for pages
        {"name": "pack_512_heads_1888", "op": "pack", "layer": "8b", "batch": 64, "rows": 1888, "len": 0, "page": 64,
         "ragged": True, "rotate": "none", "pos": 0},
        # one row over a 256-entry budget in fp32: what a call costs at least
        {"name": "attn_one_token_f32", "op": "attn", "layer": "tiny", "batch": 1, "rows": 1, "len": 256, "page": 0,
         "ragged": False, "mask": "tree"},
        # plain decoding of 16 sequences from pages: one row each, lengths around a 1024-entry budget
        {"name": "attn_one_token_batch16_pages", "op": "attn", "layer": "7b", "batch": 16, "rows": 1, "len": 1024, "page": 64,
         "ragged": True, "mask": "chain"},
        # a tree of 64 drafted tokens for one sequence at a 2048-entry budget
        {"name": "attn_tree64_single_2048", "op": "attn", "layer": "26b", "batch": 1, "rows": 64, "len": 2048, "page": 0,
         "ragged": False, "mask": "tree"},
        # trees of up to 32 tokens for 16 sequences over uncompressed lengths in pages: much memory, ragged heads
        {"name": "attn_tree32_batch16_16384", "op": "attn", "layer": "8b", "batch": 16, "rows": 32, "len": 16384, "page": 128,
         "ragged": True, "mask": "tree"},
        # the next turn's 512 tokens over a 16384-entry cache, each seeing those before it: much arithmetic
        {"name": "attn_chain512_over_16384", "op": "attn", "layer": "26b", "batch": 1, "rows": 512, "len": 16384, "page": 0,
         "ragged": False, "mask": "chain"},
        # fp32 trees of an odd size over small pages
        {"name": "attn_tree27_f32_pages", "op": "attn", "layer": "tiny", "batch": 4, "rows": 27, "len": 701, "page": 16,
         "ragged": True, "mask": "tree"},
        # after verification: one layer of one sequence, and all 32 layers of eight sequences in one call
        {"name": "commit_single_2048", "op": "commit", "layer": "26b", "batch": 1, "rows": 64, "len": 2048, "page": 0,
         "ragged": False},
        {"name": "commit_256_rows_pages", "op": "commit", "layer": "8b", "batch": 256, "rows": 32, "len": 1000, "page": 64,
         "ragged": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: an operator and a layer, then sizes spread over the range that the listed cases span."""
    op = rng.choice(["append", "append", "pack", "attn", "attn", "attn", "commit"])
    layer = rng.choice(sorted(_LAYERS))
    Hq, Hkv, hd, dt = _LAYERS[layer]
    page = rng.choice([0, 16, 32, 64, 128, 256])
    case = {"op": op, "layer": layer, "page": page, "ragged": rng.random() < 0.6}
    if op == "append":
        rows = rng.choice([1, rng.randint(2, 64), _log_int(rng, 65, 8192)])
        case.update(rows=rows, batch=max(1, min(_log_int(rng, 1, 64), 14000 // rows)), len=rng.choice([0, _log_int(rng, 1, 4096)]),
                    rotate=rng.choice(["half", "adjacent", "sections"]), pos=rng.choice([0, rng.randint(1, 40000), 900000]))
    elif op == "pack":
        rows = _log_int(rng, 33, 4096)
        case.update(page=page or 64, ragged=True, rows=rows, batch=max(1, min(_log_int(rng, 1, 64), 110000 // rows)), len=0,
                    rotate="none", pos=0)
    elif op == "attn":
        rows = rng.choice([1, rng.randint(2, 16), rng.randint(17, 64), _log_int(rng, 65, 512)])
        length = _log_int(rng, 64, 2048 if dt == "f32" else 16384)
        cells = 48 * 512 * 16384 // 4
        batch = max(1, min(_log_int(rng, 1, 32), 16 * 12000 // length, cells // (Hq * rows * length)))
        case.update(rows=rows, batch=batch, len=length, mask=rng.choice(["tree", "tree", "chain"]) if rows <= 64 else "chain")
    else:
        case.update(rows=rng.randint(2, 64), batch=_log_int(rng, 1, 256), len=_log_int(rng, 16, 1000))
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _lengths(case, r):
    """Entries per (sequence, KV head) before the call, and rows per sequence (per head where lists are packed)."""
    B, Hkv, T, n = case["batch"], _LAYERS[case["layer"]][1], case["rows"], case["len"]
    if not case["ragged"]:
        return [[n] * Hkv for _ in range(B)], [T] * B
    length = [[r.randint(n // 2, n) for _ in range(Hkv)] for _ in range(B)]
    if case["op"] == "pack":
        return length, [[r.randint(max(1, T // 4), T) for _ in range(Hkv)] for _ in range(B)]
    return length, [r.randint(max(1, T // 2), T) for _ in range(B)]


def _trees(case, r, n_rows):
    """Parents (-1: the root), depths and visibility words of the drafted rows."""
    B, T = case["batch"], case["rows"]
    W = (T + 31) // 32
    depth = torch.zeros(B, T, dtype=torch.int32)
    words = torch.zeros(B, T, W, dtype=torch.int32)
    for b in range(B):
        seen, deep = [0] * T, [0] * T
        for t in range(T):
            p = -1 if t == 0 else r.randint(max(0, t - 6), t - 1)
            seen[t] = (seen[p] if p >= 0 else 0) | 1 << t
            deep[t] = deep[p] + 1 if p >= 0 else 0
        depth[b] = torch.tensor(deep, dtype=torch.int32)
        words[b] = torch.tensor([[(((s >> (32 * w)) & 0xFFFFFFFF) ^ 0x80000000) - 0x80000000 for w in range(W)] for s in seen],
                                dtype=torch.int32)
    return depth, words


def _caches(case, g, r, slots):
    """Keys, values and the entries' small arrays, head-major or in pages drawn at random from one pool, and the table.
    slots[b][g]: entries that the head must have room for; the pool would hold all heads at their longest."""
    B = case["batch"]
    Hq, Hkv, hd, dt = _LAYERS[case["layer"]]
    most, page = case["len"] + case["rows"], case["page"]
    if page == 0:
        shape, table = (B, Hkv, (most + 15) // 16 * 16), None
    else:
        need = [[(s + page - 1) // page for s in row] for row in slots]
        wide, at = (most + page - 1) // page, 0
        n_pages = B * Hkv * wide
        order = list(range(n_pages))
        r.shuffle(order)
        table = torch.full((B, Hkv, wide), -1, dtype=torch.int32)
        for b in range(B):
            for h in range(Hkv):
                table[b, h, :need[b][h]] = torch.tensor(order[at:at + need[b][h]], dtype=torch.int32)
                at += need[b][h]
        shape = (n_pages, page)
        table = table.cuda()
    k = torch.randn(*shape, hd, generator=g, device="cuda").to(_DT[dt])
    v = torch.randn(*shape, hd, generator=g, device="cuda").to(_DT[dt])
    score = torch.rand(*shape, generator=g, device="cuda")
    kind = torch.randint(0, 3, shape, generator=g, device="cuda", dtype=torch.uint8)
    orig = torch.randint(0, 4096, shape, generator=g, device="cuda", dtype=torch.int32)
    return {"k": k, "v": v, "score": score, "kind": kind, "orig_pos": orig, "pages": table}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1_000_003 + 17) & 0x7FFFFFFFFFFF)
    r = random.Random(int(seed) * 7919 + 3)
    B, T, op = case["batch"], case["rows"], case["op"]
    Hq, Hkv, hd, dt = _LAYERS[case["layer"]]
    length, n_rows = _lengths(case, r)
    st = {"case": case, "n_rows": torch.tensor(n_rows, dtype=torch.int32).cuda() if case["ragged"] else None}
    if op == "pack":
        # the lists as the compression leaves them, in slots reserved for the longest
        src = dict(case, page=0)
        st["from"] = _caches(src, g, r, [[T] * Hkv] * B)
        st.update(_caches(case, g, r, n_rows))
        st["len"] = torch.zeros(B, Hkv, dtype=torch.int32, device="cuda")
        st["len_out"] = torch.zeros_like(st["len"])
        return st
    st.update(_caches(case, g, r, [[n + T for n in row] for row in length]))
    st["len"] = torch.tensor(length, dtype=torch.int32).cuda()
    if op == "append":
        st["k_new"], st["v_new"] = (torch.randn(B, T, Hkv, hd, generator=g, device="cuda").to(_DT[dt]) for _ in range(2))
        st["q"] = torch.randn(B, T, Hq, hd, generator=g, device="cuda").to(_DT[dt])
        st["q_out"] = torch.zeros_like(st["q"])
        st["len_out"] = torch.zeros_like(st["len"])
        axes = 3 if case["rotate"] == "sections" else 1
        if T <= 64:
            steps = _trees(case, r, n_rows)[0].unsqueeze(0).expand(axes, B, T)
        else:
            steps = torch.arange(T, dtype=torch.int32).expand(axes, B, T)
        steps = steps.contiguous().cuda()
        if axes == 3:           # rows and columns of an image grid beside the time axis
            steps = torch.stack([steps[0], steps[1] // 7 + 5, steps[2] % 7 + 3])
        st["pos"] = (steps + case["pos"]).to(torch.int32).contiguous()
        st["sections"] = (hd // 8, 3 * hd // 16, 3 * hd // 16) if axes == 3 else (hd // 2,)
        st["inv_freq"] = (_THETA ** (-torch.arange(0, hd, 2, dtype=torch.float64) / hd)).float().cuda()
    elif op == "attn":
        n = torch.tensor([n_rows] * Hkv, dtype=torch.int32).t().cuda()
        st["len"] = st["len"] + n                       # the drafted rows are in the cache
        st["bound"] = max(max(row) for row in length) + T
        st["q"] = torch.randn(B, T, Hq, hd, generator=g, device="cuda").to(_DT[dt])
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(B, Hq, T, device="cuda")
        st["mask"] = _trees(case, r, n_rows)[1].cuda() if case["mask"] == "tree" else None
    else:
        path = torch.zeros(B, T, dtype=torch.int32)
        n_path = []
        for b in range(B):
            m = r.randint(1, min(12, n_rows[b]))
            path[b, :m] = torch.tensor(sorted(r.sample(range(n_rows[b]), m)), dtype=torch.int32)
            n_path.append(m)
        st["path"], st["n_path"] = path.cuda(), torch.tensor(n_path, dtype=torch.int32).cuda()
        st["len_out"] = torch.zeros_like(st["len"])
    return st


# ---- the plain forms ------------------------------------------------------------------------------------------------


def _place(st, slot):
    """Row of the cache, seen as [rows, hd], that holds slot [B, Hkv, n] of every head."""
    if st["pages"] is None:
        B, Hkv, Lmax, _ = st["k"].shape
        head = torch.arange(B * Hkv, device=slot.device).view(B, Hkv, 1)
        return head * Lmax + slot
    page = st["k"].shape[1]
    return torch.gather(st["pages"].long(), 2, slot // page) * page + slot % page


def _small(st, name):
    return st[name].view(-1)


def _turned(x, cos, sin, adjacent):
    """Pairs of the last axis turned by the angles; x [B, T, H, hd], cos and sin [B, T, 1, hd / 2]."""
    x = x.float()
    if adjacent:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _plain_append(st):
    case, T = st["case"], st["case"]["rows"]
    dev = st["k"].device
    n = st["n_rows"]
    n = torch.full((case["batch"], 1), T, device=dev) if n is None else n.view(case["batch"], -1).long()     # [B, 1 or Hkv]
    t = torch.minimum(torch.arange(T, device=dev).view(1, 1, T), n.unsqueeze(-1) - 1)    # rows past the last one: that one again
    length = st["len"].long()
    at = _place(st, length.unsqueeze(-1) + t)                                            # [B, Hkv, T]
    if case["op"] == "pack":
        src, t = st["from"], t.expand(at.shape)
        for name in ("k", "v"):
            rows = torch.gather(src[name], 2, t.unsqueeze(-1).expand(-1, -1, -1, src[name].shape[-1]))
            st[name].view(-1, rows.shape[-1])[at] = rows
        for name in ("score", "kind", "orig_pos"):
            _small(st, name)[at] = torch.gather(src[name], 2, t)
    else:
        axis = torch.repeat_interleave(torch.arange(len(st["sections"]), device=dev), torch.tensor(st["sections"], device=dev),
                                       output_size=sum(st["sections"]))
        angle = (st["pos"].double()[axis] * st["inv_freq"].double().view(-1, 1, 1)).permute(1, 2, 0).unsqueeze(2)
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        adjacent = case["rotate"] == "adjacent"
        k = _turned(st["k_new"], cos, sin, adjacent).to(st["k"].dtype)
        q = _turned(st["q"], cos, sin, adjacent).to(st["q"].dtype)
        tb = t[:, :1].expand(-1, at.shape[1], -1)
        for name, x in (("k", k), ("v", st["v_new"])):
            rows = torch.gather(x.transpose(1, 2), 2, tb.unsqueeze(-1).expand(-1, -1, -1, x.shape[-1]))
            st[name].view(-1, rows.shape[-1])[at] = rows
        _small(st, "score")[at] = 0.0
        _small(st, "kind")[at] = 2
        _small(st, "orig_pos")[at] = torch.gather(st["pos"][0].unsqueeze(1).expand(at.shape), 2, tb)
        live = (torch.arange(T, device=dev).view(1, T) < n[:, :1]).view(case["batch"], T, 1, 1)
        st["q_out"].copy_(torch.where(live, q, st["q_out"]))
    st["len_out"].copy_(length + n)


def _plain_attn(st):
    case, T = st["case"], st["case"]["rows"]
    dev, B = st["q"].device, case["batch"]
    Hq, Hkv, hd, _ = _LAYERS[case["layer"]]
    G, L = Hq // Hkv, st["bound"]
    length = st["len"].long()
    n = torch.full((B,), T, device=dev) if st["n_rows"] is None else st["n_rows"].long()
    if st["pages"] is None:
        k, v = st["k"][:, :, :L], st["v"][:, :, :L]
    else:
        table = st["pages"].long().clamp(min=0)
        k, v = (st[name][table].flatten(2, 3)[:, :, :L] for name in ("k", "v"))
    L = k.shape[2]
    q = st["q"].float().view(B, T, Hkv, G, hd).permute(0, 2, 1, 3, 4).reshape(B * Hkv, T * G, hd)
    s = torch.bmm(q, k.float().reshape(B * Hkv, L, hd).transpose(1, 2).contiguous()).view(B, Hkv, T, G, L) * hd ** -0.5
    j = torch.arange(L, device=dev)
    i = j.view(1, 1, L) - (length - n.view(B, 1)).unsqueeze(-1)                          # drafted row of the entry, [B, Hkv, L]
    row = torch.arange(T, device=dev)
    if st["mask"] is None:
        sees = i.unsqueeze(2) <= row.view(1, 1, T, 1)
    else:
        at = i.clamp(0, T - 1)
        word = torch.gather(st["mask"].unsqueeze(1).expand(B, Hkv, T, -1), 3, (at // 32).unsqueeze(2).expand(B, Hkv, T, L))
        sees = ((word >> (at % 32).unsqueeze(2)) & 1).bool() | (i < 0).unsqueeze(2)
    sees = (sees & (j.view(1, 1, 1, L) < length.view(B, Hkv, 1, 1))).unsqueeze(3)        # [B, Hkv, T, 1, L]
    s = s.masked_fill(~sees, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(s - top)
    total = p.sum(dim=-1, keepdim=True)
    o = torch.bmm(p.view(B * Hkv, T * G, L), v.float().reshape(B * Hkv, L, hd)).view(B, Hkv, T, G, hd)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    live = (row.view(1, T) < n.view(B, 1))
    o = o.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, hd).to(st["q"].dtype)
    st["out"].copy_(torch.where(live.view(B, T, 1, 1), o, st["out"]))
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 1, 3, 2).reshape(B, Hq, T)
    st["lse"].copy_(torch.where(live.view(B, 1, T), lse, st["lse"]))


def _plain_commit(st):
    P, n = st["path"].shape[1], st["n_path"].long().view(-1, 1)
    i = torch.minimum(torch.arange(P, device=n.device).view(1, P), n - 1)                # past the last accepted row: that one again
    taken = torch.gather(st["path"].long(), 1, i)
    length = st["len"].long().unsqueeze(-1)
    to, come = _place(st, length + i.unsqueeze(1)), _place(st, length + taken.unsqueeze(1))
    for name in ("k", "v"):
        rows = st[name].view(-1, st[name].shape[-1])
        rows[to] = rows[come]
    for name in ("score", "kind", "orig_pos"):
        _small(st, name)[to] = _small(st, name)[come]
    st["len_out"].copy_(st["len"] + st["n_path"].view(-1, 1))


# ---- the framework's calls ------------------------------------------------------------------------------------------

_contexts = {}


def _context():
    device = torch.cuda.current_device()
    if device not in _contexts:
        import paper_2509_00419_amd as lv
        _contexts[device] = lv.Context(device)
    return _contexts[device]


def _own(st):
    ctx, op = _context(), st["case"]["op"]
    if op == "append":
        ctx.kv_append(st["k_new"], st["v_new"], st["k"], st["v"], st["len"], pos=st["pos"], inv_freq=st["inv_freq"],
                      sections=st["sections"], adjacent=st["case"]["rotate"] == "adjacent", q=st["q"], q_out=st["q_out"],
                      n_new=st["n_rows"], pages=st["pages"], score=st["score"], kind=st["kind"], orig_pos=st["orig_pos"],
                      length_out=st["len_out"])
    elif op == "pack":
        src = st["from"]
        ctx.kv_append(src["k"].transpose(1, 2), src["v"].transpose(1, 2), st["k"], st["v"], st["len"], n_new=st["n_rows"],
                      pages=st["pages"], score=st["score"], kind=st["kind"], orig_pos=st["orig_pos"], score_new=src["score"],
                      kind_new=src["kind"], orig_new=src["orig_pos"], length_out=st["len_out"])
    elif op == "attn":
        ctx.tree_attn(st["q"], st["k"], st["v"], st["len"], mask=st["mask"], n_rows=st["n_rows"], pages=st["pages"],
                      len_bound=st["bound"], out=st["out"], row_lse=st["lse"])
    else:
        ctx.tree_commit(st["k"], st["v"], st["len"], st["path"], st["n_path"], pages=st["pages"], score=st["score"],
                        kind=st["kind"], orig_pos=st["orig_pos"], length_out=st["len_out"])


def run(st):
    op = st["case"]["op"]
    if own:
        _own(st)
    elif op in ("append", "pack"):
        _plain_append(st)
    elif op == "attn":
        _plain_attn(st)
    else:
        _plain_commit(st)
    if op == "attn":
        return {"out": st["out"], "lse": st["lse"]}
    out = {name: st[name] for name in ("k", "v", "score", "kind", "orig_pos")}
    out["len"] = st["len_out"]
    if op == "append":
        out["q"] = st["q_out"]
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    Hq, Hkv, hd, dt = _LAYERS[case["layer"]]
    e, B, T, n, op = (2 if dt == "bf16" else 4), case["batch"], case["rows"], case["len"], case["op"]
    ragged = case["ragged"]
    if op == "append":
        rows = B * T * (0.75 if ragged else 1.0)
        axes = 3 if case["rotate"] == "sections" else 1
        return {"bytes": rows * (2 * (Hq + 2 * Hkv) * hd * e + 9 * Hkv + 4 * axes) + 8 * B * Hkv, "flops": 3.0 * rows * (Hq + Hkv) * hd}
    if op == "pack":
        rows = B * Hkv * T * 0.625
        return {"bytes": rows * 2 * (2 * hd * e + 9) + 12 * B * Hkv, "flops": 0.0}
    if op == "commit":
        rows = B * Hkv * min(12, T) * 0.5
        return {"bytes": rows * 2 * (2 * hd * e + 9) + 8 * B * Hkv, "flops": 0.0}
    m, t = (0.75 * n, max(1.0, 0.75 * T)) if ragged else (n, T)
    seen = m + (t / 2 + 1 if case["mask"] == "chain" else min(t, 6.0))
    return {"bytes": B * (Hkv * (m + t) * 2 * hd * e + 2 * t * Hq * hd * e + 4 * t * Hq), "flops": 4.0 * B * Hq * t * seen * hd}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------


def _slots_of(st, b, h, slots):
    """Row numbers of `slots` (a range) of head (b, h) in the cache seen as [rows, ...]."""
    at = torch.arange(slots.start, slots.stop, device=st["k"].device)
    if st["pages"] is None:
        _, Hkv, Lmax, _ = st["k"].shape
        return at + (b * Hkv + h) * Lmax
    size = st["k"].shape[1]
    return st["pages"][b, h].long()[torch.div(at, size, rounding_mode="floor")] * size + torch.remainder(at, size)


def exact(case, seed):
    st = prepare(case, seed)
    B, T, op = case["batch"], case["rows"], case["op"]
    Hq, Hkv, hd, _ = _LAYERS[case["layer"]]
    G = Hq // Hkv
    length = st["len"].tolist()
    n_rows = [T] * B if st["n_rows"] is None else st["n_rows"].tolist()
    flat = {name: st[name].reshape(-1, hd) if name in ("k", "v") else st[name].reshape(-1) for name in ("k", "v", "score", "kind", "orig_pos")}
    if op == "attn":
        out, lse = st["out"].double(), st["lse"].double()
        for b in range(B):
            n = n_rows[b]
            below = torch.tril(torch.ones(n, n, dtype=torch.bool, device="cuda"))
            if st["mask"] is not None:
                bit = torch.arange(n, device="cuda")
                below = torch.bitwise_right_shift(st["mask"][b, :n].long()[:, bit // 32], bit % 32).remainder(2) == 1
            for h in range(Hkv):
                at = _slots_of(st, b, h, range(length[b][h]))
                keys, values = flat["k"][at].double(), flat["v"][at].double()
                sees = torch.ones(n, length[b][h], dtype=torch.bool, device="cuda")
                sees[:, length[b][h] - n:] = below
                for x in range(h * G, h * G + G):
                    z = torch.where(sees, st["q"][b, :n, x].double() @ keys.t().contiguous() / math.sqrt(hd), -math.inf)
                    norm = torch.logsumexp(z, dim=1)
                    lse[b, x, :n] = norm
                    out[b, :n, x] = torch.exp(z - norm.unsqueeze(1)) @ values
        return {"out": out, "lse": lse}
    got = {name: x.double() if name in ("k", "v", "score") else x.clone() for name, x in flat.items()}
    new_len = [[0] * Hkv for _ in range(B)]
    q_out = None
    if op == "append":
        which = sum(([a] * s for a, s in enumerate(st["sections"])), [])
        angle = torch.stack([st["pos"][a].double() * st["inv_freq"][c].double() for c, a in enumerate(which)], dim=-1)
        turn = torch.polar(torch.ones_like(angle), angle).unsqueeze(2)

        def turned(x):
            x = x.double()
            if case["rotate"] == "adjacent":
                return torch.view_as_real(torch.view_as_complex(x.unflatten(-1, (hd // 2, 2)).contiguous()) * turn).flatten(-2)
            z = torch.complex(x[..., :hd // 2], x[..., hd // 2:]) * turn
            return torch.cat([z.real, z.imag], dim=-1)

        k_new, v_new, all_q = turned(st["k_new"]), st["v_new"].double(), turned(st["q"])
        q_out = st["q_out"].double()
        for b in range(B):
            q_out[b, :n_rows[b]] = all_q[b, :n_rows[b]]
    for b in range(B):
        for h in range(Hkv):
            first = length[b][h]
            if op == "commit":
                m = int(st["n_path"][b])
                come = _slots_of(st, b, h, range(first, first + T))[st["path"][b, :m].long()]
                to = _slots_of(st, b, h, range(first, first + m))
                for name in flat:
                    got[name][to] = flat[name][come].to(got[name].dtype)
            else:
                m = n_rows[b] if op == "append" else n_rows[b][h] if case["ragged"] else n_rows[b]
                to = _slots_of(st, b, h, range(first, first + m))
                if op == "pack":
                    for name in flat:
                        got[name][to] = st["from"][name][b, h, :m].to(got[name].dtype)
                else:
                    got["k"][to], got["v"][to] = k_new[b, :m, h], v_new[b, :m, h]
                    got["score"][to], got["kind"][to], got["orig_pos"][to] = 0.0, 2, st["pos"][0, b, :m]
            new_len[b][h] = first + m
    got = {name: x.view(st[name].shape) for name, x in got.items()}
    got["len"] = torch.tensor(new_len, dtype=torch.int32)
    if q_out is not None:
        got["q"] = q_out
    return got
