"""Decoding over a cache of pages, as calls whose time and results can be compared with their plain forms.

Three operators on one cache: keys and values in pages of `page_size` rows, found through a table of page numbers per sequence
(one page per sequence is the layout of the contiguous caches), with each row's position and accumulated attention weight beside it.

  append  the keys / values of new tokens (one token, the rows of a prompt, the accepted nodes of a tree) go into the cache
  decode  attention of one new token per sequence over its whole cache, optionally adding each row's weight to its account
  evict   the cache is cut down to a budget of rows per KV head: the newest and those with the largest accounts stay; a row that
          stays and lies beyond the budget moves into the place of one that leaves

Head layouts and types are those of the repository's workloads (the tiny single-precision instance, Llama-3-8B and Llama-2-70B
shapes, the drafter's Self-Attention layer with eight query heads per KV head).  Keys and values are N(0, 1).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

# query heads, KV heads, head dim, type
HEADS = {
    "tiny": (4, 2, 64, "f32"),
    "8b": (32, 8, 128, "bf16"),
    "70b": (64, 8, 128, "bf16"),
    "sa": (32, 4, 128, "bf16"),          # the drafter's Self-Attention layer
    "mha": (16, 16, 64, "bf16"),
    "odd": (6, 2, 80, "bf16"),
}
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_INF = float("inf")


def _decode(heads, B, P_min, P_max, page, acc=False):
    """page: rows of a page; 0 = one page per sequence."""
    return dict(kind="decode", heads=heads, B=B, P_min=P_min, P_max=P_max, page=page, acc=acc)


def _append(heads, B, P_min, P_max, page, M, n_min, n_max, path):
    """M rows handed over per sequence, n_min .. n_max of them stored; path: picked by a list of accepted nodes."""
    return dict(kind="append", heads=heads, B=B, P_min=P_min, P_max=P_max, page=page, M=M, n_min=n_min, n_max=n_max, path=path)


def _evict(heads, B, P_min, P_max, page, budget, recent):
    return dict(kind="evict", heads=heads, B=B, P_min=P_min, P_max=P_max, page=page, budget=budget, recent=recent)


def listed():
    return [
        # the smallest call: single precision, a short conversation, all latency
        dict(_decode("tiny", 1, 48, 64, 16), name="decode-tiny-fp32"),
        # one request behind a prompt of about a thousand tokens
        dict(_decode("8b", 1, 1024, 1084, 16), name="decode-8b-1k"),
        # the same on the contiguous cache that verification keeps: one page of odd size
        dict(_decode("8b", 4, 3001, 4097, 0), name="decode-8b-one-page"),
        # a serving batch of very different lengths
        dict(_decode("8b", 64, 17, 8192, 64), name="decode-8b-batch64"),
        # long context, eight query heads per KV head; with the batch above the largest call
        dict(_decode("70b", 8, 32768, 32768, 128), name="decode-70b-32k"),
        # a server that keeps accounts for eviction
        dict(_decode("8b", 16, 1900, 2112, 32, acc=True), name="decode-8b-accounts"),
        # a decoded token of every request of a batch
        dict(_append("8b", 64, 17, 1000, 16, 1, 1, 1, False), name="append-token"),
        # the accepted nodes of trees of 60, one to seven per request
        dict(_append("8b", 16, 100, 1500, 0, 60, 1, 7, True), name="append-accepted"),
        # ragged prompts into empty caches
        dict(_append("70b", 4, 0, 0, 128, 2048, 517, 2048, False), name="append-prompts"),
        # one short conversation that has grown past its budget
        dict(_evict("tiny", 1, 300, 320, 16, 256, 32), name="evict-tiny-fp32"),
        # a batch in steady state: 64 tokens decoded since the last time
        dict(_evict("8b", 16, 2112, 2112, 32, 2048, 256), name="evict-8b-steady"),
        # long prompts cut to an eighth
        dict(_evict("70b", 8, 9000, 16384, 64, 2048, 512), name="evict-70b-prompts"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 1e15


def draw(rng: random.Random):
    """One more case; it costs no more than the largest listed one."""
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["decode", "decode", "decode", "append", "evict"])
        heads = rng.choice(["8b", "8b", "8b", "70b", "sa", "mha", "tiny", "odd"])
        B = _log_int(rng, 1, 96)
        page = rng.choice([0, 16, 16, 32, 48, 64, 128, 256, rng.randint(1, 40)])
        if kind == "decode":
            P = _log_int(rng, 1, 32768)
            c = _decode(heads, B, max(1, int(P * rng.random())), P, page, acc=rng.random() < 0.3)
        elif kind == "append":
            P = _log_int(rng, 1, 2000) if rng.random() < 0.8 else 0
            M = rng.choice([1, 1, rng.randint(2, 256), _log_int(rng, 16, 2048)])
            path = 1 < M <= 256 and rng.random() < 0.6
            n = rng.randint(1, min(M, 9)) if path else M
            c = _append(heads, B, P // 2, P, page, M, rng.randint(0, n), n, path)
        else:
            budget = _log_int(rng, 16, 4096)
            P = budget + _log_int(rng, 1, 16384)
            c = _evict(heads, B, max(1, P - rng.randint(0, P // 2)), P, page, budget, rng.randint(0, budget))
        # (states of more than 8 GiB are a matter of memory, not of another kind of call)
        if _cost(c) <= most and _state_bytes(c) < 8 << 30:
            return c


# ------------------------------------------------------------------ inputs

def _geometry(case):
    H, Hkv, dh, dtype = HEADS[case["heads"]]
    need = case["P_max"] + (case["n_max"] if case["kind"] == "append" else 0)
    ps = case["page"] or need
    return H, Hkv, dh, dtype, ps, (need + ps - 1) // ps


def _state_bytes(case):
    H, Hkv, dh, dtype, ps, mp = _geometry(case)
    return case["B"] * Hkv * mp * ps * dh * 2 * (2 if dtype == "bf16" else 4)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def prepare(case, seed):
    H, Hkv, dh, dtype, ps, mp = _geometry(case)
    B, kind, dt = case["B"], case["kind"], _TORCH[dtype]
    host = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.empty(shape, dtype=dt, device="cuda").normal_(generator=g)
    n = host.integers(case["P_min"], case["P_max"] + 1, size=B).astype(np.int32)
    n[host.integers(0, B)] = case["P_max"]
    new = host.integers(case["n_min"], case["n_max"] + 1, size=B).astype(np.int32) if kind == "append" else np.zeros(B, np.int32)
    if kind == "append":
        new[host.integers(0, B)] = case["n_max"]
    # pages in the order in which a server that had them all back from others would hand them out; entries not yet needed are -1
    want = (n + new + ps - 1) // ps
    n_pages = B * mp + 3
    order = host.permutation(n_pages).astype(np.int32)
    table = np.full((B, mp), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :want[b]] = order[at:at + want[b]]
        at += int(want[b])
    cap = mp * ps
    st = dict(case=case, H=H, k=normal(n_pages, Hkv, ps, dh), v=normal(n_pages, Hkv, ps, dh), table=_dev(table), len0=_dev(n),
              status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    st["len"] = st["len0"].clone()
    st["pos"] = st["seen"] = st["score0"] = st["score"] = None
    if kind != "decode" or case["acc"]:
        _accounts(st, g, n, B, Hkv, cap)
    if kind == "decode":
        st["q"] = (1.5 * torch.randn(B, H, dh, device="cuda", generator=g)).to(dt)
        st["out"] = torch.zeros(B, H, dh, dtype=dt, device="cuda")
    if kind == "append":
        M = case["M"]
        st["k_new"], st["v_new"], st["n_new"] = normal(B, Hkv, M, dh), normal(B, Hkv, M, dh), _dev(new)
        st["path"] = None
        if case["path"]:                               # nodes of an accepted path: increasing, the root first, then -1
            path = np.full((B, M), -1, np.int32)
            for b in range(B):
                if new[b]:
                    path[b, :new[b]] = np.concatenate([[0], 1 + np.sort(host.choice(M - 1, size=new[b] - 1, replace=False))])
            st["path"] = _dev(path)
    if own:
        import paper_2410_03804_amd as moa

        st["cache"] = moa.KVCache(st["k"], st["v"], st["table"], st["len"], pos=st["pos"], seen=st["seen"], score=st["score"])
        if kind == "decode":
            nb = moa.decode_attn_workspace_bytes(st["cache"], H)
        elif kind == "evict":
            nb = moa.kv_evict_workspace_bytes(st["cache"], case["budget"])
        else:
            nb = 0
        st["ws"] = torch.empty(max(nb, 256), dtype=torch.uint8, device="cuda")
    return st


def _accounts(st, g, n, B, Hkv, cap):
    """Positions and accumulated weights as earlier decoding and eviction leave them: positions distinct and roughly in order, one
    row in 16 without any weight that single precision can hold, the others' spread over several powers of ten."""
    slot = torch.arange(cap, device="cuda")
    held = slot[None, None, :] < _dev(n)[:, None, None]
    gaps = torch.randint(1, 4, (B, Hkv, cap), device="cuda", generator=g)
    at = torch.cumsum(gaps, dim=2)
    seen = 3 * cap + 1 + torch.arange(B, device="cuda")
    last = torch.where(held, at, torch.zeros_like(at)).amax(dim=2, keepdim=True)
    pos = seen[:, None, None] - 1 - (last - at)
    shift = slot + torch.where(held, 40 * torch.rand((B, Hkv, cap), device="cuda", generator=g), torch.full((), 1e6, device="cuda"))
    pos = torch.gather(pos, 2, torch.argsort(shift, dim=2))
    weight = torch.exp(2.0 * torch.randn((B, Hkv, cap), device="cuda", generator=g) - 3.0)
    weight = torch.where(torch.rand((B, Hkv, cap), device="cuda", generator=g) < 1 / 16, torch.zeros_like(weight), weight)
    st["pos"] = torch.where(held, pos, torch.full_like(pos, -1)).to(torch.int32).contiguous()
    st["seen0"] = seen.to(torch.int32).contiguous()
    st["seen"] = st["seen0"].clone()
    st["score0"] = torch.where(held, weight, torch.zeros_like(weight)).contiguous()
    st["score"] = st["score0"].clone()
    st["pos0"] = st["pos"].clone()


# ------------------------------------------------------------------ one pass

def run(st):
    return {"decode": _run_decode, "append": _run_append, "evict": _run_evict}[st["case"]["kind"]](st)


def _reset(st, *names):
    # the call moves the cache's account on; what a program does that rolls a cache back
    for name in names:
        st[name].copy_(st[name + "0"])


def _run_decode(st):
    acc = st["case"]["acc"]
    if acc:
        _reset(st, "score")
    if own:
        import paper_2410_03804_amd as moa

        moa.decode_attn(st["cache"], st["q"], st["out"], st["ws"], accumulate=acc, dev_status=st["status"])
    else:
        _plain_decode(st, acc)
    return dict(out=st["out"], score=st["score"]) if acc else dict(out=st["out"])


def _run_append(st):
    _reset(st, "len", "seen", "pos", "score")
    if own:
        import paper_2410_03804_amd as moa

        moa.kv_append(st["cache"], st["k_new"], st["v_new"], path=st["path"], n_new=st["n_new"], dev_status=st["status"])
    else:
        _plain_append(st)
    return {name: st[name] for name in ("k", "v", "pos", "score", "len", "seen")}


def _run_evict(st):
    # the rows that moved are still where they came from, so with its accounts back the same rows move again
    _reset(st, "len", "pos", "score")
    if own:
        import paper_2410_03804_amd as moa

        moa.kv_evict(st["cache"], st["case"]["budget"], st["case"]["recent"], st["ws"], dev_status=st["status"])
    else:
        _plain_evict(st)
    return {name: st[name] for name in ("k", "v", "pos", "score", "len")}


# ------------------------------------------------------------------ plain forms

def _plain_decode(st, acc):
    k, v, table, q = st["k"], st["v"], st["table"], st["q"]
    _, Hkv, ps, dh = k.shape
    B, mp = table.shape
    cap, G = mp * ps, q.shape[1] // Hkv
    step = max(1, (1 << 28) // (Hkv * cap * dh))
    for b0 in range(0, B, step):
        sl = slice(b0, min(b0 + step, B))
        pages = table[sl].clamp(min=0).long()
        nb = pages.shape[0]
        rows = lambda pool: pool[pages].permute(0, 2, 1, 3, 4).reshape(nb, Hkv, cap, dh).float()
        held = torch.arange(cap, device=q.device)[None, :] < st["len"][sl, None]
        kf = rows(k)
        s = torch.matmul(q[sl].float().view(nb, Hkv, G, dh) * dh ** -0.5, kf.transpose(2, 3).contiguous())
        s = torch.where(held[:, None, None, :], s, torch.full((), -_INF, device=q.device))
        e = torch.exp(s - s.amax(dim=3, keepdim=True))
        p = e / e.sum(dim=3, keepdim=True)
        vf = torch.where(held[:, None, :, None], rows(v), torch.zeros((), device=q.device))
        st["out"][sl] = torch.matmul(p, vf).view(nb, Hkv * G, dh).to(q.dtype)
        if acc:
            st["score"][sl] += p.sum(dim=2)


def _pool_rows(table, slots, ps, Hkv):
    """Row numbers, in a pool of pages seen as rows, of the slots [B, Hkv, n]."""
    page = torch.gather(table.clamp(min=0).long()[:, None, :].expand(-1, Hkv, -1), 2, slots // ps)
    return (page * Hkv + torch.arange(Hkv, device=slots.device)[None, :, None]) * ps + slots % ps


def _plain_append(st):
    k, v, table, n, n_new = st["k"], st["v"], st["table"], st["len"].long(), st["n_new"].long()
    _, Hkv, ps, dh = k.shape
    B, M, cap = table.shape[0], st["k_new"].shape[2], table.shape[1] * ps
    i = torch.arange(M, device=k.device)[None, :]
    i = torch.minimum(i, (n_new - 1).clamp(min=0)[:, None])                    # beyond the last new row: that row once more
    src = torch.gather(st["path"].long(), 1, i).clamp(min=0) if st["path"] is not None else i
    slot = (n[:, None] + i).clamp(max=cap - 1)
    some = (n_new > 0)[:, None, None]                                          # without new rows a row is replaced by itself
    slots = slot[:, None, :].expand(B, Hkv, M)
    at = _pool_rows(table, slots, ps, Hkv).reshape(-1)
    for pool, rows in ((k, st["k_new"]), (v, st["v_new"])):
        flat = pool.view(-1, dh)
        new = torch.gather(rows, 2, src[:, None, :, None].expand(B, Hkv, M, dh))
        # (a sequence without new rows may own no page at all: its place is then another's, whose row stays as it is)
        keep = some.expand(B, Hkv, M).reshape(-1)
        at_kept = torch.where(keep, at, at[keep.to(torch.int32).argmax()])
        new = new.reshape(-1, dh)
        new = torch.where(keep[:, None], new, new[keep.to(torch.int32).argmax()][None, :])
        flat[at_kept] = new
    for name, value in (("pos", (st["seen"].long()[:, None] + i)[:, None, :].expand(B, Hkv, M).to(torch.int32)),
                        ("score", torch.zeros((B, Hkv, M), device=k.device))):
        t = st[name]
        t.scatter_(2, slots, torch.where(some, value, torch.gather(t, 2, slots)))
    st["len"] += st["n_new"]
    st["seen"] += st["n_new"]


def _plain_evict(st):
    k, v, table, n, pos, score = st["k"], st["v"], st["table"], st["len"].long(), st["pos"], st["score"]
    budget, recent = st["case"]["budget"], st["case"]["recent"]
    _, Hkv, ps, dh = k.shape
    B, cap = table.shape[0], table.shape[1] * ps
    slot = torch.arange(cap, device=k.device)[None, None, :].expand(B, Hkv, cap)
    held = slot < n[:, None, None]
    newest = pos.long() >= (st["seen"].long() - recent)[:, None, None]
    rank = torch.where(newest, torch.full_like(score, _INF), score)
    rank = torch.where(held, rank, torch.full_like(score, -_INF))
    order = torch.sort(rank, dim=2, descending=True, stable=True).indices[:, :, :budget]
    stays = torch.zeros((B, Hkv, cap), dtype=torch.bool, device=k.device).scatter_(2, order, True)
    cut = (n > budget)[:, None, None]
    gone = torch.full_like(slot, cap)
    moves = min(budget, cap - budget)
    if moves > 0:
        dst = torch.sort(torch.where(cut & ~stays & (slot < budget), slot, gone), dim=2).values[:, :, :moves]
        src = torch.sort(torch.where(cut & stays & (slot >= budget), slot, gone), dim=2).values[:, :, :moves]
        # beyond the last move: the first one again, or a row onto itself where there is none
        none = dst[:, :, :1] == cap
        first_d = torch.where(none, torch.zeros_like(dst[:, :, :1]), dst[:, :, :1])
        first_s = torch.where(none, torch.zeros_like(src[:, :, :1]), src[:, :, :1])
        dst, src = torch.where(dst == cap, first_d, dst), torch.where(src == cap, first_s, src)
        at, frm = _pool_rows(table, dst, ps, Hkv).reshape(-1), _pool_rows(table, src, ps, Hkv).reshape(-1)
        for pool in (k, v):
            flat = pool.view(-1, dh)
            flat[at] = flat[frm]
        pos.scatter_(2, dst, torch.gather(pos, 2, src))
        score.scatter_(2, dst, torch.gather(score, 2, src))
    st["len"].clamp_(max=budget)


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return {"decode": _exact_decode, "append": _exact_append, "evict": _exact_evict}[case["kind"]](st, case)


def _slots_of(st, b, count):
    """(page, row in the page) of the first `count` slots of sequence b, on the GPU."""
    ps = st["k"].shape[2]
    page = st["table"][b].long().repeat_interleave(ps)[:count]
    return page, torch.arange(count, device="cuda") % ps


def _exact_decode(st, case):
    q, H = st["q"].double(), st["H"]
    Hkv, dh = st["k"].shape[1], st["k"].shape[3]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    score = st["score0"].double() if case["acc"] else None
    for b, count in enumerate(st["len0"].tolist()):
        page, row = _slots_of(st, b, count)
        for h in range(Hkv):
            mine = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
            keys, values = st["k"][page, h, row].double(), st["v"][page, h, row].double()
            weight = torch.softmax(q[b, mine] @ keys.t() / math.sqrt(dh), dim=1)
            out[b, mine] = weight @ values
            if score is not None:
                score[b, h, :count] += weight.sum(0)
    return dict(out=out, score=score) if case["acc"] else dict(out=out)


def _exact_append(st, case):
    k, v, pos, score = st["k"].double(), st["v"].double(), st["pos0"].double(), st["score0"].double()
    for b, (count, new, seen) in enumerate(zip(st["len0"].tolist(), st["n_new"].tolist(), st["seen0"].tolist())):
        if new == 0:
            continue
        page, row = (x[count:] for x in _slots_of(st, b, count + new))
        rows = st["path"][b, :new].long() if st["path"] is not None else torch.arange(new, device="cuda")
        k[page, :, row] = st["k_new"][b][:, rows].transpose(0, 1).double()
        v[page, :, row] = st["v_new"][b][:, rows].transpose(0, 1).double()
        pos[b, :, count:count + new] = torch.arange(seen, seen + new, device="cuda", dtype=torch.float64)
        score[b, :, count:count + new] = 0.0
    return dict(k=k, v=v, pos=pos, score=score, len=(st["len0"] + st["n_new"]).double(), seen=(st["seen0"] + st["n_new"]).double())


def _exact_evict(st, case):
    budget, recent = case["budget"], case["recent"]
    k, v = st["k"].double(), st["v"].double()
    pos, score = st["pos0"].cpu().numpy(), st["score0"].cpu().numpy().astype(np.float64)
    new_pos, new_score = pos.copy(), score.copy()
    lens, seen = st["len0"].tolist(), st["seen0"].tolist()
    for b, count in enumerate(lens):
        if count <= budget:
            continue
        page, row = _slots_of(st, b, count)
        for h in range(st["k"].shape[1]):
            newest = pos[b, h, :count] >= seen[b] - recent
            order = np.lexsort((np.arange(count), -score[b, h, :count], ~newest))
            stays = np.zeros(count, bool)
            stays[order[:budget]] = True
            dst, src = np.flatnonzero(~stays[:budget]), budget + np.flatnonzero(stays[budget:])
            new_pos[b, h, dst], new_score[b, h, dst] = pos[b, h, src], score[b, h, src]
            d, s = _dev(dst), _dev(src)
            k[page[d], h, row[d]] = k[page[s], h, row[s]]
            v[page[d], h, row[d]] = v[page[s], h, row[s]]
    return dict(k=k, v=v, pos=_dev(new_pos).double(), score=_dev(new_score), len=st["len0"].clamp(max=budget).double())


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    H, Hkv, dh, dtype, ps, mp = _geometry(case)
    es, B = 2 if dtype == "bf16" else 4, case["B"]
    row = Hkv * dh * es
    held = B * 0.5 * (case["P_min"] + case["P_max"])
    if case["kind"] == "decode":
        # keys and values once, queries and results, the table; with accounts each is read and written
        by = held * 2 * row + B * 2 * H * dh * es + 4 * held / ps + (8 * held * Hkv if case["acc"] else 0)
        return dict(bytes=by, flops=4.0 * held * H * dh)
    if case["kind"] == "append":
        # a row of keys and one of values read and written, its position and its account
        new = B * 0.5 * (case["n_min"] + case["n_max"])
        return dict(bytes=new * (4 * row + 8 * Hkv) + B * 32, flops=0.0)
    # every account and position read; of the rows that leave, those below the budget are replaced (accounts in no order)
    over = max(0.0, held / B - case["budget"]) if case["P_min"] > case["budget"] else 0.5 * (case["P_max"] - case["budget"])
    moved = B * over * case["budget"] / max(held / B, case["budget"])
    return dict(bytes=held * 8 * Hkv + moved * (4 * row + 16 * Hkv) + B * 16, flops=0.0)
