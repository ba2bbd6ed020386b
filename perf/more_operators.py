"""Serving over a KV cache held in 8 bits, as calls whose time and results can be compared with their plain forms.

What a decoding step does around the attention, on a cache of pages whose keys and values are e4m3 numbers with one scale for every 16
tokens of a page and KV head:

  pages   pages for the new tokens of every request are taken from a list of free ones, tables, offsets, positions and slots written; the
          pages that no token came to use go back to the list
  rope    queries and keys of a packed batch get their norm per head and are rotated to their positions
  append  new rows are encoded into the cache (a block's scale is the smallest power of two that holds its rows, and grows with them),
          and the cache is read back as contiguous keys and values, as verification of a draft tree takes them
  decode  attention of one new token per sequence over its whole cache

Head layouts and types are those of the repository's workloads (the tiny single-precision instance, Llama-3-8B and Llama-2-70B
shapes, the drafter's Self-Attention layer with eight query heads per KV head).  Keys, values and queries are N(0, 1), one channel in
32 several times as large.
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
    "odd": (6, 2, 80, "bf16"),
    "odd-f32": (6, 2, 80, "f32"),
}
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_CODE = torch.float8_e4m3fn
_BLOCK = 16                              # slots that share a scale
_EPS, _THETA = 1e-6, 500000.0


def _pages(B, P_max, page, n_min, n_max, room):
    """B sequences of up to P_max tokens, n_min .. n_max new ones each; room: share of the pages wanted that is free."""
    return dict(kind="pages", B=B, P_max=P_max, page=page, n_min=n_min, n_max=n_max, room=room)


def _rope(heads, T, far, norm, part):
    """T tokens at positions below `far`; part: only the first half of a head's dims is rotated."""
    return dict(kind="rope", heads=heads, T=T, far=far, norm=norm, part=part)


def _append(heads, B, P_min, P_max, page, M, n_min, n_max, rows):
    """rows: "tree" (slabs of M nodes, of which a list says n_min .. n_max), "slab" (slabs of M, the first n_min .. n_max), "packed"
    (the rows of all sequences one behind the other)."""
    return dict(kind="append", heads=heads, B=B, P_min=P_min, P_max=P_max, page=page, M=M, n_min=n_min, n_max=n_max, rows=rows)


def _decode(heads, B, P_min, P_max, page):
    """page: rows of a page; 0 = one page per sequence."""
    return dict(kind="decode", heads=heads, B=B, P_min=P_min, P_max=P_max, page=page)


def listed():
    return [
        # a decoded token of each request of a small batch
        dict(_pages(16, 1000, 16, 1, 1, 2.0), name="pages-token"),
        # a batch of ragged prompts
        dict(_pages(64, 0, 16, 200, 2048, 1.2), name="pages-prompts"),
        # the tokens that a batch decodes in one step: latency
        dict(_rope("8b", 16, 32768, True, False), name="rope-token"),
        # the tokens of a batch of prompts
        dict(_rope("8b", 8192, 32768, True, False), name="rope-prompts"),
        # single precision, heads of 80 dims of which 40 are rotated, no norm, far positions
        dict(_rope("odd-f32", 999, 1000000, False, True), name="rope-odd-fp32"),
        # a decoded token of every request of a batch
        dict(_append("8b", 64, 17, 250, 16, 1, 1, 1, "slab"), name="append-token"),
        # the accepted nodes of trees of 60, one to seven per request
        dict(_append("8b", 16, 100, 1500, 40, 60, 1, 7, "tree"), name="append-accepted"),
        # ragged prompts into empty caches
        dict(_append("70b", 4, 0, 0, 128, 2048, 517, 2048, "packed"), name="append-prompts"),
        # the smallest attention: single precision, a short conversation, all latency
        dict(_decode("tiny", 1, 48, 64, 16), name="decode-tiny-fp32"),
        # one request behind a prompt of about a thousand tokens
        dict(_decode("8b", 1, 1024, 1084, 16), name="decode-8b-1k"),
        # a serving batch of very different lengths
        dict(_decode("8b", 64, 17, 8192, 64), name="decode-8b-batch64"),
        # long context, eight query heads per KV head; the largest call
        dict(_decode("70b", 8, 32768, 32768, 128), name="decode-70b-32k"),
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
        kind = rng.choice(["decode", "decode", "append", "rope", "pages"])
        heads = rng.choice(["8b", "8b", "8b", "70b", "sa", "tiny", "odd", "odd-f32"])
        B = _log_int(rng, 1, 96)
        page = rng.choice([16, 16, 32, 48, 64, 128, 256, rng.randint(1, 40)])
        if kind == "pages":
            n = _log_int(rng, 1, 4096)
            c = _pages(_log_int(rng, 1, 1024), rng.choice([0, _log_int(rng, 1, 8192)]), page, rng.randint(0, n), n, rng.choice([0.5, 1.0, 2.0]))
            if c["B"] * n > 1 << 18:
                continue
        elif kind == "rope":
            c = _rope(heads, _log_int(rng, 1, 16384), _log_int(rng, 16, 1000000), rng.random() < 0.7, rng.random() < 0.3)
        elif kind == "append":
            P = _log_int(rng, 1, 2000) if rng.random() < 0.8 else 0
            M = rng.choice([1, 1, rng.randint(2, 256), _log_int(rng, 16, 2048)])
            rows = rng.choice(["slab", "packed", "tree"]) if 1 < M <= 256 else rng.choice(["slab", "packed"])
            n = rng.randint(1, min(M, 9)) if rows == "tree" else M
            c = _append(heads, B, P // 2, P, page, M, rng.randint(0, n), n, rows)
        else:
            P = _log_int(rng, 1, 32768)
            c = _decode(heads, B, max(1, int(P * rng.random())), P, rng.choice([page, page, page, 0]))
        # (states of more than 6 GiB are a matter of memory, not of another kind of call)
        if _cost(c) <= most and (kind in ("pages", "rope") or _state_bytes(c) < 6 << 30):
            return c


# ------------------------------------------------------------------ inputs

def _geometry(case):
    H, Hkv, dh, dtype = HEADS[case["heads"]]
    need = case["P_max"] + (case["n_max"] if case["kind"] == "append" else 0)
    ps = case["page"] or need
    return H, Hkv, dh, dtype, ps, (need + ps - 1) // ps


def _state_bytes(case):
    H, Hkv, dh, dtype, ps, mp = _geometry(case)
    return case["B"] * Hkv * mp * ps * dh * 2 * (1 if case["kind"] == "decode" else 5)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _normal(g, *shape):
    """N(0, 1), one channel in 32 six times as large."""
    x = torch.randn(shape, device="cuda", generator=g)
    x[..., 5::32] *= 6.0
    return x


def prepare(case, seed):
    host = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"pages": _prepare_pages, "rope": _prepare_rope, "append": _prepare_cache, "decode": _prepare_cache}[case["kind"]](case, host, g)


def _lengths(case, host, lo, hi):
    n = host.integers(lo, hi + 1, size=case["B"]).astype(np.int32)
    n[host.integers(0, case["B"])] = hi
    return n


def _prepare_pages(case, host, g):
    B, ps = case["B"], case["page"]
    n = _lengths(case, host, case["P_max"] // 8, case["P_max"])
    new = _lengths(case, host, case["n_min"], case["n_max"])
    mp = (case["P_max"] + case["n_max"] + ps - 1) // ps
    held = (n + ps - 1) // ps
    wanted = int(((n + new + ps - 1) // ps - held).sum())
    free = max(1, int(case["room"] * wanted))
    n_pages = 3 * B * mp + 4                             # the others are other batches'
    order = host.permutation(n_pages).astype(np.int32)
    table = np.full((B, mp), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += int(held[b])
    listed_free = np.full(n_pages, -1, np.int32)
    listed_free[:free] = order[at:at + free]
    T = B * case["n_max"]                                # the rows that the batch has room for
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
    return dict(case=case, ps=ps, n_pages=n_pages, len=_dev(n), new=_dev(new), table=_dev(table), free=_dev(listed_free),
                n_free=torch.tensor([free], dtype=torch.int32, device="cuda"), got=i32(B), off=i32(B + 1), pos=i32(T), slot=i32(T), status=i32(1))


def _rot(case, dh):
    return dh // 2 if case["part"] else dh


def _prepare_rope(case, host, g):
    H, Hkv, dh, dtype = HEADS[case["heads"]]
    dt, T = _TORCH[dtype], case["T"]
    qkv = _normal(g, T, H + 2 * Hkv, dh).to(dt)         # as one projection leaves them
    # runs of neighbouring positions, as prompts are, from anywhere
    start = torch.randint(0, case["far"], (T,), device="cuda", generator=g)
    run = torch.arange(T, device="cuda")
    pos = ((start[run // 97] + run % 97) % case["far"]).to(torch.int32)
    weight = lambda: (1.0 + 0.2 * torch.randn(dh, device="cuda", generator=g)).to(dt)
    return dict(case=case, q=qkv[:, :H], k=qkv[:, H:H + Hkv], pos=pos, gq=weight() if case["norm"] else None, gk=weight() if case["norm"] else None,
                q_out=torch.zeros(T, H, dh, dtype=dt, device="cuda"), k_out=torch.zeros(T, Hkv, dh, dtype=dt, device="cuda"))


def _prepare_cache(case, host, g):
    H, Hkv, dh, dtype, ps, mp = _geometry(case)
    B, kind, dt = case["B"], case["kind"], _TORCH[dtype]
    n = _lengths(case, host, case["P_min"], case["P_max"])
    new = _lengths(case, host, case["n_min"], case["n_max"]) if kind == "append" else np.zeros(B, np.int32)
    # pages in the order in which a server that had them all back from others would hand them out; entries not yet needed are -1
    want = (n + new + ps - 1) // ps
    n_pages = B * mp + 3
    order = host.permutation(n_pages).astype(np.int32)
    table = np.full((B, mp), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :want[b]] = order[at:at + want[b]]
        at += int(want[b])
    bps = (ps + _BLOCK - 1) // _BLOCK
    st = dict(case=case, dt=dt, table=_dev(table), len0=_dev(n), spare=int(order[at]), status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    st["len"] = st["len0"].clone()
    for name in ("k", "v"):
        # the codes of a block reach up to between half of the largest number and all of it; scales differ by powers of two
        st[name] = torch.empty(n_pages, Hkv, ps, dh, dtype=_CODE, device="cuda")
        st[name + "_scale"] = torch.exp2(torch.randint(-5, -2, (n_pages, Hkv, bps), device="cuda", generator=g).float())
        per = st[name + "_scale"].repeat_interleave(_BLOCK, dim=2)[:, :, :ps, None]
        step = max(1, (1 << 27) // (Hkv * ps * dh))
        for p in range(0, n_pages, step):
            rows = st[name][p:p + step]
            rows.copy_((_normal(g, *rows.shape) / per[p:p + step]).clamp(-448, 448).to(_CODE))
    if kind == "decode":
        st["q"] = (1.5 * torch.randn(B, H, dh, device="cuda", generator=g)).to(dt)
        st["out"] = torch.zeros(B, H, dh, dtype=dt, device="cuda")
    else:
        st["path"] = st["n_new"] = st["off"] = None
        M, P = case["M"], case["P_max"] + case["n_max"]
        if case["rows"] == "packed":
            off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
            st["off"] = _dev(off)
            T = int(off[-1])
            qkv = _normal(g, T, H + 2 * Hkv, dh).to(dt)
            st["k_new"], st["v_new"] = qkv[:, H:H + Hkv].contiguous(), qkv[:, H + Hkv:]      # keys rotated since, values as projected
        else:
            st["k_new"], st["v_new"], st["n_new"] = _normal(g, B, Hkv, M, dh).to(dt), _normal(g, B, Hkv, M, dh).to(dt), _dev(new)
        if case["rows"] == "tree":                     # nodes of an accepted path: increasing, the root first, then -1
            path = np.full((B, M), -1, np.int32)
            for b in range(B):
                if new[b]:
                    path[b, :new[b]] = np.concatenate([[0], 1 + np.sort(host.choice(M - 1, size=new[b] - 1, replace=False))])
            st["path"] = _dev(path)
        st["k_out"], st["v_out"] = (torch.zeros(B, Hkv, P, dh, dtype=dt, device="cuda") for _ in range(2))
    if own:
        import paper_2410_03804_amd as moa

        st["cache"] = moa.QuantKVCache(st["k"], st["v"], st["k_scale"], st["v_scale"], st["table"], st["len"], dt)
        if kind == "decode":
            st["ws"] = torch.empty(max(moa.kvq_decode_attn_workspace_bytes(st["cache"], H), 256), dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    return {"pages": _run_pages, "rope": _run_rope, "append": _run_append, "decode": _run_decode}[st["case"]["kind"]](st)


def _run_pages(st):
    # the pages taken go back in the order in which they came, so that a pass leaves the list as it found it
    if own:
        import paper_2410_03804_amd as moa

        moa.kv_reserve(st["table"], st["len"], st["new"], st["ps"], st["free"], st["n_free"], st["off"], st["got"], pos=st["pos"], slot=st["slot"],
                       dev_status=st["status"])
        moa.kv_release(st["table"], st["len"], st["ps"], st["free"], st["n_free"], dev_status=st["status"])
    else:
        _plain_reserve(st)
        _plain_release(st)
    return {name: st[name] for name in ("off", "got", "pos", "slot", "table", "free", "n_free")}


def _run_rope(st):
    H, Hkv, dh, _ = HEADS[st["case"]["heads"]]
    if own:
        import paper_2410_03804_amd as moa

        moa.qk_norm_rope(st["q"], st["k"], st["q_out"], st["k_out"], st["pos"], rope_theta=_THETA, rot_dim=_rot(st["case"], dh), gq=st["gq"], gk=st["gk"],
                         rms_eps=_EPS)
    else:
        for x, g, out in ((st["q"], st["gq"], st["q_out"]), (st["k"], st["gk"], st["k_out"])):
            _plain_rope(x, g, st["pos"], _rot(st["case"], dh), out)
    return dict(q=st["q_out"], k=st["k_out"])


def _run_append(st):
    st["len"].copy_(st["len0"])                        # the call moves the lengths on; what a program does that rolls a cache back
    if own:
        import paper_2410_03804_amd as moa

        if st["off"] is not None:
            moa.kvq_append_rows(st["cache"], st["k_new"], st["v_new"], st["off"], dev_status=st["status"])
        else:
            moa.kvq_append(st["cache"], st["k_new"], st["v_new"], path=st["path"], n_new=st["n_new"], dev_status=st["status"])
        moa.kvq_read(st["cache"], st["k_out"], st["v_out"], dev_status=st["status"])
    else:
        _plain_append(st)
        _plain_read(st)
    return {name: st[name] for name in ("k_out", "v_out", "k_scale", "v_scale", "len")}


def _run_decode(st):
    if own:
        import paper_2410_03804_amd as moa

        moa.kvq_decode_attn(st["cache"], st["q"], st["out"], st["ws"], dev_status=st["status"])
    else:
        _plain_decode(st)
    return st["out"]


# ------------------------------------------------------------------ plain forms

def _plain_reserve(st):
    table, n, new, ps = st["table"], st["len"].long(), st["new"].long(), st["ps"]
    B, mp = table.shape
    T, free = st["pos"].numel(), st["free"]
    page = torch.arange(mp, device=n.device)[None, :]
    needs = (page >= (n // ps)[:, None]) & (page <= ((n + new - 1) // ps)[:, None]) & (new > 0)[:, None] & (table < 0)
    need = needs.sum(dim=1)
    upto = torch.cumsum(need, dim=0)
    ok = (need == 0) | (upto <= st["n_free"].long())
    taken = (torch.where(ok, upto, torch.zeros_like(upto))).amax()
    which = (torch.cumsum(needs.reshape(-1).long(), dim=0) - 1).view(B, mp)
    at = (st["n_free"].long() - 1 - which).clamp(min=0)
    table.copy_(torch.where(needs & ok[:, None], free[at], table))
    st["n_free"] -= taken.to(torch.int32)
    st["off"][1:] = torch.cumsum(new, dim=0).to(torch.int32)
    st["got"].copy_(torch.where(ok, new, torch.zeros_like(new)).to(torch.int32))
    t = torch.arange(T, device=n.device)
    b = torch.searchsorted(st["off"][1:].long(), t, right=True).clamp(max=B - 1)
    real = t < st["off"][B]
    i = n[b] + t - st["off"].long()[b]
    st["pos"].copy_(torch.where(real, i, torch.zeros_like(i)).to(torch.int32))
    id_ = table.view(-1)[(b * mp + i // ps).clamp(max=B * mp - 1)].long()
    st["slot"].copy_(torch.where(real & ok[b] & (id_ >= 0), id_ * ps + i % ps, torch.full_like(i, -1)).to(torch.int32))


def _plain_release(st):
    table, ps, free = st["table"], st["ps"], st["free"]
    B, mp = table.shape
    page = torch.arange(mp, device=table.device)[None, :]
    gone = (page >= ((st["len"].long() + ps - 1) // ps)[:, None]) & (table >= 0)
    which = torch.cumsum(gone.reshape(-1).long(), dim=0)
    count = which[-1]
    # the first of them is the next one to be taken: place n_free + count - its number; the others go to a place behind the list
    at = torch.where(gone.reshape(-1), st["n_free"].long() + count - which, torch.full_like(which, free.numel()))
    free.copy_(torch.cat([free, free[:1]]).scatter_(0, at, table.reshape(-1))[:-1])
    table.masked_fill_(gone, -1)
    st["n_free"] += count.to(torch.int32)


def _plain_rope(x, weight, pos, rot, out):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(dim=2, keepdim=True) + _EPS) * weight.float()
    c = torch.arange(rot // 2, device=x.device, dtype=torch.float64)
    angle = pos.double()[:, None] * torch.exp(c * (-2.0 * math.log(_THETA) / rot))[None, :]
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    a, b = y[:, :, :rot // 2], y[:, :, rot // 2:rot]
    out.copy_(torch.cat([a * cos - b * sin, b * cos + a * sin, y[:, :, rot:]], dim=2).to(out.dtype))


def _plain_append(st):
    table, ps, n0 = st["table"], st["k"].shape[2], st["len0"].long()
    _, Hkv, _, dh = st["k"].shape
    B, mp = table.shape
    case, bps = st["case"], st["k_scale"].shape[2]
    N = case["n_max"]
    i = torch.arange(N, device=table.device)[None, :].expand(B, N)
    new = (st["off"][1:] - st["off"][:-1] if st["off"] is not None else st["n_new"]).long()[:, None]
    real = i < new
    slot = (n0[:, None] + i).clamp(max=mp * ps - 1)
    # (what is no row goes to a page that no sequence has)
    page = torch.where(real, torch.gather(table.long(), 1, slot // ps), torch.full_like(slot, st["spare"]))
    head = torch.arange(Hkv, device=table.device)[None, :, None]
    row = (page[:, None, :] * Hkv + head) * ps + (slot % ps)[:, None, :]
    block = (page[:, None, :] * Hkv + head) * bps + (slot % ps // _BLOCK)[:, None, :]
    # the rows in front of the first new one in its block, which has their scale already
    first = slot[:, :1] - slot[:, :1] % ps % _BLOCK
    j = first + torch.arange(_BLOCK, device=table.device)[None, :]
    old = (j < n0[:, None]) & (new > 0)
    page_j = torch.where(old, torch.gather(table.long(), 1, (j // ps).clamp(max=mp - 1)), torch.full_like(j, st["spare"]))
    row_j = (page_j[:, None, :] * Hkv + head) * ps + (j % ps)[:, None, :]
    block_j = (page_j[:, None, :] * Hkv + head) * bps + (j % ps // _BLOCK)[:, None, :]
    for name in ("k", "v"):
        x = st[name + "_new"]
        if st["off"] is not None:
            src = (st["off"][:-1].long()[:, None] + i).clamp(max=x.shape[0] - 1)
            x = x[src].permute(0, 2, 1, 3).float()
        else:
            src = torch.gather(st["path"].long(), 1, i).clamp(min=0) if st["path"] is not None else i
            x = torch.gather(x, 2, src[:, None, :, None].expand(B, Hkv, N, dh)).float()
        scale, codes = st[name + "_scale"].view(-1), st[name].view(torch.uint8).view(-1, dh)
        most = torch.zeros_like(scale).scatter_reduce_(0, block.reshape(-1), x.abs().amax(dim=3).reshape(-1), "amax")
        bits = most.view(torch.int32)
        e = ((bits >> 23) - 135 + ((bits & 0x7fffff) > 0x600000)).clamp(-120, 120)
        fits = ((e + 127) << 23).view(torch.float32)
        mark = lambda at: torch.zeros(scale.shape, dtype=torch.bool, device=scale.device).index_fill_(0, at.reshape(-1), True)
        touched, held = mark(block), mark(block_j)
        touched.view(-1, Hkv * bps)[st["spare"]] = False
        grown = torch.where(touched, torch.where(held, torch.maximum(scale, fits), fits), scale)
        kept = codes[row_j].view(_CODE).float() * (scale / grown)[block_j][..., None]
        codes[row_j] = kept.to(_CODE).view(torch.uint8)
        codes[row] = (x / grown[block][..., None]).clamp(-448, 448).to(_CODE).view(torch.uint8)
        scale.copy_(grown)
    st["len"] += new[:, 0].to(torch.int32)


def _plain_read(st):
    table, ps = st["table"], st["k"].shape[2]
    B, mp = table.shape
    for name in ("k", "v"):
        out = st[name + "_out"]
        Hkv, P, dh = out.shape[1:]
        held = torch.arange(P, device=out.device)[None, :] < st["len"][:, None]
        values = _rows(st, name, slice(0, B))[:, :, :P]
        out.copy_(torch.where(held[:, None, :, None], values.to(out.dtype), out))


def _rows(st, name, which):
    """[sequences, Hkv, capacity, dh]: what the cache's codes stand for."""
    pages = st["table"][which].clamp(min=0).long()
    codes, scale = st[name].view(torch.uint8)[pages].view(_CODE), st[name + "_scale"][pages]
    nb, mp, Hkv, ps, dh = codes.shape
    values = codes.float() * scale.repeat_interleave(_BLOCK, dim=3)[:, :, :, :ps, None]
    return values.permute(0, 2, 1, 3, 4).reshape(nb, Hkv, mp * ps, dh)


def _plain_decode(st):
    table, q = st["table"], st["q"]
    _, Hkv, ps, dh = st["k"].shape
    B, mp = table.shape
    cap, G = mp * ps, q.shape[1] // Hkv
    step = max(1, (1 << 28) // (Hkv * cap * dh))
    for b0 in range(0, B, step):
        sl = slice(b0, min(b0 + step, B))
        held = torch.arange(cap, device=q.device)[None, :] < st["len"][sl, None]
        qf = q[sl].float().view(-1, Hkv, G, dh) * dh ** -0.5
        s = torch.matmul(qf, _rows(st, "k", sl).transpose(2, 3).contiguous())
        s = torch.where(held[:, None, None, :], s, torch.full((), -math.inf, device=q.device))
        e = torch.exp(s - s.amax(dim=3, keepdim=True))
        p = e / e.sum(dim=3, keepdim=True)
        vf = torch.where(held[:, None, :, None], _rows(st, "v", sl), torch.zeros((), device=q.device))
        st["out"][sl] = torch.matmul(p, vf).view(-1, Hkv * G, dh).to(q.dtype)


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return {"pages": _exact_pages, "rope": _exact_rope, "append": _exact_append, "decode": _exact_decode}[case["kind"]](st, case)


def _exact_pages(st, case):
    ps, n, new = st["ps"], st["len"].tolist(), st["new"].tolist()
    table, free, left = st["table"].cpu().numpy(), st["free"].tolist(), int(st["n_free"])
    off, got, pos, slot = [0], [], [], []
    stack = free[:left]
    refused = False
    for b in range(case["B"]):
        lacking = [p for p in range(n[b] // ps, (n[b] + new[b] - 1) // ps + 1) if table[b, p] < 0] if new[b] else []
        fits = not lacking or (not refused and len(lacking) <= len(stack))
        refused = refused or not fits
        pages = {p: int(table[b, p]) for p in range(table.shape[1]) if table[b, p] >= 0}
        if fits:
            pages.update({p: stack.pop() for p in lacking})
        for i in range(n[b], n[b] + new[b]):
            pos.append(i)
            slot.append(pages[i // ps] * ps + i % ps if fits else -1)
        off.append(off[-1] + new[b])
        got.append(new[b] if fits else 0)
    T = st["pos"].numel()
    return dict(off=np.array(off), got=np.array(got), pos=np.array(pos + [0] * (T - len(pos))), slot=np.array(slot + [-1] * (T - len(slot))),
                table=table, free=np.array(free), n_free=np.array([left]))


def _exact_rope(st, case):
    H, Hkv, dh, _ = HEADS[case["heads"]]
    rot = _rot(case, dh)
    half = rot // 2
    freq = torch.tensor([_THETA ** (-2.0 * c / rot) for c in range(half)], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st["pos"].double()[:, None] * freq)[:, None, :]
    found = {}
    for name, weight in (("q", st["gq"]), ("k", st["gk"])):
        y = st[name].double()
        if weight is not None:
            y = y / torch.sqrt(y.square().mean(dim=2, keepdim=True) + _EPS) * weight.double()
        z = torch.complex(y[..., :half].contiguous(), y[..., half:rot].contiguous()) * turn
        found[name] = torch.cat([z.real, z.imag, y[..., rot:]], dim=2)
    return found


def _e4m3(x):
    """The nearest number that e4m3 holds, ties to even, for |x| <= 448."""
    _, e = np.frexp(np.where(x == 0, 1.0, x))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(x / step) * step


def _smallest_scale(most):
    m, e = np.frexp(most)
    return np.ldexp(1.0, np.clip(np.where(most == 0, -120, e - 9 + (m > 0.875)), -120, 120))


def _exact_append(st, case):
    if st["k"].numel() > 1 << 27:
        return None                                                   # (minutes on the host)
    ps, table = st["k"].shape[2], st["table"].cpu().numpy()
    n0 = st["len0"].tolist()
    new = (st["off"][1:] - st["off"][:-1] if st["off"] is not None else st["n_new"]).tolist()
    found = dict(len=(st["len0"].double() + torch.tensor(new, device="cuda")))
    for name in ("k", "v"):
        codes, scale = st[name].float().cpu().numpy(), st[name + "_scale"].cpu().numpy().astype(np.float64)
        given = st[name + "_new"].float().cpu().numpy()
        out = st[name + "_out"].float().cpu().numpy().astype(np.float64)
        for b in range(case["B"]):
            if st["off"] is not None:
                o = int(st["off"][b])
                rows = given[o:o + new[b]].transpose(1, 0, 2)
            else:
                rows = given[b][:, st["path"][b, :new[b]].cpu().numpy() if st["path"] is not None else slice(0, new[b])]
            s, end = 0, n0[b] + new[b]
            while s < end:                                            # one block after the other
                page, r = table[b, s // ps], s % ps
                e = min(s + min(_BLOCK - r % _BLOCK, ps - r), end)
                was = slice(r, r + max(0, min(e, n0[b]) - s))
                x = rows[:, max(s - n0[b], 0):max(e - n0[b], 0)].astype(np.float64)
                before = scale[page, :, r // _BLOCK]
                after = before
                if x.shape[1]:
                    after = _smallest_scale(np.abs(x).max(axis=(1, 2)))
                    if was.stop > was.start:
                        after = np.maximum(after, before)
                held = codes[page, :, was].astype(np.float64) * (before / after)[:, None, None]
                both = np.concatenate([_e4m3(held), _e4m3(x / after[:, None, None])], axis=1)
                out[b, :, s:e] = both * after[:, None, None]
                scale[page, :, r // _BLOCK] = after
                s = e
        found[name + "_out"], found[name + "_scale"] = _dev(out), _dev(scale)
    return found


def _exact_decode(st, case):
    q = st["q"].double()
    Hkv, ps, dh = st["k"].shape[1:]
    G = q.shape[1] // Hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for b, count in enumerate(st["len"].tolist()):
        s = torch.arange(count, device="cuda")
        page, r = st["table"][b].long()[s // ps], s % ps
        for h in range(Hkv):
            mine = slice(h * G, (h + 1) * G)
            keys, values = (st[x].view(torch.uint8)[page, h, r].view(_CODE).double() * st[x + "_scale"][page, h, r // _BLOCK].double()[:, None] for x in "kv")
            out[b, mine] = torch.softmax(q[b, mine] @ keys.t() / math.sqrt(dh), dim=1) @ values
    return out


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    kind = case["kind"]
    if kind == "pages":
        # lengths read; offsets, counts, positions and slots written; every page handed out read from the list, written and given back
        new = case["B"] * 0.5 * (case["n_min"] + case["n_max"])
        return dict(bytes=16 * case["B"] + 8 * case["B"] * case["n_max"] + 16 * new / case["page"] + 8, flops=0.0)
    H, Hkv, dh, dtype = HEADS[case["heads"]]
    es = 2 if dtype == "bf16" else 4
    if kind == "rope":
        n = case["T"] * (H + Hkv) * dh
        return dict(bytes=2 * n * es + 4 * case["T"], flops=(6.0 if case["norm"] else 2.0) * n)
    ps = _geometry(case)[4]
    row = Hkv * dh
    held = case["B"] * 0.5 * (case["P_min"] + case["P_max"])
    if kind == "decode":
        # keys and values with their scales, queries and results, the table
        return dict(bytes=held * (2 * row + 8 * Hkv / _BLOCK + 4 / ps) + case["B"] * 2 * H * dh * es, flops=4.0 * held * H * dh)
    # new rows read and their codes written; all rows' codes read and their values written
    new = case["B"] * 0.5 * (case["n_min"] + case["n_max"])
    return dict(bytes=new * 2 * row * (es + 1) + (held + new) * (2 * row * (1 + es) + 8 * Hkv / _BLOCK), flops=0.0)
