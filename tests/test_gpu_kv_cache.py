"""moa_kv_append and moa_kv_evict on an MI355X (exact), and the three calls of a decoding loop together."""
import numpy as np
import pytest
import torch

import paper_2410_03804_amd as moa
from kv_util import TDT, Cache, check, decode_reference, evict_reference, workspace

pytestmark = pytest.mark.gpu

HEADS = {"tiny": (4, 2, 64, "f32"), "8b": (32, 8, 128, "bf16"), "d33": (3, 1, 33, "bf16"), "d5f": (2, 2, 5, "f32")}


def bits(t):
    return t.detach().cpu().contiguous().view(torch.uint8).numpy().copy()


def state(c):
    return {n: bits(getattr(c, n)) for n in ("k", "v", "pos", "seen", "score") if getattr(c, n) is not None} | {"len": bits(c.t_len)}


def append_reference(c, k_new, v_new, path, n_new, lens):
    """The pools, accounts and lengths after the append, on the CPU (in the storage type)."""
    k, v = c.k.cpu().clone(), c.v.cpu().clone()
    pos, seen, score = (None if t is None else t.cpu().clone() for t in (c.pos, c.seen, c.score))
    kn, vn = k_new.cpu(), v_new.cpu()
    M = kn.shape[2]
    out = []
    for b in range(len(lens)):
        n = M if n_new is None else int(n_new[b])
        n = min(max(n, 0), M, c.cap - lens[b])
        for i in range(n):
            src, s = i if path is None else int(path[b, i]), lens[b] + i
            page = int(c.table[b, s // c.page])
            if page < k.shape[0]:
                k[page, :, s % c.page], v[page, :, s % c.page] = kn[b, :, src], vn[b, :, src]
            if pos is not None:
                pos[b, :, s] = int(seen[b]) + i
            if score is not None:
                score[b, :, s] = 0.0
        if seen is not None:
            seen[b] += n
        out.append(lens[b] + n)
    ref = dict(k=k, v=v, pos=pos, seen=seen, score=score)
    return {n: bits(t) for n, t in ref.items() if t is not None} | {"len": bits(torch.tensor(out, dtype=torch.int32))}


def same(got, want):
    assert got.keys() == want.keys()
    for name in want:
        assert np.array_equal(got[name], want[name]), name


def new_rows(c, M, seed):
    g = torch.Generator().manual_seed(seed)
    return tuple(torch.randn(len(c.lens), c.Hkv, M, c.dh, generator=g).to(TDT[c.dtype]).cuda() for _ in range(2))


@pytest.mark.parametrize("accounts", [False, True])
@pytest.mark.parametrize("M,n_new", [(1, None), (1, [1, 0, 1]), (9, [9, 4, 0]), (300, [300, 1, 299]), (2000, None)])
@pytest.mark.parametrize("page", [16, 7, 0])
@pytest.mark.parametrize("heads", list(HEADS))
def test_append(heads, page, M, n_new, accounts):
    lens = [0, 33, 6]
    c = Cache(HEADS[heads], lens, page or 33 + M, seed=M, accounts=accounts, room=M)
    k_new, v_new = new_rows(c, M, 3)
    n = None if n_new is None else torch.tensor(n_new, dtype=torch.int32, device="cuda")
    want = append_reference(c, k_new, v_new, None, n_new, lens)
    moa.kv_append(c.moa(), k_new, v_new, n_new=n, dev_status=c.status)
    same(state(c), want)
    assert c.status.item() == 0


@pytest.mark.parametrize("heads", ["8b", "d33"])
def test_append_accepted_nodes(heads):
    """path / n_path as moa_tree_accept leaves them: -1 behind the accepted nodes; the same node may come twice."""
    lens, M = [5, 100, 0, 31], 60
    c = Cache(HEADS[heads], lens, 16, seed=2, accounts=True, room=M)
    k_new, v_new = new_rows(c, M, 4)
    path = np.full((4, M), -1, np.int32)
    n_new = [4, 1, 7, 2]
    path[0, :4], path[1, :1], path[2, :7], path[3, :2] = [0, 3, 17, 59], [0], [0, 1, 2, 3, 4, 5, 6], [8, 8]
    want = append_reference(c, k_new, v_new, path, n_new, lens)
    moa.kv_append(c.moa(), k_new, v_new, path=torch.from_numpy(path).cuda(), n_new=torch.tensor(n_new, dtype=torch.int32, device="cuda"),
                  dev_status=c.status)
    same(state(c), want)
    assert c.status.item() == 0


@pytest.mark.parametrize("M", [8, 1500])
def test_append_beyond_the_capacity_and_bad_counts(M):
    lens = [60, 64, 10, 0]
    c = Cache(HEADS["tiny"], lens, 16, seed=5, accounts=True, room=0)
    k_new, v_new = new_rows(c, M, 5)
    # sequence 2 owns pages only up to slot 16 (then BAD_PAGE), the first fills up, the second is full, the last gets nothing
    n_new = [M, 1, M + 3, -1]
    want = append_reference(c, k_new, v_new, None, n_new, lens)
    moa.kv_append(c.moa(), k_new, v_new, n_new=torch.tensor(n_new, dtype=torch.int32, device="cuda"), dev_status=c.status)
    same(state(c), want)
    assert c.status.item() == moa.DEV_CACHE_FULL | moa.DEV_BAD_LENGTH | moa.DEV_BAD_PAGE
    assert c.t_len.tolist() == [64, 64, min(64, 10 + M), 0]


def test_append_bad_path_entry():
    c = Cache(HEADS["tiny"], [3], 16, seed=6, room=4)
    k_new, v_new = new_rows(c, 2, 6)
    path = torch.tensor([[-1, 2]], dtype=torch.int32, device="cuda")
    want = append_reference(c, k_new, v_new, np.array([[0, 1]]), None, [3])
    moa.kv_append(c.moa(), k_new, v_new, path=path, dev_status=c.status)
    same(state(c), want)
    assert c.status.item() == moa.DEV_BAD_PARENT


def test_append_unaligned_rows():
    c = Cache(HEADS["8b"], [3, 20], 16, seed=7, room=4)
    k_new, v_new = new_rows(c, 3, 7)
    flat = torch.empty(k_new.numel() + 1, dtype=k_new.dtype, device="cuda")
    flat[1:].copy_(k_new.view(-1))
    want = append_reference(c, k_new, v_new, None, None, [3, 20])
    moa.kv_append(c.moa(), flat[1:].view(k_new.shape), v_new)
    same(state(c), want)


def evict_expected(c, budget, recent, lens):
    k, v, pos, seen, score = (t.cpu().clone() for t in (c.k, c.v, c.pos, c.seen, c.score))
    out = []
    for b, n in enumerate(lens):
        out.append(min(n, budget))
        for h in range(c.Hkv):
            dst, src = evict_reference(pos[b, h].numpy(), score[b, h].numpy(), seen[b], n, budget, recent)
            for d, s in zip(dst, src):
                pd, ps = int(c.table[b, d // c.page]), int(c.table[b, s // c.page])
                k[pd, h, d % c.page], v[pd, h, d % c.page] = k[ps, h, s % c.page], v[ps, h, s % c.page]
                pos[b, h, d], score[b, h, d] = pos[b, h, s], score[b, h, s]
    ref = dict(k=k, v=v, pos=pos, seen=seen, score=score)
    return {n: bits(t) for n, t in ref.items()} | {"len": bits(torch.tensor(out, dtype=torch.int32))}


def evict(c, budget, recent):
    k = c.moa()
    ws = workspace(moa.kv_evict_workspace_bytes(k, budget))
    ws.fill_(255)
    moa.kv_evict(k, budget, recent, ws, dev_status=c.status)
    torch.cuda.synchronize()


@pytest.mark.parametrize("budget,recent", [(1, 0), (1, 1), (7, 3), (64, 0), (64, 64), (500, 100), (2000, 9), (5000, 10)])
@pytest.mark.parametrize("page", [16, 7, 0])
@pytest.mark.parametrize("heads", ["tiny", "8b", "d33"])
def test_evict(heads, page, budget, recent):
    lens = [2300, 1, 0, 64, 65, 777, 2000]
    c = Cache(HEADS[heads], lens, page or 2300, seed=budget, accounts=True)
    want = evict_expected(c, budget, recent, lens)
    evict(c, budget, recent)
    same(state(c), want)
    assert c.status.item() == 0


@pytest.mark.parametrize("n,budget", [(1025, 1024), (16384, 2048), (33000, 100), (20001, 20000), (70001, 5000), (40000, 39990)])
def test_evict_long(n, budget):
    c = Cache((2, 2, 8, "f32"), [n, n // 2], 64, seed=n, accounts=True)
    want = evict_expected(c, budget, budget // 4, [n, n // 2])
    evict(c, budget, budget // 4)
    same(state(c), want)


@pytest.mark.parametrize("kind", ["equal", "nan", "infinite", "negative", "tiny", "random", "octave", "pairs", "few_bits"])
def test_evict_kinds_of_accounts(kind):
    lens = [900, 70]
    c = Cache((4, 2, 16, "f32"), lens, 16, seed=21, accounts=True)
    rng = np.random.default_rng(21)
    s = rng.random(c.score.shape).astype(np.float32)
    if kind == "equal":
        s[:] = 0.25
    elif kind == "nan":
        s[rng.random(s.shape) < 0.95] = np.nan
    elif kind == "infinite":
        s[rng.random(s.shape) < 0.3] = np.inf
        s[rng.random(s.shape) < 0.3] = -np.inf
    elif kind == "negative":
        s -= 0.5
    elif kind == "tiny":
        s *= 1e-40                                   # denormals keep their order
    elif kind == "octave":
        s = (1.0 + s / 8192).astype(np.float32)      # one first digit, and second ones, for hundreds of slots
    elif kind == "pairs":
        s = np.repeat(s[..., ::2], 2, axis=-1)[..., : s.shape[-1]]
    elif kind == "few_bits":
        s = (np.floor(s * 3) / 4 + 1.0).astype(np.float32)
    c.score.copy_(torch.from_numpy(np.ascontiguousarray(s)))
    for budget in (600, 60):                         # the second time on what the first has left
        want = evict_expected(c, budget, 5, lens)
        evict(c, budget, 5)
        same(state(c), want)
        lens = c.t_len.tolist()


def test_evict_random_sizes():
    rng = np.random.default_rng(24)
    for i in range(40):
        n = int(np.exp(rng.uniform(np.log(2), np.log(9000))))
        budget = int(rng.integers(1, n + 1))
        c = Cache((2, 2, 4, "f32"), [n, int(rng.integers(0, n + 1))], int(rng.integers(1, 80)), seed=i, accounts=True)
        if i % 2:
            c.score.copy_(torch.exp(2 * torch.randn(c.score.shape, generator=torch.Generator().manual_seed(i))))
        lens, recent = c.t_len.tolist(), int(rng.integers(0, budget + 1))
        want = evict_expected(c, budget, recent, lens)
        evict(c, budget, recent)
        same(state(c), want)


def test_evict_more_protected_than_the_budget_holds():
    """Positions that are not distinct can make every slot one of the newest: the lowest ones stay."""
    c = Cache((2, 1, 16, "f32"), [200], 16, seed=22, accounts=True)
    c.pos.fill_(int(c.seen[0]))
    want = evict_expected(c, 50, 50, [200])
    evict(c, 50, 50)
    same(state(c), want)


def test_evict_lengths_outside_the_capacity_and_bad_pages():
    c = Cache((2, 2, 16, "f32"), [160, 160], 16, seed=23, accounts=True)
    c.t_len.copy_(torch.tensor([161, -1], dtype=torch.int32))
    before_k, before = c.k.clone(), c.pos.clone()
    c.t_table[0, 2] = -1
    evict(c, 100, 10)
    assert c.t_len.tolist() == [100, -1]
    assert c.status.item() == moa.DEV_BAD_LENGTH | moa.DEV_BAD_PAGE
    assert torch.equal(c.pos[1], before[1]) and not torch.equal(c.pos[0], before[0])
    rows = torch.from_numpy(c.table[1].astype(np.int64)).cuda()
    assert torch.equal(c.k[rows], before_k[rows])


def test_decoding_loop():
    """Prompts appended, then tokens decoded one by one with accounts and an eviction whenever a sequence is 16 over the budget: every
    call against the definition, from the state it found."""
    B, M, budget, recent = 3, 70, 64, 16
    c = Cache(HEADS["8b"], [0] * B, 16, seed=31, accounts=True, room=112)
    cache = c.moa()
    c.seen.zero_()
    ws = workspace(max(moa.decode_attn_workspace_bytes(cache, c.H), moa.kv_evict_workspace_bytes(cache, budget)))
    k_new, v_new = new_rows(c, M, 31)
    n_new = [70, 3, 41]
    lens = [0] * B
    want = append_reference(c, k_new, v_new, None, n_new, lens)
    moa.kv_append(cache, k_new, v_new, n_new=torch.tensor(n_new, dtype=torch.int32, device="cuda"), dev_status=c.status)
    same(state(c), want)
    out = torch.zeros(B, c.H, c.dh, dtype=torch.bfloat16, device="cuda")
    evicted = 0
    for step in range(40):
        lens = c.t_len.tolist()
        k1, v1 = new_rows(c, 1, 100 + step)
        want = append_reference(c, k1, v1, None, None, lens)
        moa.kv_append(cache, k1, v1, dev_status=c.status)
        same(state(c), want)
        c.lens = c.t_len.tolist()
        q = torch.randn(B, c.H, c.dh, generator=torch.Generator().manual_seed(step)).to(torch.bfloat16).cuda()
        before = c.score.cpu().double().numpy()
        ref, tol, weight, wtol = decode_reference(c, q)
        moa.decode_attn(cache, q, out, ws, accumulate=True, dev_status=c.status)
        check(out, ref, tol, f"step {step}")
        check(c.score, before + weight, wtol + 2.0 ** -23 * (np.abs(before) + weight), f"accounts {step}")
        if max(c.lens) >= budget + 16:
            want = evict_expected(c, budget, recent, c.lens)
            moa.kv_evict(cache, budget, recent, ws, dev_status=c.status)
            same(state(c), want)
            evicted += 1
    assert evicted >= 2 and c.status.item() == 0
    assert c.seen.tolist() == [n + 40 for n in n_new]


def test_verified_tree_committed_and_decoded_on():
    """A tree verified over the contiguous caches, its accepted nodes' keys and values committed by the path of the accept walk, the next
    token decoded over the same caches as pages of their capacity, and these cut down to a budget."""
    B, H, dh, M, cap = 2, 4, 64, 9, 330
    lens, budget = [300, 17], 200
    g = torch.Generator().manual_seed(51)
    bf16, i32 = torch.bfloat16, torch.int32
    rand = lambda *shape: torch.randn(shape, generator=g).to(bf16).cuda()
    c = Cache((H, H, dh, "bf16"), lens, cap, seed=51, accounts=True, spare=0)
    c.table = np.arange(B, dtype=np.int32)[:, None]
    c.t_table = torch.from_numpy(c.table).cuda()
    c.k, c.v = rand(B, H, cap, dh), rand(B, H, cap, dh)
    parent = torch.tensor([[-1, 0, 0, 1, 1, 2, 3, 3, 6], [-1, 0, 0, 0, 1, 2, 3, 4, 5]], dtype=i32, device="cuda")
    tok = torch.arange(B * M, dtype=i32, device="cuda").view(B, M)
    tgt = torch.full((B, M), 99, dtype=i32, device="cuda")
    for b, path in enumerate(([0, 1, 3, 6], [0, 2])):           # each node's successor on the path is the LLM's token
        for x, y in zip(path, path[1:]):
            tgt[b, x] = tok[b, y]
    mask, depth = torch.zeros(B, M, 1, dtype=torch.int64, device="cuda"), torch.zeros(B, M, dtype=i32, device="cuda")
    moa.tree_build(parent, mask, depth, c.status)
    shape = moa.Shape(1, H * dh, H, H, dh, H * dh, H, H, moa.BF16)
    x, out = rand(B, M, H * dh), torch.zeros(B, M, H * dh, dtype=bf16, device="cuda")
    kt, vt = (torch.zeros(B, H, M, dh, dtype=bf16, device="cuda") for _ in range(2))
    moa.tree_verify_attn(shape, x, None, None, None, None, c.k, c.v, c.t_len, cap, mask, out, kt, vt,
                         workspace(moa.workspace_bytes(shape, B, cap, M, 0)), c.status)
    path, n_path, bonus = torch.zeros(B, M, dtype=i32, device="cuda"), torch.zeros(B, dtype=i32, device="cuda"), torch.zeros(B, dtype=i32, device="cuda")
    moa.tree_accept(parent, tok, tgt, path, n_path, bonus)
    cache = c.moa()
    want = append_reference(c, kt, vt, path.cpu().numpy(), n_path.tolist(), lens)
    moa.kv_append(cache, kt, vt, path=path, n_new=n_path, dev_status=c.status)
    same(state(c), want)
    assert c.t_len.tolist() == [304, 19] and n_path.tolist() == [4, 2]
    for b, nodes in enumerate(([0, 1, 3, 6], [0, 2])):          # (without projections a node's key is its own row)
        assert torch.equal(c.k[b, :, lens[b]:lens[b] + len(nodes)], x[b, nodes].view(-1, H, dh).transpose(0, 1))
    ws = workspace(max(moa.decode_attn_workspace_bytes(cache, H), moa.kv_evict_workspace_bytes(cache, budget)))
    for step in range(2):                                       # over the whole cache, then over what eviction leaves
        c.lens = c.t_len.tolist()
        q = rand(B, H, dh)
        o = torch.zeros_like(q)
        before = c.score.cpu().double().numpy()
        ref, tol, weight, wtol = decode_reference(c, q)
        moa.decode_attn(cache, q, o, ws, accumulate=True, dev_status=c.status)
        check(o, ref, tol, f"step {step}")
        check(c.score, before + weight, wtol + 2.0 ** -23 * (np.abs(before) + weight), "accounts")
        want = evict_expected(c, budget, 20, c.lens)
        moa.kv_evict(cache, budget, 20, ws, dev_status=c.status)
        same(state(c), want)
    assert c.t_len.tolist() == [200, 19] and c.status.item() == 0


def test_captured_step_replayed():
    """Append, decode and evict captured into one graph; each replay against the same calls made eagerly on a copy."""
    budget = 600
    a, b = (Cache(HEADS["8b"], [620, 599, 0], 16, seed=41, accounts=True, room=20) for _ in range(2))
    k1, v1 = new_rows(a, 1, 41)
    q = torch.randn(3, a.H, a.dh, generator=torch.Generator().manual_seed(41)).to(torch.bfloat16).cuda()

    def step(c, cache, out, ws):
        moa.kv_append(cache, k1, v1, dev_status=c.status)
        moa.decode_attn(cache, q, out, ws, accumulate=True, dev_status=c.status)
        moa.kv_evict(cache, budget, 50, ws, dev_status=c.status)

    ca, cb = a.moa(), b.moa()
    wa, wb = (workspace(max(moa.decode_attn_workspace_bytes(ca, a.H), moa.kv_evict_workspace_bytes(ca, budget))) for _ in range(2))
    oa, ob = (torch.zeros(3, a.H, a.dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step(a, ca, oa, wa)
    for _ in range(4):
        g.replay()
        step(b, cb, ob, wb)
        torch.cuda.synchronize()
        same(state(a), state(b))
        assert torch.equal(oa, ob)
        k1.normal_()
        q.normal_()
    assert a.status.item() == 0 and a.t_len.tolist() == [600, 600, 4]
