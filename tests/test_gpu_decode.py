"""moa_decode_attn on an MI355X against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2410_03804_amd as moa
from kv_util import TDT, Cache, check, decode_reference, workspace

pytestmark = pytest.mark.gpu

HEADS = {
    "tiny": (4, 2, 64, "f32"), "8b": (32, 8, 128, "bf16"), "mha64": (8, 8, 64, "bf16"), "g8": (16, 2, 128, "bf16"),
    "g20": (20, 1, 128, "bf16"), "g32": (64, 2, 64, "bf16"), "g9f": (9, 1, 128, "f32"), "d80": (6, 2, 80, "bf16"),
    "d33f": (5, 5, 33, "f32"), "d33": (3, 1, 33, "bf16"), "d256f": (2, 1, 256, "f32"), "d256": (8, 2, 256, "bf16"), "d1": (2, 2, 1, "f32"),
    "g16": (16, 1, 128, "bf16"), "g9": (9, 1, 64, "bf16"), "d8": (4, 1, 8, "bf16"), "d72": (8, 2, 72, "bf16"), "d96": (12, 2, 96, "bf16"), "d120": (7, 1, 120, "bf16"), "d56": (4, 4, 56, "bf16"), "g3f": (6, 2, 100, "f32"), "d192": (4, 4, 192, "bf16"), "d136": (10, 1, 136, "bf16"), "d248": (18, 1, 248, "bf16"),
    "g64": (64, 1, 128, "bf16"), "g33": (33, 1, 64, "bf16"), "g31d256": (31, 1, 256, "bf16"), "g24d72": (48, 2, 72, "bf16"),
    "d255": (3, 1, 255, "bf16"), "d130": (4, 2, 130, "bf16"),
}
LENS = {
    "one": [1], "few": [5, 1, 17], "edges": [127, 128, 129, 31, 33], "edges512": [511, 512, 513], "ragged": [1000, 3, 0, 2500, 64],
}


def run(c, q, accumulate=False, ws=None, out=None):
    k = c.moa()
    if ws is None:
        ws = workspace(moa.decode_attn_workspace_bytes(k, c.H))
    if out is None:
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    moa.decode_attn(k, q, out, ws, accumulate=accumulate, dev_status=c.status)
    torch.cuda.synchronize()
    return out


def queries(c, seed, scale=1.5):
    g = torch.Generator().manual_seed(seed + 1000)
    return (scale * torch.randn(len(c.lens), c.H, c.dh, generator=g)).to(TDT[c.dtype]).cuda()


@pytest.mark.parametrize("page", [16, 7, 0])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("heads", list(HEADS))
def test_against_definition(heads, lens, page):
    n = LENS[lens]
    c = Cache(HEADS[heads], n, page or max(n), seed=len(heads) + page)
    q = queries(c, 1)
    want, tol, _, _ = decode_reference(c, q)
    check(run(c, q), want, tol, f"{heads} {lens} page {page}")
    assert c.status.item() == (moa.DEV_EMPTY_KEYS if 0 in n else 0)


@pytest.mark.parametrize("page", [1, 50, 128, 256])
@pytest.mark.parametrize("heads", ["8b", "tiny", "mha64"])
def test_page_sizes(heads, page):
    c = Cache(HEADS[heads], [700, 255, 1], page, seed=page)
    q = queries(c, 2)
    want, tol, _, _ = decode_reference(c, q)
    check(run(c, q), want, tol, f"{heads} page {page}")
    assert c.status.item() == 0


@pytest.mark.parametrize("heads,lens,page", [("8b", [33001], 64), ("g8", [16385, 9], 16), ("tiny", [20000, 1, 4097], 16),
                                             ("g32", [30000, 900, 0], 16), ("g33", [40000, 3, 1025, 129], 64), ("g24d72", [17000, 17000, 5, 0], 50),
                                             ("g64", [33001, 31, 32, 900], 128)])
def test_long(heads, lens, page):
    c = Cache(HEADS[heads], lens, page, seed=3)
    q = queries(c, 3)
    want, tol, _, _ = decode_reference(c, q)
    check(run(c, q), want, tol, f"long {heads}")


@pytest.mark.parametrize("heads", ["8b", "tiny", "d80"])
def test_many_sequences(heads):
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 90, 150).tolist()
    lens[70], lens[149] = 900, 600
    c = Cache(HEADS[heads], lens, 16, seed=5)
    q = queries(c, 5)
    want, tol, _, _ = decode_reference(c, q)
    check(run(c, q), want, tol, f"150 sequences {heads}")


@pytest.mark.parametrize("lens", [[1], [300, 0, 17], [2100, 1, 0, 640], [129]])
@pytest.mark.parametrize("heads", ["8b", "tiny", "g20", "g32", "g9f", "d80", "mha64", "g16", "g9", "d33", "d72", "d256", "d248", "d255", "g64", "g33",
                                   "g31d256", "g24d72"])
def test_accounts(heads, lens):
    c = Cache(HEADS[heads], lens, 16, seed=7, accounts=True)
    q = queries(c, 7)
    before = c.score.cpu().double().numpy()
    want, tol, weight, wtol = decode_reference(c, q)
    check(run(c, q, accumulate=True), want, tol, f"{heads} {lens}")
    # an addition of a weight to an account and one more where there are several row tiles
    check(c.score, before + weight, wtol + 2.0 ** -23 * (np.abs(before) + weight), f"accounts {heads} {lens}")
    for b, n in enumerate(lens):
        assert np.array_equal(c.score.cpu().numpy()[b, :, n:], before[b, :, n:].astype(np.float32))


@pytest.mark.parametrize("heads,lens", [("g64", [33000, 31, 0, 1500]), ("g32", [30000, 900, 3]), ("g33", [33100, 5, 1025, 129]), ("8b", [9000, 1, 3000])])
def test_accounts_of_long_sequences(heads, lens):
    c = Cache(HEADS[heads], lens, 64, seed=23, accounts=True)
    q = queries(c, 23)
    before = c.score.cpu().double().numpy()
    want, tol, weight, wtol = decode_reference(c, q)
    check(run(c, q, accumulate=True), want, tol, f"{heads} {lens}")
    check(c.score, before + weight, wtol + 2.0 ** -23 * (np.abs(before) + weight), "accounts")


def test_accounts_are_left_alone_without_accumulate():
    c = Cache(HEADS["8b"], [600, 20], 16, seed=8, accounts=True)
    before = c.score.clone()
    run(c, queries(c, 8))
    assert torch.equal(c.score, before)


@pytest.mark.parametrize("heads", ["8b", "tiny", "mha64", "d256", "d72"])
def test_rows_that_are_not_16_byte_aligned(heads):
    c = Cache(HEADS[heads], [513, 40], 16, seed=9, offset=1)
    q = queries(c, 9)
    want, tol, _, _ = decode_reference(c, q)
    check(run(c, q), want, tol, f"offset {heads}")


@pytest.mark.parametrize("heads", ["8b", "tiny", "mha64"])
@pytest.mark.parametrize("bad", [-1, 1 << 30, -(1 << 31)])
def test_pages_that_do_not_exist_are_left_out(heads, bad):
    c = Cache(HEADS[heads], [900, 40], 16, seed=10, accounts=True)
    q = queries(c, 10)
    skip = {(0, 3), (0, 55), (1, 0), (1, 1), (1, 2)}
    want, tol, weight, wtol = decode_reference(c, q, skip=skip)
    for b, p in skip:
        c.t_table[b, p] = bad
    before = c.score.cpu().double().numpy()
    check(run(c, q, accumulate=True), want, tol, f"bad pages {heads}")            # sequence 1 has no keys left: zeros
    check(c.score, before + weight, wtol + 2.0 ** -23 * (np.abs(before) + weight), "accounts")
    assert c.status.item() == moa.DEV_BAD_PAGE | moa.DEV_EMPTY_KEYS


@pytest.mark.parametrize("heads", ["8b", "tiny"])
def test_lengths_outside_the_capacity(heads):
    c = Cache(HEADS[heads], [640, 640, 640], 16, seed=11)
    q = queries(c, 11)
    want, tol, _, _ = decode_reference(c, q, lens=[640, 0, 640])
    c.t_len.copy_(torch.tensor([641, -5, 640], dtype=torch.int32))
    check(run(c, q), want, tol, "clamped")
    assert c.status.item() == moa.DEV_BAD_LENGTH | moa.DEV_EMPTY_KEYS


@pytest.mark.parametrize("heads", ["8b", "tiny", "mha64"])
def test_peaked_and_far_scores(heads):
    """Scores of hundreds: the running maximum moves by far more than an exponential can hold."""
    c = Cache(HEADS[heads], [1500, 200], 16, seed=12)
    c.k[:] = c.k * torch.linspace(0.1, 12.0, c.k.shape[0], device="cuda").to(c.k.dtype)[:, None, None, None]
    q = queries(c, 12, scale=8.0)
    want, tol, _, _ = decode_reference(c, q)
    check(run(c, q), want, tol, f"peaked {heads}")


@pytest.mark.parametrize("heads", ["8b", "tiny", "mha64", "d96", "d72", "d256", "d136"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_query_that_is_no_number_stays_with_its_head(heads, bad):
    c = Cache(HEADS[heads], [700, 37, 0], 16, seed=16)
    q = queries(c, 16)
    want, tol, _, _ = decode_reference(c, q)
    heads_hit = torch.zeros(c.H, dtype=torch.bool)
    heads_hit[0] = heads_hit[c.H - 1] = True
    q[:, heads_hit.cuda(), 0] = bad
    out = run(c, q)
    check(out[:, (~heads_hit).cuda()], want[:, (~heads_hit).numpy()], tol[:, (~heads_hit).numpy()], "the other heads")
    assert not torch.isfinite(out[:2, heads_hit.cuda()]).any()
    assert (out[2] == 0).all()


@pytest.mark.parametrize("seed", range(60))
def test_random_calls(seed):
    rng = np.random.default_rng(1000 + seed)
    dtype = "bf16" if seed % 3 else "f32"
    Hkv, G = int(rng.integers(1, 9)), int(rng.choice([1, 2, 3, 4, 5, 8, 16, 17, 32, 40]))
    dh = int(rng.choice([64, 128, 8 * rng.integers(1, 33), rng.integers(1, 257)]))
    top = int(np.exp(rng.uniform(0, np.log(3000 if Hkv * dh > 400 else 9000))))
    lens = rng.integers(0, top + 1, int(rng.integers(1, 8))).tolist()
    lens[0] = top
    c = Cache((Hkv * G, Hkv, dh, dtype), lens, int(rng.choice([1, 16, 64, top, rng.integers(2, 300)])), seed=seed, accounts=bool(rng.integers(0, 2)))
    q = queries(c, seed)
    what = f"{dtype} Hkv {Hkv} G {G} dh {dh} lens {lens} page {c.page}"
    print(what, flush=True)
    want, tol, weight, wtol = decode_reference(c, q)
    if c.score is None:
        check(run(c, q), want, tol, what)
        return
    before = c.score.cpu().double().numpy()
    check(run(c, q, accumulate=True), want, tol, what)
    check(c.score, before + weight, wtol + 2.0 ** -23 * (np.abs(before) + weight), "accounts")


@pytest.mark.parametrize("heads", ["8b", "tiny"])
def test_same_bits_again_and_on_another_stream(heads):
    c = Cache(HEADS[heads], [3000, 2, 777], 16, seed=13)
    q = queries(c, 13)
    first = run(c, q)
    assert torch.equal(run(c, q), first)
    s = torch.cuda.Stream()
    out = torch.zeros_like(first)
    k = c.moa()
    ws = workspace(moa.decode_attn_workspace_bytes(k, c.H))
    ws.fill_(255)                                   # nothing in the workspace has to start at anything
    s.wait_stream(torch.cuda.current_stream())
    moa.decode_attn(k, q, out, ws, stream=s)
    s.synchronize()
    assert torch.equal(out, first)


@pytest.mark.parametrize("heads", ["8b", "tiny"])
def test_sequences_that_share_pages(heads):
    """A common prompt: the first pages of all sequences are the same ones."""
    c = Cache(HEADS[heads], [600, 601, 700, 5], 16, seed=18)
    for b in (1, 2):
        c.table[b, :30] = c.table[0, :30]
    c.t_table.copy_(torch.from_numpy(c.table))
    q = queries(c, 18)
    want, tol, _, _ = decode_reference(c, q)
    check(run(c, q), want, tol, f"shared pages {heads}")


@pytest.mark.parametrize("heads", [(1, 1, 8, "f32"), (2, 1, 16, "bf16")])
def test_thousands_of_sequences(heads):
    rng = np.random.default_rng(19)
    lens = rng.integers(0, 20, 3000).tolist()
    lens[2999], lens[64], lens[1000] = 600, 530, 0
    c = Cache(heads, lens, 8, seed=19, accounts=True)
    q = queries(c, 19)
    before = c.score.cpu().double().numpy()
    want, tol, weight, wtol = decode_reference(c, q)
    check(run(c, q, accumulate=True), want, tol, "3000 sequences")
    check(c.score, before + weight, wtol + 2.0 ** -23 * (np.abs(before) + weight), "accounts")


@pytest.mark.parametrize("heads", ["8b", "tiny", "d256"])
def test_queries_that_are_not_16_byte_aligned(heads):
    c = Cache(HEADS[heads], [900, 64, 0], 16, seed=22, accounts=True)
    q = queries(c, 22)
    flat = torch.empty(q.numel() + 1, dtype=q.dtype, device="cuda")
    flat[1:].copy_(q.view(-1))
    before = c.score.cpu().double().numpy()
    want, tol, weight, wtol = decode_reference(c, q)
    check(run(c, flat[1:].view(q.shape), accumulate=True), want, tol, f"queries {heads}")
    check(c.score, before + weight, wtol + 2.0 ** -23 * (np.abs(before) + weight), "accounts")


@pytest.mark.parametrize("heads", ["8b", "tiny"])
def test_two_calls_at_once(heads):
    """On two streams, over one cache, with a workspace and an output each."""
    c = Cache(HEADS[heads], [9000, 700, 3], 16, seed=20)
    k = c.moa()
    qs = [queries(c, 20), queries(c, 21)]
    want = [run(c, q) for q in qs]
    n = moa.decode_attn_workspace_bytes(k, c.H)
    ws, out = [workspace(n) for _ in qs], [torch.zeros_like(q) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in (0, 1):
            moa.decode_attn(k, qs[i], out[i], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_more_blocks_of_accounts_than_a_launch_is_wide():
    """Room for 2^28 slots, a few in use: blocks of 256 accounts in two rows of the second launch."""
    B, Hkv, dh, ps = 1, 1, 8, 16
    cap = 256 * ((1 << 20) + 5)
    c = Cache((1, Hkv, dh, "f32"), [70], ps, seed=17)
    table = torch.full((B, cap // ps), -1, dtype=torch.int32, device="cuda")
    table[:, :c.mp] = c.t_table
    score = torch.zeros(B, Hkv, cap, device="cuda")
    cache = moa.KVCache(c.k, c.v, table, c.t_len, score=score)
    q = queries(c, 17)
    want, tol, weight, wtol = decode_reference(c, q)
    out = torch.zeros_like(q)
    moa.decode_attn(cache, q, out, workspace(moa.decode_attn_workspace_bytes(cache, 1)), accumulate=True, dev_status=c.status)
    check(out, want, tol, "out")
    check(score[:, :, :70], weight[:, :, :70], wtol[:, :, :70] + 2.0 ** -23 * weight[:, :, :70], "accounts")
    assert float(score[:, :, 70:].abs().max()) == 0.0 and c.status.item() == 0


def test_pool_of_more_than_4_gib():
    Hkv, ps, dh = 8, 64, 128
    n_pages = (5 << 30) // (Hkv * ps * dh * 2) + 1
    k = torch.empty(n_pages, Hkv, ps, dh, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    c = Cache((32, Hkv, dh, "bf16"), [600, 700], ps, seed=14, spare=0)
    small_k, small_v = c.k, c.v
    far = torch.from_numpy(np.random.default_rng(14).permutation(n_pages)[:small_k.shape[0]].astype(np.int64)).cuda()
    far[0], far[1] = n_pages - 1, n_pages - 2
    far = torch.unique(far)
    assert far.numel() == small_k.shape[0]
    k[far], v[far] = small_k, small_v
    q = queries(c, 14)
    want, tol, _, _ = decode_reference(c, q)
    table = c.t_table.long().clamp(max=small_k.shape[0] - 1)
    c.k, c.v, c.t_table = k, v, far[table].to(torch.int32)
    check(run(c, q), want, tol, "far pages")


def test_contiguous_cache_of_the_verification():
    """A root-only tree on a contiguous cache is the token's own row appended and then decoded: moa_tree_verify_attn without
    projections against kv_append + decode_attn on the same cache seen as one page per sequence."""
    B, H, dh, cap = 3, 8, 64, 700
    lens = [650, 1, 0]
    g = torch.Generator().manual_seed(15)
    kc, vc = (torch.randn(B, H, cap, dh, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    x = torch.randn(B, 1, H * dh, generator=g).to(torch.bfloat16).cuda()
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    shape = moa.Shape(1, H * dh, H, H, dh, H * dh, H, H, moa.BF16)
    mask = torch.ones(B, 1, 1, dtype=torch.int64, device="cuda")
    want = torch.zeros_like(x)
    kt, vt = (torch.zeros(B, H, 1, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    moa.tree_verify_attn(shape, x, None, None, None, None, kc, vc, n, cap, mask, want, kt, vt,
                         workspace(moa.workspace_bytes(shape, B, cap, 1, 0)))
    cache = moa.KVCache(kc, vc, torch.arange(B, dtype=torch.int32, device="cuda")[:, None], n)
    moa.kv_append(cache, kt, vt)
    out = torch.zeros(B, H, dh, dtype=torch.bfloat16, device="cuda")
    moa.decode_attn(cache, x.view(B, H, dh), out, workspace(moa.decode_attn_workspace_bytes(cache, H)))
    assert n.tolist() == [651, 2, 1]
    # the verification rounds its weights (2^-8) and its partial results (2^-12); either rounds its result (2^-8) of |o| <= max |v|
    top = float(vc.float().abs().max())
    assert float((out.view(B, -1).float() - want.view(B, -1).float()).abs().max()) <= (3 * 2.0 ** -8 + 2.0 ** -11) * top
