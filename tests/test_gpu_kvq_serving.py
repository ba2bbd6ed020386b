"""The calls as a server makes them, one behind the other: pages for a ragged batch, norm and rotation of what its projection gave, rows
into the cache held in 8 bits, attention of the next token, drafts verified against the cache read back, pages given back.  Every step is held
to the same computation in 64 bits, which keeps a cache of its own."""
import numpy as np
import pytest
import torch

import kvq_util as U
import paper_2410_03804_amd as moa
from test_gpu_qk_norm_rope import reference as rope_reference

pytestmark = pytest.mark.gpu


class Server:
    def __init__(self, heads, B, n_pages, page, mp, seed):
        self.H, self.Hkv, self.dh, self.dtype = heads
        self.dt, self.B, self.page, self.mp = U.TDT[self.dtype], B, page, mp
        self.rng = np.random.default_rng(seed)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        # the host's cache: its pages are the device's, read back after each reservation
        self.ref = U.QCache(heads, [0] * B, page, seed=seed, spare=n_pages, mp=mp)
        self.ref.table[:] = -1
        self.ref.upload()
        self.cache = self.ref.moa()
        self.table, self.len = self.ref.t_table, self.ref.t_len
        self.free, self.n_free = torch.arange(n_pages, dtype=torch.int32, device="cuda"), torch.tensor([n_pages], dtype=torch.int32, device="cuda")
        self.off, self.got, self.status = i32(B + 1), i32(B), i32(1)
        self.n_pages = n_pages
        g = lambda: torch.from_numpy((1 + 0.2 * self.rng.standard_normal(self.dh)).astype(np.float32)).to(self.dt).cuda()
        self.gq, self.gk = g(), g()
        self.ws = U.workspace(moa.kvq_decode_attn_workspace_bytes(self.cache, self.H))

    def step(self, n, what, keep=None):
        """n[b] new tokens each; keep: of these, the ones that stay (a draft's)."""
        T = int(sum(n)) + 2
        new = torch.tensor(n, dtype=torch.int32, device="cuda")
        pos, slot = (torch.full((T,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
        x = torch.from_numpy(self.rng.standard_normal((T, self.H + 2 * self.Hkv, self.dh)).astype(np.float32)).to(self.dt).cuda()
        q, k, v = x[:, :self.H], x[:, self.H:self.H + self.Hkv], x[:, self.H + self.Hkv:]
        moa.kv_reserve(self.table, self.len, new, self.page, self.free, self.n_free, self.off, self.got, pos=pos, slot=slot, dev_status=self.status)
        q_rot, k_rot = torch.empty(q.shape, dtype=self.dt, device="cuda"), torch.empty(k.shape, dtype=self.dt, device="cuda")
        moa.qk_norm_rope(q, k, q_rot, k_rot, pos, rope_theta=10000.0, gq=self.gq, gk=self.gk, rms_eps=1e-5)
        moa.kvq_append_rows(self.cache, k_rot, v, self.off, n_new=self.got, dev_status=self.status)
        # the last token of each sequence that has new ones attends
        last = (self.off[1:].long() - 1).clamp(min=0)
        qd = q_rot[last].contiguous()
        out = torch.empty(self.B, self.H, self.dh, dtype=self.dt, device="cuda")
        moa.kvq_decode_attn(self.cache, qd, out, self.ws, dev_status=self.status)
        torch.cuda.synchronize()
        # on the host: positions are where the sequences are, rows as the formula has them
        got = self.got.tolist()
        off = np.concatenate([[0], np.cumsum(n)])
        want_pos = np.concatenate([np.arange(l, l + m) for l, m in zip(self.ref.lens, n)] + [np.zeros(2)]).astype(np.int32)
        assert pos.tolist() == want_pos.tolist() and self.off.tolist() == off.tolist()
        for rows, g, done in ((q, self.gq, q_rot), (k, self.gk, k_rot)):
            want, tol = rope_reference(rows.cpu().double().numpy(), g.cpu().double().numpy(), float(np.float32(1e-5)), want_pos, 10000.0, self.dh)
            step = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24
            assert np.all(np.abs(U.host(done) - want) <= 1.01 * tol + step * (np.abs(want) + tol) + 2.0 ** -149), what
        table = self.table.cpu().numpy()
        held = table[table >= 0]
        assert len(set(held.tolist())) == len(held) == self.n_pages - self.n_free.item(), "a page is somebody's alone"
        s = slot.tolist()
        for b in range(self.B):
            for i in range(got[b]):
                p = self.ref.lens[b] + i
                assert s[off[b] + i] == table[b, p // self.page] * self.page + p % self.page
        self.ref.table = np.where(table >= 0, table, 1 << 29).astype(np.int32)
        kd, vd = U.host(k_rot), U.host(v)
        self.ref.append([(kd[off[b]:off[b] + got[b]].transpose(1, 0, 2), vd[off[b]:off[b] + got[b]].transpose(1, 0, 2)) for b in range(self.B)])
        self.same(what)
        want, tol = U.decode_reference(self.ref, qd)
        U.check(out, want, tol, what)
        if keep is not None:
            # a draft of which less stays: the cache is cut back, its pages go back
            for b, (m, stay) in enumerate(zip(got, keep)):
                self.ref.lens[b] -= m - min(m, stay)
            self.len.copy_(torch.tensor(self.ref.lens, dtype=torch.int32))
            self.release(what)
        return got

    def same(self, what):
        """Codes and scales of the slots in use, and the lengths.  (Pages that went back keep what they held.)"""
        codes, scales = self.ref.downloaded()
        for w in range(2):
            for b, n in enumerate(self.ref.lens):
                s = np.arange(n)
                p, r = self.ref.table[b, s // self.page], s % self.page
                assert np.array_equal(codes[w][p, :, r], self.ref.codes[w][p, :, r]), what
                assert np.array_equal(scales[w][p, :, r // 16], self.ref.scales[w][p, :, r // 16]), what
        assert self.len.tolist() == self.ref.lens, what

    def release(self, what):
        moa.kv_release(self.table, self.len, self.page, self.free, self.n_free, dev_status=self.status)
        table = self.table.cpu().numpy()
        for b, n in enumerate(self.ref.lens):
            assert np.all(table[b, -(-n // self.page):] == -1), what
            assert np.all(table[b, :-(-n // self.page)] >= 0), what


@pytest.mark.parametrize("heads,page", [((8, 2, 64, "f32"), 16), ((32, 8, 128, "bf16"), 16), ((16, 2, 128, "bf16"), 40), ((6, 2, 80, "bf16"), 7)], ids=str)
def test_a_server_s_steps(heads, page):
    B, mp = 5, -(-700 // page)
    s = Server(heads, B, 2 * mp, page, mp, seed=page)
    s.step([37, 1, 200, 0, 90], "prompts")
    for i in range(3):
        s.step([1, 1, 1, 0, 1], f"token {i}")
    s.step([8, 8, 8, 0, 8], "draft", keep=[3, 8, 1, 0, 0])
    s.step([1, 1, 1, 350, 1], "a prompt beside tokens")
    assert s.status.item() & ~moa.DEV_EMPTY_KEYS == 0
    # sequence 2 is done; its pages serve the next
    s.ref.lens[2] = 0
    s.len[2] = 0
    s.release("done")
    s.step([1, 30, 250, 1, 1], "another in its place")
    # more than there is: who does not fit goes without, the others go on
    got = s.step([1, 1, 300, 300, 200], "no room")
    assert 0 in got and got[0] == got[1] == 1 and s.status.item() & moa.DEV_CACHE_FULL
    s.step([1, 1, 0, 1, 0], "on")


def test_a_tree_behind_a_cache_held_in_8_bits():
    """moa_tree_verify_attn over the caches that moa_kvq_read gives back, and its accepted nodes appended to the cache held in 8 bits."""
    heads = (8, 2, 64, "f32")
    H, Hkv, dh, _ = heads
    d, B, M, P = H * dh, 2, 9, 128
    c = U.QCache(heads, [100, 37], 16, seed=3, room=10)
    cache = c.moa()
    kc, vc = (torch.zeros(B, Hkv, P, dh, device="cuda") for _ in range(2))
    moa.kvq_read(cache, kc, vc, dev_status=c.status)
    parent = torch.tensor([[-1, 0, 0, 1, 1, 2, 3, 3, 5]] * B, dtype=torch.int32, device="cuda")
    mask, depth = torch.zeros(B, M, 1, dtype=torch.int64, device="cuda"), torch.zeros(B, M, dtype=torch.int32, device="cuda")
    moa.tree_build(parent, mask, depth, c.status)
    shape = moa.Shape(4, d, H, Hkv, dh, 2 * d, H, Hkv, moa.F32)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(B, M, d, device="cuda", generator=g)
    w = [torch.randn(n, d, device="cuda", generator=g) * d ** -0.5 for n in (H * dh, Hkv * dh, Hkv * dh, d)]
    out, kt, vt = torch.empty(B, M, d, device="cuda"), torch.empty(B, Hkv, M, dh, device="cuda"), torch.empty(B, Hkv, M, dh, device="cuda")
    ws = U.workspace(moa.workspace_bytes(shape, B, P, M, 0))
    moa.tree_verify_attn(shape, x, *w, kc, vc, c.t_len, P, mask, out, kt, vt, ws, c.status)
    # node 0 attends the cache and itself: the attention of one token of a cache that has it, but for that one row's encoding
    torch.cuda.synchronize()
    for b in range(B):
        n = c.lens[b]
        for h in range(Hkv):
            q = (x[b, 0].double() @ w[0].double().t()).view(H, dh)[h * (H // Hkv):(h + 1) * (H // Hkv)].cpu().numpy()
            keys = np.concatenate([c.rows(0, b, h, n), U.host(kt)[b, h, :1]])
            s = q @ keys.T / np.sqrt(dh)
            p = np.exp(s - s.max(1, keepdims=True))
            head = (p / p.sum(1, keepdims=True)) @ np.concatenate([c.rows(1, b, h, n), U.host(vt)[b, h, :1]])
            if h == 0:
                whole = np.zeros((H, dh))
            whole[h * (H // Hkv):(h + 1) * (H // Hkv)] = head
        want = whole.reshape(-1) @ U.host(w[3]).T
        # single precision from end to end: the bound of the repository's fp32 attention calls
        assert np.max(np.abs(U.host(out)[b, 0] - want)) <= 1e-4
    tok, tgt = torch.tensor([[0, 5, 6, 7, 8, 9, 1, 2, 3]] * B, dtype=torch.int32, device="cuda"), torch.tensor([[5, 7, 0, 2, 0, 0, 0, 4, 0], [6, 0, 9, 0, 0, 11, 0, 0, 0]], dtype=torch.int32, device="cuda")
    path, n_path, bonus = torch.zeros(B, M, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    moa.tree_accept(parent, tok, tgt, path, n_path, bonus)
    moa.kvq_append(cache, kt, vt, path=path, n_new=n_path, dev_status=c.status)
    torch.cuda.synchronize()
    assert n_path.tolist() == [4, 3] and path[0, :4].tolist() == [0, 1, 3, 7] and path[1, :3].tolist() == [0, 2, 5]
    p = path.cpu().numpy()
    c.append([tuple(U.host(t)[b][:, p[b, :n]] for t in (kt, vt)) for b, n in enumerate(n_path.tolist())])
    c.check_state("accepted")
    assert c.status.item() == 0


def test_a_captured_decoding_step():
    """One token of every sequence as a graph: pages, norm and rotation, append, attention, lengths moving on within it."""
    heads = (16, 4, 128, "bf16")
    s = Server(heads, 4, 80, 16, 20, seed=9)
    s.step([15, 30, 1, 64], "prompts")
    B, H, Hkv, dh = 4, s.H, s.Hkv, s.dh
    x = torch.zeros(B, H + 2 * Hkv, dh, dtype=s.dt, device="cuda")
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    q_rot, k_rot, out = (torch.zeros(B, h, dh, dtype=s.dt, device="cuda") for h in (H, Hkv, H))

    def step():
        moa.kv_reserve(s.table, s.len, one, 16, s.free, s.n_free, s.off, s.got, pos=pos, dev_status=s.status)
        moa.qk_norm_rope(x[:, :H], x[:, H:H + Hkv], q_rot, k_rot, pos, rope_theta=10000.0, gq=s.gq, gk=s.gk)
        moa.kvq_append_rows(s.cache, k_rot, x[:, H + Hkv:], s.off, n_new=s.got, dev_status=s.status)
        moa.kvq_decode_attn(s.cache, q_rot, out, s.ws, dev_status=s.status)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(40):
        x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay() if i % 4 else step()
        torch.cuda.synchronize()
        assert pos.tolist() == s.ref.lens
        s.ref.table = np.where(s.table.cpu().numpy() >= 0, s.table.cpu().numpy(), 1 << 29).astype(np.int32)
        kd, vd = U.host(k_rot), U.host(x[:, H + Hkv:])
        s.ref.append([(kd[b][:, None], vd[b][:, None]) for b in range(B)])
        s.same(f"replay {i}")
        want, tol = U.decode_reference(s.ref, q_rot)
        U.check(out, want, tol, f"replay {i}")
    assert s.status.item() == 0
