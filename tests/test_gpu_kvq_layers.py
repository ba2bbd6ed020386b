"""The cache held in 8 bits as several layers use it, one table and list of pages and a len of each layer's own, and the attention at the ends of
the numbers that it is said to be precise for."""
import numpy as np
import pytest
import torch

import kvq_util as U
import paper_2410_03804_amd as moa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,page", [((8, 2, 64, "f32"), 16), ((32, 8, 128, "bf16"), 40)], ids=str)
def test_layers_share_a_table(heads, page):
    B, mp, n_layers = 4, -(-300 // page), 3
    H, Hkv, dh, dtype = heads
    n_pages = B * mp // 2
    layers = [U.QCache(heads, [0] * B, page, seed=i, spare=n_pages, mp=mp) for i in range(n_layers)]
    table = layers[0].t_table
    table.fill_(-1)
    for c in layers:
        c.t_table = table
    caches = [c.moa() for c in layers]
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    free, n_free = torch.arange(n_pages, dtype=torch.int32, device="cuda"), torch.tensor([n_pages], dtype=torch.int32, device="cuda")
    off, got, status = i32(B + 1), i32(B), i32(1)
    ws = U.workspace(moa.kvq_decode_attn_workspace_bytes(caches[0], H))
    rng = np.random.default_rng(1)
    for step, n in enumerate(([30, 1, 0, 90], [1, 1, 1, 1], [5, 0, 160, 7], [1, 1, 1, 1], [280, 250, 1, 1])):
        T = sum(n)
        pos, slot = i32(T), i32(T)
        which = step % n_layers                                # any layer's lengths
        moa.kv_reserve(table, layers[which].t_len, torch.tensor(n, dtype=torch.int32, device="cuda"), page, free, n_free, off, got, pos=pos, slot=slot, dev_status=status)
        for c, cache in zip(layers, caches):
            x = torch.from_numpy(rng.standard_normal((T, 2 * Hkv, dh)).astype(np.float32)).to(U.TDT[dtype]).cuda()
            moa.kvq_append_rows(cache, x[:, :Hkv], x[:, Hkv:], off, n_new=got, dev_status=status)
            q = torch.from_numpy(rng.standard_normal((B, H, dh)).astype(np.float32)).to(U.TDT[dtype]).cuda()
            out = torch.empty_like(q)
            moa.kvq_decode_attn(cache, q, out, ws, dev_status=status)
            torch.cuda.synchronize()
            first, g, d = off.tolist(), got.tolist(), U.host(x)
            c.table = np.where(table.cpu().numpy() >= 0, table.cpu().numpy(), 1 << 29).astype(np.int32)
            rows = lambda b, a: d[first[b]:first[b] + g[b], a:a + Hkv].transpose(1, 0, 2)
            c.append([(rows(b, 0), rows(b, Hkv)) for b in range(B)])
            want, tol = U.decode_reference(c, q)
            U.check(out, want, tol, f"step {step}")
            assert c.t_len.tolist() == c.lens
        assert all(c.lens == layers[0].lens for c in layers)
        for b in range(B):
            assert pos.tolist()[first[b]:first[b] + g[b]] == list(range(layers[0].lens[b] - g[b], layers[0].lens[b]))
        moa.kv_release(table, layers[-1].t_len, page, free, n_free, dev_status=status)
        assert n_free.item() == n_pages - sum(-(-n // page) for n in layers[0].lens)
    assert 0 in got.tolist() and status.item() & moa.DEV_CACHE_FULL          # the last step asked for more than there is
    assert status.item() & ~moa.DEV_EMPTY_KEYS == moa.DEV_CACHE_FULL


@pytest.mark.parametrize("n", [50, 1100])
@pytest.mark.parametrize("heads", [(4, 2, 64, "f32"), (32, 8, 128, "bf16"), (6, 2, 80, "f32"), (3, 1, 33, "bf16"), (3, 1, 33, "f32")], ids=str)
def test_numbers_at_the_ends(heads, n):
    """Queries of 1e33 over keys as small as that makes them, and values of about 1e-30 and of up to 1e38 / len.

    The bounds are those of any call (kvq_util.decode_reference): a sum of dh products q c with c <= 448 is below 256 * 448 * 1e33 = 1.2e38, and
    a weight times its scale, 2^-100, has a rounding of 2^-24 of itself down to weights of 2^-10, whose last part is 2^-126; smaller ones add up
    to n 2^-10 2^-16 at most."""
    for values in (2.0 ** -100, 2.0 ** 106):                  # 448 2^106 1100 = 2^125
        c = U.QCache(heads, [n, n // 3], 16, seed=n)
        held = np.isfinite(c.scales[0])
        e = c.rng.integers(-2, 1, c.scales[0].shape)
        c.scales[0] = np.where(held, np.ldexp(2.0 ** -117, e), np.nan).astype(np.float32)
        c.scales[1] = np.where(held, np.ldexp(values, e), np.nan).astype(np.float32)
        c.upload()
        q = torch.from_numpy(np.clip(c.rng.standard_normal((2, c.H, c.dh)), -3, 3) * 3.3e32).to(U.TDT[c.dtype]).cuda()
        out = torch.empty_like(q)
        cache = c.moa()
        moa.kvq_decode_attn(cache, q, out, U.workspace(moa.kvq_decode_attn_workspace_bytes(cache, c.H)), dev_status=c.status)
        want, tol = U.decode_reference(c, q)
        U.check(out, want, tol, f"{heads} {n} values by {values:.0e}")
        assert c.status.item() == 0
