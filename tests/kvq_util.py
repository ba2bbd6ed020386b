"""Caches held in 8 bits for the tests of the moa_kvq_* calls, and their definitions in 64 bits on the CPU (numpy, no torch arithmetic)."""
from __future__ import annotations

import numpy as np
import torch

import paper_2410_03804_amd as moa

TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 16
NAN = 0x7F


def code_values():
    """What the 256 codes stand for: sign, exponent of bias 7, mantissa of three bits; exponent 0 has no leading one; 0x7f is NaN."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, np.ldexp(1.0 + m / 8.0, e - 7), np.ldexp(m / 8.0, -6))
    v = np.where(c & 0x80, -v, v)
    return np.where((c & 0x7F) == NAN, np.nan, v)


VALUES = code_values()
_POSITIVE = VALUES[:NAN]                              # 0 .. 448, ascending


def encode(x):
    """Codes of the numbers nearest to x (|x| <= 448 or not finite), the even code of two; NaN for what is not finite."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, NAN - 1)
    lo = hi - 1
    to_hi, to_lo = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where((to_hi < to_lo) | ((to_hi == to_lo) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isfinite(x), code, NAN)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def smallest_scale(x):
    """The smallest power of two within 2^-120 .. 2^120 by which the finite numbers of x are at most 448."""
    x = np.abs(np.asarray(x, np.float64))
    most = np.max(x[np.isfinite(x)], initial=0.0)
    e = -120
    while e < 120 and most > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class QCache:
    """A pool with NaN in every row that no sequence holds and NaN scales in blocks that hold none, pages handed out in random order, table
    entries behind the last page in use beyond any pool.  `room`: slots kept free (and backed by pages) behind each sequence; `offset`:
    bytes in front of the codes, so that their rows are not aligned."""

    def __init__(self, heads, lens, page, seed, room=0, spare=2, offset=0, dev="cuda", mp=None):
        self.H, self.Hkv, self.dh, self.dtype = heads
        self.lens, self.page, self.offset, self.dev = list(lens), page, offset, dev
        rng = self.rng = np.random.default_rng(seed)
        B = len(self.lens)
        self.mp = mp or max(1, -(-(max(self.lens) + room) // page))
        self.cap, self.bps = self.mp * page, -(-page // BLOCK)
        want = [-(-(n + room) // page) for n in self.lens]
        n_pages = sum(want) + spare
        order = rng.permutation(n_pages)
        table = np.full((B, self.mp), 1 << 29, np.int32)
        at = 0
        for b in range(B):
            table[b, :want[b]] = order[at:at + want[b]]
            at += want[b]
        self.table = table
        shape = (n_pages, self.Hkv, page, self.dh)
        held = np.zeros((n_pages, page), bool)
        blocks = np.zeros((n_pages, self.bps), bool)
        for b in range(B):
            s = np.arange(self.lens[b])
            held[table[b, s // page], s % page] = True
            blocks[table[b, s // page], s % page // BLOCK] = True
        self.codes, self.scales = [], []
        for _ in range(2):
            c = encode(np.clip(rng.standard_normal(shape) * 100.0, -448, 448))
            c = np.where(held[:, None, :, None], c, np.uint8(NAN))
            s = np.ldexp(1.0, rng.integers(-9, -5, (n_pages, self.Hkv, self.bps)))
            self.codes.append(c)
            self.scales.append(np.where(blocks[:, None, :], s, np.nan).astype(np.float32))
        self.upload()
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)

    def upload(self):
        pools = []
        for c in self.codes:
            flat = torch.zeros(c.size + self.offset, dtype=torch.uint8, device=self.dev)
            flat[self.offset:].copy_(torch.from_numpy(c.reshape(-1)))
            pools.append(flat[self.offset:].view(torch.float8_e4m3fn).view(c.shape))
        self.k, self.v = pools
        self.ks, self.vs = (torch.from_numpy(s.copy()).to(self.dev) for s in self.scales)
        self.t_table = torch.from_numpy(self.table).to(self.dev)
        self.t_len = torch.tensor(self.lens, dtype=torch.int32, device=self.dev)

    def moa(self):
        return moa.QuantKVCache(self.k, self.v, self.ks, self.vs, self.t_table, self.t_len, TDT[self.dtype])

    def downloaded(self):
        """(codes, scales) as the device holds them."""
        codes = [p.view(torch.uint8).cpu().numpy() for p in (self.k, self.v)]
        return codes, [s.cpu().numpy() for s in (self.ks, self.vs)]

    def rows(self, w, b, h, n):
        """[n, dh] in 64 bits: what the first n slots stand for, of keys (w = 0) or values."""
        s = np.arange(n)
        page, r = self.table[b, s // self.page], s % self.page
        return VALUES[self.codes[w][page, h, r]] * self.scales[w][page, h, r // BLOCK].astype(np.float64)[:, None]

    def append(self, rows):
        """rows[b] = (k, v) [Hkv, n, dh] in 64 bits: the same on the host, block by block."""
        for b, both in enumerate(rows):
            n = both[0].shape[1]
            for w in range(2):
                s, end = self.lens[b], self.lens[b] + n
                while s < end:
                    page, r = int(self.table[b, s // self.page]), s % self.page
                    r0 = r // BLOCK * BLOCK
                    stop = min(min(r0 + BLOCK, self.page) - r, end - s)
                    for h in range(self.Hkv):
                        x = both[w][h, s - self.lens[b]:s - self.lens[b] + stop]
                        scale = smallest_scale(x)
                        if r > r0:
                            old = float(self.scales[w][page, h, r // BLOCK])
                            if scale > old:
                                held = VALUES[self.codes[w][page, h, r0:r]] * (old / scale)
                                self.codes[w][page, h, r0:r] = encode(held)
                            else:
                                scale = old
                        self.scales[w][page, h, r // BLOCK] = scale
                        self.codes[w][page, h, r:r + stop] = encode(x / scale)
                    s += stop
            self.lens[b] += n

    def check_state(self, what):
        """The device's cache is this one, to the last bit, also where nothing was to be written.  (A NaN's sign is nobody's.)"""
        codes, scales = self.downloaded()
        for w, name in enumerate("kv"):
            want = np.where((self.codes[w] & 0x7F) == NAN, NAN, self.codes[w])
            got = np.where((codes[w] & 0x7F) == NAN, NAN, codes[w])
            assert np.array_equal(scales[w], self.scales[w], equal_nan=True), (what, name, "scales")
            assert np.array_equal(got, want), (what, name, "codes", np.argwhere(got != want)[:4])
        assert self.t_len.tolist() == self.lens, (what, "len")


def host(t):
    return t.detach().cpu().double().numpy()


def workspace(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


def decode_reference(c, q, skip=()):
    """out and its bounds.

    Bounds (u = 2^-24, half a step of the result's type 2^-8 or u): a score is a sum of dh products in single precision, then scaled twice:
    off by at most (dh + 8) u S, S = the largest sum of |q_d k_d| / sqrt(dh) of the row; its weight is then off by that, and by a few u of the
    exponential, relative, and so is their sum; a sum over n keys adds n u; a weight times its scale, u, and split into two bf16 parts where the
    result is bf16, 2^-16.  Together at most eps = 2 (dh + 8) u S + (n + 64) u + 2^-15 [bf16] of sum p |v|; then the result is rounded."""
    u = 2.0 ** -24
    G = c.H // c.Hkv
    qd = host(q)
    out, tol = np.zeros_like(qd), np.zeros_like(qd)
    for b, n in enumerate(c.lens):
        keep = np.array([s for s in range(n) if (b, s // c.page) not in skip], dtype=np.int64)
        if not len(keep):
            continue
        for h in range(c.Hkv):
            page, r = c.table[b, keep // c.page], keep % c.page
            k, v = (VALUES[c.codes[w][page, h, r]] * c.scales[w][page, h, r // BLOCK].astype(np.float64)[:, None] for w in range(2))
            qh = qd[b, h * G:(h + 1) * G] / np.sqrt(c.dh)
            s = qh @ k.T
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            S = (np.abs(qh) @ np.abs(k).T).max(1, keepdims=True)
            eps = 2 * (c.dh + 8) * u * S + (n + 64) * u + (2.0 ** -15 if c.dtype == "bf16" else 0.0)
            out[b, h * G:(h + 1) * G] = p @ v
            tol[b, h * G:(h + 1) * G] = (2.0 ** -8 if c.dtype == "bf16" else u) * np.abs(p @ v) + eps * (p @ np.abs(v))
    return out, tol


def check(got, want, tol, what):
    got = host(got)
    assert np.all(np.isfinite(got)), f"{what}: non-finite"
    ratio = float(np.max(np.abs(got - want) / np.maximum(tol, 1e-300))) if got.size else 0.0
    print(f"[kvq] {what}: largest error / bound {ratio:.3f}", flush=True)
    assert np.all(np.abs(got - want) <= tol), (what, ratio)
