"""moa_qk_norm_rope against its formula in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2410_03804_amd as moa

pytestmark = pytest.mark.gpu

TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
U24 = 2.0 ** -24


def reference(x, g, eps, pos, theta, rot):
    """The result and its bounds, x [T, heads, dh] in 64 bits.

    Bounds (u = 2^-24): the sum of dh squares is off by at most (dh + 1) u, its root by half of that, and 1 / sqrt, the products with it and with g
    by 5 u; an element of y by cy = (dh / 2 + 8) u of itself, and eps is single precision.  Cosine and sine are off by u and by the angle's own
    error: pos times a frequency that is good to 2^-48 or better.  A rotated element is two products and a sum, 3 u of |a| + |b|."""
    T, _, dh = x.shape
    cy = 0.0
    y = x
    if g is not None:
        y = x / np.sqrt(np.mean(x * x, axis=2, keepdims=True) + eps) * g
        cy = (dh / 2 + 8) * U24
    out, tol = y.copy(), cy * np.abs(y)
    half = rot // 2
    if half:
        ang = pos.astype(np.longdouble)[:, None] * np.longdouble(theta) ** (-2 * np.arange(half, dtype=np.longdouble) / rot)
        c, s = np.cos(ang).astype(np.float64)[:, None], np.sin(ang).astype(np.float64)[:, None]
        a, b = y[..., :half], y[..., half:rot]
        out[..., :half], out[..., half:rot] = a * c - b * s, b * c + a * s
        t = (np.abs(a) + np.abs(b)) * (cy + 4 * U24 + np.abs(pos.astype(np.float64))[:, None, None] * 2.0 ** -48)
        tol[..., :half] = tol[..., half:rot] = t
    return out, tol


def check(got, want, tol, dtype, what):
    got = got.detach().cpu().double().numpy()
    tol = tol * 1.01 + (2.0 ** -8 if dtype == "bf16" else U24) * (np.abs(want) + tol) + 2.0 ** -149
    ratio = float(np.max(np.abs(got - want) / tol)) if got.size else 0.0
    print(f"[rope] {what}: largest error / bound {ratio:.3f}", flush=True)
    assert np.all(np.abs(got - want) <= tol), (what, ratio)


class Case:
    def __init__(self, H, Hkv, dh, dtype, T, seed, norm=True, far=40000, theta=500000.0, packed=True, offset=0, pad=0):
        rng = np.random.default_rng(seed)
        self.H, self.Hkv, self.dh, self.dtype, self.theta = H, Hkv, dh, dtype, float(np.float32(theta))
        dt = TDT[dtype]
        width = (H + 2 * Hkv) * dh + pad
        flat = torch.from_numpy((rng.standard_normal(T * width + offset) * 2).astype(np.float32)).to(dt).cuda()
        qkv = flat[offset:].view(T, width)[:, :(H + 2 * Hkv) * dh].unflatten(1, (H + 2 * Hkv, dh))
        self.q, self.k = qkv[:, :H], qkv[:, H:H + Hkv]
        if not packed:
            self.q, self.k = self.q.contiguous(), self.k.contiguous()
        g = lambda: torch.from_numpy((1 + 0.3 * rng.standard_normal(dh)).astype(np.float32)).to(dt).cuda() if norm else None
        self.gq, self.gk = g(), g()
        self.pos_h = rng.integers(0, far, T).astype(np.int32)
        self.pos = torch.from_numpy(self.pos_h).cuda()

    def want(self, x, g, rot, eps=1e-6):
        gd = None if g is None else g.cpu().double().numpy()
        return reference(x.cpu().double().numpy(), gd, float(np.float32(eps)), self.pos_h, self.theta, rot)

    def run(self, rot=None, what="", inplace=False):
        rot_n = self.dh if rot is None else rot
        wq, wk = self.want(self.q, self.gq, rot_n), self.want(self.k, self.gk, rot_n)
        qo, ko = (self.q, self.k) if inplace else (torch.full(x.shape, 99.0, dtype=x.dtype, device="cuda") for x in (self.q, self.k))
        moa.qk_norm_rope(self.q, self.k, qo, ko, self.pos, rope_theta=self.theta, rot_dim=rot, gq=self.gq, gk=self.gk, rms_eps=1e-6)
        torch.cuda.synchronize()
        check(qo, *wq, self.dtype, f"q {what}")
        check(ko, *wk, self.dtype, f"k {what}")


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("T", [1, 2, 3, 17, 260])
@pytest.mark.parametrize("heads", [(4, 2, 64, "f32"), (32, 8, 128, "bf16"), (32, 4, 128, "bf16"), (6, 2, 80, "bf16"), (6, 2, 80, "f32"), (3, 1, 256, "bf16"),
                                   (2, 1, 256, "f32"), (5, 1, 34, "bf16"), (7, 3, 16, "bf16"), (1, 1, 2, "f32"), (5, 2, 96, "f32"), (64, 8, 128, "f32"),
                                   (3, 2, 72, "bf16"), (3, 2, 248, "bf16"), (3, 2, 20, "f32"), (3, 2, 252, "f32"), (3, 2, 8, "bf16")], ids=str)
def test_sizes(heads, T, norm):
    Case(*heads, T, seed=T, norm=norm).run(what=f"{heads} {T}")


@pytest.mark.parametrize("rot", [0, 2, 16, 30, 32, 64, 96, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_part_of_the_dims_is_rotated(dtype, rot):
    Case(8, 2, 128, dtype, 50, seed=rot).run(rot=rot, what=f"{dtype} {rot}")
    Case(8, 2, 128, dtype, 50, seed=rot, norm=False).run(rot=rot, what=f"{dtype} {rot} no norm")


@pytest.mark.parametrize("heads,rot", [((6, 2, 80, "bf16"), 40), ((6, 2, 80, "bf16"), 8), ((6, 2, 80, "f32"), 20), ((6, 2, 80, "f32"), 36), ((3, 1, 256, "bf16"), 72), ((3, 1, 256, "f32"), 4),
                                       ((3, 1, 64, "bf16"), 0), ((9, 2, 12, "f32"), 4)], ids=str)
@pytest.mark.parametrize("T", [5, 2300])
def test_parts_in_pieces_of_every_width(heads, rot, T):
    Case(*heads, T, seed=rot).run(rot=rot, what=f"{heads} {rot}")


@pytest.mark.parametrize("dh", [1, 3, 33, 129, 255])
def test_odd_heads(dh):
    for dtype in ("f32", "bf16"):
        c = Case(3, 2, dh, dtype, 20, seed=dh)
        c.run(rot=0, what=f"{dh} norm alone")
        c.run(rot=dh // 2 * 2, what=f"{dh}")


@pytest.mark.parametrize("heads", [(8, 2, 128, "bf16"), (4, 2, 64, "f32"), (5, 1, 34, "bf16")], ids=str)
def test_in_place_and_contiguous(heads):
    Case(*heads, 70, seed=1).run(inplace=True, what="in place")
    Case(*heads, 70, seed=1, packed=False).run(what="contiguous")
    Case(*heads, 70, seed=1, packed=False).run(inplace=True, what="contiguous in place")


@pytest.mark.parametrize("offset,pad", [(1, 0), (8, 0), (0, 1), (0, 8), (3, 5)])
def test_rows_that_are_not_aligned(offset, pad):
    Case(8, 2, 128, "bf16", 30, seed=2, offset=offset, pad=pad).run(what=f"{offset} {pad}")
    Case(4, 2, 64, "f32", 30, seed=2, offset=offset, pad=pad).run(what=f"{offset} {pad}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_positions(dtype):
    c = Case(8, 2, 128, dtype, 64, seed=3, norm=False, theta=10000.0)
    c.pos_h[:8] = (0, 1, 2 ** 31 - 1, -1, -2 ** 31, 10 ** 6, 131071, 2 ** 24 + 1)
    c.pos.copy_(torch.from_numpy(c.pos_h))
    c.run(what=f"{dtype} far")


def test_queries_or_keys_alone():
    c = Case(8, 2, 128, "bf16", 30, seed=4)
    qo = torch.zeros(c.q.shape, dtype=torch.bfloat16, device="cuda")
    ko = torch.zeros(c.k.shape, dtype=torch.bfloat16, device="cuda")
    moa.qk_norm_rope(c.q, None, qo, None, c.pos, rope_theta=c.theta, gq=c.gq)
    moa.qk_norm_rope(None, c.k, None, ko, c.pos, rope_theta=c.theta, gk=None)
    check(qo, *c.want(c.q, c.gq, 128), "bf16", "q alone")
    check(ko, *c.want(c.k, None, 128), "bf16", "k alone, no norm")
    moa.qk_norm_rope(c.q, c.k, qo, ko, None, rot_dim=0, gk=c.gk)
    assert torch.equal(qo, c.q)                                                # neither norm nor rotation
    check(ko, *c.want(c.k, c.gk, 0), "bf16", "k's norm")


def test_rows_of_zeros_and_what_is_not_finite_stays_in_its_head():
    c = Case(4, 2, 128, "bf16", 8, seed=5)
    c.q[0, 1] = 0.0
    c.q[2, 0, 5] = float("inf")
    c.k[3, 1, 7] = float("nan")
    qo, ko = (torch.zeros(x.shape, dtype=x.dtype, device="cuda") for x in (c.q, c.k))
    moa.qk_norm_rope(c.q, c.k, qo, ko, c.pos, rope_theta=c.theta, gq=c.gq, gk=c.gk)
    assert torch.all(qo[0, 1] == 0) and torch.isnan(ko[3, 1]).all() and torch.isnan(qo[2, 0, 5])
    bad_q, bad_k = torch.zeros(8, 4, dtype=torch.bool), torch.zeros(8, 2, dtype=torch.bool)
    bad_q[2, 0] = bad_k[3, 1] = True
    assert torch.isfinite(qo.cpu()[~bad_q]).all() and torch.isfinite(ko.cpu()[~bad_k]).all()


def test_no_rows_and_captured_replays():
    c = Case(8, 2, 128, "bf16", 40, seed=6)
    moa.qk_norm_rope(c.q[:0], c.k[:0], c.q[:0], c.k[:0], c.pos[:0])
    qo, ko = (torch.zeros(x.shape, dtype=x.dtype, device="cuda") for x in (c.q, c.k))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moa.qk_norm_rope(c.q, c.k, qo, ko, c.pos, rope_theta=c.theta, gq=c.gq, gk=c.gk)
    for step in range(4):
        c.pos_h = (c.pos_h + 977).astype(np.int32)
        c.pos.copy_(torch.from_numpy(c.pos_h))
        c.q.mul_(1.25)
        graph.replay()
        torch.cuda.synchronize()
        check(qo, *c.want(c.q, c.gq, 128), "bf16", f"replay {step}")
        check(ko, *c.want(c.k, c.gk, 128), "bf16", f"replay {step}")


