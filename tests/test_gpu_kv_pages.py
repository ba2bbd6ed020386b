"""moa_kv_reserve and moa_kv_release against the same on the host, entry by entry."""
import numpy as np
import pytest
import torch

import paper_2410_03804_amd as moa

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Pages:
    """The host's copy of table, list and lengths, and the device's."""

    def __init__(self, B, n_pages, page, mp, seed, free=None):
        self.rng = np.random.default_rng(seed)
        self.B, self.n_pages, self.page, self.mp, self.cap = B, n_pages, page, mp, mp * page
        self.table = np.full((B, mp), -1, np.int32)
        free = n_pages if free is None else free
        self.stack = [int(p) for p in self.rng.permutation(n_pages)[:free]]
        self.len = np.zeros(B, np.int32)
        self.free = i32(np.concatenate([self.stack, np.full(n_pages - free, -9)]).astype(np.int32))
        self.n_free, self.t_table, self.t_len, self.status = i32([free]), i32(self.table), i32(self.len), i32([0])
        self.tail = None

    def reserve(self, n, T, seen=None, pos=True, slot=True, alias=False):
        n = np.asarray(n, np.int32)
        off, got = torch.full((self.B + 1,), -5, dtype=torch.int32, device="cuda"), torch.full((self.B,), -5, dtype=torch.int32, device="cuda")
        tp, ts = (torch.full((T,), -5, dtype=torch.int32, device="cuda") if on else None for on in (pos, slot))
        new = i32(n)
        if alias:
            got = new
        moa.kv_reserve(self.t_table, self.t_len, new, self.page, self.free, self.n_free, off, got, pos=tp, slot=ts, seen=None if seen is None else i32(seen),
                       rows=T, dev_status=self.status)
        torch.cuda.synchronize()
        # the host's
        status, at, w_off, w_got, w_pos, w_slot, refused = 0, 0, [], [], [], [], False
        for b in range(self.B):
            k, ln = int(n[b]), int(np.clip(self.len[b], 0, self.cap))
            if ln != self.len[b] or k < 0:
                status |= moa.DEV_BAD_LENGTH
            k = max(k, 0)
            if k > self.cap - ln:
                status |= moa.DEV_CACHE_FULL
                k = self.cap - ln
            if k > T - at:
                status |= moa.DEV_BAD_LENGTH
                k = T - at
            pages = range(ln // self.page, (ln + k - 1) // self.page + 1) if k else []
            lacks = [p for p in pages if self.table[b, p] < 0]
            ok = not lacks or (not refused and len(lacks) <= len(self.stack))
            if not ok:
                refused = True
                status |= moa.DEV_CACHE_FULL
            else:
                for p in lacks:
                    self.table[b, p] = self.stack.pop()
            if any(self.table[b, p] >= self.n_pages for p in pages):
                status |= moa.DEV_BAD_PAGE
            w_off.append(at)
            w_got.append(k if ok else 0)
            for i in range(k):
                w_pos.append((ln if seen is None else int(seen[b])) + i)
                page = int(self.table[b, (ln + i) // self.page])
                w_slot.append(page * self.page + (ln + i) % self.page if ok and 0 <= page < self.n_pages else -1)
            at += k
        w_off.append(at)
        assert off.tolist() == w_off
        assert got.tolist() == w_got
        if pos:
            assert tp.tolist() == w_pos + [0] * (T - at)
        if slot:
            assert ts.tolist() == w_slot + [-1] * (T - at)
        self.same(status)
        return w_got

    def release(self, status=0):
        moa.kv_release(self.t_table, self.t_len, self.page, self.free, self.n_free, dev_status=self.status)
        torch.cuda.synchronize()
        gone = []
        for b in range(self.B):
            keep = -(-int(np.clip(self.len[b], 0, self.cap)) // self.page)
            for p in range(keep, self.mp):
                if self.table[b, p] >= 0:
                    gone.append(int(self.table[b, p]))
                    self.table[b, p] = -1
        self.stack += [p for p in gone[::-1] if p < self.n_pages]
        self.same(status)

    def same(self, status):
        assert np.array_equal(self.t_table.cpu().numpy(), self.table)
        assert self.n_free.item() == len(self.stack) and self.free.tolist()[:len(self.stack)] == self.stack
        assert self.t_len.tolist() == self.len.tolist()
        assert self.status.item() == status
        self.status.zero_()

    def grow(self, n):
        self.len = (self.len + np.asarray(n, np.int32)).astype(np.int32)
        self.t_len.copy_(i32(self.len))


@pytest.mark.parametrize("pad", [0, 8192])
@pytest.mark.parametrize("page", [1, 16, 40])
@pytest.mark.parametrize("B", [1, 2, 63, 64, 300])
def test_a_batch_s_life(B, page, pad):
    """Prompts, decoded tokens, drafts that are mostly rejected, sequences that end, until the pool runs out now and then.  pad: rows of the
    batch that no token comes to use; beyond 8192 rows it is several launches."""
    mp = -(-400 // page)
    s = Pages(B, max(8, B * mp // 3), page, mp, seed=B * 100 + page)
    rng = s.rng
    for step in range(12):
        n = rng.integers(0, 120, B) if step % 4 == 0 else np.ones(B, int) if step % 2 else rng.integers(0, 9, B)
        n = np.minimum(n, s.cap - s.len)
        got = s.reserve(n, int(n.sum()) + pad + int(rng.integers(0, 5)), seen=rng.integers(0, 10 ** 6, B) if step % 3 == 0 else None, alias=step % 5 == 2)
        accepted = np.minimum(got, rng.integers(0, 5, B)) if step % 2 == 0 and step else np.asarray(got)
        s.grow(accepted)
        if step % 3 == 2:
            s.len[rng.random(B) < 0.4] = 0
            s.grow(np.zeros(B))
            s.release()
    s.len[:] = 0
    s.grow(np.zeros(B))
    s.release()
    assert len(set(s.stack)) == len(s.stack) and np.all(s.table == -1)


@pytest.mark.parametrize("B,T", [(3000, 9000), (1025, 1025), (1024, 8192), (1024, 8193), (2500, 500), (7, 40000), (1, 100000), (2100, 2000)])
def test_many_sequences_and_many_rows(B, T):
    page = 16
    s = Pages(B, 3 * B + T // page, page, 40 if B > 7 else 600 if B > 1 else 7000, seed=T)
    n = s.rng.integers(0, 2 * T // B + 1, B)
    s.reserve(n, T)
    s.release()                                  # what was taken, back in its order
    s.reserve(n, T)


@pytest.mark.parametrize("pad", [0, 9000])
def test_pages_run_out_in_order(pad):
    s = Pages(6, 10, 16, 8, seed=1, free=4)
    assert s.reserve([30, 16, 20, 0, 1, 0], 67 + pad) == [30, 16, 0, 0, 0, 0]      # 2 + 1; two are wanted, one is left; then who needs one waits too
    s.grow([30, 16, 0, 0, 0, 0])
    assert s.reserve([2, 1, 0, 0, 0, 0], 8 + pad) == [2, 1, 0, 0, 0, 0]            # the first has room in its page, the second takes the last one
    s.grow([2, 1, 0, 0, 0, 0])
    assert s.reserve([1, 15, 0, 0, 0, 0], 17 + pad) == [0, 15, 0, 0, 0, 0]         # none is left; who lacks none goes on


def test_the_same_room_asked_for_twice_takes_no_more():
    s = Pages(4, 50, 16, 9, seed=2)
    n = [17, 0, 40, 1]
    s.reserve(n, 58)
    left = len(s.stack)
    s.reserve(n, 58)
    assert len(s.stack) == left


def test_a_batch_too_small_for_a_prompt_of_a_large_one():
    """Rows run out in the middle of a sequence whose pages were counted, and of more than one round of sequences."""
    for alias in (False, True):
        s = Pages(1500, 4000, 16, 9, seed=8)
        n = s.rng.integers(0, 20, 1500)
        n[1100] = 130
        T = int(n[:1100].sum()) + 20
        got = s.reserve(n, T, alias=alias)
        assert got[1100] == 20 and not any(got[1101:])
        s = Pages(3, 700, 16, 900, seed=9)
        assert s.reserve([9000, 200, 5], 9100, alias=alias) == [9000, 100, 0]
        s.release()
        assert len(s.stack) == 700


def test_numbers_outside_their_ranges_in_a_large_batch():
    s = Pages(4, 50, 16, 4, seed=3)
    s.reserve([-3, 70, 5, 2], 9000)
    s.grow([-2, 100, 3, 0])
    s.reserve([1, 1, 1, 1], 9000)
    s.table[1, 0], s.table[2, 1] = 50, 10 ** 9
    s.t_table.copy_(i32(s.table))
    s.grow([2, -100, 0, 0])
    s.reserve([5, 20, 20, 0], 9000)
    big = Pages(40, 30, 16, 500, seed=4)                      # two launches of the release
    big.table[3, 7], big.table[20, 499], big.table[20, 2] = 30, 10 ** 9, 17
    big.stack.remove(17)
    big.free[:29].copy_(i32(big.stack))
    big.n_free.fill_(29)
    big.t_table.copy_(i32(big.table))
    big.grow([-4] + [0] * 39)
    big.release(status=moa.DEV_BAD_PAGE | moa.DEV_BAD_LENGTH)
    for claim, left in ((-7, 2), (31, 30), (30, 30)):
        big.n_free.fill_(claim)
        big.t_len.zero_()
        big.t_table[5, 100:102] = i32([4, 9])
        moa.kv_release(big.t_table, big.t_len, 16, big.free, big.n_free, dev_status=big.status)
        assert big.n_free.item() == left and torch.all(big.t_table == -1)
        assert big.status.item() == (moa.DEV_BAD_LENGTH if claim != 30 else 0) | (moa.DEV_BAD_PAGE if claim >= 30 else 0)
        big.status.zero_()


def test_numbers_outside_their_ranges():
    s = Pages(4, 50, 16, 4, seed=3)
    s.reserve([-3, 70, 5, 2], 200)                          # beyond the capacity of 64
    s.reserve([3, 3, 3, 3], 8)                              # beyond the batch's rows
    s.reserve([3, 3, 3, 3], 0, pos=False, slot=False)
    s.grow([-2, 100, 3, 0])
    s.reserve([1, 1, 1, 1], 4)
    s.release(status=moa.DEV_BAD_LENGTH)


def test_entries_that_name_no_page():
    s = Pages(3, 20, 16, 5, seed=4)
    s.table[1, 0], s.table[1, 3], s.table[2, 4] = 20, 10 ** 9, 55
    s.t_table.copy_(i32(s.table))
    s.reserve([5, 5, 5], 20)
    s.grow([5, 5, 5])
    s.release(status=moa.DEV_BAD_PAGE)
    assert s.table[1, 0] == 20 and s.table[1, 3] == -1


def test_without_positions_or_slots():
    s = Pages(5, 40, 16, 5, seed=5)
    s.reserve([5, 20, 0, 1, 2], 40, pos=False)
    s.reserve([5, 20, 0, 1, 2], 40, slot=False)
    s.reserve([5, 20, 0, 1, 2], 30, pos=False, slot=False)


def test_a_list_that_claims_more_than_there_is():
    s = Pages(2, 10, 16, 4, seed=6, free=10)
    s.n_free.fill_(99)
    off, got = i32([0] * 3), i32([0] * 2)
    moa.kv_reserve(s.t_table, s.t_len, i32([1, 1]), 16, s.free, s.n_free, off, got, dev_status=s.status)
    assert s.status.item() == moa.DEV_BAD_LENGTH and s.n_free.item() == 8
    assert s.t_table[:, 0].tolist() == [s.stack[9], s.stack[8]]
    s.t_table[0, 1:] = 3                                      # a page in three places more than there is
    s.t_table[1, 1:] = 3
    s.status.zero_()
    moa.kv_release(s.t_table, s.t_len, 16, s.free, s.n_free, dev_status=s.status)
    assert s.status.item() == moa.DEV_BAD_PAGE and s.n_free.item() == 10 and torch.all(s.t_table == -1)


def test_captured():
    s = Pages(8, 100, 16, 10, seed=7)
    n, off, got, pos, slot = i32([3] * 8), i32([0] * 9), i32([0] * 8), i32([0] * 24), i32([0] * 24)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moa.kv_reserve(s.t_table, s.t_len, n, 16, s.free, s.n_free, off, got, pos=pos, slot=slot, dev_status=s.status)
        s.t_len.add_(got)
        moa.kv_release(s.t_table, s.t_len, 16, s.free, s.n_free, dev_status=s.status)
    for step in range(6):
        graph.replay()
        torch.cuda.synchronize()
        taken = 8 * -(-3 * (step + 1) // 16)
        assert s.n_free.item() == 100 - taken and s.t_len.tolist() == [3 * (step + 1)] * 8
        assert pos.tolist() == [3 * step + i for _ in range(8) for i in range(3)]
        table = s.t_table.cpu().numpy()
        assert slot.tolist() == [int(table[b, (3 * step + i) // 16]) * 16 + (3 * step + i) % 16 for b in range(8) for i in range(3)]
    assert s.status.item() == 0


@pytest.mark.parametrize("claims,holds", [(-(2 ** 31), 0), (-1, 0), (99, 10), (2 ** 31 - 1, 10)])
@pytest.mark.parametrize("B", [2, 60])                        # one launch; two, whose additions come from several workgroups
def test_a_release_to_a_list_that_claims_the_impossible(B, claims, holds):
    s = Pages(B, 10, 16, 400, seed=8, free=10)
    s.n_free.fill_(claims)
    s.t_table[0, 5], s.t_table[B - 1, 399] = 3, 4
    moa.kv_release(s.t_table, s.t_len, 16, s.free, s.n_free, dev_status=s.status)
    more = moa.DEV_BAD_PAGE if holds == 10 else 0
    assert s.status.item() == moa.DEV_BAD_LENGTH | more and torch.all(s.t_table == -1)
    assert s.n_free.item() == min(holds + 2, 10)
    if holds == 0:
        assert s.free[:2].tolist() == [4, 3]
