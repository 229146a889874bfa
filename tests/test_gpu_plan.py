"""A step's tables made on the GPU (include/qqq_serve.h) against the host's loops: whole numbers, equal everywhere, and nothing else written."""
import numpy as np
import pytest
import torch

from oracle import qqq_serve_oracle as ref
from paper_2406_09904_amd import binding as qqq

pytestmark = pytest.mark.gpu


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Both:
    """Sessions on the host and their twins on the device; every call is made on both and everything compared."""

    def __init__(self, seed, sessions, columns, pages, page, stride=0):
        self.rng = np.random.default_rng(seed)
        self.host = ref.Sessions(sessions, columns, pages, page)
        self.host.free = self.rng.permutation(pages).astype(np.int32)
        wide = torch.full((sessions, columns + stride), -7, dtype=torch.int32, device="cuda")
        wide[:, :columns] = 0
        self.wide, self.columns, self.P = wide, columns, page
        self.dev = qqq.KV8Sessions(wide[:, :columns], torch.zeros(sessions, dtype=torch.int32, device="cuda"), _dev(self.host.free),
                                   torch.tensor([pages], dtype=torch.int32, device="cuda"))
        self.max_len = columns * page + page - 1

    def hold(self, held):
        """Sessions that hold so much already."""
        self.host.held[:] = held
        for s, h in enumerate(held):
            for j in range(min(h // self.P, self.columns)):
                self.host.count -= 1
                self.host.pages[s, j] = self.host.free[self.host.count]
        self.dev.pages.copy_(_dev(self.host.pages))
        self.dev.held.copy_(_dev(self.host.held))
        self.dev.free_count.fill_(self.host.count)

    def step(self, new, ids=None, max_new=None, max_len=None, tokens=None, spare=0, apart=False, pad=0):
        new = np.asarray(new, np.int32)
        B, max_new, max_len = len(new), int(max(new.max(initial=0), 0)) if max_new is None else max_new, self.max_len if max_len is None else max_len
        rows = int(np.maximum(new, 0).sum()) + spare if tokens is None else tokens
        wide = np.full((B, self.columns + pad), -5, np.int32)
        table, sequence, positions = wide[:, :self.columns], np.full(rows, -6, np.int32), np.full(rows, -6, np.int32)
        before = [t.clone() for t in self.dev]
        d_ids = None if ids is None else _dev(np.asarray(ids, np.int32))
        d_wide, d_seq, d_pos = _dev(wide), _dev(sequence), _dev(positions)
        batch = qqq.KV8Batch(d_wide[:, :self.columns], torch.full((B,), -8, dtype=torch.int32, device="cuda"), torch.full((B + 1,), -8, dtype=torch.int32, device="cuda"), d_ids,
                             max_new, max_len)
        lacking = torch.full((1,), -9, dtype=torch.int32, device="cuda")
        after = (self.dev.held.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")) if apart else None
        assert qqq.qqq_kv8_plan(self.dev, batch, _dev(new), self.P, d_seq, d_pos, lacking, after=after) is batch
        kv_len, cu, lack = self.host.plan(ids, new, max_new, max_len, table, sequence, positions)
        for got, want, what in ((d_wide, wide, "page_table"), (batch.kv_len, kv_len, "kv_len"), (batch.cu, cu, "cu"), (d_seq, sequence, "sequence"), (d_pos, positions, "positions"),
                                (lacking, [lack], "lacking")):
            assert np.array_equal(got.cpu().numpy(), want), what
        if apart:
            assert torch.equal(before[1], self.dev.held) and torch.equal(before[3], self.dev.free_count)
            self.dev.held.copy_(after[0])
            self.dev.free_count.copy_(after[1])
        self.check()
        return batch

    def check(self):
        for got, want, what in ((self.dev.pages, self.host.pages, "pages"), (self.dev.held, self.host.held, "held"), (self.dev.free, self.host.free, "stack"),
                                (self.dev.free_count, [self.host.count], "free_count")):
            assert np.array_equal(got.cpu().numpy(), want), what
        assert (self.wide[:, self.columns:] == -7).all()


# one sequence, one wave's and a wave and one, a workgroup's and one more, several turns of the scan; single tokens, ragged, none
@pytest.mark.parametrize("B,new_hi,held_hi,page", [(1, 1, 0, 16), (1, 1, 63, 64), (1, 1000, 5000, 16), (2, 3, 100, 32), (63, 1, 500, 64), (64, 5, 300, 16), (65, 90, 40, 16),
                                                   (256, 1, 300, 64), (257, 2, 300, 16), (300, 2, 700, 64), (512, 1, 90, 16), (513, 40, 90, 16), (1023, 1, 90, 32), (1024, 3, 33, 16), (1025, 2, 50, 16), (2500, 4, 200, 16), (4096, 1, 40, 16),
                                                   (4097, 2, 40, 16), (9001, 3, 60, 16), (5, 4000, 9000, 16), (20, 1, 5000, 16), (1, 1, 90000, 16)])
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("slots", [False, True])
def test_plan(B, new_hi, held_hi, page, slots, apart):
    rng = np.random.default_rng(B * 7 + new_hi)
    sessions = B + (B // 3 + 1 if slots else 0)
    both = Both(B, sessions, (held_hi + new_hi) // page + 2, sessions * ((held_hi + new_hi) // page + 1) + 3, page, stride=3)
    both.hold(rng.integers(0, held_hi + 1, sessions))
    ids = rng.permutation(sessions)[:B] if slots else None
    both.step(rng.integers(0, new_hi + 1, B), ids, max_new=new_hi, spare=5, apart=apart, pad=B % 3)


@pytest.mark.parametrize("B,columns", [(40, 30), (40, 150), (300, 200)])   # in one launch and in two
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("apart", [False, True])
def test_steps_and_releases_in_turn(B, columns, page, apart):
    both = Both(B + page, B + 9, columns, (B + 9) * columns // 2, page)
    rng = both.rng
    for turn in range(8):
        ids = rng.permutation(B + 9)[:B]
        new = np.minimum(rng.integers(0, 3 * page, B) * (rng.random(B) < 0.7), both.max_len - both.host.held[ids])
        both.step(new, ids, max_new=3 * page, apart=apart)
        ends = np.concatenate([rng.permutation(B + 9)[:B // 3], [-1, B + 9]])     # (two that do not exist)
        qqq.qqq_kv8_release(both.dev, page, _dev(ends.astype(np.int32)))
        both.host.release(ends)
        both.check()
    qqq.qqq_kv8_release(both.dev, page)
    both.host.release(range(B + 9))
    both.check()
    assert both.host.count == (B + 9) * columns // 2 and sorted(both.host.free) == list(range(both.host.count))    # every page is back, once


@pytest.mark.parametrize("B", [7, 500, 1500])
@pytest.mark.parametrize("apart", [False, True])
def test_pages_that_are_lacking(B, apart):
    """Entries without a page are -1, the stack stays at its bottom, and a release gives back only what is one."""
    both = Both(B, B, 12, 3 * B, 16)
    both.step(np.full(B, 16 * 8 + 3), apart=apart)
    assert both.host.count == 0 and (both.host.pages == -1).any()
    both.step(np.full(B, 40), apart=apart)
    both.host.release(range(B))
    qqq.qqq_kv8_release(both.dev, 16)
    both.check()
    assert both.host.count == 3 * B


@pytest.mark.parametrize("B", [50, 700, 1300])
@pytest.mark.parametrize("apart", [False, True])
def test_what_is_out_of_bounds_is_cut(B, apart):
    """More tokens than the bounds, the rows or the cache allow, fewer than none, sessions that do not exist, numbers that no program writes."""
    both = Both(B, B, 6, 4 * B, 16)
    both.hold(np.arange(B) % 90)
    rng = both.rng
    both.step(rng.integers(-5, 60, B), max_new=31, max_len=100, apart=apart)
    both.step(rng.integers(0, 60, B), tokens=10 * B, max_new=1 << 30, apart=apart)
    ids = rng.permutation(B)
    ids[::5], ids[1::11] = -3, B
    both.step(rng.integers(0, 4, B), ids, tokens=0, apart=apart)
    both.step(rng.integers(0, 4, B), ids, max_len=0, apart=apart)
    for held, count in ((np.full(B, -2 ** 31), -5), (np.full(B, 2 ** 31 - 1), 2 ** 31 - 1)):
        both.host.held[:], both.host.count = held.astype(np.int32), count
        both.dev.held.copy_(_dev(both.host.held))
        both.dev.free_count.fill_(count)
        if count < 0:
            both.step(rng.integers(0, 40, B), apart=apart)
        else:
            both.step(np.full(B, 2 ** 31 - 1, np.int64).astype(np.int32), tokens=3, max_new=1 << 30, apart=apart)


def test_no_sequence_and_no_page():
    both = Both(1, 3, 2, 4, 16)
    both.step([], max_new=0)
    both.step([0, 0, 0])
    short = Both(2, 4, 0, 0, 64)                     # no table at all: sequences shorter than a page
    short.step([1, 5, 0, 63], max_new=63)
    short.step([62, 5, 63, 1], max_new=63)


@pytest.mark.parametrize("apart", [False, True])
def test_the_sessions_own_table(apart):
    """Without slots the step's table can be the sessions' own: only fresh pages are written."""
    both = Both(4, 30, 20, 400, 16, stride=4)
    both.hold(both.rng.integers(0, 200, 30))
    new = both.rng.integers(0, 50, 30).astype(np.int32)
    batch = qqq.new_kv8_batch(30, 20, 50, both.max_len)._replace(page_table=both.dev.pages)
    after = (both.dev.held.clone(), both.dev.free_count.clone()) if apart else None
    qqq.qqq_kv8_plan(both.dev, batch, _dev(new), 16, after=after)
    if apart:
        both.dev.held.copy_(after[0])
        both.dev.free_count.copy_(after[1])
    kv_len, cu, _ = both.host.plan(None, new, 50, both.max_len, np.zeros((30, 20), np.int32), np.zeros(9999, np.int32), np.zeros(9999, np.int32))
    assert np.array_equal(batch.kv_len.cpu(), kv_len) and np.array_equal(batch.cu.cpu(), cu)
    both.check()


def test_sessions_that_end_twice_are_released_once():
    both = Both(5, 70, 4, 200, 16)
    both.hold(both.rng.integers(0, 46, 70))
    ids = np.concatenate([np.arange(70), np.arange(70)])
    qqq.qqq_kv8_release(both.dev, 16, _dev(ids.astype(np.int32)))
    free = both.dev.free.cpu().numpy()
    assert int(both.dev.free_count) == 200 and sorted(free) == list(range(200)) and not both.dev.held.any()


@pytest.mark.parametrize("sessions,listed", [(3, 50), (70, 140), (40, 1024), (900, 3000), (1500, 5000)])
def test_sessions_that_are_listed_twice_are_released_in_the_first_places(sessions, listed):
    """In any order, within a wave, a workgroup's turn and beyond: the stack is the oracle's, entry by entry; numbers that are no session and lengths below 0 among them."""
    both = Both(sessions, sessions, 6, 6 * sessions, 16)
    both.hold(both.rng.integers(0, 6 * 16, sessions))
    for _ in range(3):
        ids = both.rng.integers(-1, sessions + 1, listed)
        both.host.held[::7] = -5
        both.dev.held[::7] = -5
        qqq.qqq_kv8_release(both.dev, 16, _dev(ids.astype(np.int32)))
        both.host.release(ids)
        both.check()
        both.host.held[::7] = 0
        both.dev.held[::7] = 0
        both.step(both.rng.integers(0, 40, sessions), max_new=40)


@pytest.mark.parametrize("lowest", [1, 37, 10 ** 6])
def test_pages_of_a_part_of_the_cache(lowest):
    """The stack holds pages from some number on, others have the rest: their numbers may pass its size, and every one comes back."""
    both = Both(lowest, 9, 5, 40, 16)
    both.host.free += lowest
    both.dev.free.copy_(_dev(both.host.free))
    for turn in range(4):
        both.step(both.rng.integers(0, 80, 9), max_new=80)
        ends = both.rng.permutation(9)[:6]
        qqq.qqq_kv8_release(both.dev, 16, _dev(ends.astype(np.int32)))
        both.host.release(ends)
        both.check()
    qqq.qqq_kv8_release(both.dev, 16)
    assert int(both.dev.free_count) == 40 and sorted(both.dev.free.tolist()) == list(range(lowest, lowest + 40)) and not both.dev.held.any()


@pytest.mark.parametrize("B,columns", [(8, 40), (200, 300)])
def test_captured_steps(B, columns):
    """A step is captured once and replayed: each replay carries on from what the one before left, beside eager work of the same tensors' copies."""
    both, eager = Both(6, B, columns, B * columns, 16), Both(6, B, columns, B * columns, 16)
    for b in (both, eager):
        b.hold(np.arange(B) % 300 if columns > 30 else np.zeros(B, int))
    new = torch.zeros(B, dtype=torch.int32, device="cuda")
    batch = qqq.new_kv8_batch(B, columns, 20, both.max_len)
    sequence, positions = (torch.zeros(20 * B, dtype=torch.int32, device="cuda") for _ in range(2))
    work = torch.empty(max(qqq.qqq_kv8_plan_workspace_bytes(both.dev, batch, 16), 4), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qqq.qqq_kv8_plan(both.dev, batch, new, 16, sequence, positions, workspace=work)
    for turn in range(5):
        n = both.rng.integers(0, 21, B).astype(np.int32)
        new.copy_(_dev(n))
        graph.replay()
        torch.cuda.synchronize()
        want = eager.step(n, max_new=20)
        rows = int(n.sum())
        assert torch.equal(batch.kv_len, want.kv_len) and torch.equal(batch.cu, want.cu)
        closed = torch.arange(columns, device="cuda")[None] < (batch.kv_len // 16)[:, None]
        assert torch.equal(batch.page_table[closed], want.page_table[closed])
        assert np.array_equal(sequence[:rows].cpu().numpy(), np.repeat(np.arange(B), n))
        both.host = eager.host
        both.check()


def test_on_a_stream_of_its_own():
    both = Both(9, 33, 9, 300, 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both.step(np.arange(33))
        both.step(np.arange(33)[::-1].copy())
    torch.cuda.current_stream().wait_stream(side)
