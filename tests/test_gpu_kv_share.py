"""Forking, freeing, copying and compacting pages against the lists of kvb_ref.Books."""
import numpy as np
import pytest
import torch

import kvb_ref as ref
from paper_2505_13204_b200 import binding

pytestmark = pytest.mark.gpu
PAGE = ref.PAGE


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32)).cuda()


class Device:
    """Books on the GPU beside a model's."""

    def __init__(self, books, layers=2, size=(2, 48), rng=None):
        self.m = books
        N = len(books.shares)
        self.raw = rng.integers(0, 256, (layers, N) + size).astype(np.uint8) if rng is not None else np.zeros((layers, N) + size, np.uint8)
        self.pages = torch.as_tensor(self.raw).cuda()
        self.t = [i32(x) for x in self.arrays()]

    def arrays(self):
        m, N = self.m, len(self.m.shares)
        table = np.full((len(m.table), m.width), -1, np.int32)
        for b, r in enumerate(m.table):
            table[b, :len(r)] = r
        return table, [len(r) for r in m.table], m.cached, m.stack + [-1] * (N - len(m.stack)), [len(m.stack)], m.shares

    def check(self):
        for name, x, y in zip(("block_table", "seq_pages", "cached_len", "free_pages", "n_free", "page_shares"), self.t, self.arrays()):
            assert np.array_equal(x.cpu().numpy(), np.asarray(y, np.int32)), name
        assert np.array_equal(self.pages.cpu().numpy(), self.raw)
        # every page is on the stack, or has as many holders as tables name it
        count = np.bincount([p for r in self.m.table for p in r], minlength=len(self.m.shares))
        for p in range(len(self.m.shares)):
            assert (count[p] == 0) == (p in set(self.m.stack)) and max(count[p] - 1, 0) == self.m.shares[p]

    def fork(self, ctx, src, dst, length=None):
        table, held, cached, free, n, shares = self.t
        o = ctx.kv_fork(self.pages, i32(src), i32(dst), table, held, cached, free, n, shares, None if length is None else i32(length))
        out, full, bad = self.m.fork(src, dst, length)
        for s, d in {(a, b) for _, a, b in out if a >= 0}:
            self.raw[:, d] = self.raw[:, s]
        status = ctx.poll_status()
        assert status == (binding.STATUS_KV_FULL if full else 0) | (binding.STATUS_BAD_OFFSETS if bad else 0)
        got = np.stack([o[k].cpu().numpy() for k in ("new_len", "copy_src", "copy_dst")], 1)
        assert np.array_equal(got, np.asarray(out).reshape(-1, 3))
        self.check()

    def free(self, ctx, keep, new=None):
        table, held, cached, free, n, shares = self.t
        ctx.kv_free(i32(keep), table, held, free, n, shares, None if new is None else i32(new))
        self.m.free(keep, new)
        for b, x in enumerate(keep):
            if x != ref.NONE:
                self.m.cached[b] = min(x, self.m.cached[b])
        cached.copy_(i32(self.m.cached))
        assert ctx.poll_status() == 0
        self.check()

    def compact(self, ctx):
        table, held, cached, free, n, shares = self.t
        o = ctx.kv_compact(self.pages, table, held, free, n, shares)
        to, moves = self.m.compact()
        before = self.raw.copy()
        for s, d in moves:
            self.raw[:, d] = before[:, s]
        assert ctx.poll_status() == 0
        assert o["page_map"].tolist() == to and o["n_moved"].tolist() == [len(moves)]
        self.check()


def books(rng, B, longest, spare, live):
    """B sequences, the first `live` of them with 0 .. longest tokens."""
    cached = [int(rng.integers(0, longest + 1)) if b < live else 0 for b in range(B)]
    need = [-(-n // PAGE) for n in cached]
    N = sum(need) + spare
    order, at, table = [int(x) for x in rng.permutation(N)], 0, []
    for n in need:
        table.append(order[at:at + n])
        at += n
    return ref.Books(table, need, order[at:], [0] * N, cached, longest // PAGE + 3)


@pytest.mark.parametrize("B,live,longest,spare", [(2, 1, 10, 1), (8, 3, 300, 20), (40, 10, 1000, 100), (1500, 300, 200, 1300), (6, 2, 64, 0), (30, 9, 700, 7),
                                                  (12, 4, 300, 2600), (64, 20, 500, 9000)])   # pools of more than one round of a scan
def test_fork_free_compact(ctx, B, live, longest, spare):
    rng = np.random.default_rng(B + longest)
    d = Device(books(rng, B, longest, spare, live), rng=rng)
    dst = live + rng.permutation(B - live)
    src = rng.integers(0, live, len(dst))
    half = len(dst) // 2 + 1
    d.fork(ctx, src[:half].tolist(), dst[:half].tolist())
    length = [int(rng.integers(0, d.m.cached[s] + 1)) for s in src[half:]]
    length = [n // PAGE * PAGE if i % 3 == 0 else n for i, n in enumerate(length)]
    if length:
        d.fork(ctx, src[half:].tolist(), dst[half:].tolist(), length)
    # forks of forks
    empty = [b for b in range(B) if not d.m.table[b] and d.m.cached[b] == 0][:5]
    full = [b for b in range(B) if d.m.table[b]]
    if empty and full:
        d.fork(ctx, [full[i % len(full)] for i in range(len(empty))], empty)
    keep = [int(rng.integers(0, n + 1)) if rng.random() < 0.6 else ref.NONE for n in d.m.cached]
    d.free(ctx, keep)
    d.compact(ctx)
    d.compact(ctx)                                        # nothing is left to move
    d.free(ctx, [0] * B, [0] * B)
    assert len(d.m.stack) == len(d.m.shares)
    d.compact(ctx)


def test_fork_refuses_what_cannot_be(ctx):
    rng = np.random.default_rng(0)
    d = Device(books(rng, 8, 200, 5, 3), rng=rng)
    n = d.m.cached[0]
    assert n > 70
    # destinations that hold pages, named twice, outside; sources outside, that are destinations; lengths that the source has not
    d.fork(ctx, [0, 0, 0, 0, -1, 9, 5, 0, 0, 0], [1, 4, 4, 8, 5, 6, 7, -3, 0, 3], [n, 10, 10, 10, 1, 1, 0, 1, 1, n])
    d.fork(ctx, [0, 0, 0], [5, 6, 7], [n + 1, -4, 64])
    with pytest.raises(binding.AasdError):
        table, held, cached, free, top, shares = d.t
        ctx.kv_fork(d.pages, i32([0, 1]), i32([2]), table, held, cached, free, top, shares)
    with pytest.raises(AssertionError):
        ctx.kv_fork(d.pages, i32([0]).long(), i32([2]), table, held, cached, free, top, shares)
    with pytest.raises(binding.AasdError):
        ctx.kv_fork(d.pages[:, :1].contiguous(), i32([0]), i32([2]), table, held, cached, free, top, shares)
    src, dst = i32([0]), i32([5])
    with pytest.raises(binding.AasdError):               # outputs over what the fork is made from
        ctx.kv_fork(d.pages, src, dst, table, held, cached, free, top, shares, outputs=dict(new_len=dst, copy_src=i32([0]), copy_dst=i32([0])))
    with pytest.raises(binding.AasdError):
        ctx.kv_compact(d.pages, table, held, free, top, shares, outputs=dict(page_map=shares, n_moved=i32([0])))
    with pytest.raises(binding.AasdError):
        ctx.kv_free(i32([0]), table, held, free, top, shares)
    with pytest.raises(binding.AasdError):
        ctx.kv_compact(d.pages, table, held, free, top, shares[:2].contiguous())
    d.check()


def test_inconsistent_books_are_reported_and_nothing_outside_is_touched(ctx):
    guard = torch.full((64,), 77, dtype=torch.int32, device="cuda")

    def inside(values, n):
        x = guard.clone()
        x[16:16 + n] = i32(values)
        return x, x[16:16 + n]

    def check(*whole):
        for x, n in whole:
            assert (x[:16] == 77).all() and (x[16 + n:] == 77).all()

    for stack, top in (([9, 3, 3, -1], 3), ([0, 1, 2, 3], 9), ([0, -4, 2, 3], 4)):
        wt, t = inside([1, 50, -1, 2, -7, -1], 6)
        wf, f = inside(stack, 4)
        wh, h = inside([2, 2], 2)
        ws, s = inside([0, 0, 0, 0], 4)
        n, pages = i32([top]), torch.zeros((1, 4, 1, 16), dtype=torch.uint8, device="cuda")
        ctx.kv_compact(pages, t.view(2, 3), h, f, n, s)
        assert ctx.poll_status() & binding.STATUS_BAD_OFFSETS
        ctx.kv_free(i32([0, 0]), t.view(2, 3), h, f, n, s)
        assert ctx.poll_status() & binding.STATUS_BAD_OFFSETS
        check((wt, 6), (wf, 4), (wh, 2), (ws, 4))
    for held in ([-1, 9], [2 ** 31 - 1, -2 ** 31]):
        wt, t = inside([1, 2, -1, 0, -1, -1], 6)
        wh, h = inside(held, 2)
        wf, f = inside([3, -1, -1, -1], 4)
        ws, s = inside([0, 0, 0, 0], 4)
        ctx.kv_free(i32([0, 0]), t.view(2, 3), h, f, i32([1]), s)
        assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS
        check((wt, 6), (wf, 4), (wh, 2), (ws, 4))


@pytest.mark.parametrize("layers,N,H,size,n", [(1, 3, 1, 16, 1), (3, 9, 2, 8208, 4), (2, 40, 8, 16400, 17), (5, 6, 1, 4608, 3), (1, 300, 3, 48, 150)])
def test_copy(ctx, layers, N, H, size, n):
    rng = np.random.default_rng(N)
    raw = rng.integers(0, 256, (layers, N, H, size)).astype(np.uint8)
    pages = torch.as_tensor(raw).cuda()
    order = rng.permutation(N)
    src, dst = order[:n].astype(np.int32), order[n:2 * n].astype(np.int32)
    if n > 2:
        src[1], dst[2] = -1, -1
    ctx.kv_copy(pages, i32(src), i32(dst))
    assert ctx.poll_status() == 0
    for s, d in zip(src, dst):
        if s >= 0 and d >= 0:
            raw[:, d] = raw[:, s]
    assert np.array_equal(pages.cpu().numpy(), raw)
    ctx.kv_copy(pages, i32([N, 0, -2]), i32([0, N + 3, 1]))
    assert ctx.poll_status() == binding.STATUS_ID_RANGE and np.array_equal(pages.cpu().numpy(), raw)


def test_steps_with_shared_pages(ctx):
    """kv_plan with holders: samples of one prompt go on, end and come again; no page is lost or has two owners that write it."""
    rng = np.random.default_rng(3)
    B, P, N = 6, 12, 40
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")                    # noqa: E731
    table, held, cached, shares = i(B, P) - 1, i(B), i(B), i(N)
    free, top = torch.arange(N, dtype=torch.int32, device="cuda"), i32([N])
    pages = torch.zeros((1, N, 1, 16), dtype=torch.uint8, device="cuda")
    new = i(B)
    new[0] = 200
    plan = ctx.kv_plan(cached, new, table, held, free, top, 200, page_shares=shares)
    cached = plan["kv_len"]
    ctx.kv_fork(pages, i32([0] * 5), i32([1, 2, 3, 4, 5]), table, held, cached, free, top, shares)
    for step in range(40):
        new = i32(rng.integers(0, 9, B))
        plan = ctx.kv_plan(cached, new, table, held, free, top, B * 9, rows_per_seq=9, page_shares=shares)
        assert (plan["kv_len"] == cached + new).all()
        cached = cached + torch.minimum(new, i32(rng.integers(0, 9, B)))
        if step % 7 == 6:
            end = int(rng.integers(1, B))
            cached[end] = 0
            ctx.kv_free(cached, table, held, free, top, shares)
            ctx.kv_fork(pages, i32([0]), i32([end]), table, held, cached, free, top, shares, i32([192]))
        if step % 11 == 10:
            ctx.kv_compact(pages, table, held, free, top, shares)
        t, h, f, s = (x.cpu().numpy() for x in (table, held, free, shares))
        count = np.bincount([p for b in range(B) for p in t[b, :h[b]]], minlength=N)
        stack = f[:int(top)]
        assert len(set(stack)) == len(stack) and (count[stack] == 0).all() and (count > 0).sum() + len(stack) == N
        assert np.array_equal(s, np.maximum(count - 1, 0))
        for b in range(B):                              # what is written from here on is the sequence's own
            for pg in range(int(cached[b]) // PAGE, h[b]):
                assert count[t[b, pg]] == 1
    assert ctx.poll_status() == 0
