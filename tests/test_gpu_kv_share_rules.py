"""What the page calls refuse and report."""
import numpy as np
import pytest
import torch

from paper_2505_13204_b200 import binding

pytestmark = pytest.mark.gpu
BOOKS = ("block_table", "seq_pages", "free_pages", "n_free", "page_shares")


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def small_books():
    """Two sequences with tokens, two without, six pages free; every array is longer than any output."""
    table = np.full((4, 4), -1)
    table[0, :3], table[1, :1] = (0, 1, 2), (7,)
    return dict(block_table=i32(table), seq_pages=i32([3, 1, 0, 0]), free_pages=i32([3, 4, 5, 6, 8, 9, -1, -1, -1, -1]), n_free=i32([6]), page_shares=i32([0] * 10))


def pages():
    return torch.zeros((2, 10, 1, 48), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("which", BOOKS + ("cached_len", "src_seq", "dst_seq", "fork_len", "pages", "new_len"))
@pytest.mark.parametrize("out", ["new_len", "copy_src", "copy_dst"])
def test_fork_refuses_outputs_over_its_arrays(ctx, which, out):
    b = small_books()
    given = dict(b, cached_len=i32([150, 20, 0, 0]), src_seq=i32([0]), dst_seq=i32([2]), fork_len=i32([70]), pages=pages(), new_len=i32([9]))
    outputs = {k: i32([9]) for k in ("new_len", "copy_src", "copy_dst")}
    if which == "new_len":
        if out == "new_len":
            return
        outputs["new_len"] = given["new_len"]
    over = given[which].view(-1)
    outputs[out] = over.view(torch.int32)[-1:] if which == "pages" else over[-1:]
    kept = {k: v.clone() for k, v in given.items()}
    with pytest.raises(binding.AasdError):
        ctx.kv_fork(given["pages"], given["src_seq"], given["dst_seq"], b["block_table"], b["seq_pages"], given["cached_len"], b["free_pages"], b["n_free"], b["page_shares"],
                    given["fork_len"], outputs=outputs)
    assert all(torch.equal(given[k], kept[k]) for k in kept) and ctx.poll_status() == 0


@pytest.mark.parametrize("which", BOOKS + ("pages", "page_map"))
@pytest.mark.parametrize("out", ["page_map", "n_moved"])
def test_compact_refuses_outputs_over_its_arrays(ctx, which, out):
    b = small_books()
    given = dict(b, pages=pages(), page_map=i32([9] * 10))
    outputs = dict(page_map=given["page_map"], n_moved=i32([9]))
    if which == out:
        return
    over = given[which].view(torch.int32).view(-1) if which == "pages" else given[which].view(-1)
    if out == "n_moved":
        outputs["n_moved"] = over[-1:]
    else:                                     # page_map ends where the array begins: both are parts of one
        joint = torch.zeros(9 + over.numel(), dtype=torch.int32, device="cuda")
        joint[9:] = over
        part = joint[9:]
        if which == "pages":
            if part.data_ptr() % 16:          # (pools start on 16-byte boundaries)
                joint = torch.zeros(12 + over.numel(), dtype=torch.int32, device="cuda")
                part = joint[12:]
            given["pages"] = part.view(torch.uint8).view(2, 10, 1, 48)
        else:
            given[which] = b[which] = part.view(given[which].shape)
        at = part.storage_offset() - 9
        outputs["page_map"] = joint[at:at + 10]
    kept = {k: v.clone() for k, v in given.items()}
    with pytest.raises(binding.AasdError):
        ctx.kv_compact(given["pages"], b["block_table"], b["seq_pages"], b["free_pages"], b["n_free"], b["page_shares"], outputs=outputs)
    assert all(torch.equal(given[k], kept[k]) for k in kept) and ctx.poll_status() == 0


def test_neighbouring_arrays_and_empty_ones_are_no_overlap(ctx):
    """Outputs that begin where the books end, in one allocation, and calls without sequences."""
    b = small_books()
    sizes = [b[k].numel() for k in BOOKS]
    joint = torch.empty(sum(sizes) + 4 + 3, dtype=torch.int32, device="cuda")
    at, part = 0, {}
    for k, n in zip(BOOKS, sizes):
        part[k] = joint[at:at + n].view(b[k].shape)
        part[k].copy_(b[k])
        at += n
    cached = joint[at:at + 4]
    cached.copy_(i32([150, 20, 0, 0]))
    outputs = {k: joint[at + 4 + i:at + 5 + i] for i, k in enumerate(("new_len", "copy_src", "copy_dst"))}
    ctx.kv_fork(pages(), i32([0]), i32([3]), part["block_table"], part["seq_pages"], cached, part["free_pages"], part["n_free"], part["page_shares"], i32([64]), outputs=outputs)
    assert ctx.poll_status() == 0 and outputs["new_len"].item() == 64 and part["seq_pages"].tolist() == [3, 1, 0, 1] and part["page_shares"].tolist() == [1] + [0] * 9
    none = joint[2:2]                         # an empty array inside another one
    ctx.kv_compact(pages(), part["block_table"][:0], none, part["free_pages"], part["n_free"], part["page_shares"])
    assert ctx.poll_status() == 0


def test_compact_looks_at_tables_when_nothing_moves(ctx):
    """Table entries that name a free page, or none of the pool, are reported and stay, whether pages move or not."""
    for entry in (5, 77, -9):
        for moves in (False, True):
            free = [2, 3, 4, 5] if not moves else [0, 3, 4, 5]
            used = [0, 1] if not moves else [1, 2]
            table = i32([used + [entry], [-1, -1, -1]])
            o = ctx.kv_compact(torch.zeros((1, 6, 1, 16), dtype=torch.uint8, device="cuda"), table, i32([3, 0]), i32(free + [-1, -1]), i32([4]), i32([0] * 6))
            assert o["n_moved"].tolist() == [int(moves)] and ctx.poll_status() == binding.STATUS_BAD_OFFSETS
            assert table.tolist() == [[1, 0, entry] if moves else [0, 1, entry], [-1, -1, -1]]


@pytest.mark.parametrize("B", [4, 40, 1500])      # the tables looked through by the collecting CTA, or by a launch of their own; few threads
def test_a_shared_page_that_is_about_to_be_written_is_reported(ctx, B):
    """Sequences cut inside what others hold too: a step that stores to such a page is reported in front of it, by kv_free and by kv_plan with
    page_shares; steps that store to pages of their own are not."""
    N, P = 12, 5

    def start():
        cached = i32([0] * B)
        books = [i32(np.full((B, P), -1)), i32([0] * B), i32(np.arange(N)[::-1]), i32([N]), i32([0] * N)]
        p = ctx.kv_plan(cached, i32([150] + [0] * (B - 1)), *books[:4], 150)
        cached = p["kv_len"].clone()
        ctx.kv_fork(torch.zeros((1, N, 1, 16), dtype=torch.uint8, device="cuda"), i32([0]), i32([B - 1]), *books[:2], cached, *books[2:])
        assert ctx.poll_status() == 0
        return books

    def at(first, last):
        return i32([first] + [0] * (B - 2) + [last])

    def keep(first, last):
        return i32([first] + [binding.NONE] * (B - 2) + [last])

    bad = binding.STATUS_BAD_OFFSETS
    # (kept, new) of the sequence and of its sample; the status.  Pages 0 and 1 are shared, the third is each one's own.
    cases = [((150, 150), (3, 3), 0), ((100, 150), (3, 1), bad), ((150, 100), (3, 1), bad), ((150, 127), (0, 1), bad), ((128, 150), (5, 0), 0), ((128, 128), (1, 70), 0),
             ((100, 150), (0, 1), 0),                     # nothing is stored
             ((100, 0), (3, 0), 0), ((0, 64), (0, 9), 0), # the other one ends in the same call
             ((64, 150), (64, 0), bad), ((64, 150), (1, 0), bad)]   # (page 1 is kept for the new tokens)
    for kept, new, status in cases:
        books = start()
        ctx.kv_free(keep(*kept), *books, at(*new))
        assert ctx.poll_status() == status, (kept, new)
        books = start()
        p = ctx.kv_plan(at(*kept), at(*new), *books[:4], sum(new), page_shares=books[4])
        assert ctx.poll_status() == status, (kept, new)
        assert p["kv_len"].tolist() == at(kept[0] + new[0], kept[1] + new[1]).tolist()
    # a sequence that is left alone is not looked at, and neither is one without new tokens in a call without them
    books = start()
    ctx.kv_free(keep(binding.NONE, 150), *books, at(3, 3))
    ctx.kv_free(keep(100, 150), *books)
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("call", ["compact", "fork"])
def test_what_a_call_gives_back_is_not_handed_to_another_stream(call):
    """The context works on another stream than torch's current one, and what the call returns is dropped: what its kernels read again is not
    handed to the current stream, which is not behind them."""
    rng = np.random.default_rng(0)
    N = 4000
    c = binding.Context()
    side = torch.cuda.Stream()
    try:
        order = rng.permutation(N)
        used, rest = order[:N // 2], order[N // 2:]
        raw = rng.integers(0, 256, (1, N, 1, 64)).astype(np.uint8)
        pool = torch.as_tensor(raw).cuda()
        n = 1 if call == "compact" else N // 2             # sequences of one page; or one sequence that holds all of them
        table = np.full((2 * n, N // 2 // n), -1)
        table[:n] = used.reshape(n, -1)
        books = [i32(table), i32([N // 2 // n] * n + [0] * n), i32(np.concatenate([rest, np.full(N // 2, -1)])), i32([N - N // 2]), i32([0] * N)]
        cached, src, dst = i32([63] * n + [0] * n), i32(np.arange(n)), i32(n + np.arange(n))
        torch.cuda.synchronize()
        c.set_stream(side)
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        if call == "compact":
            c.kv_compact(pool, *books)
        else:
            c.kv_fork(pool, src, dst, *books[:2], cached, *books[2:])
        found = [torch.full((len(src) if call == "fork" else N,), 3, dtype=torch.int32, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        assert c.poll_status() == 0 and all((x == 3).all() for x in found)
        got = pool.cpu().numpy()[0]
        if call == "compact":
            far = np.sort(used[used >= N // 2])
            to = np.arange(N)
            to[far] = np.setdiff1d(np.arange(N // 2), used)
            assert np.array_equal(books[0].cpu().numpy()[0], to[used]) and np.array_equal(got[to[used]], raw[0, used])
        else:
            assert books[0].cpu().numpy()[n:, 0].tolist() == rest[::-1].tolist() and cached.tolist() == [63] * (2 * n)
            assert np.array_equal(got[rest[::-1]], raw[0, used])
    finally:
        c.close()
