"""The 8-bit cache's attention where it can go wrong in other ways: waits that run out, graphs, scratch that both caches use."""
import numpy as np
import pytest
import torch

import test_gpu_kvb as kvb
from paper_2505_13204_b200 import binding

pytestmark = pytest.mark.gpu
i32 = kvb.i32


@pytest.fixture(scope="module")
def long_pools():
    rng = np.random.default_rng(20)
    return {D: kvb.Pool(rng, [2000], 2, D) for D in (64, 128, 256)}


@pytest.mark.parametrize("new,D,dtype,page", [(1, 128, "bf16", 1), (1, 64, "f32", 0), (40, 128, "bf16", 2), (200, 128, "bf16", 0), (40, 64, "bf16", 4), (200, 64, "bf16", 1),
                                             (40, 256, "bf16", 1)])
def test_a_wait_that_runs_out_ends_the_call_and_the_context_recovers(long_pools, new, D, dtype, page):
    """One of the first CTA's pages never arrives: its waits run out, the call ends by itself and the status word says so.  Nothing
    faults; with the scratch registered again the same call gives what it gave."""
    c = binding.Context()
    try:
        B, n, pool = 200, 2000, long_pools[D]
        g = torch.Generator(device="cuda").manual_seed(page)
        q = torch.randn((B * new, 4, D), generator=g, device="cuda").to(kvb.DT[dtype])
        args = (q, pool.pages, i32(np.tile(pool.table, (B, 1))), i32([n - new] * B), i32([n] * B))
        want = c.kvb_attend(*args, rows_per_seq=new)["out"].clone()
        assert c.poll_status() == 0
        c.debug_withhold_tile(page, 0, 1 << 14)
        c.kvb_attend(*args, rows_per_seq=new)
        torch.cuda.synchronize()                   # the call ended by itself
        assert c.poll_status() == binding.STATUS_TIMEOUT
        c.reinit_workspace()
        assert torch.equal(c.kvb_attend(*args, rows_per_seq=new)["out"], want) and c.poll_status() == 0
    finally:
        c.close()


def test_both_caches_take_turns_on_one_scratch():
    """Calls on 4-bit and 8-bit pools, few rows and many, one after the other on a context's one scratch: each gives what it gives alone."""
    import test_gpu_kv as kv
    rng = np.random.default_rng(21)
    c = binding.Context()
    try:
        four, eight = kv.Pool(rng, [700, 90], 2, 128), kvb.Pool(rng, [700, 90], 2, 128)
        calls = []
        for new in (1, 60):
            q = torch.as_tensor(rng.standard_normal((2 * new, 8, 128)).astype(np.float32)).bfloat16().cuda()
            for call, pool in ((c.kv_attend, four), (c.kvb_attend, eight)):
                calls.append((call, (q, pool.pages, i32(pool.table), i32([700 - new, 90 - new]), i32([700, 90])), new))
        alone = []
        for call, args, new in calls:
            alone.append(call(*args, rows_per_seq=new)["out"].clone())
            torch.cuda.synchronize()
        for _ in range(5):
            got = [call(*args, rows_per_seq=new)["out"] for call, args, new in calls]
            assert all(torch.equal(a, b) for a, b in zip(got, alone))
        assert c.poll_status() == 0
    finally:
        c.close()


def test_a_step_is_replayed_from_a_graph():
    """Plan (with holders), store, attention, commit, fork, free and compact captured once and replayed: what the calls give one by one."""
    rng = np.random.default_rng(22)
    B, Hq, Hkv, D, new, P, N = 3, 8, 2, 64, 5, 4, 16
    c = binding.Context()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    c.set_stream(side)
    try:
        with torch.cuda.stream(side):
            x = torch.as_tensor(rng.standard_normal((B * new, Hq + 2 * Hkv, D)).astype(np.float32)).cuda()
            pages = binding.kvb_pages(N, Hkv, D, layers=1)
            old = torch.as_tensor(rng.standard_normal((150, 2 * Hkv, D)).astype(np.float32)).cuda()
            parent = i32([[-1, 0, 0, 1, 3]] * B)
            best, n_new = i32([4, 2, 0]), i32([new] * B)

            def start():
                books = [i32(np.full((B + 1, P), -1)), i32([0] * (B + 1)), i32(np.arange(N)[::-1]), i32([N]), i32([0] * N)]
                cached = i32([0] * (B + 1))
                lens = i32([60, 64, 26, 0])
                p = c.kv_plan(cached, lens, *books[:4], 150)
                c.kvb_write(pages[0], old[:, :0], old[:, :Hkv], old[:, Hkv:], books[0], cached, p["kv_len"], p["positions"], p["tok_offsets"], outputs=dict(q=old[:, :0]))
                return books, p["kv_len"]

            def step(books, cached):
                n4 = torch.cat([n_new, n_new.new_zeros(1)])
                p = c.kv_plan(cached, n4, *books[:4], B * new, page_shares=books[4])
                q = c.kvb_write(pages[0], x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], books[0], cached, p["kv_len"], p["positions"], p["tok_offsets"])["q"]
                o = c.kvb_attend(q, pages[0], books[0], cached, p["kv_len"], p["tok_offsets"], node_parent=parent.view(-1))["out"]
                length = c.kvb_commit(pages, books[0][:B].contiguous(), cached[:B].contiguous(), p["kv_len"], best, parent)
                cached = torch.cat([length, length.new_zeros(1)])
                f = c.kv_fork(pages, i32_one, i32_last, *books[:2], cached, *books[2:])
                m = c.kv_compact(pages, *books)
                return o, cached, f["new_len"], m["page_map"]

            i32_one, i32_last = i32([1]), i32([B])
            books, cached = start()
            c.kv_workspace(D)
            want = [t.clone() for t in step(books, cached)] + [t.clone() for t in books] + [pages.clone()]
            side.synchronize()
            books, cached = start()
            kept = [t.clone() for t in books] + [pages.clone()]
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = step(books, cached)
            for _ in range(3):
                for t, k in zip(books + [pages], kept):
                    t.copy_(k)
                graph.replay()
                side.synchronize()
                live = want[-1].view(-1)[: int(N - want[4 + 3]) * Hkv * pages.shape[-1]]
                for a, b in zip(list(got) + books, want[:-1]):
                    assert torch.equal(a, b)
                assert torch.equal(pages.view(-1)[:live.numel()], live)
        assert c.poll_status() == 0
    finally:
        c.close()
