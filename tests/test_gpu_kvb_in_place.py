"""The 8-bit store and its outputs: the rows of q and k in place, what is refused, and the keys on another stream."""
import numpy as np
import pytest
import torch

import kvb_ref as ref
from paper_2505_13204_b200 import binding
from test_gpu_kvb import DT, PAGE, garbage, i32, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


# sequences, new tokens, query heads, key heads, D: a warp per page, head and half whose rows take several passes (8, 4 or 2 at 64, 128, 256
# channels), one pass, and a CTA for each
CASES = [(64, 8, 4, 8, 128), (160, 20, 2, 2, 64), (160, 5, 2, 2, 256), (300, 31, 1, 1, 128), (160, 2, 2, 2, 128), (3, 70, 4, 2, 128), (2, 150, 2, 2, 64)]


@pytest.mark.parametrize("B,new,Hq,Hkv,D", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot", ["all", "part"])
def test_queries_and_keys_in_place(ctx, B, new, Hq, Hkv, D, dtype, rot):
    """q and k overwritten by what they become: the same outputs and the same bytes in the cache as with outputs of their own."""
    rng = np.random.default_rng(B + new + D)
    cached = rng.integers(0, 100, B)
    cached[0] = PAGE - 1 if new > 1 else 0              # (rows on both sides of a page's end)
    rows, table, pool = tables(rng, cached + new)
    raw = garbage(rng, pool, Hkv, D)
    make = lambda h: torch.as_tensor((rng.standard_normal((B * new, h, D)) * 2.0 ** rng.integers(-2, 3, (B * new, 1, 1))).astype(np.float32)).to(DT[dtype]).cuda()   # noqa: E731
    q, k, v = make(Hq), make(Hkv), make(Hkv)
    k[3, 0, 5] = float("nan")                            # a row that is stored as zeros
    w = [torch.as_tensor((1 + 0.1 * rng.standard_normal(D)).astype(np.float32)).to(DT[dtype]).cuda() for _ in range(2)]
    r = D if rot == "all" else D // 2
    ang = np.arange(400)[:, None] * 10000.0 ** (-np.arange(r // 2) / (r // 2))
    cs = torch.as_tensor(np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)).cuda()
    pos = i32((cached[:, None] + np.arange(new)).ravel())
    got = []
    for place in (False, True):
        a, b = q.clone(), k.clone()
        pages = torch.as_tensor(raw).cuda()
        outputs = dict(q=a, k=b) if place else None
        o = ctx.kvb_write(pages, a, b, v, i32(table), i32(cached), i32(cached + new), pos, None, new, cs, *w, keep_k=True, outputs=outputs)
        assert ctx.poll_status() == binding.STATUS_BAD_ROW
        got.append((o["q"], o["k"], pages))
    for x, y in zip(*got):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))     # (NaN rows too)


def test_outputs_over_anything_else_are_refused(ctx):
    D, T = 64, 8
    t, z, n = i32([[0]]), i32([0]), i32([T])
    pos = i32(np.arange(T))
    pages = torch.full((1, 2, ref.head_bytes(D)), 7, dtype=torch.uint8, device="cuda")
    buf = torch.randn((3 * T + 1, 2, D), device="cuda")
    kept = buf.clone()
    q, k, v = buf[:T], buf[T:2 * T], buf[2 * T:3 * T]
    own = lambda: torch.empty((T, 2, D), device="cuda")                                    # noqa: E731
    wide = torch.randn((T, 6, D), device="cuda")          # heads of a fused projection: the rows of dense outputs fall among others'
    cases = [(q, k, v, own(), v), (q, k, v, own(), q), (q, k, v, k, None), (q, k, v, v, own()), (q, k, v, own(), buf[T + 1:2 * T + 1]),
             (q, k, v, buf[1:T + 1], own()), (q, k, v, own(), buf[2 * T - 1:3 * T - 1])]
    same = own()
    cases.append((q, k, v, same, same))
    flat = wide.view(-1)[:T * 2 * D].view(T, 2, D)
    cases += [(wide[:, :2], wide[:, 2:4], wide[:, 4:], flat, None), (wide[:, 2:4], wide[:, :2], wide[:, 4:], own(), flat)]
    for a, b, c, qo, ko in cases:
        with pytest.raises(binding.AasdError):
            ctx.kvb_write(pages, a, b, c, t, z, n, pos, rows_per_seq=T, outputs=dict(q=qo, k=ko))
    assert torch.equal(buf, kept) and (pages == 7).all() and ctx.poll_status() == 0
    # rows in place, a single token whatever its stride says, and no queries at all
    ctx.kvb_write(pages, q, k, v, t, z, n, pos, rows_per_seq=T, outputs=dict(q=q, k=k))
    ctx.kvb_write(pages, wide[:1, :2], wide[:1, 2:4], wide[:1, 4:], t, z, i32([1]), pos[:1].contiguous(), rows_per_seq=1, outputs=dict(q=wide[:1, :2], k=wide[:1, 2:4]))
    ctx.kvb_write(pages, k[:, :0], k, v, t, z, n, pos, rows_per_seq=T, outputs=dict(q=k[3:, :0], k=k))
    assert ctx.poll_status() == 0


def test_zeros_of_rows_without_a_place_do_not_come_after_the_keys():
    """The context works on another stream than torch's current one, whose own work ends after the call's: keep_k's rows are the keys."""
    rng = np.random.default_rng(3)
    D, T = 64, 8
    c = binding.Context()
    try:
        x = torch.as_tensor(rng.standard_normal((T + 2, 3, D)).astype(np.float32)).cuda()
        args = (x[:, :1], x[:, 1:2], x[:, 2:], i32([[0]]), i32([0]), i32([T]), i32(np.arange(T + 2)), i32([0, T + 2]))
        pages = binding.kvb_pages(1, 1, D)
        want = c.kvb_write(pages, *args, keep_k=True)["k"].clone()
        assert (want[:T] != 0).any(-1).all() and (want[T:] == 0).all()
        torch.cuda.synchronize()
        c.set_stream(torch.cuda.Stream())
        torch.cuda._sleep(20_000_000)
        got = c.kvb_write(pages, *args, keep_k=True)["k"]
        torch.cuda.synchronize()
        assert torch.equal(got, want) and c.poll_status() == 0
    finally:
        c.close()
