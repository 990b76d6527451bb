"""8-bit attention over pages whose values' scales lie as far apart as the format lets them: what a page weighs does not depend on how small
its values are."""
import numpy as np
import pytest
import torch

import kv_ref
import kvb_ref as ref
import test_gpu_kvb as kvb
from paper_2505_13204_b200 import binding

pytestmark = pytest.mark.gpu
PAGE = ref.PAGE


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


# sizes of the pages' values: zeros have a scale of 2^-64, 1e33 one of about 2^103 (so the scales' exponents differ by 167, 119, 100, 30 ..)
SIZES = [(0.0, 1e33), (1e33, 0.0), (1e33, 0.0, 1e-3, 1e3, 1e26), (1e-3, 1e3, 1e33, 0.0, 1e28, 1e33), (1e24, 0.0, 1e24, 1e-9, 1e24, 1e-12, 1e24)]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("G,D", [(3, 64), (3, 256), (60, 64), (60, 128), (60, 256), (200, 64), (200, 128)])   # few rows; one tile, in one group or two; two tiles
@pytest.mark.parametrize("qscale", [1.0, 30.0])                                                            # even weights, and sharp ones
def test_pages_of_small_values_keep_their_weight(ctx, sizes, G, D, qscale):
    rng = np.random.default_rng(len(sizes) + D)
    n = len(sizes) * PAGE - 3
    pool = kvb.Pool(rng, [0], 1, D)
    pool.rows, pool.table, pages = kvb.tables(rng, [n])
    raw = np.full((pages, 1, ref.head_bytes(D)), 0x7F, np.uint8)
    k = rng.standard_normal((n, 1, D)).astype(np.float32)
    v = (rng.standard_normal((n, 1, D)) * np.repeat(sizes, PAGE)[:n, None, None]).astype(np.float32)
    ref.write(raw, pool.rows, [0], [n], [0], k, v, D)
    e = [ref.load(raw, pool.rows[0][c // PAGE] * PAGE + c % PAGE, D) for c in range(n)]
    pool.k, pool.v, pool.kv_len = [np.asarray([x[0] for x in e])], [np.asarray([x[1] for x in e])], [n]
    pool.pages = torch.as_tensor(raw).cuda()
    B = 300                       # (the same sequence again and again, so that a CTA goes from page to page, and segments are cut in many ways)
    for dtype in ("bf16", "f32"):
        q = torch.as_tensor((rng.standard_normal((1, G, D)) * qscale).astype(np.float32)).to(kvb.DT[dtype]).cuda()
        o = ctx.kvb_attend(q.repeat(B, 1, 1), pool.pages, kvb.i32(np.tile(pool.table, (B, 1))), kvb.i32([n - 1] * B), kvb.i32([n] * B), rows_per_seq=1, want_lse=True)
        assert ctx.poll_status() == 0
        want, wl, size = kv_ref.attend(kvb.f64(q[0]), pool.k[0], pool.v[0], range(n), 1 / np.sqrt(D))
        lim, lim_lse = kvb.limits(want, wl, size, np.abs(kvb.f64(q[0])).max(-1), np.abs(pool.k[0]).sum(-1).max(), 1 / np.sqrt(D), np.ptp(pool.v[0]), np.abs(pool.v[0]).max(),
                                  dtype == "f32")
        assert (np.abs(kvb.f64(o["lse"]) - wl) <= lim_lse).all(), dtype
        assert (np.abs(kvb.f64(o["out"]) - want) <= lim[:, None] + np.abs(want) * kvb.HALF[dtype]).all(), dtype


@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_cut_segment_with_pages_of_zeros(ctx, D):
    """Long sequences that the CTAs share, two pages of three without values: results and lse against 64-bit sums."""
    g = torch.Generator(device="cuda").manual_seed(D)
    B, n, new, Hq = 4, 20000, 40, 4
    per = -(-n // PAGE)
    pages = binding.kvb_pages(per, 1, D)
    k = torch.randn((n, 1, D), generator=g, device="cuda")
    v = torch.randn((n, 1, D), generator=g, device="cuda") * 1e30
    v[(torch.arange(n, device="cuda") // PAGE) % 3 != 0] = 0
    table = torch.arange(per, dtype=torch.int32, device="cuda")[None].contiguous()
    ctx.kvb_write(pages, k[:, :0], k, v, table, kvb.i32([0]), kvb.i32([n]), torch.zeros(n, dtype=torch.int32, device="cuda"), rows_per_seq=n, outputs=dict(q=k[:, :0]))
    q = torch.randn((B * new, Hq, D), generator=g, device="cuda").bfloat16()
    o = ctx.kvb_attend(q, pages, table.repeat(B, 1), kvb.i32([n - new] * B), kvb.i32([n] * B), rows_per_seq=new, want_lse=True)
    e = ctx.kvb_read(pages, torch.arange(n, dtype=torch.int32, device="cuda"), D, torch.float32)
    assert ctx.poll_status() == 0
    kd, vd = e["k"][:, 0].double(), e["v"][:, 0].double()
    w = torch.einsum("nhd,td->nht", q.double(), kd) / np.sqrt(D)
    w = w.masked_fill(torch.arange(n, device="cuda") > (n - new + torch.arange(B * new, device="cuda") % new)[:, None, None], float("-inf"))
    lse = torch.logsumexp(w, -1)
    want = torch.einsum("nht,td->nhd", torch.exp(w - lse[..., None]), vd)
    size = torch.einsum("nhd,td->nht", q.double().abs(), kd.abs()).amax(-1) / np.sqrt(D)
    lim, lim_lse = kvb.limits(None, kvb.f64(lse), kvb.f64(size), kvb.f64(q.double().abs().amax(-1)), float(kd.abs().sum(-1).max()), 1 / np.sqrt(D),
                              float(vd.max() - vd.min()), float(vd.abs().max()), False)
    assert (np.abs(kvb.f64(o["lse"]) - kvb.f64(lse)) <= lim_lse).all()
    assert (np.abs(kvb.f64(o["out"]) - kvb.f64(want)) <= lim[..., None] + np.abs(kvb.f64(want)) * kvb.HALF["bf16"]).all()
