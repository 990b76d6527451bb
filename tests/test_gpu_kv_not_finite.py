"""Attention of rows whose queries are not finite, in both caches: NaN in out and lse, however the work was cut; -inf is left to rows that
see nothing."""
import numpy as np
import pytest
import torch

import test_gpu_kv as kv
import test_gpu_kvb as kvb
from paper_2505_13204_b200 import binding

pytestmark = pytest.mark.gpu
i32 = kvb.i32


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


# query heads, token rows, D, dtype: the split kernels (eight rows at a time and sixteen), one tile, two tiles
SHAPES = [(4, 1, 128, "bf16"), (4, 1, 64, "f32"), (8, 2, 64, "bf16"), (16, 2, 128, "f32"), (4, 2, 256, "bf16"), (4, 20, 128, "bf16"), (4, 20, 64, "bf16"), (4, 20, 256, "bf16"),
          (4, 50, 128, "bf16"), (4, 50, 64, "bf16")]


@pytest.mark.parametrize("Hq,new,D,dtype", SHAPES)
@pytest.mark.parametrize("lens", ["one long", "many short"])          # segments that the CTAs share, and whole ones
@pytest.mark.parametrize("bits", [4, 8])
def test_rows_with_nan(ctx, Hq, new, D, dtype, lens, bits):
    g = torch.Generator(device="cuda").manual_seed(Hq + new)
    B, n = (1, 12000) if lens == "one long" else (400, 130)
    per = -(-n // 64)
    pages = (binding.kvb_pages if bits == 8 else binding.kv_pages)(per, 1, D)        # (the sequences of a batch have the same pages)
    k = torch.randn((n, 1, D), generator=g, device="cuda")
    v = torch.randn((n, 1, D), generator=g, device="cuda")
    row = torch.arange(per, dtype=torch.int32, device="cuda")[None].contiguous()
    zero = torch.zeros(n, dtype=torch.int32, device="cuda")
    if bits == 8:
        ctx.kvb_write(pages, k[:, :0], k, v, row, i32([0]), i32([n]), zero, rows_per_seq=n, outputs=dict(q=k[:, :0]))
    else:
        ctx.kv_write(pages, k[:, :0], k, v, torch.arange(n, dtype=torch.int32, device="cuda"), zero, outputs=dict(q=k[:, :0]))
    table = row.repeat(B, 1)
    T = B * new
    q = torch.randn((T, Hq, D), generator=g, device="cuda").to(kvb.DT[dtype])
    bad = torch.zeros((T, Hq), dtype=torch.bool, device="cuda")
    for t, h, d in ((0, 0, 0), (T - 1, Hq - 1, D - 1), (T // 2, 1, 17)):
        q[t, h, d] = float("nan")
        bad[t, h] = True
    if bits == 8:                                        # (infinities likewise; all the row's products may be -inf)
        q[T // 2, 2] = 0
        q[T // 2, 2, 3] = float("inf")
        bad[T // 2, 2] = True
    fresh = [new] * B
    if new > 1:
        fresh[0] = new - 1                               # the first sequence has a row without a token
        q[new - 1] = float("nan")
    attend = ctx.kvb_attend if bits == 8 else ctx.kv_attend
    o = attend(q, pages, table, i32([n - new] * B), i32([n - new + f for f in fresh]), rows_per_seq=new, want_lse=True)
    assert ctx.poll_status() == 0
    none = torch.zeros(T, dtype=torch.bool, device="cuda")
    if new > 1:
        none[new - 1] = True
        bad[new - 1] = False
    assert (o["out"][none] == 0).all() and torch.isneginf(o["lse"][none]).all()
    assert torch.isnan(o["out"][bad]).all() and torch.isnan(o["lse"][bad]).all()
    good = ~bad & ~none[:, None]
    assert torch.isfinite(o["out"][good]).all() and torch.isfinite(o["lse"][good]).all()
