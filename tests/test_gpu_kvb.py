"""The paged 8-bit cache on the GPU against the plain model of kvb_ref.py."""
import numpy as np
import pytest
import torch

import kv_ref
import kvb_ref as ref
from paper_2505_13204_b200 import binding

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}          # unit roundoffs
PAGE = ref.PAGE


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


def tables(rng, lens, extra=2):
    """Block tables over a shuffled pool: lists, the padded array, pages of the pool."""
    need = [-(-int(n) // PAGE) for n in lens]
    pool = sum(need) + extra
    order, at, rows = rng.permutation(pool), 0, []
    for n in need:
        rows.append([int(x) for x in order[at:at + n]])
        at += n
    t = np.full((len(need), max(need + [1]) + 1), -1, np.int32)
    for b, r in enumerate(rows):
        t[b, :len(r)] = r
    return rows, t, pool


def garbage(rng, pool, Hkv, D):
    """A pool that was in use: any codes, scales of ordinary sizes."""
    raw = rng.integers(0, 256, (pool, Hkv, ref.head_bytes(D))).astype(np.uint8)
    raw[:, :, 2 * PAGE * D:] = np.array([2.0 ** -7, 2.0 ** -8, np.nan, np.inf], "<f4").view(np.uint8)
    return raw


def fill(rng, raw, rows, lens, D, kscale=1.0, vscale=1.0):
    """Stores random tokens in 64-page bites of each sequence; returns their values, [n, Hkv, D] per sequence."""
    Hkv = raw.shape[1]
    ks, vs = [], []
    for b, n in enumerate(lens):
        n = int(n)
        k = (rng.standard_normal((n, Hkv, D)) * kscale).astype(np.float32)
        v = (rng.standard_normal((n, Hkv, D)) * vscale).astype(np.float32)
        if n:
            ref.write(raw, [rows[b]], [0], [n], [0], k, v, D)
        e = [ref.load(raw, rows[b][c // PAGE] * PAGE + c % PAGE, D) for c in range(n)]
        ks.append(np.asarray([x[0] for x in e]).reshape(n, Hkv, D))
        vs.append(np.asarray([x[1] for x in e]).reshape(n, Hkv, D))
    return ks, vs


# ---- store -----------------------------------------------------------------------------------------------

WRITES = [  # sequences, new tokens (most), longest context, query heads, key heads, D, dtype, rotated channels, neighbours, norm, padded
    (1, 1, 0, 1, 1, 64, "bf16", 64, False, True, True), (3, 1, 200, 8, 2, 128, "bf16", 128, False, True, True),
    (4, 9, 130, 8, 2, 128, "f32", 128, False, True, True), (2, 150, 70, 4, 2, 64, "bf16", 32, True, False, False),
    (3, 70, 64, 6, 3, 128, "f32", 64, False, True, False), (2, 130, 1, 2, 1, 256, "bf16", 256, False, True, False),
    (5, 5, 63, 7, 1, 256, "f32", 128, True, True, True), (1, 300, 300, 5, 5, 64, "f32", 0, False, True, False),
    (40, 3, 500, 4, 2, 128, "bf16", 128, True, True, True), (300, 2, 40, 2, 1, 64, "bf16", 64, False, True, False),
    # more pages than CTAs at a time, few rows each (a warp per page), in one pass and in several; and many rows each
    (160, 5, 300, 4, 2, 128, "bf16", 128, False, True, True), (160, 9, 130, 2, 1, 64, "f32", 64, False, True, False),
    (160, 3, 70, 2, 1, 256, "bf16", 256, False, True, True), (160, 30, 100, 3, 1, 64, "bf16", 32, True, True, False),
    (160, 40, 60, 2, 1, 256, "f32", 128, False, False, False), (160, 30, 100, 2, 1, 128, "f32", 0, False, True, False),
    (120, 90, 64, 2, 1, 64, "bf16", 64, False, True, False)]


@pytest.mark.parametrize("B,new,longest,Hq,Hkv,D,dtype,rot,inter,norm,padded", WRITES)
def test_write(ctx, B, new, longest, Hq, Hkv, D, dtype, rot, inter, norm, padded):
    rng = np.random.default_rng(B * 13 + new + D)
    cached = rng.integers(0, longest + 1, B)
    cached[0] = longest
    fresh = rng.integers(0, new + 1, B)
    fresh[0] = new
    rows, table, pool = tables(rng, cached + fresh)
    raw = garbage(rng, pool, Hkv, D)
    fill(rng, raw, rows, cached, D, kscale=0.5)
    offs = np.arange(B + 1) * new if padded else np.concatenate([[0], np.cumsum(fresh)])
    T = int(offs[-1]) if padded else int(offs[-1]) + 1       # packed: a row that no sequence owns
    # heads inside a fused projection; sizes differ by token, so that scales grow in the middle of pages
    buf = rng.standard_normal((T, Hq + 2 * Hkv, D)) * 2.0 ** rng.integers(-2, 3, (T, 1, 1))
    buf = torch.as_tensor(buf.astype(np.float32)).to(DT[dtype]).cuda()
    q, k, v = buf[:, :Hq], buf[:, Hq:Hq + Hkv], buf[:, Hq + Hkv:]
    w = [torch.as_tensor((1 + 0.1 * rng.standard_normal(D)).astype(np.float32)).to(DT[dtype]).cuda() if norm else None for _ in range(2)]
    limit = longest + new + 1
    ang = np.arange(limit)[:, None] * 10000.0 ** (-np.arange(rot // 2) / max(1, rot // 2))
    cs = torch.as_tensor(np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)).cuda() if rot else None
    pos = np.full(T, -1, np.int32)
    for b in range(B):
        pos[offs[b]:offs[b] + fresh[b]] = cached[b] + np.arange(fresh[b])
    pages = torch.as_tensor(raw).cuda()
    o = ctx.kvb_write(pages, q, k, v, i32(table), i32(cached), i32(cached + fresh), i32(pos), None if padded else i32(offs), new if padded else 0,
                      cs, *w, eps=1e-6, interleaved=inter, keep_k=True)
    assert ctx.poll_status() == 0
    # what is stored is a function of the keys as normed and rotated in fp32: those of the 4-bit call in fp32, to the bit
    side = ctx.kv_write(torch.empty((T // PAGE + 1, Hkv, kv_ref.head_bytes(D)), dtype=torch.uint8, device="cuda"), *(x.float() for x in (q, k, v)),
                        i32(np.arange(T)), i32(pos), cs, *(None if x is None else x.float() for x in w), eps=1e-6, interleaved=inter, keep_k=True)
    assert ctx.poll_status() == 0
    used = torch.as_tensor(pos >= 0).cuda()
    assert torch.equal(o["q"], side["q"].to(DT[dtype]))
    assert torch.equal(o["k"][used], side["k"][used].to(DT[dtype]))
    ref.write(raw, rows, cached, cached + fresh, offs, side["k"].cpu().numpy(), v.float().cpu().numpy(), D)
    assert np.array_equal(pages.cpu().numpy(), raw)
    # and that is the formula's result
    eps, cos = float(np.float32(1e-6)), None if cs is None else f64(cs)
    for t in np.flatnonzero(pos >= 0)[:40]:
        for got, x, ww in ((f64(side["q"][t]), f64(q[t]), w[0]), (f64(side["k"][t]), f64(k[t]), w[1])):
            want = kv_ref.norm_rotate(x, None if ww is None else f64(ww), cos[pos[t]] if rot else None, rot, inter, eps)
            # fp32: the norm's factor 8 roundings, the products and the sum of a pair 4 more, relative to the pair's size
            assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 12 * 2.0 ** -24 * np.abs(want).max(-1, keepdims=True)).all()


@pytest.mark.parametrize("B,new", [(3, 70), (160, 12)])
@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "f32"), (256, "bf16")])
def test_write_of_unaligned_rows(ctx, B, new, D, dtype):
    rng = np.random.default_rng(B + D)
    cached, T = rng.integers(0, 100, B), B * new
    rows, table, pool = tables(rng, cached + new)
    raw = garbage(rng, pool, 1, D)
    x = torch.as_tensor(rng.standard_normal((T, 3 * D)).astype(np.float32)).to(DT[dtype]).cuda()
    flat = torch.zeros(T * (3 * D + 1) + 1, dtype=DT[dtype], device="cuda")
    odd = flat[1:].view(T, 3 * D + 1)[:, :3 * D]          # every row starts somewhere else
    odd.copy_(x)
    ang = np.arange(200)[:, None] * 10000.0 ** (-np.arange(D // 2) / (D // 2))
    cs = torch.as_tensor(np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)).cuda()
    pos = i32((cached[:, None] + np.arange(new)).ravel())
    got = []
    for y in (x, odd):
        pages = torch.as_tensor(raw).cuda()
        q, k, v = (y[:, i * D:(i + 1) * D].unflatten(1, (1, D)) for i in range(3))
        o = ctx.kvb_write(pages, q, k, v, i32(table), i32(cached), i32(cached + new), pos, None, new, cs, keep_k=True)
        assert ctx.poll_status() == 0
        got.append((pages, o["q"], o["k"]))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_write_of_rows_that_are_not_finite_or_have_no_position(ctx):
    rng = np.random.default_rng(6)
    D, n = 128, 70
    rows, table, pool = tables(rng, [n])
    raw = garbage(rng, pool, 1, D)
    x = torch.as_tensor(rng.standard_normal((n, 4, D)).astype(np.float32)).cuda()
    q, k, v = x[:, :2], x[:, 2:3], x[:, 3:]
    k[1, 0, 17], k[2, 0, 3], v[3, 0, 127], v[66, 0, 0] = float("nan"), float("inf"), float("-inf"), float("nan")
    k[4, 0, 0], v[5, 0, 1] = 3.4e38, -3.4e38             # finite, however large
    v[6] = 0
    q[5, 0, 0] = float("nan")
    pos = np.arange(n, dtype=np.int32)
    pos[7] = -1                                          # placed, but without a position: zeros
    pages = torch.as_tensor(raw).cuda()
    o = ctx.kvb_write(pages, q, k, v, i32(table), i32([0]), i32([n]), i32(pos), i32([0, n]))
    assert ctx.poll_status() == binding.STATUS_BAD_ROW
    assert torch.isnan(o["q"][5, 0, 0]) and torch.isfinite(o["q"][6]).all() and (o["q"][7] == 0).all()
    ref.write(raw, rows, [0], [n], [0], k.cpu().numpy(), v.cpu().numpy(), D, placed=pos >= 0)
    assert np.array_equal(pages.cpu().numpy(), raw)


def test_write_in_steps_keeps_older_entries(ctx):
    """Token by token and in bites, with rows that are larger each time: the bytes follow the model's; what was stored moves by half a step
    of the final scale's subnormals at most."""
    rng = np.random.default_rng(7)
    D, Hkv, total = 64, 2, 200
    rows, table, pool = tables(rng, [total])
    raw = garbage(rng, pool, Hkv, D)
    pages = torch.as_tensor(raw).cuda()
    x = (rng.standard_normal((total, 2 * Hkv, D)) * np.exp(np.arange(total) / 20.0)[:, None, None]).astype(np.float32)
    at = 0
    for n in [1, 1, 1, 5, 20, 36, 1, 70, 65]:
        part = torch.as_tensor(x[at:at + n]).cuda()
        ctx.kvb_write(pages, part[:, :1], part[:, :Hkv], part[:, Hkv:], i32(table), i32([at]), i32([at + n]), i32(at + np.arange(n)), rows_per_seq=n)
        ref.write(raw, rows, [at], [at + n], [0], x[at:at + n, :Hkv], x[at:at + n, Hkv:], D)
        at += n
    assert ctx.poll_status() == 0 and np.array_equal(pages.cpu().numpy(), raw)
    e = ctx.kvb_read(pages, i32([rows[0][c // PAGE] * PAGE + c % PAGE for c in range(total)]), D, torch.float32)
    for half, got in enumerate((f64(e["k"]), f64(e["v"]))):
        for h in range(Hkv):
            for c in range(total):
                s = 2.0 ** ref.Block(raw[rows[0][c // PAGE], h], half, D).e
                want = x[c, half * Hkv + h].astype(np.float64)
                assert (np.abs(got[c, h] - want) <= 2.0 ** -4 * np.abs(want) + s * 2.0 ** -9).all()


def test_write_reports_bad_pages_and_positions_and_stays_in_bounds(ctx):
    rng = np.random.default_rng(8)
    D = 64
    x = torch.as_tensor(rng.standard_normal((8, 3, D)).astype(np.float32)).cuda()
    q, k, v = x[:, :1], x[:, 1:2], x[:, 2:]
    cs = torch.ones((10, D), device="cuda")
    pages = torch.full((3, 1, ref.head_bytes(D)), 9, dtype=torch.uint8, device="cuda")
    table = i32([[3, -1], [-5, 0]])
    o = ctx.kvb_write(pages, q, k, v, table, i32([0, 60]), i32([4, 64]), i32([0, 1, 2, 3, 4, 10, -7, 7]), rows_per_seq=4, cos_sin=cs)
    assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS | binding.STATUS_ID_RANGE
    assert (pages == 9).all() and (o["q"][5] == 0).all() and (o["q"][6] == 0).all() and (o["q"][0] != 0).any()
    # a sequence that claims more tokens than it has rows, offsets past the rows, a table that is too narrow
    for kv, offs in (([100, 0], [0, 4, 8]), ([4, 4], [0, 4, 9]), ([4, 4], [-3, 4, 8])):
        ctx.kvb_write(pages, q, k, v, i32([[0], [1]]), i32([0, 0]), i32(kv), i32(np.arange(8)), i32(offs))
        ctx.poll_status()
    assert (pages[2] == 9).all()
    ctx.kvb_write(pages, q, k, v, i32([[0]]), i32([62]), i32([70]), i32(np.arange(8)), rows_per_seq=8)
    assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS and (pages[2] == 9).all()


# ---- attention -----------------------------------------------------------------------------------------

class Pool:
    """A cache with random entries for B sequences, on both sides.  Past the sequences' ends: NaN codes and infinite scales."""

    def __init__(self, rng, kv_len, Hkv, D, kscale=1.0, vscale=1.0):
        self.kv_len, self.D, self.Hkv = [int(x) for x in kv_len], D, Hkv
        self.rows, self.table, pool = tables(rng, self.kv_len)
        raw = np.full((pool, Hkv, ref.head_bytes(D)), 0x7F, np.uint8)
        raw[:, :, 2 * PAGE * D:] = np.array([np.inf, np.nan, np.nan, np.inf], "<f4").view(np.uint8)
        self.k, self.v = fill(rng, raw, self.rows, self.kv_len, D, kscale, vscale)
        self.pages = torch.as_tensor(raw).cuda()


def _visible(cached, i, parent):
    if parent is None:
        return list(range(cached + i + 1))
    return list(range(cached)) + [cached + x for x in ref.path_of(i, parent)]


def limits(want, lse, size, qmax, kl1, scale, vspread, vmax, f32):
    """How far the result and the lse may be off.  `size`: largest sum of |q_d k_d| (scaled); qmax: the row's largest query; kl1: largest sum of
    |k_d|.  A product's fp32 sum: at most 2^-21 of the sum of its terms' sizes (fp32 queries: their halves leave out 2^-22 of each
    term as well), carried into base 2 and the exponential with 2^-21 more of the exponent's size.  bf16 queries of many rows are
    two e4m3 numbers: what lies below 2^-17 of the row's largest is left out."""
    wrong = size * 2.0 ** -20 + 2.0 ** -20 + np.abs(lse) * 2.0 ** -22
    if not f32:
        wrong = wrong + qmax * kl1 * scale * 2.0 ** -17
    # the weights move by that relative to each other; probabilities have 11 bits (fp32: 22)
    lim = vspread * (2 * wrong + (2.0 ** -21 if f32 else 2.0 ** -11) + 2.0 ** -20) + 2.0 ** -20 * vmax
    return lim, wrong + 2.0 ** -21 * np.abs(lse)


def check_attend(ctx, pool, q, cached, offs, rows, parent, scale=None):
    D = pool.D
    s = 1.0 / np.sqrt(D) if scale is None else scale
    o = ctx.kvb_attend(q, pool.pages, i32(pool.table), i32(cached), i32(pool.kv_len), tok_offsets=None if rows else i32(offs),
                       rows_per_seq=rows, node_parent=None if parent is None else i32(parent), scale=0.0 if scale is None else scale,
                       want_lse=True)
    assert ctx.poll_status() == 0
    got, lse, qn = f64(o["out"]), f64(o["lse"]), f64(q)
    f32 = q.dtype == torch.float32
    G = q.shape[1] // pool.Hkv
    for b in range(len(cached)):
        fresh = pool.kv_len[b] - cached[b]
        for t in range(offs[b], offs[b + 1]):
            i = t - offs[b]
            par = None if parent is None else parent.reshape(-1)[offs[b]:offs[b + 1]]
            vis = _visible(cached[b], i, par) if i < fresh else []
            want, wl, size = kv_ref.attend(qn[t], pool.k[b], pool.v[b], vis, s)
            if not vis:
                assert (got[t] == 0).all() and np.isneginf(lse[t]).all()
                continue
            kl1 = np.abs(pool.k[b][vis]).sum(-1).max(0).repeat(G)
            lim, lim_lse = limits(want, wl, size, np.abs(qn[t]).max(-1), kl1, abs(s), np.ptp(pool.v[b][vis], axis=(0, 2)).repeat(G), np.abs(pool.v[b][vis]).max(), f32)
            lim = lim[:, None] + np.abs(want) * HALF["f32" if f32 else "bf16"] + 1e-44
            err = np.abs(got[t] - want)
            assert (err <= lim).all(), (b, i, float((err / lim).max()))
            assert (np.abs(lse[t] - wl) <= lim_lse).all(), (b, i, float((np.abs(lse[t] - wl) / lim_lse).max()))


def tree(rng, n):
    return np.array([-1] + [int(rng.integers(0, i)) for i in range(1, n)], np.int32)


ATTENDS = [  # sequences, new tokens (most), longest context, query heads, key heads, D, dtype
    (1, 1, 0, 1, 1, 64, "bf16"), (1, 1, 1, 4, 1, 128, "bf16"), (3, 1, 200, 8, 2, 128, "bf16"), (2, 1, 700, 5, 5, 64, "f32"),
    (2, 1, 130, 28, 4, 128, "f32"), (1, 1, 1500, 16, 2, 128, "bf16"), (5, 9, 150, 8, 2, 128, "bf16"), (3, 17, 140, 7, 1, 64, "bf16"),
    (2, 33, 64, 8, 2, 128, "bf16"), (2, 33, 65, 4, 4, 256, "bf16"), (2, 20, 63, 6, 2, 256, "f32"), (1, 70, 100, 8, 1, 128, "bf16"),
    (2, 150, 30, 4, 2, 64, "bf16"), (1, 200, 1, 2, 1, 128, "f32"), (1, 300, 500, 2, 1, 128, "bf16"), (9, 2, 128, 40, 8, 64, "bf16"),
    (2, 90, 127, 3, 1, 256, "bf16"), (1, 70, 100, 8, 1, 256, "bf16"), (5, 9, 300, 6, 2, 256, "bf16"), (1, 300, 500, 2, 1, 256, "bf16")]


@pytest.mark.parametrize("B,new,longest,Hq,Hkv,D,dtype", ATTENDS)
@pytest.mark.parametrize("trees", [False, True])
def test_attend(ctx, B, new, longest, Hq, Hkv, D, dtype, trees):
    rng = np.random.default_rng(B * 31 + new + longest + Hq)
    cached = rng.integers(0, longest + 1, B)
    cached[0] = longest
    fresh = rng.integers(0, new + 1, B)                 # some sequences have fewer nodes than rows, some none
    fresh[0] = new
    pool = Pool(rng, cached + fresh, Hkv, D)
    rows = new if trees else 0
    offs = np.arange(B + 1) * new if trees else np.concatenate([[0], np.cumsum(fresh)])
    parent = None
    if trees:
        parent = np.full((B, new), -1, np.int32)
        for b in range(B):
            if fresh[b]:
                parent[b, :fresh[b]] = tree(rng, fresh[b])
    T = int(offs[-1])
    # rows of q inside a wider buffer
    q = torch.as_tensor(rng.standard_normal((T, Hq + 1, D)).astype(np.float32) * 1.5).to(DT[dtype]).cuda()[:, :Hq]
    check_attend(ctx, pool, q, cached, offs, rows, parent)


LONG = [  # sequences, new tokens, contexts from .. to, query heads, key heads, D, dtype, trees: every CTA passes many pages and segments
    (64, 1, 100, 3000, 28, 4, 128, "bf16", False), (33, 1, 1, 4000, 16, 8, 64, "bf16", False), (40, 1, 500, 1500, 8, 8, 256, "bf16", False),
    (64, 2, 0, 2000, 32, 4, 128, "bf16", True), (48, 33, 700, 2200, 16, 8, 128, "bf16", True), (60, 33, 0, 1800, 32, 8, 128, "bf16", True),
    (70, 17, 1, 2500, 10, 5, 64, "bf16", True), (3, 1500, 0, 700, 16, 4, 128, "bf16", False), (2, 1100, 300, 900, 16, 8, 64, "bf16", False),
    (9, 65, 1000, 1400, 8, 8, 128, "bf16", False), (40, 5, 600, 1900, 8, 2, 128, "f32", True), (20, 1, 10, 2000, 32, 8, 64, "f32", False),
    (2, 400, 100, 600, 4, 2, 256, "bf16", False), (1, 64, 20000, 20000, 8, 2, 128, "bf16", False),
    (1, 40, 20000, 20000, 4, 2, 256, "bf16", False), (48, 33, 700, 2200, 8, 4, 256, "bf16", True), (3, 1500, 0, 700, 4, 1, 256, "bf16", False),
    (60, 3, 0, 1800, 16, 4, 256, "bf16", True)]


@pytest.mark.parametrize("B,new,lo,hi,Hq,Hkv,D,dtype,trees", LONG)
def test_attend_long(ctx, B, new, lo, hi, Hq, Hkv, D, dtype, trees):
    """Larger batches, stored by the call and read back through kvb_read (fp32, exact), against 64-bit sums on the same device."""
    g = torch.Generator(device="cuda")
    g.manual_seed(B * 7 + new)
    cached = torch.randint(lo, hi + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    kv = cached + new
    need = (kv + PAGE - 1) // PAGE
    P, n = int(need.max()) + 1, int(need.sum()) + 3
    start = torch.cumsum(need, 0) - need
    j = torch.arange(P, device="cuda")
    order = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
    table = torch.where(j < need[:, None], order[(start[:, None] + j).clamp(max=n - 1)], -1).to(torch.int32).contiguous()
    pages = binding.kvb_pages(n, Hkv, D)
    pages.fill_(255)
    off = torch.cumsum(kv, 0) - kv
    b = torch.repeat_interleave(torch.arange(B, device="cuda"), kv.long())
    t = torch.arange(b.numel(), device="cuda") - off[b]
    slots = (table[b, t // PAGE] * PAGE + t % PAGE).to(torch.int32)
    offs = torch.cat([off, kv.sum(0, keepdim=True)]).to(torch.int32)
    size = torch.exp2(torch.randint(-2, 3, (b.numel(), 1, 1), generator=g, device="cuda").float())
    k = torch.randn((b.numel(), Hkv, D), generator=g, device="cuda")
    v = torch.randn((b.numel(), Hkv, D), generator=g, device="cuda") * size
    ctx.kvb_write(pages, k[:, :0], k, v, table, torch.zeros_like(kv), kv, torch.zeros_like(slots), offs, outputs=dict(q=k[:, :0]))
    q = (torch.randn((B * new, Hq, D), generator=g, device="cuda") * 1.3).to(DT[dtype])
    rng = np.random.default_rng(B)
    parent = np.stack([tree(rng, new) for _ in range(B)]) if trees else None
    o = ctx.kvb_attend(q, pages, table, cached, kv, rows_per_seq=new, node_parent=None if parent is None else i32(parent), want_lse=True)
    assert ctx.poll_status() == 0
    for s in range(B):
        lo_t, n_t, c = int(off[s]), int(kv[s]), int(cached[s])
        e = ctx.kvb_read(pages, slots[lo_t:lo_t + n_t].contiguous(), D, torch.float32)
        ks, vs = e["k"].double(), e["v"].double()
        see = torch.zeros((new, n_t), dtype=torch.bool)
        see[:, :c] = True
        for i in range(new):
            see[i, [c + x for x in (range(i + 1) if parent is None else ref.path_of(i, parent[s]))]] = True
        see = see.cuda()
        qs = q[s * new:(s + 1) * new].double().view(new, Hkv, Hq // Hkv, D)
        w = torch.einsum("nhgd,thd->hgnt", qs, ks) / np.sqrt(D)
        sz = torch.einsum("nhgd,thd->hgnt", qs.abs(), ks.abs()).amax(-1) / np.sqrt(D)
        w = w.masked_fill(~see, float("-inf"))
        lse = torch.logsumexp(w, -1)
        want = torch.einsum("hgnt,thd->nhgd", torch.exp(w - lse[..., None]), vs).reshape(new, Hq, D)
        kl1 = ks.abs().sum(-1).amax(0)[:, None, None]
        spread = (vs.amax((0, 2)) - vs.amin((0, 2)))[:, None, None]
        lim, lim_lse = limits(None, lse.cpu().numpy(), sz.cpu().numpy(), qs.abs().amax(-1).permute(1, 2, 0).cpu().numpy(), kl1.cpu().numpy(), 1 / np.sqrt(D),
                              spread.cpu().numpy(), float(vs.abs().max()), dtype == "f32")
        got = f64(o["out"][s * new:(s + 1) * new])
        lim = lim.transpose(2, 0, 1).reshape(new, Hq)[..., None] + np.abs(f64(want)) * HALF[dtype]
        err = np.abs(got - f64(want))
        assert (err <= lim).all(), (s, float((err / lim).max()))
        gl, le = f64(o["lse"][s * new:(s + 1) * new]), f64(lse.permute(2, 0, 1).reshape(new, Hq))
        assert (np.abs(gl - le) <= lim_lse.transpose(2, 0, 1).reshape(new, Hq)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,D", [(3, 128), (60, 128), (60, 256)])                   # few rows, and many
def test_attend_with_large_products_and_values_of_any_size(ctx, dtype, G, D):
    """Sharp softmaxes, scales of the pages far from 1 and from each other."""
    rng = np.random.default_rng(3)
    for kscale, vscale, qscale in ((4.0, 1e-4, 3.0), (0.01, 3e4, 1.0), (1.0, 1.0, 1e3), (1e-3, 1.0, 1e-3), (1.0, 1e30, 1.0), (1e-15, 1e-25, 1e15), (300.0, 1.0, 300.0)):
        pool = Pool(rng, [300, 70], 2, D, kscale, vscale)
        q = torch.as_tensor(rng.standard_normal((2, 2 * G, D)).astype(np.float32) * qscale).to(DT[dtype]).cuda()
        check_attend(ctx, pool, q, [299, 69], [0, 1, 2], 1, None)


@pytest.mark.parametrize("G,D", [(3, 64), (60, 64), (60, 256)])
def test_attend_where_a_pages_values_dwarf_the_others(ctx, G, D):
    rng = np.random.default_rng(4)
    for sizes in ((1.0, 1e5, 1e-5), (1e-6, 1.0, 1e6), (1e4, 1.0, 1e-8)):
        pool = Pool(rng, [0], 1, D)
        pool.rows, pool.table, n = tables(rng, [190])
        raw = np.full((n, 1, ref.head_bytes(D)), 0x7F, np.uint8)
        k = rng.standard_normal((190, 1, D)).astype(np.float32)
        v = rng.standard_normal((190, 1, D)).astype(np.float32)
        for pg, s in enumerate(sizes):
            v[pg * PAGE:(pg + 1) * PAGE] *= s
        ref.write(raw, pool.rows, [0], [190], [0], k, v, D)
        e = [ref.load(raw, pool.rows[0][c // PAGE] * PAGE + c % PAGE, D) for c in range(190)]
        pool.k, pool.v, pool.kv_len = [np.asarray([x[0] for x in e])], [np.asarray([x[1] for x in e])], [190]
        pool.pages = torch.as_tensor(raw).cuda()
        for dtype in ("bf16", "f32"):
            q = torch.as_tensor(rng.standard_normal((1, G, D)).astype(np.float32)).to(DT[dtype]).cuda()
            check_attend(ctx, pool, q, [189], [0, 1], 1, None)


@pytest.mark.parametrize("G,D", [(2, 64), (64, 64), (64, 256)])
def test_attend_scale_and_unaligned_queries(ctx, G, D):
    rng = np.random.default_rng(8)
    pool = Pool(rng, [90, 10], 2, D)
    for dtype in ("bf16", "f32"):
        buf = torch.as_tensor(rng.standard_normal((2, 2 * G * D + 3)).astype(np.float32)).to(DT[dtype]).cuda()
        q = buf[:, 1:1 + 2 * G * D].unflatten(1, (2 * G, D))
        check_attend(ctx, pool, q, [89, 9], [0, 1, 2], 1, None, scale=0.37)


@pytest.mark.parametrize("new,Hq", [(1, 8), (40, 8)])
def test_attend_is_the_same_on_a_second_call_another_stream_and_from_a_graph(ctx, new, Hq):
    rng = np.random.default_rng(9)
    pool = Pool(rng, [900 + new, 40 + new, 700 + new], 2, 128)
    q = torch.as_tensor(rng.standard_normal((3 * new, Hq, 128)).astype(np.float32)).to(torch.bfloat16).cuda()
    args = (q, pool.pages, i32(pool.table), i32([900, 40, 700]), i32(pool.kv_len))
    one = ctx.kvb_attend(*args, rows_per_seq=new)["out"]
    assert torch.equal(one, ctx.kvb_attend(*args, rows_per_seq=new)["out"])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ctx.set_stream(side)
    try:
        with torch.cuda.stream(side):
            assert torch.equal(one, ctx.kvb_attend(*args, rows_per_seq=new)["out"])
            side.synchronize()
            graph, out = torch.cuda.CUDAGraph(), torch.empty_like(one)
            with torch.cuda.graph(graph, stream=side):
                ctx.kvb_attend(*args, rows_per_seq=new, outputs=dict(out=out))
            for _ in range(3):
                out.zero_()
                graph.replay()
                side.synchronize()
                assert torch.equal(out, one)
    finally:
        ctx.set_stream(torch.cuda.current_stream())


@pytest.mark.parametrize("rows", [5, 60])
def test_attend_reports_bad_tables_and_parents(ctx, rows):
    rng = np.random.default_rng(10)
    n = 2 * rows
    pool = Pool(rng, [65 + rows, rows], 1, 64)
    q = torch.as_tensor(rng.standard_normal((n, 2, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
    for bad in (pool.pages.shape[0] + 5, -2, -1, 2 ** 30):
        table = pool.table.copy()
        table[0, 0] = bad
        o = ctx.kvb_attend(q, pool.pages, i32(table), i32([65, 0]), i32(pool.kv_len), rows_per_seq=rows, want_lse=True)
        assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS
        # what lies in that page is not seen; the other sequence is as it was
        keep = [c for c in range(64, 66)]
        want, wl, _ = kv_ref.attend(f64(q[0]), pool.k[0], pool.v[0], keep, 0.125)
        assert np.abs(f64(o["out"][0]) - want).max() <= 0.02 * np.abs(pool.v[0]).max() and np.abs(f64(o["lse"][0]) - wl).max() < 0.01
        want, _, _ = kv_ref.attend(f64(q[rows]), pool.k[1], pool.v[1], [0], 0.125)
        assert np.abs(f64(o["out"][rows]) - want).max() <= 2.0 ** -8 * np.abs(want).max()
    parent = np.full((2, rows), -1, np.int32)
    parent[0, 1], parent[1, 2] = 1, 700
    ctx.kvb_attend(q, pool.pages, i32(pool.table), i32([65, 0]), i32(pool.kv_len), rows_per_seq=rows, node_parent=i32(parent))
    assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS
    table = pool.table[:, :1].copy()                     # a table that is too narrow for what is cached
    o = ctx.kvb_attend(q, pool.pages, i32(table), i32([65, 0]), i32(pool.kv_len), rows_per_seq=rows)
    assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS and torch.isfinite(o["out"]).all()


@pytest.mark.parametrize("rows,D", [(1, 128), (30, 128), (30, 256)])
def test_rows_that_no_sequence_owns_give_zeros(ctx, rows, D):
    rng = np.random.default_rng(11)
    pool = Pool(rng, [64 + rows, rows], 2, D)
    T = 2 * rows + 7
    q = torch.as_tensor(rng.standard_normal((T, 8, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    q[-2:] = float("nan")
    out = dict(out=torch.full((T, 8, D), 3.0, dtype=torch.bfloat16, device="cuda"), lse=torch.full((T, 8), 3.0, device="cuda"))
    offs = [3, 3 + rows, 3 + 2 * rows]
    ctx.kvb_attend(q, pool.pages, i32(pool.table), i32([64, 0]), i32(pool.kv_len), tok_offsets=i32(offs), outputs=out)
    assert ctx.poll_status() == 0
    owned = np.zeros(T, bool)
    owned[3:3 + 2 * rows] = True
    got, lse = f64(out["out"]), f64(out["lse"])
    assert (got[~owned] == 0).all() and np.isneginf(lse[~owned]).all() and np.isfinite(lse[owned]).all() and (np.abs(got[owned]).max((1, 2)) > 0).all()
    # no sequence at all
    ctx.kvb_attend(q, pool.pages, i32(pool.table)[:0], i32([0])[:0], i32([0])[:0], tok_offsets=i32([0]), outputs=out)
    assert (out["out"] == 0).all() and torch.isneginf(out["lse"]).all()


# ---- the accepted path, read-back -----------------------------------------------------------------------------

COMMITS = [(1, 9, 0, 1, 1, 64), (3, 9, 100, 2, 2, 128), (5, 33, 63, 3, 1, 256), (2, 150, 64, 2, 3, 128), (8, 70, 300, 1, 2, 64), (1, 300, 7, 1, 1, 128)]


@pytest.mark.parametrize("B,new,longest,layers,Hkv,D", COMMITS)
@pytest.mark.parametrize("packed", [False, True])
def test_commit(ctx, B, new, longest, layers, Hkv, D, packed):
    rng = np.random.default_rng(B * 5 + new + D)
    cached = rng.integers(0, longest + 1, B)
    cached[0] = longest
    fresh = rng.integers(1, new + 1, B)
    fresh[0] = new
    rows, table, pool = tables(rng, cached + fresh)
    raw = np.stack([garbage(rng, pool, Hkv, D) for _ in range(layers)])
    raw[..., :2 * PAGE * D] &= 0x77                      # (no NaN codes)
    for one in raw:                                      # scales of all sizes, page by page
        for pg in range(pool):
            for h in range(Hkv):
                for half in range(2):
                    ref.Block(one[pg, h], half, D).e = int(rng.integers(-9, 3))
    parent = np.full((B, new), -1, np.int32)
    best = np.zeros(B, np.int32)
    for b in range(B):
        parent[b, :fresh[b]] = tree(rng, fresh[b]) if b % 3 else np.maximum(np.arange(fresh[b]) - 1 - rng.integers(0, 2, fresh[b]), np.where(np.arange(fresh[b]) > 0, 0, -1))
        best[b] = rng.integers(0, fresh[b]) if b else fresh[b] - 1
    if B > 2:
        best[2] = -1
    offs = np.concatenate([[0], np.cumsum(fresh)])
    par = np.concatenate([parent[b, :fresh[b]] for b in range(B)]) if packed else parent
    pages = torch.as_tensor(raw).cuda()
    new_len = ctx.kvb_commit(pages, i32(table), i32(cached), i32(cached + fresh), i32(best), i32(par), i32(offs) if packed else None)
    assert ctx.poll_status() == 0
    for b in range(B):
        path = ref.path_of(best[b], parent[b]) if best[b] >= 0 else []
        assert int(new_len[b]) == cached[b] + len(path)
        for one in raw:
            if path:
                ref.commit(one, rows[b], int(cached[b]), path, D)
    assert np.array_equal(pages.cpu().numpy(), raw)


def test_commit_reports_bad_parents_and_moves_nothing(ctx):
    rng = np.random.default_rng(12)
    raw = garbage(rng, 2, 1, 64)[None]
    pages = torch.as_tensor(raw).cuda()
    for parent, best, table in (([-1, 2, 1, 0], 2, [[0, 1]]), ([-1, 0, 0, 1], 3, [[0, 7]]), ([-1, 0, -5, 1], 2, [[0, 1]])):
        new_len = ctx.kvb_commit(pages, i32(table), i32([62]), i32([66]), i32([best]), i32([parent]))
        assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS and new_len.tolist() == [62]
    assert np.array_equal(pages.cpu().numpy(), raw)
    # (parents that the path does not come by are not looked at: 3 hangs on the root)
    assert ctx.kvb_commit(pages, i32([[0, 1]]), i32([62]), i32([66]), i32([3]), i32([[-1, 2, 1, 0]])).tolist() == [64]
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_read(ctx, D, dtype):
    rng = np.random.default_rng(D)
    raw = garbage(rng, 5, 3, D)
    raw[1, :, 2 * PAGE * D:2 * PAGE * D + 8] = np.array([2.0 ** -64, 2.0 ** 100], "<f4").view(np.uint8)
    pages = torch.as_tensor(raw).cuda()
    slots = rng.integers(0, 5 * PAGE, 333)
    slots[5] = -1
    e = ctx.kvb_read(pages, i32(slots), D, DT[dtype])
    assert ctx.poll_status() == 0
    for i, s in enumerate(slots):
        want = ref.load(raw, int(s), D) if s >= 0 else [np.zeros((3, D))] * 2
        for got, w in zip((e["k"][i], e["v"][i]), want):
            assert np.array_equal(f64(got), w, equal_nan=True)
    o = dict(k=torch.empty((3, 3, D), dtype=DT[dtype], device="cuda"), v=torch.empty((3, 3, D), dtype=DT[dtype], device="cuda"))
    ctx.kvb_read(pages, i32([5 * PAGE, -2, 7]), D, DT[dtype], outputs=o)
    assert ctx.poll_status() == binding.STATUS_ID_RANGE and (o["k"][:2] == 0).all() and (o["v"][:2] == 0).all()


# ---- refusals ------------------------------------------------------------------------------------------------------

def test_calls_refuse_what_does_not_fit(ctx):
    t = i32([[0, 1]])
    z, one = i32([0]), i32([4])
    pages = torch.zeros((2, 2, ref.head_bytes(64)), dtype=torch.uint8, device="cuda")
    x = torch.zeros((4, 6, 64), dtype=torch.bfloat16, device="cuda")
    q, k, v = x[:, :2], x[:, 2:4], x[:, 4:]
    pos = i32(np.arange(4))
    ok = dict(rows_per_seq=4)
    ctx.kvb_write(pages, q, k, v, t, z, one, pos, **ok)
    ctx.kvb_attend(q, pages, t, z, one, **ok)
    four = binding.kv_pages(2, 2, 64)
    with pytest.raises((AssertionError, binding.AasdError)):
        ctx.kvb_write(four, q, k, v, t, z, one, pos, **ok)            # a 4-bit pool
    with pytest.raises((AssertionError, binding.AasdError)):
        ctx.kv_attend(q, pages, t, z, one, **ok)                      # an 8-bit pool in the 4-bit call
    for bad in (dict(rows_per_seq=3), dict(rows_per_seq=-1)):
        with pytest.raises(binding.AasdError):
            ctx.kvb_write(pages, q, k, v, t, z, one, pos, **bad)
        with pytest.raises(binding.AasdError):
            ctx.kvb_attend(q, pages, t, z, one, **bad)
    with pytest.raises(binding.AasdError):
        ctx.kvb_write(pages, q, k, v, t, z, one, pos[:3], **ok)
    with pytest.raises(binding.AasdError):
        ctx.kvb_write(pages, q, k, v, t, z[:0], one, pos, **ok)
    with pytest.raises(binding.AasdError):
        ctx.kvb_write(pages, q, k, v, t, z, one, pos)                 # packed, without offsets
    with pytest.raises(AssertionError):
        ctx.kvb_write(pages, q, k, v, t.long(), z, one, pos, **ok)
    with pytest.raises(AssertionError):
        ctx.kvb_write(pages, q, k.float(), v, t, z, one, pos, **ok)
    with pytest.raises(binding.AasdError):
        ctx.kvb_write(pages, q.half(), k.half(), v.half(), t, z, one, pos, **ok)
    with pytest.raises(binding.AasdError):
        ctx.kvb_write(pages, q, k, v, t, z, one, pos, eps=-1.0, **ok)
    with pytest.raises(binding.AasdError):
        ctx.kvb_attend(q, pages, t, z, one, scale=float("nan"), **ok)
    with pytest.raises(binding.AasdError):
        ctx.kvb_attend(x[:, :3], pages, t, z, one, **ok)              # query heads that are no multiple
    with pytest.raises(binding.AasdError):
        ctx.kvb_commit(pages[None], t, z, one, i32([0]), i32([[-1, 0, 1, 2]]), outputs=z)
    with pytest.raises(AssertionError):
        ctx.kvb_read(pages, z, 128)
    assert ctx.poll_status() == 0


def test_pools_past_4_gb(ctx):
    """Pages whose bytes lie behind 2^32: store, read, attention, a moved path, a copied page."""
    D, Hkv = 128, 8
    n = (5 << 30) // (Hkv * ref.head_bytes(D))
    pages = binding.kvb_pages(n, Hkv, D, layers=1)
    rng = np.random.default_rng(13)
    x = torch.as_tensor(rng.standard_normal((70, 16 + 2 * Hkv, D)).astype(np.float32)).bfloat16().cuda()
    q, k, v = x[:, :16], x[:, 16:16 + Hkv], x[:, 16 + Hkv:]
    got = []
    for table in ([[0, 1]], [[n - 1, n - 2]]):
        t = i32(table)
        o = ctx.kvb_write(pages[0], q, k, v, t, i32([0]), i32([70]), i32(np.arange(70)), rows_per_seq=70)
        slots = i32([table[0][c // PAGE] * PAGE + c % PAGE for c in range(70)])
        e = ctx.kvb_read(pages[0], slots, D)
        a = ctx.kvb_attend(o["q"], pages[0], t, i32([0]), i32([70]), rows_per_seq=70)["out"]
        one = ctx.kvb_attend(o["q"][69:], pages[0], t, i32([69]), i32([70]), rows_per_seq=1)["out"]
        parent = np.full((1, 6), -1, np.int32)
        parent[0, 3], parent[0, 5] = 0, 3
        ctx.kvb_commit(pages, t, i32([60]), i32([66]), i32([5]), i32(parent))
        m = ctx.kvb_read(pages[0], slots[60:63].contiguous(), D)
        got.append((e["k"], e["v"], a, one, m["k"], m["v"]))
    for x, y in zip(*got):
        assert torch.equal(x, y)
    ctx.kv_copy(pages, i32([n - 1]), i32([3]))
    assert torch.equal(pages[0, 3], pages[0, n - 1]) and ctx.poll_status() == 0
