"""The paged 4-bit cache on the GPU against the plain model of kv_ref.py."""
import numpy as np
import pytest
import torch

import kv_ref as ref
from paper_2505_13204_b200 import binding

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
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


# ---- page tables -----------------------------------------------------------------------------------

def _books(rng, B, P, pool, held):
    pages = rng.permutation(pool)
    table, at = [], 0
    for b in range(B):
        table.append([int(x) for x in pages[at:at + held[b]]])
        at += held[b]
    return table, [int(x) for x in pages[at:]]


def _upload(table, stack, held, P, pool):
    t = np.full((len(table), P), -1, np.int32)
    for b, row in enumerate(table):
        t[b, :len(row)] = row
    f = np.full(pool, -1, np.int32)
    f[:len(stack)] = stack
    return i32(t), i32(np.asarray(held)), i32(f), i32([len(stack)])


def _check_plan(ctx, cached, new, table, held, stack, P, pool, rows, total, depth=None, full=None):
    dev = _upload(table, stack, held, P, pool)
    got = ctx.kv_plan(i32(cached), i32(new), *dev, total, rows_per_seq=rows, node_depth=None if depth is None else i32(depth))
    want = ref.plan(list(cached), list(new), table, held, stack, P, rows, total, depth)
    status = ctx.poll_status()
    assert status == (binding.STATUS_KV_FULL if want["full"] else 0)
    if full is not None:
        assert want["full"] == full
    after = [t.cpu().numpy() for t in _upload(table, stack, held, P, pool)]
    for name, d, w in zip(("block_table", "seq_pages", "free_pages", "n_free"), dev, after):
        assert np.array_equal(d.cpu().numpy(), w), name
    for k in ("kv_len", "tok_offsets", "slot_map", "positions"):
        assert np.array_equal(got[k].cpu().numpy(), want[k]), k
    return got, dev


PLANS = [  # sequences, widest table, longest sequence, padded rows (0: packed)
    (1, 1, 30, 1), (1, 40, 2000, 0), (5, 9, 500, 9), (32, 70, 4000, 33), (256, 20, 1100, 17), (300, 12, 700, 0),
    (1000, 3, 150, 3), (257, 40, 2300, 0), (2, 400, 25000, 0)]


@pytest.mark.parametrize("B,P,longest,rows", PLANS)
@pytest.mark.parametrize("kind", ["step", "fresh", "scarce", "churn"])
def test_plan(ctx, B, P, longest, rows, kind):
    rng = np.random.default_rng(B * 7 + P + len(kind))
    cached = rng.integers(0, longest + 1, B)
    new = rng.integers(0, rows + 1, B) if rows else rng.integers(0, max(2, longest // 3), B)
    if kind == "fresh":
        cached[:] = 0
        if not rows:
            new = rng.integers(0, longest, B)
    if kind == "churn":                                # sequences end, others shrink
        gone = rng.random(B) < 0.4
        cached[gone] = 0
        new[gone] = 0
    spare = rng.integers(0, 3, B) if kind != "churn" else rng.integers(0, P + 1, B)
    held = np.minimum(-(-cached // PAGE) + spare * (kind != "fresh"), P)
    cached = np.minimum(cached, held * PAGE)
    slack = 0 if kind == "scarce" else int((-(-(cached + new) // PAGE)).sum()) + 3
    pool = int(held.sum()) + max(1, slack if kind != "scarce" else B // 3)
    table, stack = _books(rng, B, P, pool, held)
    total = B * rows if rows else int(new.sum()) + int(rng.integers(0, 5))
    depth = rng.integers(0, 9, total) if rows > 1 else None
    _check_plan(ctx, cached, new, table, list(map(int, held)), stack, P, pool, rows, total, depth)


def test_plan_with_nothing_to_do(ctx):
    _check_plan(ctx, [0, 0], [0, 0], [[], []], [0, 0], [3, 2, 1, 0], 4, 4, 1, 2, full=False)
    _check_plan(ctx, [64, 128], [0, 0], [[3], [2, 1]], [1, 2], [0], 4, 4, 0, 0, full=False)


def test_plan_leaves_out_packed_tokens_that_do_not_fit(ctx):
    got, _ = _check_plan(ctx, [0, 0, 0], [5, 6, 0], [[], [], []], [0, 0, 0], [0, 1, 2], 4, 3, 0, 10, full=True)
    assert got["kv_len"].tolist() == [5, 0, 0]


def test_plan_reports_inconsistent_books_and_stays_in_bounds(ctx):
    B, P, pool = 4, 3, 8
    table = i32(np.array([[0, 1, -1], [2, 99, -1], [3, -1, -1], [4, -1, -1]]))
    held = i32([2, 2, 9, 1])                           # a page id outside the pool, a count outside the table
    free, n = i32([5, 6, 7, -1, -1, -1, -1, -1]), i32([3])
    got = ctx.kv_plan(i32([70, 10, 64, 10]), i32([1, 1, 1, -4]), table, held, free, n, 4, rows_per_seq=1)
    assert ctx.poll_status() & binding.STATUS_BAD_OFFSETS
    assert got["slot_map"].tolist()[0] == 1 * 64 + 6 and got["slot_map"].tolist()[2:] == [-1, -1]
    assert got["kv_len"].tolist() == [71, 11, 64, 10]


# ---- norm, rotation, store ------------------------------------------------------------------------

WRITES = [  # tokens, query heads, key heads, D, dtype, rotated channels, neighbours, norm, element offset of the projection
    (1, 1, 1, 64, "bf16", 64, False, True, 0), (13, 32, 8, 128, "bf16", 128, False, True, 0),
    (77, 5, 5, 128, "f32", 128, True, True, 0), (130, 6, 2, 64, "f32", 32, True, False, 0),
    (65, 7, 1, 256, "bf16", 128, False, True, 0), (64, 4, 2, 256, "f32", 256, False, False, 0),
    (33, 3, 1, 128, "bf16", 48, False, True, 3), (9, 2, 2, 64, "f32", 10, False, True, 1),
    (21, 4, 4, 128, "bf16", 0, False, True, 0), (300, 14, 2, 128, "bf16", 128, False, False, 8)]


def _projection(rng, T, Hq, Hkv, D, dtype, shift, spread=1.0):
    """q, k, v as views into one fused projection output whose rows start `shift` elements off."""
    width = (Hq + 2 * Hkv) * D + shift
    x = torch.as_tensor(rng.standard_normal((T, width)).astype(np.float32) * spread).to(DT[dtype]).cuda()
    cut = [shift, shift + Hq * D, shift + (Hq + Hkv) * D, width]
    return [x[:, a:b].unflatten(1, ((b - a) // D, D)) for a, b in zip(cut[:-1], cut[1:])]


@pytest.mark.parametrize("T,Hq,Hkv,D,dtype,rot,inter,norm,shift", WRITES)
def test_write(ctx, T, Hq, Hkv, D, dtype, rot, inter, norm, shift):
    rng = np.random.default_rng(T + D + rot)
    q, k, v = _projection(rng, T, Hq, Hkv, D, dtype, shift)
    w = [torch.as_tensor((1 + 0.2 * rng.standard_normal(D)).astype(np.float32)).to(DT[dtype]).cuda() if norm else None for _ in range(2)]
    limit = 5000
    ang = np.arange(limit)[:, None] * 10000.0 ** (-np.arange(rot // 2) / max(1, rot // 2))
    cs = torch.as_tensor(np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)).cuda() if rot else None
    pool = T // PAGE + 4
    slots = rng.permutation(pool * PAGE)[:T].astype(np.int32)
    pos = rng.integers(0, limit, T).astype(np.int32)
    pos[T // 2] = -1 if T > 3 else pos[T // 2]          # a padding row
    slots[T // 3] = -1 if T > 5 else slots[T // 3]      # a token that was not placed
    raw = rng.integers(0, 256, (pool, Hkv, ref.head_bytes(D))).astype(np.uint8)
    pages = torch.as_tensor(raw).cuda()
    o = ctx.kv_write(pages, q, k, v, i32(slots), i32(pos), cs, *w, eps=1e-6, interleaved=inter, keep_k=True)
    assert ctx.poll_status() == 0
    got = pages.cpu().numpy()
    half = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}[dtype]      # unit roundoff: 24 and 8 bits
    csn = None if cs is None else f64(cs)
    eps = float(np.float32(1e-6))
    gq, gk, nq, nk, nv = f64(o["q"]), f64(o["k"]), f64(q), f64(k), f64(v)
    used = np.ones(got.shape, bool)
    for t in range(T):
        if pos[t] < 0:
            assert (gq[t] == 0).all() and (gk[t] == 0).all()
            continue
        c = csn[pos[t]] if rot else None
        wq, wk = (None, None) if not norm else (f64(w[0]), f64(w[1]))
        rq = ref.norm_rotate(nq[t], wq, c, rot, inter, eps)
        rk = ref.norm_rotate(nk[t], wk, c, rot, inter, eps)
        # fp32 arithmetic: the norm's factor 8 roundings, the products and the sum of a pair 4 more, relative to the
        # pair's size; then one rounding to the output's type
        for g, r, x, ww in ((gq[t], rq, nq[t], wq), (gk[t], rk, nk[t], wk)):
            size = np.abs(r).max(-1, keepdims=True)
            assert (np.abs(g - r) <= half * np.abs(r) + 12 * 2.0 ** -24 * size).all()
        if slots[t] < 0:
            continue
        kk, vv = ref.load(got, slots[t], D)
        e = ref.Entry(rk.astype(np.float32), nv[t].astype(np.float32))
        assert np.array_equal(vv, e.values("v"))                     # the values are quantised from exact inputs
        step = e.k[1][:, None].astype(np.float64)
        # keys: fp32 rounding of the rotated row may move a code that lies on a boundary, and the scale by one bfloat16 step
        assert (np.abs(kk - rk) <= step * (0.5 + 15 * 2.0 ** -7) + np.abs(e.k[2][:, None]) * 2.0 ** -7 + 1e-5 * np.abs(rk).max()).all()
    # what was not a destination keeps its bytes
    page, off, h, kb = slots // PAGE, slots % PAGE, D // 2, PAGE * D // 2
    for t in range(T):
        if slots[t] >= 0 and pos[t] >= 0:
            used[page[t], :, off[t] * h:(off[t] + 1) * h] = False
            used[page[t], :, kb + off[t]:2 * kb + off[t]:PAGE] = False
            for i in range(2):
                at = 2 * kb + i * PAGE * 4 + off[t] * 4
                used[page[t], :, at:at + 4] = False
    assert np.array_equal(got[used], raw[used])


def test_write_is_bit_exact_for_given_keys(ctx):
    """Without norm and rotation the keys are exact inputs: their bytes have to be the model's."""
    rng = np.random.default_rng(5)
    for dtype, D, spread in (("bf16", 128, 3.0), ("f32", 64, 1e-3), ("f32", 256, 1e6), ("bf16", 64, 1.0)):
        T = 100
        q, k, v = _projection(rng, T, 2, 2, D, dtype, 0, spread)
        k[3], v[4] = 2.5, 0.0                            # rows without a range
        k[5, 0, 1:] = 1e-30
        raw = rng.integers(0, 256, (3, 2, ref.head_bytes(D))).astype(np.uint8)
        pages = torch.as_tensor(raw).cuda()
        slots = rng.permutation(3 * PAGE)[:T]
        ctx.kv_write(pages, q, k, v, i32(slots), i32(np.arange(T)))
        for t in range(T):
            ref.store(raw, int(slots[t]), ref.Entry(f64(k[t]).astype(np.float32), f64(v[t]).astype(np.float32)), D)
        assert np.array_equal(pages.cpu().numpy(), raw)
    assert ctx.poll_status() == 0


def test_write_of_rows_that_are_not_finite(ctx):
    rng = np.random.default_rng(6)
    q, k, v = _projection(rng, 8, 2, 1, 128, "f32", 0)
    k[1, 0, 17], k[2, 0, 3], v[3, 0, 127], v[4, 0, 0] = float("nan"), float("inf"), float("-inf"), 3e38
    v[4, 0, 1] = -3e38                                  # finite, but their difference is not
    q[5, 0, 0] = float("nan")
    pages = binding.kv_pages(1, 1, 128)
    o = ctx.kv_write(pages, q, k, v, i32(np.arange(8)), i32(np.arange(8)))
    assert ctx.poll_status() == binding.STATUS_BAD_ROW
    got = pages.cpu().numpy()
    for t, (kz, vz) in enumerate([(0, 0), (1, 0), (1, 0), (0, 1), (0, 1), (0, 0), (0, 0), (0, 0)]):
        kk, vv = ref.load(got, t, 128)
        assert (kk == 0).all() == bool(kz) and (vv == 0).all() == bool(vz) and np.isfinite(kk).all() and np.isfinite(vv).all()
    assert torch.isnan(o["q"][5, 0, 0]) and torch.isfinite(o["q"][6]).all()


def test_write_reports_positions_and_slots_out_of_range(ctx):
    rng = np.random.default_rng(7)
    q, k, v = _projection(rng, 4, 1, 1, 64, "bf16", 0)
    cs = torch.ones((10, 64), device="cuda")
    pages = torch.zeros((1, 1, ref.head_bytes(64)), dtype=torch.uint8, device="cuda")
    o = ctx.kv_write(pages, q, k, v, i32([64, 5, -7, 6]), i32([1, 10, 2, -3]), cs)
    assert ctx.poll_status() == binding.STATUS_ID_RANGE
    assert int(pages.sum()) == 0
    assert (o["q"][1] == 0).all() and (o["q"][3] == 0).all() and (o["q"][0] != 0).any()


# ---- attention -----------------------------------------------------------------------------------------

class Pool:
    """A cache with random entries for B sequences, on both sides."""

    def __init__(self, rng, kv_len, Hkv, D, kscale=1.0, vscale=1.0, garbage=True):
        self.kv_len, self.D, self.Hkv = [int(x) for x in kv_len], D, Hkv
        need = [-(-n // PAGE) for n in self.kv_len]
        pool = sum(need) + 2
        order, at = rng.permutation(pool), 0
        P = max(need + [1]) + 1
        self.table = np.full((len(need), P), -1, np.int32)
        raw = rng.integers(0, 256, (pool, Hkv, ref.head_bytes(D))).astype(np.uint8)
        meta = raw[:, :, PAGE * D:].view("<u4")
        meta[...] = 0x7FC07F80 if garbage else 0        # NaN minima and infinite scales wherever nothing is stored
        raw[:, :, PAGE * D:] = meta.view(np.uint8)
        self.k, self.v = [], []
        for b, n in enumerate(self.kv_len):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
            ks, vs = [], []
            for c in range(n):
                e = ref.Entry(rng.standard_normal((Hkv, D)).astype(np.float32) * kscale,
                              rng.standard_normal((Hkv, D)).astype(np.float32) * vscale)
                ref.store(raw, int(self.table[b, c // PAGE]) * PAGE + c % PAGE, e, D)
                ks.append(e.values("k"))
                vs.append(e.values("v"))
            self.k.append(np.asarray(ks).reshape(n, Hkv, D))
            self.v.append(np.asarray(vs).reshape(n, Hkv, D))
        self.pages = torch.as_tensor(raw).cuda()


def _visible(cached, i, parent):
    if parent is None:
        return list(range(cached + i + 1))
    return list(range(cached)) + [cached + x for x in ref.path_of(i, parent)]


def _check_attend(ctx, pool, q, cached, offs, rows, parent, scale=None):
    D = pool.D
    s = 1.0 / np.sqrt(D) if scale is None else scale
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32(cached), i32(pool.kv_len), tok_offsets=None if rows else i32(offs),
                      rows_per_seq=rows, node_parent=None if parent is None else i32(parent), scale=0.0 if scale is None else scale,
                      want_lse=True)
    assert ctx.poll_status() == 0
    got, lse, qn = f64(o["out"]), f64(o["lse"]), f64(q)
    f32 = q.dtype == torch.float32
    worst = 0.0
    for b in range(len(cached)):
        fresh = pool.kv_len[b] - cached[b]
        for t in range(offs[b], offs[b + 1]):
            i = t - offs[b]
            par = None if parent is None else parent.reshape(-1)[offs[b]:offs[b + 1]]
            vis = _visible(cached[b], i, par) if i < fresh else []
            want, wl, size = ref.attend(qn[t], pool.k[b], pool.v[b], vis, s)
            if not vis:
                assert (got[t] == 0).all() and np.isneginf(lse[t]).all()
                continue
            spread = np.ptp(pool.v[b][vis], axis=(0, 2)).repeat(q.shape[1] // pool.Hkv) + 2.0 ** -60
            # a product's fp32 sum: at most 2^-21 of the sum of its terms' sizes (fp32 queries: their two 11-bit
            # halves leave out 2^-22 of each term as well), carried into base 2 and the exponential with 2^-21 more
            # of the exponent's size; the exponentials' weights move by that much relative to each other
            wrong = size * 2.0 ** -20 + 2.0 ** -20 + np.abs(wl) * 2.0 ** -22
            # probabilities: 11 bits, 2^-11 relative (fp32: 22 bits), of codes whose span is the values'
            prob = 2.0 ** -21 if f32 else 2.0 ** -11
            lim = spread * (2 * wrong + prob + 2.0 ** -20) + 2.0 ** -21 * np.abs(pool.v[b][vis]).max()
            lim = lim[:, None] + np.abs(want) * (2.0 ** -24 if f32 else 2.0 ** -8)
            err = np.abs(got[t] - want)
            worst = max(worst, float((err / lim).max()))
            assert (err <= lim).all(), (b, i, float((err / lim).max()))
            assert (np.abs(lse[t] - wl) <= wrong + 2.0 ** -21 * np.abs(wl)).all()
    return worst


def _tree(rng, n):
    """Parents of a tree of n nodes; None of them is in order but that parents come first."""
    return np.array([-1] + [int(rng.integers(0, i)) for i in range(1, n)], np.int32)


ATTENDS = [  # sequences, new tokens (most), longest context, query heads, key heads, D, dtype
    (1, 1, 0, 1, 1, 64, "bf16"), (1, 1, 1, 4, 1, 128, "bf16"), (3, 1, 200, 8, 2, 128, "bf16"), (2, 1, 700, 5, 5, 64, "f32"),
    (2, 1, 130, 28, 4, 128, "f32"), (1, 1, 3000, 16, 2, 128, "bf16"), (5, 9, 150, 8, 2, 128, "bf16"), (3, 17, 140, 7, 1, 64, "bf16"),
    (2, 33, 64, 8, 2, 128, "bf16"), (2, 33, 65, 4, 4, 256, "bf16"), (2, 20, 63, 6, 2, 256, "f32"), (1, 70, 100, 8, 1, 128, "bf16"),
    (2, 150, 30, 4, 2, 64, "bf16"), (1, 200, 1, 2, 1, 128, "f32"), (1, 300, 500, 2, 1, 128, "bf16"), (9, 2, 128, 40, 8, 64, "bf16")]


@pytest.mark.parametrize("B,new,longest,Hq,Hkv,D,dtype", ATTENDS)
@pytest.mark.parametrize("tree", [False, True])
def test_attend(ctx, B, new, longest, Hq, Hkv, D, dtype, tree):
    rng = np.random.default_rng(B * 31 + new + longest + Hq)
    cached = rng.integers(0, longest + 1, B)
    cached[0] = longest
    fresh = rng.integers(0, new + 1, B)                 # some sequences have fewer nodes than rows, some none
    fresh[0] = new
    pool = Pool(rng, cached + fresh, Hkv, D)
    rows = new if tree else 0
    offs = np.arange(B + 1) * new if tree else np.concatenate([[0], np.cumsum(fresh)])
    parent = None
    if tree:
        parent = np.full((B, new), -1, np.int32)
        for b in range(B):
            if fresh[b]:
                parent[b, :fresh[b]] = _tree(rng, fresh[b])
    T = int(offs[-1])
    # rows of q inside a wider buffer
    q = torch.as_tensor(rng.standard_normal((T, Hq + 1, D)).astype(np.float32) * 1.5).to(DT[dtype]).cuda()[:, :Hq]
    _check_attend(ctx, pool, q, cached, offs, rows, parent)


LONG = [  # sequences, new tokens, contexts from .. to, query heads, key heads, D, dtype, trees: every CTA passes many pages and segments
    (64, 1, 100, 3000, 28, 4, 128, "bf16", False), (33, 1, 1, 4000, 16, 8, 64, "bf16", False), (40, 1, 500, 1500, 8, 8, 256, "bf16", False),
    (64, 2, 0, 2000, 32, 4, 128, "bf16", True), (48, 33, 700, 2200, 16, 8, 128, "bf16", True), (60, 33, 0, 1800, 32, 8, 128, "bf16", True),
    (70, 17, 1, 2500, 10, 5, 64, "bf16", True), (3, 1500, 0, 700, 16, 4, 128, "bf16", False), (2, 1100, 300, 900, 16, 8, 64, "bf16", False),
    (9, 65, 1000, 1400, 8, 8, 128, "bf16", False), (40, 5, 600, 1900, 8, 2, 128, "f32", True), (20, 1, 10, 2000, 32, 8, 64, "f32", False)]


@pytest.mark.parametrize("B,new,lo,hi,Hq,Hkv,D,dtype,tree", LONG)
def test_attend_long(ctx, B, new, lo, hi, Hq, Hkv, D, dtype, tree):
    """Larger batches against 64-bit sums on the same device; the entries come through kv_read (fp32, one rounding)."""
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
    pages = binding.kv_pages(n, Hkv, D)
    pages.fill_(255)
    b = torch.repeat_interleave(torch.arange(B, device="cuda"), kv.long())
    t = torch.arange(b.numel(), device="cuda") - (torch.cumsum(kv, 0) - kv)[b]
    slots = (table[b, t // PAGE] * PAGE + t % PAGE).to(torch.int32)
    for i in range(0, b.numel(), 50000):
        m = min(50000, b.numel() - i)
        k = torch.randn((m, Hkv, D), generator=g, device="cuda")
        v = torch.randn((m, Hkv, D), generator=g, device="cuda")
        ctx.kv_write(pages, k[:, :0], k, v, slots[i:i + m].contiguous(), torch.zeros(m, dtype=torch.int32, device="cuda"),
                     outputs=dict(q=k[:, :0]))
    q = (torch.randn((B * new, Hq, D), generator=g, device="cuda") * 1.3).to(DT[dtype])
    rng = np.random.default_rng(B)
    parent = None
    if tree:
        parent = np.stack([_tree(rng, new) for _ in range(B)])
    o = ctx.kv_attend(q, pages, table, cached, kv, rows_per_seq=new, node_parent=None if parent is None else i32(parent), want_lse=True)
    assert ctx.poll_status() == 0
    off = torch.cumsum(kv, 0) - kv
    for s in range(B):
        lo_t, n_t, c = int(off[s]), int(kv[s]), int(cached[s])
        e = ctx.kv_read(pages, slots[lo_t:lo_t + n_t].contiguous(), D, torch.float32)
        k, v = e["k"].double(), e["v"].double()
        see = torch.zeros((new, n_t), dtype=torch.bool)
        see[:, :c] = True
        for i in range(new):
            see[i, [c + x for x in (range(i + 1) if parent is None else ref.path_of(i, parent[s]))]] = True
        see = see.cuda()
        qs = q[s * new:(s + 1) * new].double().view(new, Hkv, Hq // Hkv, D)
        w = torch.einsum("nhgd,thd->hgnt", qs, k) / np.sqrt(D)
        size = torch.einsum("nhgd,thd->hgnt", qs.abs(), k.abs()).amax(-1) / np.sqrt(D)
        w = w.masked_fill(~see, float("-inf"))
        lse = torch.logsumexp(w, -1)
        want = torch.einsum("hgnt,thd->nhgd", torch.exp(w - lse[..., None]), v).reshape(new, Hq, D)
        wrong = size * 2.0 ** -20 + 2.0 ** -20 + lse.abs() * 2.0 ** -22               # as in _check_attend
        spread = v.amax((0, 2)) - v.amin((0, 2))
        lim = spread[:, None, None] * (2 * wrong + (2.0 ** -21 if dtype == "f32" else 2.0 ** -11) + 2.0 ** -20) + 2.0 ** -21 * v.abs().max()
        lim = lim.permute(2, 0, 1).reshape(new, Hq)[..., None] + want.abs() * (2.0 ** -24 if dtype == "f32" else 2.0 ** -8)
        got = o["out"][s * new:(s + 1) * new].double()
        assert bool(((got - want).abs() <= lim).all()), (s, float(((got - want).abs() / lim).max()))
        gl = o["lse"][s * new:(s + 1) * new].double()
        le, lw = lse.permute(2, 0, 1).reshape(new, Hq), wrong.permute(2, 0, 1).reshape(new, Hq)
        assert bool(((gl - le).abs() <= lw + 2.0 ** -21 * le.abs()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_with_large_products_and_values_of_any_size(ctx, dtype):
    """Sharp softmaxes, scales of the values far from 1 and different by token, rows without a range."""
    rng = np.random.default_rng(3)
    for kscale, vscale, qscale in ((4.0, 1e-4, 3.0), (0.01, 3e4, 1.0), (1.0, 1.0, 1e3), (1e-3, 1.0, 1e-3)):
        pool = Pool(rng, [300, 70], 2, 128, kscale, vscale)
        q = torch.as_tensor(rng.standard_normal((2, 6, 128)).astype(np.float32) * qscale).to(DT[dtype]).cuda()
        _check_attend(ctx, pool, q, [299, 69], [0, 1, 2], 1, None)


def test_attend_where_a_tokens_values_dwarf_the_others(ctx):
    rng = np.random.default_rng(4)
    pool = Pool(rng, [130], 1, 64)
    e = ref.Entry(np.full((1, 64), 0.5, np.float32), rng.standard_normal((1, 64)).astype(np.float32) * 1e5)
    flat = ref.Entry(np.zeros((1, 64), np.float32), np.full((1, 64), 7.0, np.float32))
    raw = pool.pages.cpu().numpy()
    for c, x in ((3, e), (100, flat), (128, flat)):
        ref.store(raw, int(pool.table[0, c // PAGE]) * PAGE + c % PAGE, x, 64)
        pool.k[0][c], pool.v[0][c] = x.values("k"), x.values("v")
    pool.pages = torch.as_tensor(raw).cuda()
    for dtype in ("bf16", "f32"):
        q = torch.as_tensor(rng.standard_normal((1, 3, 64)).astype(np.float32)).to(DT[dtype]).cuda()
        _check_attend(ctx, pool, q, [129], [0, 1], 1, None)


def test_attend_scale_and_unaligned_queries(ctx):
    rng = np.random.default_rng(8)
    pool = Pool(rng, [90, 10], 2, 64)
    for dtype in ("bf16", "f32"):
        buf = torch.as_tensor(rng.standard_normal((2, 4 * 64 + 3)).astype(np.float32)).to(DT[dtype]).cuda()
        q = buf[:, 1:257].unflatten(1, (4, 64))
        _check_attend(ctx, pool, q, [89, 9], [0, 1, 2], 1, None, scale=0.37)


def test_attend_is_the_same_on_a_second_call_and_on_another_stream(ctx):
    rng = np.random.default_rng(9)
    pool = Pool(rng, [2500, 40, 700], 2, 128)
    q = torch.as_tensor(rng.standard_normal((3, 8, 128)).astype(np.float32)).to(torch.bfloat16).cuda()
    args = (q, pool.pages, i32(pool.table), i32([2499, 39, 699]), i32(pool.kv_len))
    one = ctx.kv_attend(*args, rows_per_seq=1)["out"]
    two = ctx.kv_attend(*args, rows_per_seq=1)["out"]
    assert torch.equal(one, two)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ctx.set_stream(side)
    try:
        with torch.cuda.stream(side):
            three = ctx.kv_attend(*args, rows_per_seq=1)["out"]
        side.synchronize()
    finally:
        ctx.set_stream(torch.cuda.current_stream())
    assert torch.equal(one, three)


def test_attend_reports_bad_tables_and_parents(ctx):
    rng = np.random.default_rng(10)
    pool = Pool(rng, [70, 5], 1, 64)
    q = torch.as_tensor(rng.standard_normal((10, 2, 64)).astype(np.float32)).cuda()
    table = pool.table.copy()
    table[0, 0] = pool.pages.shape[0] + 5
    o = ctx.kv_attend(q, pool.pages, i32(table), i32([65, 0]), i32(pool.kv_len), rows_per_seq=5)
    assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS and torch.isfinite(o["out"]).all()
    parent = np.array([[-1, 0, 3, 2, 1], [-1, 0, 0, 2, 9]], np.int32)
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([65, 0]), i32(pool.kv_len), rows_per_seq=5, node_parent=i32(parent))
    assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS and torch.isfinite(o["out"]).all()


# ---- the accepted path ------------------------------------------------------------------------------------

@pytest.mark.parametrize("B,cap,longest,Hkv,D,layers", [(1, 1, 100, 1, 64, 1), (6, 9, 200, 2, 128, 3), (40, 33, 130, 4, 64, 2), (3, 70, 64, 1, 256, 5)])
@pytest.mark.parametrize("packed", [False, True])
def test_commit(ctx, B, cap, longest, Hkv, D, layers, packed):
    rng = np.random.default_rng(B + cap)
    cached = rng.integers(0, longest + 1, B)
    nodes = rng.integers(1, cap + 1, B)
    nodes[0] = cap
    kv = cached + nodes
    if B > 3:
        kv[2] = cached[2]                                # its tokens were not placed
    pools = [Pool(rng, kv, Hkv, D) for _ in range(1)]
    table, pages = pools[0].table, pools[0].pages
    raw = np.stack([rng.permutation(pages.cpu().numpy().reshape(-1)).reshape(pages.shape) for _ in range(layers)])
    offs = np.concatenate([[0], np.cumsum(nodes)]) if packed else np.arange(B + 1) * cap
    parent = np.full(int(offs[-1]), -1, np.int32)
    best = np.zeros(B, np.int32)
    for b in range(B):
        parent[offs[b]:offs[b] + nodes[b]] = _tree(rng, nodes[b])
        best[b] = rng.integers(0, nodes[b])
    if B > 3:
        best[1] = -1
    dev = torch.as_tensor(raw).cuda()
    new = ctx.kv_commit(dev, i32(table), i32(cached), i32(kv), i32(best), i32(parent if packed else parent.reshape(B, cap)),
                        tok_offsets=i32(offs) if packed else None)
    assert ctx.poll_status() == 0
    want, lens = raw.copy(), []
    slot = lambda b, c: (int(table[b, c // PAGE]), c % PAGE)  # noqa: E731
    h, kb = D // 2, PAGE * D // 2
    for b in range(B):
        if best[b] < 0 or kv[b] == cached[b]:
            lens.append(cached[b])
            continue
        path = ref.path_of(best[b], parent[offs[b]:offs[b] + nodes[b]])
        lens.append(cached[b] + len(path))
        for i, x in enumerate(path):
            (sp, so), (dp, do) = slot(b, cached[b] + x), slot(b, cached[b] + i)
            want[:, dp, :, do * h:(do + 1) * h] = raw[:, sp, :, so * h:(so + 1) * h]
            want[:, dp, :, kb + do:2 * kb + do:PAGE] = raw[:, sp, :, kb + so:2 * kb + so:PAGE]
            for j in range(2):
                at = 2 * kb + j * PAGE * 4
                want[:, dp, :, at + 4 * do:at + 4 * do + 4] = raw[:, sp, :, at + 4 * so:at + 4 * so + 4]
    assert new.tolist() == [int(x) for x in lens]
    assert np.array_equal(dev.cpu().numpy(), want)


def test_commit_reports_bad_parents_and_moves_nothing(ctx):
    rng = np.random.default_rng(12)
    pool = Pool(rng, [20, 20], 1, 64)
    raw = pool.pages.cpu().numpy()[None].copy()
    dev = torch.as_tensor(raw).cuda()
    parent = np.array([[-1, 2, 1, 0], [-1, 0, 1, 5]], np.int32)
    new = ctx.kv_commit(dev, i32(pool.table), i32([16, 16]), i32([20, 20]), i32([2, 3]), i32(parent))
    assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS
    assert new.tolist() == [16, 16] and np.array_equal(dev.cpu().numpy(), raw)


# ---- entries as values --------------------------------------------------------------------------------------

@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_read(ctx, D, dtype):
    rng = np.random.default_rng(D)
    pool = Pool(rng, [100, 7], 3, D)
    slots = [int(pool.table[b, c // PAGE]) * PAGE + c % PAGE for b, c in ((0, 0), (0, 99), (1, 6), (0, 64), (0, 63))] + [-1]
    o = ctx.kv_read(pool.pages, i32(slots), D, DT[dtype])
    assert ctx.poll_status() == 0
    raw = pool.pages.cpu().numpy()
    for i, s in enumerate(slots):
        k, v = ref.load(raw, s, D) if s >= 0 else (np.zeros((3, D)), np.zeros((3, D)))
        # scale * code is exact in fp32; the sum is rounded once, then once more to bf16
        for g, w in ((f64(o["k"][i]), k), (f64(o["v"][i]), v)):
            assert (np.abs(g - w) <= np.abs(w) * (2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0))).all()
    ctx.kv_read(pool.pages, i32([pool.pages.shape[0] * PAGE, -9]), D, DT[dtype])
    assert ctx.poll_status() == binding.STATUS_ID_RANGE


# ---- refusals ------------------------------------------------------------------------------------------------

def test_refusals(ctx):
    rng = np.random.default_rng(11)
    pool = Pool(rng, [70], 1, 64)
    q = torch.zeros((1, 3, 64), device="cuda")
    ok = dict(tok_offsets=None, rows_per_seq=1)
    args = (pool.pages, i32(pool.table), i32([69]), i32([70]))

    def refused(code, f, *a, **kw):
        before = ctx.launch_count()
        with pytest.raises(binding.AasdError) as e:
            f(*a, **kw)
        assert e.value.code == code and ctx.launch_count() == before

    refused(3, ctx.kv_attend, q.half(), *args, **ok)                              # a type it does not have
    refused(2, ctx.kv_attend, q, *args, rows_per_seq=2)                           # rows that do not add up
    refused(1, ctx.kv_attend, q, *args)                                           # packed rows without offsets
    refused(1, ctx.kv_attend, q, *args, **ok, scale=-1.0)
    two = torch.zeros((2, 2, ref.head_bytes(64)), dtype=torch.uint8, device="cuda")
    refused(2, ctx.kv_attend, q, two, *args[1:], **ok)                            # 3 query heads over 2 key heads
    wide = torch.zeros((1, 1, 96), device="cuda")
    other = torch.zeros((2, 1, ref.head_bytes(96)), dtype=torch.uint8, device="cuda")
    refused(binding.ERR_UNSUPPORTED, ctx.kv_attend, wide, other, *args[1:], **ok, )
    shifted = torch.zeros(2 * ref.head_bytes(64) + 16, dtype=torch.uint8, device="cuda")[8:8 + 2 * ref.head_bytes(64)].view(2, 1, -1)
    refused(1, ctx.kv_attend, q, shifted, *args[1:], **ok)                        # a pool off its 16-byte boundary
    k = torch.zeros((1, 1, 64), device="cuda")
    cs = torch.zeros((4, 66), device="cuda")
    refused(2, ctx.kv_write, pool.pages, q, k, k, i32([0]), i32([0]), cs)         # more rotated channels than there are
    refused(2, ctx.kv_write, pool.pages, q, k, k, i32([0]), i32([0]), cs[:, :3].contiguous())   # an odd number
    refused(1, ctx.kv_write, pool.pages, q, k, k, i32([0]), i32([0]), eps=-1.0)
    refused(3, ctx.kv_read, pool.pages, i32([0]), 64, torch.float16)
    books = (i32([[0, -1]]), i32([1]), i32([1, -1]), i32([1]))
    refused(2, ctx.kv_plan, i32([10]), i32([1]), *books, 3, rows_per_seq=2)
    new_len = i32([69])
    refused(1, ctx.kv_commit, pool.pages[None], args[1], new_len, args[3], i32([0]), i32([[-1]]), outputs=new_len)
    lib, h = ctx.lib, ctx._h
    assert lib.aasd_kv_workspace_init(h, None, 0, 64) == 1
    assert lib.aasd_kv_workspace_init(h, ctx.kv_workspace(64).data_ptr(), 8, 64) == 4
    assert lib.aasd_kv_workspace_init(h, ctx.kv_workspace(64).data_ptr(), 1 << 40, 65) == binding.ERR_UNSUPPORTED
    assert ctx.poll_status() == 0


def test_empty_calls(ctx):
    pages = binding.kv_pages(2, 1, 64)
    z = torch.zeros((0, 2, 64), device="cuda")
    e = i32([])
    assert ctx.kv_attend(z, pages, i32([[0]]), i32([0]), i32([0]), tok_offsets=i32([0, 0]))["out"].shape == (0, 2, 64)
    ctx.kv_write(pages, z, z[:, :1], z[:, :1], e, e)
    ctx.kv_read(pages, e, 64)
    assert ctx.poll_status() == 0
