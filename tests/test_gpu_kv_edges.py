"""Edges of the paged 4-bit cache's calls: rows that no sequence owns, aliased and misshapen
arguments, captured graphs, and the branches of the attention kernels that ordinary inputs do not
take."""
import numpy as np
import pytest
import torch

import kv_ref as ref
from paper_2505_13204_b200 import binding
from test_gpu_kv import DT, PAGE, Pool, _tree, f64, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.close()


def nan_outputs(T, Hq, D, dtype, shift=0):
    """Outputs that hold NaN before the call; out starts `shift` elements past a 16-byte boundary."""
    out = torch.full((T * Hq * D + shift,), float("nan"), dtype=DT[dtype], device="cuda")[shift:].view(T, Hq, D)
    return dict(out=out, lse=torch.full((T, Hq), float("nan"), device="cuda"))


def queries(rng, T, Hq, D, dtype, size=1.0):
    return torch.as_tensor((rng.standard_normal((T, Hq, D)) * size).astype(np.float32)).to(DT[dtype]).cuda()


def check_rows(pool, q, o, rows, scale=None):
    """rows: {token row: (sequence, visible places)}; every other row is zeros with an lse of -inf.
    The bounds are those of test_gpu_kv._check_attend, which derives them."""
    s = 1.0 / np.sqrt(pool.D) if scale is None else scale
    got, lse, qn, f32 = f64(o["out"]), f64(o["lse"]), f64(q), q.dtype == torch.float32
    for t in range(q.shape[0]):
        b, vis = rows.get(t, (0, []))
        if not vis:
            assert (got[t] == 0).all() and np.isneginf(lse[t]).all(), t
            continue
        want, wl, size = ref.attend(qn[t], pool.k[b], pool.v[b], vis, s)
        spread = np.ptp(pool.v[b][vis], axis=(0, 2)).repeat(q.shape[1] // pool.Hkv) + 2.0 ** -60
        wrong = size * 2.0 ** -20 + 2.0 ** -20 + np.abs(wl) * 2.0 ** -22
        lim = spread * (2 * wrong + (2.0 ** -21 if f32 else 2.0 ** -11) + 2.0 ** -20) + 2.0 ** -21 * np.abs(pool.v[b][vis]).max()
        lim = lim[:, None] + np.abs(want) * (2.0 ** -24 if f32 else 2.0 ** -8)
        err = np.abs(got[t] - want)
        assert (err <= lim).all(), (t, float((err / lim).max()))
        assert (np.abs(lse[t] - wl) <= wrong + 2.0 ** -21 * np.abs(wl)).all(), t


# query heads per key head: the split kernel, one tile, the pair of tiles (bf16, at 4 token rows per sequence on average)
GROUPS = [(3, "f32"), (3, "bf16"), (16, "bf16"), (40, "bf16")]


# ---- rows that no sequence owns --------------------------------------------------------------------

@pytest.mark.parametrize("G,dtype", GROUPS)
@pytest.mark.parametrize("new", [(5, 6, 0), (5, 7, 2), (0, 11, 3)])
def test_tokens_of_a_sequence_that_passes_the_end_give_zeros(ctx, G, dtype, new):
    """kv_plan leaves the whole sequence out; its rows that do exist see nothing."""
    rng = np.random.default_rng(G)
    T = 10
    table, held = i32(np.full((3, 3), -1)), i32([0, 0, 0])
    plan = ctx.kv_plan(i32([0, 0, 0]), i32(new), table, held, i32([0, 1, 2, 3]), i32([4]), T)
    assert ctx.poll_status() == binding.STATUS_KV_FULL
    assert plan["tok_offsets"].tolist() == [0, new[0], new[0] + new[1], sum(new)] and plan["kv_len"].tolist() == [new[0], 0, 0]
    pool = Pool(rng, [new[0], 0, 0], 1, 64)
    q = queries(rng, T, G, 64, dtype)
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([0, 0, 0]), plan["kv_len"], plan["tok_offsets"], want_lse=True,
                      outputs=nan_outputs(T, G, 64, dtype))
    assert ctx.poll_status() == 0
    check_rows(pool, q, o, {i: (0, list(range(i + 1))) for i in range(new[0])})


@pytest.mark.parametrize("G,dtype", GROUPS)
def test_rows_in_front_of_the_first_sequence_and_behind_the_last_give_zeros(ctx, G, dtype):
    rng = np.random.default_rng(G + 1)
    pool = Pool(rng, [70, 5], 1, 64)
    q = queries(rng, 11, G, 64, dtype)
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([67, 2]), i32(pool.kv_len), i32([2, 5, 8]), want_lse=True,
                      outputs=nan_outputs(11, G, 64, dtype))
    assert ctx.poll_status() == 0
    rows = {2 + i: (0, list(range(68 + i))) for i in range(3)}
    rows.update({5 + i: (1, list(range(3 + i))) for i in range(3)})
    check_rows(pool, q, o, rows)


@pytest.mark.parametrize("G,dtype", [(3, "f32"), (4, "bf16"), (40, "bf16")])
@pytest.mark.parametrize("B,rows", [(1, 5000), (5, 900), (300, 17), (4000, 3), (7, 0)])
def test_padding_of_any_length_gives_zeros(ctx, G, dtype, B, rows):
    """Few sequences with much padding, more sequences than warps, and (rows 0) packed ones with room behind them."""
    rng = np.random.default_rng(B)
    table, kv = np.zeros((B, 2), np.int32), rng.integers(0, 3, B)
    kv[0], table[:, 1] = 2, 1
    pool = Pool(rng, [100], 1, 64)
    pool.k, pool.v = [pool.k[0]] * B, [pool.v[0]] * B
    table[:] = pool.table[0, :2]                            # (every sequence the same tokens)
    offs = np.arange(B + 1) * rows if rows else np.concatenate([[0], np.cumsum(kv)])
    T = B * rows if rows else int(offs[-1]) + 3001
    q = queries(rng, T, G, 64, dtype)
    used = torch.zeros(T, dtype=torch.bool, device="cuda")
    live = {int(offs[b]) + i: (b, list(range(51 + i))) for b in range(B) for i in range(kv[b])}
    used[list(live)] = True
    q[~used] = float("nan")                                 # (whatever the queries of such rows hold)
    o = ctx.kv_attend(q, pool.pages, i32(table), i32([50] * B), i32(50 + kv), None if rows else i32(offs), rows_per_seq=rows, want_lse=True,
                      outputs=nan_outputs(T, G, 64, dtype))
    assert ctx.poll_status() == 0
    assert bool((o["out"][~used] == 0).all()) and bool((o["lse"][~used] == float("-inf")).all())
    some = sorted(live)[:3] + sorted(live)[-3:]
    check_rows(pool, q[some], dict(out=o["out"][some], lse=o["lse"][some]), {n: live[t] for n, t in enumerate(some)})


@pytest.mark.parametrize("dtype,width,H", [("f32", 1 << 20, 8), ("bf16", 1 << 24, 16)])
def test_more_pages_than_a_call_can_count_give_zeros(ctx, dtype, width, H):
    """(The table names no page, so there would be nothing to see either.)"""
    T = 4096
    kv = width * PAGE
    pages = binding.kv_pages(1, H, 64)
    q = torch.ones((T, H, 64), dtype=DT[dtype], device="cuda")
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    o = ctx.kv_attend(q, pages, table, i32([kv - T]), i32([kv]), rows_per_seq=T, want_lse=True, outputs=nan_outputs(T, H, 64, dtype))
    assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS
    assert bool((o["out"] == 0).all()) and bool((o["lse"] == float("-inf")).all())


# ---- arguments -----------------------------------------------------------------------------------------

def refused(ctx, f, *a, **kw):
    before = ctx.launch_count()
    with pytest.raises(binding.AasdError) as e:
        f(*a, **kw)
    assert ctx.launch_count() == before
    return e.value.code


def test_commit_refuses_results_over_its_inputs(ctx):
    """Every CTA reads the lengths and the chosen node on its own, in no order with the new length."""
    pages = binding.kv_pages(2, 1, 64, layers=1)
    table, cached, kv, best, parent = i32([[0, -1]]), i32([3]), i32([5]), i32([1]), i32([[-1, 0]])
    offs = i32([0, 2])
    args = (pages, table, cached, kv, best)
    for out in (cached, kv, best):
        assert refused(ctx, ctx.kv_commit, *args, parent, outputs=out) == 1
    flat = i32([-1])
    assert refused(ctx, ctx.kv_commit, pages, table, i32([3]), i32([4]), i32([0]), flat, i32([0, 1]), outputs=flat) == 1
    prm = binding.KvCommitParams(1, 1, 64, 2, 2, 0, 1, 0)
    lib, h = ctx.lib, ctx._h
    call = [pages.data_ptr(), table.data_ptr(), cached.data_ptr(), kv.data_ptr(), offs.data_ptr(), best.data_ptr(), parent.data_ptr(), prm]
    for out in (table, offs, pages):
        assert lib.aasd_kv_commit(h, *call, out.data_ptr()) == 1
    assert ctx.poll_status() == 0


def test_plan_refuses_the_new_length_over_the_old_one(ctx):
    """The slots are found from both."""
    cached, books = i32([10]), (i32([[0, -1]]), i32([1]), i32([1, -1]), i32([1]))
    new = torch.empty(1, dtype=torch.int32, device="cuda")
    o = dict(kv_len=cached, tok_offsets=i32([0, 0]), slot_map=new, positions=new.clone())
    assert refused(ctx, ctx.kv_plan, cached, i32([1]), *books, 1, rows_per_seq=1, outputs=o) == 1
    assert ctx.poll_status() == 0


def test_tables_wider_than_a_sequence_can_be_are_refused(ctx):
    """Places of a sequence are 32-bit numbers: ceil(2^31 / 64) - 1 pages at most."""
    one = i32([0, 0]).data_ptr()
    lib, h = ctx.lib, ctx._h
    prm = binding.KvPlanParams(1, 1, 1 << 25, 1, 1)
    before = ctx.launch_count()
    assert lib.aasd_kv_plan(h, one, one, None, prm, binding.KvPlanState(one, one, one, one), binding.KvPlanOut(one + 4, one, one, one)) == 2
    prm = binding.KvCommitParams(1, 1, 64, 1, 1 << 25, 1, 0, 0)
    assert lib.aasd_kv_commit(h, None, one, one, one, None, one, one, prm, one + 4) == 2
    assert ctx.launch_count() == before


def test_lengths_that_do_not_go_together_are_refused(ctx):
    """Every array is read or written by the counts of the others."""
    B, T = 3, 6
    table, held, free, n = i32(np.full((B, 2), -1)), i32([0] * B), i32([0, 1, 2, 3]), i32([4])
    z3, z2, z5, z7 = i32([0] * 3), i32([0] * 2), i32([0] * 5), i32([0] * 7)

    def plan(**kw):
        a = dict(cached_len=z3, n_new=i32([0] * 3), block_table=table, seq_pages=held, free_pages=free, n_free=n, n_tokens=T, rows_per_seq=2)
        a.update(kw)
        return lambda: ctx.kv_plan(**a)

    new = dict(kv_len=i32([0] * 3), tok_offsets=i32([0] * 4), slot_map=i32([0] * T), positions=i32([0] * T))
    bad = [plan(cached_len=z2), plan(n_new=z2), plan(seq_pages=z2), plan(n_free=i32([])), plan(node_depth=z5)]
    bad += [plan(outputs=dict(new, kv_len=z2)), plan(outputs=dict(new, tok_offsets=z3)), plan(outputs=dict(new, slot_map=z5)),
            plan(outputs=dict(new, positions=z5))]

    pages = binding.kv_pages(4, 1, 64)
    q = torch.zeros((T, 2, 64), device="cuda")
    k = torch.zeros((T, 1, 64), device="cuda")
    z6 = i32([0] * 6)

    def attend(**kw):
        a = dict(q=q, pages=pages, block_table=table, cached_len=z3, kv_len=z3, rows_per_seq=2)
        a.update(kw)
        return lambda: ctx.kv_attend(**a)

    bad += [attend(cached_len=z2), attend(kv_len=z2), attend(node_parent=z5), attend(tok_offsets=z3, rows_per_seq=0),
            attend(outputs=dict(out=q[:5])), attend(outputs=dict(out=q.to(torch.bfloat16))), attend(outputs=dict(out=torch.zeros((T, 4, 64), device="cuda")[:, :2])),
            attend(outputs=dict(out=torch.empty_like(q), lse=torch.zeros((T, 1), device="cuda"))),
            attend(outputs=dict(out=torch.empty_like(q), lse=torch.zeros((T, 2), device="cuda", dtype=torch.float64)))]
    # blocks that are not a whole number of channels
    odd = torch.zeros((4, 1, ref.head_bytes(64) + 32), dtype=torch.uint8, device="cuda")
    bad += [attend(pages=odd), lambda: ctx.kv_read(odd, z6, 64), lambda: ctx.kv_commit(odd[None], table, z3, z3, z3, i32(np.zeros((3, 2)))),
            lambda: ctx.kv_write(odd, q, k, k, z6, z6)]

    def write(**kw):
        a = dict(pages=pages, q=q, k=k, v=k, slot_map=z6, positions=z6)
        a.update(kw)
        return lambda: ctx.kv_write(**a)

    bad += [write(slot_map=z5), write(positions=z7), write(k=k[:5], v=k[:5]), write(v=k[:5]), write(q_weight=torch.ones(63, device="cuda")),
            write(cos_sin=torch.ones((0, 64), device="cuda")[:, :, None]),
            write(outputs=dict(q=q[:5])), write(outputs=dict(q=torch.empty_like(q), k=k[:5])), write(outputs=dict(q=torch.empty_like(q, dtype=torch.bfloat16)))]

    layers = pages[None]
    tree = i32(np.zeros((3, 2)))

    def commit(**kw):
        a = dict(pages=layers, block_table=table, cached_len=i32([0] * 3), kv_len=z3, best_node=z3, node_parent=tree)
        a.update(kw)
        return lambda: ctx.kv_commit(**a)

    bad += [commit(cached_len=z2), commit(kv_len=z2), commit(best_node=z2), commit(node_parent=tree[:2]), commit(node_parent=tree.view(-1)), commit(tok_offsets=z3, node_parent=z6),
            commit(outputs=z2)]

    def read(**kw):
        a = dict(pages=pages, slots=z6, head_dim=64, dtype=torch.float32)
        a.update(kw)
        return lambda: ctx.kv_read(**a)

    bad += [read(outputs=dict(k=k[:5], v=k)), read(outputs=dict(k=k, v=k[:5])), read(outputs=dict(k=k, v=k.to(torch.bfloat16))), read(head_dim=128)]
    # int32, on the device, one after another
    bad += [plan(cached_len=z3.long()), attend(kv_len=z3.cpu()), commit(best_node=i32([0] * 6)[::2]), read(slots=z6.long()),
            plan(outputs=dict(new, positions=torch.zeros(T, device="cuda")))]
    before = ctx.launch_count()
    for i, f in enumerate(bad):
        with pytest.raises((binding.AasdError, AssertionError)):
            f()
            raise RuntimeError("call %d was not refused" % i)
    assert ctx.launch_count() == before and ctx.poll_status() == 0
    # what goes together still goes
    plan(outputs=new)()
    attend(outputs=dict(out=torch.empty_like(q), lse=torch.zeros((T, 2), device="cuda")), kv_len=z7, node_parent=z7)()
    write(outputs=dict(q=torch.empty_like(q)), slot_map=i32([-1] * 6))()
    commit(best_node=i32([-1] * 3))()
    read()()
    assert ctx.poll_status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_of_single_tokens_and_heads_do_not_matter(ctx, dtype):
    """One token, or one head, is contiguous whatever the stride of that dimension says."""
    rng = np.random.default_rng(21)
    D, Hq, Hkv = 64, 4, 1
    q = queries(rng, Hq, 1, D, dtype).transpose(0, 1)                  # one token: strides (D, D, 1)
    k, v = (queries(rng, 1, 5, D, dtype)[:, 2:3].transpose(0, 1) for _ in range(2))     # one head: strides (D, 5 D, 1)
    assert q.stride(0) < Hq * D and k.stride(1) != D
    pages, same = (torch.zeros((1, Hkv, ref.head_bytes(D)), dtype=torch.uint8, device="cuda") for _ in range(2))
    a = ctx.kv_write(pages, q, k, v, i32([7]), i32([0]), keep_k=True)
    b = ctx.kv_write(same, q.contiguous().clone(memory_format=torch.contiguous_format).reshape(1, Hq, D), k.reshape(1, 1, D).clone(),
                     v.reshape(1, 1, D).clone(), i32([7]), i32([0]), keep_k=True)
    assert torch.equal(a["q"], b["q"]) and torch.equal(a["k"], b["k"]) and torch.equal(pages, same)
    pool = Pool(rng, [9], 1, D)
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([8]), i32([9]), rows_per_seq=1, want_lse=True)
    check_rows(pool, q, o, {0: (0, list(range(9)))})
    one = queries(rng, 1, 3, D, dtype).transpose(0, 1)                 # three tokens of one head: strides (D, 3 D, 1)
    assert one.shape == (3, 1, D) and one.stride(1) == 3 * D
    o = ctx.kv_attend(one, pool.pages, i32(pool.table), i32([6]), i32([9]), rows_per_seq=3, want_lse=True)
    check_rows(pool, one, o, {i: (0, list(range(7 + i))) for i in range(3)})
    assert ctx.poll_status() == 0


# ---- roundings --------------------------------------------------------------------------------------------

def rounded32(x, w, cs, rot, inter, eps):
    """Norm and rotation in numpy's fp32, whose every operation is rounded by itself: [T, H, D]."""
    f = np.float32
    D = x.shape[-1]
    if w is not None:
        s = x * x
        s = s[..., :D // 2] + s[..., D // 2:]
        while s.shape[-1] > 1:
            s = s[..., 0::2] + s[..., 1::2]
        x = (x * (f(1) / np.sqrt(s * f(1.0 / D) + f(eps)))) * w
    half = rot // 2
    y = x.copy()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, half), slice(half, rot))
    c, n = cs[:, None, :half], cs[:, None, half:rot]
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * n, x[..., b] * c + x[..., a] * n
    return y


@pytest.mark.parametrize("D,rot,inter", [(64, 64, False), (128, 128, False), (256, 256, False), (128, 128, True), (128, 48, False), (64, 32, True)])
@pytest.mark.parametrize("norm", [False, True])
def test_write_rounds_every_operation_by_itself(ctx, D, rot, inter, norm):
    """Whatever the form of the rotation: the outputs, and with them the keys' bytes, are numpy's to the bit."""
    rng = np.random.default_rng(D + rot + norm)
    T, Hq, Hkv = 70, 3, 2
    x = rng.standard_normal((T, Hq + 2 * Hkv, D)).astype(np.float32)
    w = [(1 + 0.2 * rng.standard_normal(D)).astype(np.float32) for _ in range(2)] if norm else [None, None]
    cs = rng.standard_normal((T, rot)).astype(np.float32)
    dev = torch.as_tensor(x).cuda()
    pages = torch.zeros((2, Hkv, ref.head_bytes(D)), dtype=torch.uint8, device="cuda")
    wd = [None if y is None else torch.as_tensor(y).cuda() for y in w]
    o = ctx.kv_write(pages, dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:], i32(np.arange(T)), i32(np.arange(T)), torch.as_tensor(cs).cuda(),
                     *wd, interleaved=inter, keep_k=True)
    assert ctx.poll_status() == 0
    k = rounded32(x[:, Hq:Hq + Hkv], w[1], cs, rot, inter, 1e-6)
    assert np.array_equal(o["q"].cpu().numpy(), rounded32(x[:, :Hq], w[0], cs, rot, inter, 1e-6))
    assert np.array_equal(o["k"].cpu().numpy(), k)
    raw = np.zeros(pages.shape, np.uint8)
    for t in range(T):
        ref.store(raw, t, ref.Entry(k[t], x[t, Hq + Hkv:]), D)
    assert np.array_equal(pages.cpu().numpy(), raw)


@pytest.mark.parametrize("new,dtype", [(3, "f32"), (3, "bf16"), (20, "bf16"), (40, "bf16")])
def test_attend_with_products_far_below_zero(ctx, new, dtype):
    """Sums near -10^33, that is, far below anything but -inf: the largest of them still wins."""
    rng = np.random.default_rng(new)
    pool = Pool(rng, [150], 1, 64, garbage=False)
    raw = pool.pages.cpu().numpy()
    for c in range(150):
        e = ref.Entry(np.abs(rng.standard_normal((1, 64))).astype(np.float32) * 1e16, rng.standard_normal((1, 64)).astype(np.float32))
        ref.store(raw, int(pool.table[0, c // PAGE]) * PAGE + c % PAGE, e, 64)
        pool.k[0][c], pool.v[0][c] = e.values("k"), e.values("v")
    pool.pages = torch.as_tensor(raw).cuda()
    q = -queries(rng, new, 4, 64, dtype, 1e16).abs()
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([150 - new]), i32([150]), rows_per_seq=new, want_lse=True)
    assert ctx.poll_status() == 0
    qn, got, lse = f64(q), f64(o["out"]), f64(o["lse"])
    for i in range(new):
        _, wl, size = ref.attend(qn[i], pool.k[0], pool.v[0], list(range(151 - new + i)), 0.125)
        assert (wl < -1e31).all() and (np.abs(lse[i] - wl) <= size * 2.0 ** -20 + 2.0 ** -21 * np.abs(wl)).all()
        assert (np.abs(got[i]).max(-1) > 0).all() and np.abs(got[i]).max() <= np.abs(pool.v[0]).max() * (1 + 2.0 ** -7)


# ---- captured graphs and scratch -----------------------------------------------------------------------

def attend_case(rng, D=64, dtype="bf16"):
    """One long sequence: many CTAs meet in the scratch."""
    pool = Pool(rng, [4000], 1, D)
    q = queries(rng, 1, 4, D, dtype)
    return pool, q, (pool.pages, i32(pool.table), i32([3999]), i32([4000]))


def test_scratch_is_cleared_by_registering_it_again(ctx):
    """What a call that timed out leaves behind: tickets that are not zero."""
    pool, q, args = attend_case(np.random.default_rng(30))
    want = ctx.kv_attend(q, *args, rows_per_seq=1)["out"].clone()
    torch.cuda.synchronize()
    ctx.kv_workspace(64).fill_(0x5A)
    ctx.reinit_workspace()
    o = ctx.kv_attend(q, *args, rows_per_seq=1, want_lse=True, outputs=nan_outputs(1, 4, 64, "bf16"))
    assert torch.equal(o["out"], want) and ctx.poll_status() == 0


@pytest.fixture(scope="module")
def long_pools():
    rng = np.random.default_rng(35)
    return {D: Pool(rng, [4000], 1, D) for D in (64, 128, 256)}


@pytest.mark.parametrize("new,D,dtype", [(1, 64, "bf16"), (1, 128, "f32"), (1, 256, "bf16"), (16, 128, "bf16"), (35, 64, "bf16")])
@pytest.mark.parametrize("page", [0, 1, 3])
def test_a_wait_that_runs_out_ends_the_call_and_the_context_recovers(long_pools, new, D, dtype, page):
    """One of the first CTA's pages never arrives: its waits run out, the call ends by itself and the status
    word says so.  Nothing faults; with the scratch registered again the same call gives what it gave."""
    c = binding.Context()
    try:
        B, n, pool = 200, 4000, long_pools[D]      # several pages for every warp, and sequences that CTAs share
        q = queries(np.random.default_rng(page), B * new, 4, D, dtype)
        args = (q, pool.pages, i32(np.tile(pool.table, (B, 1))), i32([n - new] * B), i32([n] * B))
        want = c.kv_attend(*args, rows_per_seq=new)["out"].clone()
        assert c.poll_status() == 0
        c.debug_withhold_tile(page, 0, 1 << 14)
        c.kv_attend(*args, rows_per_seq=new)
        torch.cuda.synchronize()                   # the call ended by itself
        assert c.poll_status() == binding.STATUS_TIMEOUT
        c.reinit_workspace()
        assert torch.equal(c.kv_attend(*args, rows_per_seq=new)["out"], want) and c.poll_status() == 0
        # used up by one call; there is no page of that number
        c.debug_withhold_tile(10 ** 12, 0, 1 << 22)
        assert torch.equal(c.kv_attend(*args, rows_per_seq=new)["out"], want) and c.poll_status() == 0
    finally:
        c.close()


def test_a_captured_call_keeps_its_scratch():
    """A graph holds the scratch's address: calls with a larger head dimension do not move it."""
    c = binding.Context()
    try:
        pool, q, args = attend_case(np.random.default_rng(31))
        o = nan_outputs(1, 4, 64, "bf16")
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            c.set_stream(side)
            want = c.kv_attend(q, *args, rows_per_seq=1)["out"].clone()
            size = c.kv_workspace(64).numel()
            side.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                c.kv_attend(q, *args, rows_per_seq=1, outputs=dict(out=o["out"]))
            wide, wq, wargs = attend_case(np.random.default_rng(32), 256)
            c.kv_attend(wq, *wargs, rows_per_seq=1)
            others = [torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]
            for _ in range(2):
                g.replay()
            side.synchronize()
        assert torch.equal(o["out"], want) and c.poll_status() == 0
        assert all(bool((x == 0x5A).all()) for x in others)
    finally:
        c.close()


def test_scratch_of_a_call_that_is_captured_first_is_not_taken_for_cleared():
    """Its clearing is part of the graph and has not run when the next call is made."""
    c = binding.Context()
    try:
        pool, q, args = attend_case(np.random.default_rng(33))
        first, second = nan_outputs(1, 4, 64, "bf16"), nan_outputs(1, 4, 64, "bf16")
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            c.set_stream(side)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                c.kv_attend(q, *args, rows_per_seq=1, outputs=dict(out=first["out"]))
            assert c._kv_ws == {}
            c.kv_attend(q, *args, rows_per_seq=1, outputs=dict(out=second["out"]))
            for _ in range(2):
                g.replay()
            side.synchronize()
        assert torch.equal(first["out"], second["out"]) and bool(torch.isfinite(first["out"]).all()) and c.poll_status() == 0
    finally:
        c.close()


def test_a_steps_calls_replayed_from_a_graph(ctx):
    """Plan, write, attend and commit as one graph: two replays over changed inputs give what the calls give."""
    rng = np.random.default_rng(34)
    B, cap, Hq, Hkv, D = 3, 9, 8, 2, 64
    P, pool = 6, 20
    parent = i32(np.stack([_tree(rng, cap) for _ in range(B)]))
    depth = i32([[len(ref.path_of(i, parent.cpu().numpy()[b])) - 1 for i in range(cap)] for b in range(B)])
    cs = torch.as_tensor(rng.standard_normal((400, D)).astype(np.float32)).cuda()

    def state(seed):
        r = np.random.default_rng(seed)
        x = torch.as_tensor(r.standard_normal((B * cap, Hq + 2 * Hkv, D)).astype(np.float32)).to(torch.bfloat16).cuda()
        return dict(x=x, best=i32(r.integers(0, cap, B)))

    def books():
        return dict(pages=torch.zeros((1, pool, Hkv, ref.head_bytes(D)), dtype=torch.uint8, device="cuda"), table=i32(np.full((B, P), -1)),
                    held=i32([0] * B), free=i32(np.arange(pool)), n_free=i32([pool]), length=i32([0] * B), new=i32([cap] * B))

    def step(s, k):
        plan = ctx.kv_plan(k["length"], k["new"], k["table"], k["held"], k["free"], k["n_free"], B * cap, cap, depth.view(-1))
        x = s["x"]
        q = ctx.kv_write(k["pages"][0], x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], plan["slot_map"], plan["positions"], cs)["q"]
        out = ctx.kv_attend(q, k["pages"][0], k["table"], k["length"], plan["kv_len"], rows_per_seq=cap, node_parent=parent.view(-1))["out"]
        k["length"].copy_(ctx.kv_commit(k["pages"], k["table"], k["length"], plan["kv_len"], s["best"], parent))
        return out

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    try:
        with torch.cuda.stream(side):
            ctx.set_stream(side)
            a, want = books(), []
            inputs = [state(40 + i) for i in range(3)]
            for s in inputs:
                want.append(step(s, a).clone())
            b, held = books(), {k: v.clone() for k, v in inputs[0].items()}
            side.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                out = step(held, b)
            for s, w in zip(inputs, want):
                for k in held:
                    held[k].copy_(s[k])
                g.replay()
                side.synchronize()
                assert torch.equal(out, w)
            assert all(torch.equal(a[k], b[k]) for k in a)
    finally:
        ctx.set_stream(torch.cuda.current_stream())
    assert ctx.poll_status() == 0


# ---- branches of the many-row kernel ------------------------------------------------------------------

# tokens, query heads of one key head: one tile of 128 rows (two groups on alternate pages), a pair of tiles
TILES = [(16, 4), (35, 4)]


def replace(pool, which, entry):
    """Other entries at places {(sequence, place)}."""
    raw = pool.pages.cpu().numpy()
    for b, c in which:
        e = entry(b, c)
        ref.store(raw, int(pool.table[b, c // PAGE]) * PAGE + c % PAGE, e, pool.D)
        pool.k[b][c], pool.v[b][c] = e.values("k"), e.values("v")
    pool.pages = torch.as_tensor(raw).cuda()


def causal(kv, new):
    return {b * new + i: (b, list(range(n - new + i + 1))) for b, n in enumerate(kv) for i in range(new)}


@pytest.mark.parametrize("new,G", TILES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kscale,vscale,qscale", [(4.0, 1e-4, 3.0), (0.01, 3e4, 1.0), (1.0, 1.0, 1e3), (1e-3, 1.0, 1e-3)])
def test_tiles_with_large_products_and_values_of_any_size(ctx, new, G, D, kscale, vscale, qscale):
    rng = np.random.default_rng(50)
    kv = [300, 70]
    pool = Pool(rng, kv, 2, D, kscale, vscale)
    q = queries(rng, 2 * new, 2 * G, D, "bf16", qscale)
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([n - new for n in kv]), i32(kv), rows_per_seq=new, want_lse=True,
                      outputs=nan_outputs(2 * new, 2 * G, D, "bf16"))
    assert ctx.poll_status() == 0
    check_rows(pool, q, o, causal(kv, new))


@pytest.mark.parametrize("new,G", TILES)
@pytest.mark.parametrize("page", [0, 1, 3])
def test_tiles_whose_values_grow_by_2_to_the_20_on_one_page(ctx, new, G, page):
    rng = np.random.default_rng(51)
    pool = Pool(rng, [390], 1, 128)
    replace(pool, [(0, page * PAGE + 17)], lambda b, c: ref.Entry(rng.standard_normal((1, 128)), rng.standard_normal((1, 128)).astype(np.float32) * 2.0 ** 20))
    q = queries(rng, new, G, 128, "bf16")
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([390 - new]), i32([390]), rows_per_seq=new, want_lse=True)
    assert ctx.poll_status() == 0
    check_rows(pool, q, o, causal([390], new))


@pytest.mark.parametrize("new,G", TILES)
def test_tiles_whose_products_rise_from_page_to_page(ctx, new, G):
    """Every later page's products are far above all that came before: O is rescaled each time."""
    rng = np.random.default_rng(52)
    pool = Pool(rng, [390], 1, 64)
    grow = [1, 30, 200, 1000, 3000, 10000, 30000]
    replace(pool, [(0, c) for c in range(390)], lambda b, c: ref.Entry(np.abs(rng.standard_normal((1, 64))).astype(np.float32) * grow[c // PAGE],
                                                                        rng.standard_normal((1, 64)).astype(np.float32)))
    q = queries(rng, new, G, 64, "bf16").abs()
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([390 - new]), i32([390]), rows_per_seq=new, want_lse=True)
    assert ctx.poll_status() == 0
    check_rows(pool, q, o, causal([390], new))


@pytest.mark.parametrize("new,G", TILES)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", [1e4, 1e7, 1e15])
def test_tiles_whose_products_are_larger_than_fp32_counts(ctx, new, G, sign, size):
    """At 2^24 and more the products' own roundings decide the weights: the results stay means of the values,
    and the lse the largest product."""
    rng = np.random.default_rng(56)
    pool = Pool(rng, [390], 1, 64)
    replace(pool, [(0, c) for c in range(390)], lambda b, c: ref.Entry(np.abs(rng.standard_normal((1, 64))).astype(np.float32) * size,
                                                                        rng.standard_normal((1, 64)).astype(np.float32)))
    q = queries(rng, new, G, 64, "bf16", size).abs() * sign
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([390 - new]), i32([390]), rows_per_seq=new, want_lse=True)
    assert ctx.poll_status() == 0
    got, lse, qn, top = f64(o["out"]), f64(o["lse"]), f64(q), np.abs(pool.v[0]).max()
    for i in range(new):
        _, wl, most = ref.attend(qn[i], pool.k[0], pool.v[0], list(range(391 - new + i)), 0.125)
        assert (np.abs(lse[i] - wl) <= most * 2.0 ** -20 + 2.0 ** -21 * np.abs(wl)).all()
        assert (np.abs(got[i]).max(-1) > 0).all() and np.abs(got[i]).max() <= top * (1 + 2.0 ** -7)


@pytest.mark.parametrize("new,G", TILES)
def test_tiles_with_a_scale_and_unaligned_queries_and_results(ctx, new, G):
    rng = np.random.default_rng(53)
    kv = [130, 41]
    pool = Pool(rng, kv, 2, 64)
    buf = queries(rng, 2 * new, 1, 2 * G * 64 + 3, "bf16")[:, 0]
    q = buf[:, 1:1 + 2 * G * 64].unflatten(1, (2 * G, 64))
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([n - new for n in kv]), i32(kv), rows_per_seq=new, scale=0.37, want_lse=True,
                      outputs=nan_outputs(2 * new, 2 * G, 64, "bf16", shift=1))
    assert ctx.poll_status() == 0
    check_rows(pool, q, o, causal(kv, new), scale=0.37)


@pytest.mark.parametrize("new,G", TILES + [(3, 4)])
@pytest.mark.parametrize("gone", [(0,), (1,), (2, 3), (0, 1, 2, 3, 4, 5, 6)])
def test_pages_that_the_table_does_not_name_are_not_seen(ctx, new, G, gone):
    rng = np.random.default_rng(54)
    pool = Pool(rng, [390], 1, 64)
    table = pool.table.copy()
    for p in gone:
        table[0, p] = -1 if p % 2 else pool.pages.shape[0] + 3
    q = queries(rng, new, G, 64, "bf16")
    o = ctx.kv_attend(q, pool.pages, i32(table), i32([390 - new]), i32([390]), rows_per_seq=new, want_lse=True,
                      outputs=nan_outputs(new, G, 64, "bf16"))
    assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS
    check_rows(pool, q, o, {t: (b, [c for c in vis if c // PAGE not in gone]) for t, (b, vis) in causal([390], new).items()})


@pytest.mark.parametrize("new,G", TILES + [(3, 4)])
def test_parents_that_do_not_precede_their_children_end_the_path(ctx, new, G):
    rng = np.random.default_rng(55)
    pool = Pool(rng, [200], 1, 64)
    parent = _tree(rng, new)
    parent[1], parent[new - 1] = 1, new + 5
    q = queries(rng, new, G, 64, "bf16")
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32([200 - new]), i32([200]), rows_per_seq=new, node_parent=i32(parent), want_lse=True)
    assert ctx.poll_status() == binding.STATUS_BAD_OFFSETS
    rows = {}
    for i in range(new):
        path, x = [], i
        while x >= 0:
            path.append(x)
            x = int(parent[x]) if parent[x] < x else -1
        rows[i] = (0, list(range(200 - new)) + [200 - new + x for x in sorted(path)])
    check_rows(pool, q, o, rows)


@pytest.mark.parametrize("new", [(1,) * 12 + (200,), (200,) + (1,) * 70, (1, 90, 1, 0, 33, 1, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_chunks_and_single_tokens_in_one_packed_call(ctx, new, D):
    """Whichever kernel the mean length chooses, with room left behind the last sequence."""
    rng = np.random.default_rng(sum(new))
    cached = rng.integers(0, 200, len(new))
    kv = cached + np.array(new)
    pool = Pool(rng, kv, 1, D)
    offs = np.concatenate([[0], np.cumsum(new)])
    T = int(offs[-1]) + 9
    q = queries(rng, T, 4, D, "bf16")
    o = ctx.kv_attend(q, pool.pages, i32(pool.table), i32(cached), i32(kv), i32(offs), want_lse=True, outputs=nan_outputs(T, 4, D, "bf16"))
    assert ctx.poll_status() == 0
    check_rows(pool, q, o, {int(offs[b]) + i: (b, list(range(int(cached[b]) + i + 1))) for b in range(len(new)) for i in range(new[b])})


def test_pools_of_more_than_4_gb(ctx):
    """Every call on pages whose bytes lie past 32-bit offsets, in a second layer: what a small pool gives, to the bit."""
    g = torch.Generator(device="cuda").manual_seed(60)
    Hq, Hkv, D, B, cap = 32, 8, 128, 2, 24
    n, P = 66000, 4                                         # 4.6 GB a layer
    big, small = binding.kv_pages(n, Hkv, D, layers=2), binding.kv_pages(B * P, Hkv, D, layers=2)
    assert big[0].numel() > 1 << 32
    big[:, -B * P:].fill_(85)
    small.fill_(85)
    cached, kv = i32([130, 70]), i32([130 + cap, 70 + cap])
    parent = i32(np.stack([_tree(np.random.default_rng(b), cap) for b in range(B)]))
    got = []
    for pages, at in ((small, 0), (big, n - B * P)):
        g.manual_seed(61)
        table = (torch.arange(B * P, dtype=torch.int32, device="cuda") + at).view(B, P).contiguous()
        place = torch.cat([table[b, torch.arange(int(kv[b]), device="cuda") // PAGE] * PAGE + torch.arange(int(kv[b]), device="cuda") % PAGE for b in range(B)])
        slots = place.to(torch.int32).contiguous()
        out = []
        for layer in range(2):
            x = torch.randn((slots.numel(), Hq + 2 * Hkv, D), generator=g, device="cuda").bfloat16()
            ctx.kv_write(pages[layer], x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], slots, torch.zeros_like(slots))
            for new, dtype in ((cap, torch.bfloat16), (1, torch.bfloat16), (1, torch.float32)):
                q = torch.randn((B * new, Hq, D), generator=g, device="cuda").to(dtype)
                out.append(ctx.kv_attend(q, pages[layer], table, kv - new, kv, rows_per_seq=new, node_parent=parent if new == cap else None)["out"])
        new_len = ctx.kv_commit(pages, table, cached, kv, i32([cap - 1, cap - 2]), parent)
        e = ctx.kv_read(pages[1], slots, D)
        got.append(out + [new_len, e["k"], e["v"], pages[:, at:at + B * P].clone()])
    assert ctx.poll_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(*got))
