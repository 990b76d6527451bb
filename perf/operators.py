"""Cases that measure the paged 4-bit cache's operators, and their plain forms.

The operators sit between drafting and verification of a decoding step: page book-keeping
(``plan``), norm + rotation of queries and keys and the store into the cache (``write``),
attention of the new tokens over the cache (``attend``), moving the accepted path's entries
(``commit``); entries are read back as values where the cache itself is an output.

A page holds 64 tokens of every key/value head.  Bytes of one head of a page, D channels:
  [64][D/2]  keys: byte i of a token holds channel i (low half) and channel i + D/2 (high half)
  [D/2][64]  values: byte t of row i holds channels i and i + D/2 of token t
  [64] u32   keys' scale (bf16, low 16 bits) and minimum (bf16, high 16 bits) per token
  [64] u32   values' scale and minimum per token
A code c stands for scale * c + minimum.
"""
from __future__ import annotations

import math

import torch

own = False          # set from outside: False = the plain forms, True = the framework's operators

PAGE = 64
TINY = 2.0 ** -60    # smallest scale
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one decoding step's book-keeping for four sequences with draft trees of 8 tokens
        dict(name="plan_step_4", op="plan", n_seqs=4, tree=9, ctx_lo=400, ctx_hi=520, pool=64, fresh=0),
        # 256 prompts of ragged lengths arrive at once: tables and slots of ~260k tokens, room for twice that
        dict(name="plan_prompts_256", op="plan", n_seqs=256, tree=0, ctx_lo=1, ctx_hi=2047, pool=5200, fresh=1),
        # the draft tree of one long sequence (12 draft tokens at 16k), one layer
        dict(name="write_tree_1", op="write", n_tokens=13, hq=32, hkv=8, dim=128, dtype="bf16", pos=16384, rot=128, inter=0, norm=1, pool=64),
        # a prefill block of 4 prompts x 1024 tokens (a serving step's arrivals)
        dict(name="write_prefill_4k", op="write", n_tokens=4096, hq=32, hkv=8, dim=128, dtype="bf16", pos=1024, rot=128, inter=0, norm=1, pool=80),
        # fp32 model, odd token count, half of each head rotated in neighbouring pairs, no norm
        dict(name="write_f32_odd", op="write", n_tokens=1021, hq=6, hkv=2, dim=64, dtype="f32", pos=2048, rot=32, inter=1, norm=0, pool=24),
        # one fp32 sequence of the smallest configuration decodes one token
        dict(name="attend_f32_512", op="attend", n_seqs=1, new=1, tree=0, hq=8, hkv=2, dim=64, dtype="f32", ctx_lo=512, ctx_hi=512),
        # one long sequence decodes one token
        dict(name="attend_one_16k", op="attend", n_seqs=1, new=1, tree=0, hq=32, hkv=8, dim=128, dtype="bf16", ctx_lo=16384, ctx_hi=16384),
        # a full serving batch, ragged, one token each, seven query heads per key head
        dict(name="attend_batch_256", op="attend", n_seqs=256, new=1, tree=0, hq=28, hkv=4, dim=128, dtype="bf16", ctx_lo=100, ctx_hi=4000),
        # 32 sequences verify draft trees of 4 x 8 tokens over ~4k of context
        dict(name="attend_tree_32", op="attend", n_seqs=32, new=33, tree=1, hq=32, hkv=8, dim=128, dtype="bf16", ctx_lo=3500, ctx_hi=4096),
        # two prompts continue their prefill by 2048 tokens each
        dict(name="attend_chunk_2k", op="attend", n_seqs=2, new=2048, tree=0, hq=32, hkv=8, dim=128, dtype="bf16", ctx_lo=0, ctx_hi=2048),
        # the accepted path of one tree, 16 layers
        dict(name="commit_1", op="commit", n_seqs=1, cands=4, draft=8, layers=16, hkv=8, dim=128, ctx_lo=2048, ctx_hi=2048),
        # a serving step's accepted paths, 8 layers
        dict(name="commit_256", op="commit", n_seqs=256, cands=2, draft=8, layers=8, hkv=4, dim=128, ctx_lo=200, ctx_hi=1024),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(["plan", "write", "attend", "attend", "commit"])
    dim = rng.choice([64, 128, 128, 256])
    hkv = rng.choice([1, 2, 4, 5, 8])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "plan":
        n, fresh, hi = log(1, 400), rng.choice([0, 1]), log(8, 2000)
        pool = n * (hi // 64 + 2)
        if fresh:
            pool = pool // rng.choice([1, 1, 2]) + 1          # some prompts may find no room
        return dict(op=op, n_seqs=n, tree=0 if fresh else rng.choice([0, 2, 9, 17, 33]), ctx_lo=1, ctx_hi=hi, pool=pool, fresh=fresh)
    if op == "write":
        n, hkv = log(1, 4000), min(hkv, 4)
        return dict(op=op, n_tokens=n, hq=hkv * rng.choice([2, 5, 7, 8]), hkv=hkv, dim=dim, dtype=dtype, pos=log(64, 30000),
                    rot=rng.choice([dim, dim, dim // 2, 0]), inter=rng.choice([0, 0, 1]), norm=rng.choice([0, 1, 1]),
                    pool=n // 64 + 3 + log(1, 50))
    hq = hkv * rng.choice([1, 2, 4, 5, 7, 8])
    if op == "attend":
        kind = rng.choice(["one", "tree", "chunk"])
        while True:
            n = log(1, 200 if kind == "one" else 40 if kind == "tree" else 4)
            new = 1 if kind == "one" else rng.randint(2, 65) if kind == "tree" else log(2, 2000)
            hi = log(1, 40000 if n < 4 else 4000)
            keys = hi + new
            if n * keys * hkv * dim <= 4e8 and n * new * keys * hq * dim <= 3.5e10 / (1 if dtype == "bf16" else 8):
                break
        return dict(op=op, n_seqs=n, new=new, tree=int(kind == "tree"), hq=hq, hkv=hkv, dim=dim, dtype=dtype,
                    ctx_lo=rng.choice([0, hi // 2, hi]), ctx_hi=hi)
    while True:
        n, layers, hi = log(1, 200), rng.choice([1, 2, 5, 16]), log(1, 2000)
        if n * (hi + 100) * layers * hkv * dim <= 1.2e9:
            break
    return dict(op=op, n_seqs=n, cands=rng.choice([1, 2, 4]), draft=rng.randint(1, 12), layers=layers, hkv=hkv, dim=dim,
                ctx_lo=hi // 2, ctx_hi=hi)


# ---- inputs ------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)


def page_bytes(dim):
    return PAGE * dim + 2 * PAGE * 4


def quantise(x):
    """fp32 rows [..., D] -> codes (uint8), scale, minimum (bf16)."""
    lo, hi = x.amin(-1), x.amax(-1)
    m = lo.to(torch.bfloat16)
    s = ((hi - m.float()) * (1.0 / 15.0)).to(torch.bfloat16).clamp(min=TINY)
    inv = 1.0 / s.float()
    c = torch.round((x - m.float()[..., None]) * inv[..., None]).clamp(0, 15).to(torch.uint8)
    return c, s, m


def _meta(s, m):
    return torch.stack([s, m], -1).view(torch.int32)[..., 0]


def make_pages(g, n, hkv, dim):
    """A pool in use: keys with a few channels that stand out, values around zero."""
    out = torch.empty((n, hkv, page_bytes(dim)), dtype=torch.uint8, device="cuda")
    lift = torch.randn((hkv, 1, dim), generator=g, device="cuda")
    lift = lift * (lift.abs() > 1.5)
    for a in range(0, n, 512):
        b = min(n, a + 512)
        k = torch.randn((b - a, hkv, PAGE, dim), generator=g, device="cuda") + lift
        v = torch.randn((b - a, hkv, PAGE, dim), generator=g, device="cuda") * 0.7
        fill_pages(out[a:b], k, v, dim)
    return out


def fill_pages(out, k, v, dim):
    n, hkv = out.shape[:2]
    h, kb = dim // 2, PAGE * dim // 2
    c, s, m = quantise(k)
    out[:, :, :kb] = (c[..., :h] | (c[..., h:] << 4)).reshape(n, hkv, kb)
    out[:, :, 2 * kb:2 * kb + 4 * PAGE] = _meta(s, m).view(torch.uint8).reshape(n, hkv, 4 * PAGE)
    c, s, m = quantise(v)
    out[:, :, kb:2 * kb] = (c[..., :h] | (c[..., h:] << 4)).transpose(-1, -2).reshape(n, hkv, kb)
    out[:, :, 2 * kb + 4 * PAGE:] = _meta(s, m).view(torch.uint8).reshape(n, hkv, 4 * PAGE)


def make_parents(g, n, nodes):
    """Draft trees in which every node hangs on one of the few before it."""
    i = torch.arange(nodes, device="cuda", dtype=torch.int32)
    back = torch.randint(1, 5, (n, nodes), generator=g, device="cuda", dtype=torch.int32)
    par = (i - back).clamp(min=0)
    par[:, 0] = -1
    return par


def make_cands(g, n, cands, draft):
    """Parents of trees merged from `cands` candidates of `draft` tokens: the first one whole, the
    others leave it at some depth.  Node ids grow candidate by candidate; slots left over are unused."""
    cap = 1 + cands * draft
    par = torch.full((n, cap), -1, dtype=torch.int32, device="cuda")
    j = torch.arange(draft, device="cuda", dtype=torch.int32)
    par[:, 1:1 + draft] = j
    used = torch.full((n,), 1 + draft, dtype=torch.int32, device="cuda")
    for _ in range(1, cands):
        at = torch.randint(0, draft, (n, 1), generator=g, device="cuda", dtype=torch.int32)     # depth it leaves at
        new = draft - at
        node = used[:, None] + j                                                              # its own nodes
        ok = j < new
        col = torch.where(ok, node, torch.zeros_like(node)).long()
        val = torch.where(j == 0, at, node - 1)
        par.scatter_(1, col, torch.where(ok, val, torch.full_like(val, -1)))
        used = used + new[:, 0]
    par[:, 0] = -1
    return par, used


def make_table(g, lens, pool, width):
    """Block tables over a shuffled pool; entries past a sequence's pages are -1."""
    need = (lens + PAGE - 1) // PAGE
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    start = torch.cumsum(need, 0) - need
    j = torch.arange(width, device="cuda", dtype=torch.int32)
    at = (start[:, None] + j).clamp(max=pool - 1).long()
    table = torch.where(j < need[:, None], order[at], torch.full_like(order[at], -1))
    return table.to(torch.int32).contiguous(), need.to(torch.int32), order


def prepare(case, seed):
    g, c = _gen(seed), case
    if c["op"] == "plan":
        n = c["n_seqs"]
        lens = _ints(g, c["ctx_lo"], c["ctx_hi"], n)
        width = (c["ctx_hi"] + max(c["tree"], 1)) // PAGE + 1
        if c["fresh"]:
            cached, new = torch.zeros_like(lens), lens
            total, rows, depth = n * c["ctx_hi"], 0, None     # room for the longest prompts
        else:
            cached = lens
            rows = max(c["tree"], 1)
            total = n * rows
            new = _ints(g, 1, rows, n)
            depth = None
            if c["tree"]:
                depth = torch.arange(rows, device="cuda", dtype=torch.int32).repeat(n, 1) // 2
                depth = depth.reshape(-1).contiguous()
        # what the sequences hold: pages of a longer draft region of the step before for some, none for fresh ones
        held = cached if c["fresh"] else cached + _ints(g, 0, 40, n)
        held = torch.minimum(held, torch.full_like(held, width * PAGE))
        table, need, order = make_table(g, held, c["pool"], width)
        used = int(need.sum())
        free = torch.full((c["pool"],), -1, dtype=torch.int32, device="cuda")
        free[:c["pool"] - used] = order[used:]
        count = torch.tensor([c["pool"] - used], dtype=torch.int32, device="cuda")
        book = torch.cat([table.reshape(-1), need, free, count])
        return dict(case=c, cached=cached, new=new, depth=depth, rows=rows, total=total, book=book, width=width)
    if c["op"] == "write":
        n, hq, hkv, d = c["n_tokens"], c["hq"], c["hkv"], c["dim"]
        dt = DTYPES[c["dtype"]]
        qkv = torch.randn((n, (hq + 2 * hkv) * d), generator=g, device="cuda").to(dt)
        q, k, v = qkv[:, :hq * d], qkv[:, hq * d:(hq + hkv) * d], qkv[:, (hq + hkv) * d:]
        q, k, v = q.view(n, hq, d), k.view(n, hkv, d), v.view(n, hkv, d)
        w = [(1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dt) for _ in range(2)] if c["norm"] else [None, None]
        rot = c["rot"]
        ang = torch.arange(c["pos"] + n, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(rot // 2, device="cuda", dtype=torch.float64) / max(rot // 2, 1))
        cs = torch.cat([ang.cos(), ang.sin()], 1).float().contiguous() if rot else None
        run = max(1, min(n, c["pos"]))
        pos = (c["pos"] - run + torch.arange(n, device="cuda") % run).to(torch.int32)
        page = torch.randperm(c["pool"], generator=g, device="cuda")
        at = torch.arange(n, device="cuda") + int(_ints(g, 0, 60, 1))
        slots = (page[at // PAGE] * PAGE + at % PAGE).to(torch.int32)
        pages = torch.randint(0, 256, (c["pool"], hkv, page_bytes(d)), generator=g, device="cuda", dtype=torch.uint8)
        return dict(case=c, q=q, k=k, v=v, w=w, cs=cs, pos=pos, slots=slots, pages=pages)
    if c["op"] == "attend":
        n, new, hq, hkv, d = c["n_seqs"], c["new"], c["hq"], c["hkv"], c["dim"]
        cached = _ints(g, c["ctx_lo"], c["ctx_hi"], n)
        kv = cached + new
        width = (c["ctx_hi"] + new + PAGE - 1) // PAGE
        pool = int(((kv + PAGE - 1) // PAGE).sum())
        table, need, _ = make_table(g, kv, pool, width)
        pages = make_pages(g, pool, hkv, d)
        # places past a sequence's end hold whatever was there: NaN scales here
        meta = pages[:, :, PAGE * d:].view(torch.int32).view(pool, hkv, 2, PAGE)
        last = table.gather(1, (need - 1).long()[:, None])[:, 0].long()
        past = torch.arange(PAGE, device="cuda") >= (kv - (need - 1) * PAGE)[:, None]
        meta[last] = meta[last].masked_fill(past[:, None, None, :], 0x7FC07FC0)
        q = torch.randn((n * new, hq, d), generator=g, device="cuda") * 1.5
        par = make_parents(g, n, new) if c["tree"] else None
        return dict(case=c, q=q.to(DTYPES[c["dtype"]]), pages=pages, table=table, cached=cached, kv=kv, par=par, width=width)
    n, cap = c["n_seqs"], 1 + c["cands"] * c["draft"]
    cached = _ints(g, c["ctx_lo"], c["ctx_hi"], n)
    par, used = make_cands(g, n, c["cands"], c["draft"])
    kv = cached + used
    width = (c["ctx_hi"] + cap + PAGE - 1) // PAGE
    pool = int(((kv + PAGE - 1) // PAGE).sum())
    table, need, _ = make_table(g, kv, pool, width)
    best = (torch.rand(n, generator=g, device="cuda") * used).to(torch.int32)
    pages = torch.empty((c["layers"], pool, c["hkv"], page_bytes(c["dim"])), dtype=torch.uint8, device="cuda")
    for one in pages:
        one.copy_(make_pages(g, pool, c["hkv"], c["dim"]))
    # the entries to read back: the region that an accepted path can reach, in every layer
    at = cached[:, None] + torch.arange(c["draft"] + 1, device="cuda", dtype=torch.int32)
    slots = table.gather(1, (at // PAGE).long()) * PAGE + at % PAGE
    slots = (slots.reshape(1, -1) + torch.arange(c["layers"], device="cuda", dtype=torch.int32)[:, None] * (pool * PAGE)).reshape(-1)
    return dict(case=c, pages=pages, table=table, cached=cached, kv=kv, par=par, best=best, slots=slots.to(torch.int32).contiguous(), cap=cap)


# ---- plain forms ---------------------------------------------------------------------------------

def read_plain(pages, slots, dim, dtype):
    """Values at the slots: [n, hkv, D] keys and values, slots of -1 read as zeros."""
    n, hkv = pages.shape[0], pages.shape[1]
    h, kb = dim // 2, PAGE * dim // 2
    ok = (slots >= 0)[:, None, None]
    s = slots.clamp(min=0).long()
    page, off = s // PAGE, s % PAGE
    kc = pages[:, :, :kb].unflatten(2, (PAGE, h))[page, :, off]
    vc = pages[:, :, kb:2 * kb].unflatten(2, (h, PAGE))[page, :, :, off]
    meta = pages[:, :, 2 * kb:].view(torch.bfloat16).view(n, hkv, 2, PAGE, 2)[page, :, :, off].float()
    out = []
    for b, i in ((kc, 0), (vc, 1)):
        code = torch.cat([b & 15, b >> 4], -1).float()
        x = code * meta[:, :, i, 0, None] + meta[:, :, i, 1, None]
        out.append(torch.where(ok, x, torch.zeros_like(x)).to(dtype))
    return out


def rotate_plain(x, cs, rot, inter):
    """fp32 [n, H, D] rotated by the rows of cos/sin [n, rot]."""
    if not rot:
        return x
    cos, sin = cs[:, None, :rot // 2], cs[:, None, rot // 2:]
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :rot // 2], r[..., rot // 2:])
    p, q = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([p, q], -1).flatten(-2) if inter else torch.cat([p, q], -1)
    return torch.cat([r, x[..., rot:]], -1)


def norm_plain(x, w, eps=1e-6):
    """x / sqrt(mean(x^2) + eps) * w.  The order of the sum is fixed: the halves of the row are added,
    then neighbours until one value is left."""
    x = x.float()
    if w is None:
        return x
    s, d = x * x, x.shape[-1]
    s = s[..., :d // 2] + s[..., d // 2:]
    for _ in range((d // 2).bit_length() - 1):
        s = s[..., 0::2] + s[..., 1::2]
    r = 1.0 / torch.sqrt(s / d + eps)
    return x * r * w.float()


def run_plan_plain(s):
    c, width, rows = s["case"], s["width"], s["rows"]
    n, pool = c["n_seqs"], c["pool"]
    book = s["book"].clone()
    table, held, free, count = (t.clone() for t in book.split([n * width, n, pool, 1]))
    table = table.view(n, width)
    cached, new = s["cached"].long(), s["new"].long()
    held, count = held.long(), count.long()
    j = torch.arange(width, device="cuda")
    need = (cached + new + PAGE - 1) // PAGE
    want = torch.where(need > width, torch.zeros_like(need), (need - held).clamp(min=0))
    # pages that are no longer needed go onto the stack, in order
    back = (j >= need[:, None]) & (j < held[:, None])
    rank = torch.cumsum(back.reshape(-1), 0).view(n, width) - 1
    room = torch.cat([free, free.new_zeros(1)])
    room.scatter_(0, torch.where(back, count + rank, torch.full_like(rank, pool)).reshape(-1), table.reshape(-1))
    table = torch.where(back, torch.full_like(table, -1), table)
    count = count + back.sum()
    held = torch.minimum(held, need)
    # missing ones come off it, sequence by sequence
    total = torch.cumsum(want, 0)
    served = ((want == 0) | (total <= count)) & (need <= width)
    take = (j >= held[:, None]) & (j < need[:, None]) & served[:, None]
    src = count - 1 - ((total - want)[:, None] + (j - held[:, None]))
    table = torch.where(take, room[torch.where(take, src, torch.zeros_like(src))], table)
    count = count - torch.where(served & (want > 0), total, torch.zeros_like(total)).amax()
    free = torch.where(torch.arange(pool, device="cuda") < count, room[:pool], torch.full_like(free, -1))
    held = torch.where(served, torch.maximum(held, need), held)
    kv = cached + torch.where(served, new, torch.zeros_like(new))
    t = torch.arange(s["total"], device="cuda")
    if rows:
        offs = torch.arange(n + 1, device="cuda") * rows
    else:
        offs = torch.cat([new.new_zeros(1), torch.cumsum(new, 0)])
    b = (torch.searchsorted(offs, t, right=True) - 1).clamp(max=n - 1)
    i = t - offs[b]
    at = cached[b] + i
    ok = served[b] & (i < new[b])
    slot = table[b, (at // PAGE).clamp(max=width - 1)].long() * PAGE + at % PAGE
    pos = cached[b] + (s["depth"].long() if s["depth"] is not None else i)
    slot, pos = torch.where(ok, slot, torch.full_like(slot, -1)), torch.where(ok, pos, torch.full_like(pos, -1))
    return dict(block_table=table, seq_pages=held.int(), free_pages=free, n_free=count.int(), kv_len=kv.int(),
                tok_offsets=offs.int(), slot_map=slot.int(), positions=pos.int())


def run_write_plain(s):
    c = s["case"]
    dt, d, rot = DTYPES[c["dtype"]], c["dim"], c["rot"]
    cs = s["cs"][s["pos"].long()] if rot else None
    q = rotate_plain(norm_plain(s["q"], s["w"][0]), cs, rot, c["inter"]).to(dt)
    k = rotate_plain(norm_plain(s["k"], s["w"][1]), cs, rot, c["inter"])
    pages, h, kb = s["pages"], d // 2, PAGE * d // 2
    page, off = s["slots"].long() // PAGE, s["slots"].long() % PAGE
    meta = pages[:, :, 2 * kb:].view(torch.int32).view(-1, c["hkv"], 2, PAGE)
    x, sc, mn = quantise(k)
    pages[:, :, :kb].unflatten(2, (PAGE, h))[page, :, off] = x[..., :h] | (x[..., h:] << 4)
    meta[page, :, 0, off] = _meta(sc, mn)
    x, sc, mn = quantise(s["v"].float())
    pages[:, :, kb:2 * kb].unflatten(2, (h, PAGE))[page, :, :, off] = x[..., :h] | (x[..., h:] << 4)
    meta[page, :, 1, off] = _meta(sc, mn)
    k, v = read_plain(pages, s["slots"], d, dt)
    return dict(q=q, k=k, v=v)


def ancestors(par, depth):
    """[n, N, N] truth: node j lies on the path from the root to node i (itself included)."""
    n, size = par.shape
    step = torch.eye(size, device="cuda").repeat(n, 1, 1)
    step.scatter_add_(2, par.clamp(min=0).long()[..., None], (par >= 0).float()[..., None])
    return torch.linalg.matrix_power(step, depth) > 0


def run_attend_plain(s):
    c, par = s["case"], s["par"]
    n, new, hq, hkv, d = c["n_seqs"], c["new"], c["hq"], c["hkv"], c["dim"]
    h, kb, width = d // 2, PAGE * d // 2, s["width"]
    raw = s["pages"][s["table"].clamp(min=0).long()].transpose(1, 2)         # [n, hkv, width, bytes]
    meta = raw[..., 2 * kb:].contiguous().view(torch.bfloat16).view(n, hkv, width, 2, PAGE, 2).float()
    t = torch.arange(width * PAGE, device="cuda")
    live = t < s["kv"][:, None]                                             # [n, T]
    kc = raw[..., :kb].unflatten(3, (PAGE, h))
    k = torch.cat([kc & 15, kc >> 4], -1).float() * meta[..., 0, :, 0, None] + meta[..., 0, :, 1, None]
    vc = raw[..., kb:2 * kb].unflatten(3, (h, PAGE)).transpose(-1, -2)
    v = torch.cat([vc & 15, vc >> 4], -1).float() * meta[..., 1, :, 0, None] + meta[..., 1, :, 1, None]
    k = k.flatten(2, 3).masked_fill(~live[:, None, :, None], 0.0)
    v = v.flatten(2, 3).masked_fill(~live[:, None, :, None], 0.0)
    q = s["q"].float().view(n, new, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).flatten(2, 3)
    i = torch.arange(new, device="cuda")
    if par is None:
        seen = t <= s["cached"][:, None, None] + i[:, None]                 # [n, new, T]
    else:
        anc = torch.nn.functional.pad(ancestors(par, new), (0, 1))          # one more column: not a new token
        rel = (t - s["cached"][:, None]).clamp(min=-1)
        pick = torch.where((rel < 0) | (rel >= new), torch.full_like(rel, new), rel).long()
        seen = anc.gather(2, pick[:, None].expand(n, new, -1)) | (rel < 0)[:, None]
    w = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    w = w.unflatten(2, (hq // hkv, new)).masked_fill_(~(seen & live[:, None])[:, None, None], float("-inf"))
    w = torch.exp(w - w.amax(-1, keepdim=True))
    o = torch.matmul(w.flatten(2, 3), v) / w.flatten(2, 3).sum(-1, keepdim=True)
    o = o.unflatten(2, (hq // hkv, new)).permute(0, 3, 1, 2, 4).reshape(n * new, hq, d)
    return dict(out=o.to(s["q"].dtype))


def run_commit_plain(s):
    c = s["case"]
    n, cap, d, pool = c["n_seqs"], s["cap"], c["dim"], s["pages"].shape[1]
    h, kb = d // 2, PAGE * d // 2
    path = ancestors(s["par"], c["draft"])[torch.arange(n, device="cuda"), s["best"].long()]   # [n, cap]
    rank = torch.cumsum(path, 1) - 1
    node = torch.arange(cap, device="cuda")
    at = lambda x: (s["table"].gather(1, x // PAGE).long() * PAGE + x % PAGE).reshape(-1)      # noqa: E731
    base = s["cached"].long()[:, None]
    src = at(torch.where(path, base + node, base))
    dst = at(torch.where(path, base + rank, base))
    pages = s["pages"].flatten(0, 1)
    lay = torch.arange(c["layers"], device="cuda")[:, None] * (pool * PAGE)
    src, dst = (lay + src).reshape(-1), (lay + dst).reshape(-1)
    keys, vals = pages[:, :, :kb].unflatten(2, (PAGE, h)), pages[:, :, kb:2 * kb].unflatten(2, (h, PAGE))
    meta = pages[:, :, 2 * kb:].view(torch.int32).view(-1, c["hkv"], 2, PAGE)
    sp, so, dp, do = src // PAGE, src % PAGE, dst // PAGE, dst % PAGE
    keys[dp, :, do] = keys[sp, :, so]
    vals[dp, :, :, do] = vals[sp, :, :, so]
    meta[dp, :, :, do] = meta[sp, :, :, so]
    k, v = read_plain(pages, s["slots"], d, torch.bfloat16)
    return dict(new_len=(s["cached"] + path.sum(1)).int(), k=k, v=v)


# ---- the framework's operators -------------------------------------------------------------------

_handle = None


def _context():
    """The program's one context, on torch's current stream."""
    global _handle
    if _handle is None:
        from paper_2505_13204_b200 import binding
        _handle = binding.Context()
    return _handle


def run_own(s):
    c, ctx = s["case"], _context()
    if c["op"] == "plan":
        n, width, pool = c["n_seqs"], s["width"], c["pool"]
        table, held, free, count = s["book"].clone().split([n * width, n, pool, 1])
        table = table.view(n, width)
        o = ctx.kv_plan(s["cached"], s["new"], table, held, free, count, s["total"], rows_per_seq=s["rows"],
                        node_depth=s["depth"])
        return dict(block_table=table, seq_pages=held, free_pages=free, n_free=count, **o)
    if c["op"] == "write":
        o = ctx.kv_write(s["pages"], s["q"], s["k"], s["v"], s["slots"], s["pos"], s["cs"], q_weight=s["w"][0],
                         k_weight=s["w"][1], interleaved=bool(c["inter"]))
        kv = ctx.kv_read(s["pages"], s["slots"], c["dim"], DTYPES[c["dtype"]])
        return dict(q=o["q"], k=kv["k"], v=kv["v"])
    if c["op"] == "attend":
        return ctx.kv_attend(s["q"], s["pages"], s["table"], s["cached"], s["kv"], rows_per_seq=c["new"], node_parent=s["par"])
    new_len = ctx.kv_commit(s["pages"], s["table"], s["cached"], s["kv"], s["best"], s["par"])
    kv = ctx.kv_read(s["pages"].flatten(0, 1), s["slots"], c["dim"], torch.bfloat16)
    return dict(new_len=new_len, k=kv["k"], v=kv["v"])


def run(state):
    if own:
        return run_own(state)
    return {"plan": run_plan_plain, "write": run_write_plain, "attend": run_attend_plain, "commit": run_commit_plain}[
        state["case"]["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "plan":
        mean = (c["ctx_lo"] + c["ctx_hi"]) / 2
        tokens = c["n_seqs"] * (c["ctx_hi"] if c["fresh"] else max(c["tree"], 1))
        used = c["n_seqs"] * (mean / PAGE + 1)
        return dict(bytes=tokens * 8 + used * 8 + c["n_seqs"] * 24 + (tokens * 4 if c["tree"] else 0), flops=0)
    size = 4 if c.get("dtype") == "f32" else 2
    if c["op"] == "write":
        n, d = c["n_tokens"], c["dim"]
        entry = 2 * c["hkv"] * (d // 2 + 4)                   # one token's codes and scales
        return dict(bytes=n * (d * size * (2 * c["hq"] + 4 * c["hkv"]) + 2 * entry + 8) + min(n, c["pos"]) * c["rot"] * 4,
                    flops=n * d * 10 * (c["hq"] + 2 * c["hkv"]))
    if c["op"] == "attend":
        ctx = (c["ctx_lo"] + c["ctx_hi"]) / 2
        seen = ctx + (c["new"] + 1) / 2                       # keys a query sees, on average
        n, d = c["n_seqs"], c["dim"]
        return dict(bytes=n * ((ctx + c["new"]) * 2 * c["hkv"] * (d // 2 + 4) + 2 * c["new"] * c["hq"] * d * size),
                    flops=4 * n * c["new"] * seen * c["hq"] * d)
    n, d = c["n_seqs"] * c["layers"], c["dim"]
    entry = 2 * c["hkv"] * (d // 2 + 4)
    moved = c["draft"] / 4                                    # nodes off the first candidate that an average path moves
    return dict(bytes=n * (2 * moved * entry + (c["draft"] + 1) * (entry + 4 * c["hkv"] * d)), flops=0)


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _entry64(pages, page, off, dim):
    """Keys and values of one token of one page per row, straight from the layout: [n, hkv, D] each."""
    n, hkv, size = pages.shape
    flat, h, dev = pages.reshape(-1), dim // 2, pages.device
    lane, four = torch.arange(h, device=dev), torch.arange(4, device=dev)
    head = (page.long()[:, None] * hkv + torch.arange(hkv, device=dev))[..., None] * size      # first byte of each head
    off = off.long()[:, None, None]
    res = []
    for i, at in enumerate((off * h + lane, PAGE * h + lane * PAGE + off)):
        b = flat[head + at].to(torch.int64)
        m = flat[head + PAGE * dim + i * PAGE * 4 + off * 4 + four].to(torch.int64)
        lo = ((m[..., 0] | (m[..., 1] << 8)) << 16).to(torch.int32).view(torch.float32).double()
        hi = ((m[..., 2] | (m[..., 3] << 8)) << 16).to(torch.int32).view(torch.float32).double()
        res.append(torch.cat([b % 16, b // 16], -1).double() * lo[..., None] + hi[..., None])
    return res


def _nearest_bf16(x):
    return x.to(torch.bfloat16).double()


def _coded64(x):
    """What the 4-bit cache holds for rows x (64 bits)."""
    m = _nearest_bf16(x.min(-1, keepdim=True).values)
    s = _nearest_bf16((x.max(-1, keepdim=True).values - m) / 15).clamp(min=TINY)
    return s * ((x - m) / s).round().clamp(0, 15) + m


def _rotated64(x, angle_cos, angle_sin, inter):
    """Each pair as a complex number times cos + i sin."""
    half = angle_cos.shape[-1]
    y = x.clone()
    idx = torch.arange(half, device=x.device)
    ia, ib = (2 * idx, 2 * idx + 1) if inter else (idx, idx + half)
    z = torch.complex(x[..., ia], x[..., ib]) * torch.complex(angle_cos, angle_sin)[:, None]
    y[..., ia], y[..., ib] = z.real, z.imag
    return y


def exact(case, seed):
    c = case
    if c["op"] == "plan":
        return None                                            # whole numbers only
    s = prepare(case, seed)
    if c["op"] == "write":
        d, rot = c["dim"], c["rot"]
        res = []
        for x, w in ((s["q"], s["w"][0]), (s["k"], s["w"][1])):
            x = x.double()
            if w is not None:
                x = x * w.double() / (x.square().sum(-1, keepdim=True) / d + 1e-6).sqrt()
            if rot:
                cs = s["cs"].double()[s["pos"].long()]
                x = _rotated64(x, cs[:, :rot // 2], cs[:, rot // 2:], c["inter"])
            res.append(x)
        return dict(q=res[0], k=_coded64(res[1]), v=_coded64(s["v"].double()))
    if c["op"] == "attend":
        n, new, hq, hkv, d = c["n_seqs"], c["new"], c["hq"], c["hkv"], c["dim"]
        out = torch.zeros((n * new, hq, d), dtype=torch.float64, device="cuda")
        par = s["par"].tolist() if s["par"] is not None else None
        for b, (ctx, end) in enumerate(zip(s["cached"].tolist(), s["kv"].tolist())):
            t = torch.arange(end, device="cuda")
            k, v = _entry64(s["pages"], s["table"][b][t // PAGE], t % PAGE, d)
            see = torch.ones((new, end), dtype=torch.bool)
            see[:, ctx:] = False
            for i in range(new):
                if par is None:
                    see[i, ctx:ctx + i + 1] = True
                else:
                    x = i
                    while x >= 0:
                        see[i, ctx + x] = True
                        x = par[b][x]
            see = see.cuda()
            for hh in range(hq):
                g = hh // (hq // hkv)
                w = s["q"][b * new:(b + 1) * new, hh].double() @ k[:, g].T / math.sqrt(d)
                w = w.masked_fill(~see, float("-inf")).softmax(-1)
                out[b * new:(b + 1) * new, hh] = w @ v[:, g]
        return dict(out=out)
    n, span = c["n_seqs"], c["draft"] + 1
    par, best, cached, table = s["par"].tolist(), s["best"].tolist(), s["cached"].tolist(), s["table"].tolist()
    where, lens = [], []
    for b in range(n):
        path, x = [], best[b]
        while x >= 0:
            path.append(x)
            x = par[b][x]
        path.reverse()
        lens.append(cached[b] + len(path))
        for i in range(span):
            p = cached[b] + (path[i] if i < len(path) else i)
            where.append(table[b][p // PAGE] * PAGE + p % PAGE)
    where = torch.tensor(where, device="cuda")
    got = [_entry64(layer, where // PAGE, where % PAGE, c["dim"]) for layer in s["pages"]]
    return dict(new_len=torch.tensor(lens, dtype=torch.int32), k=torch.cat([x[0] for x in got]), v=torch.cat([x[1] for x in got]))
