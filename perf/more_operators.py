"""Cases that measure the 8-bit cache's operators and the page operators, and their plain forms.

``write`` norms, rotates and stores a step's keys and values in a cache of 8 bits with one scale per page, head
and half; ``attend`` is the attention of the new tokens over it; ``commit`` moves an accepted path's entries.
``fork`` makes sequences that share another's pages; ``compact`` frees the pages of ended sequences and moves the others'
to the front of the pool.  Both work on pools of either format.

A page holds 64 tokens of every key/value head.  Bytes of one head of an 8-bit page, D channels:
  keys    [64][D] e4m3 codes (see places())
  values  [64][D]
  scales  of the keys, of the values: fp32 powers of two;  8 bytes of nothing
A code c stands for scale * c.  A scale is the least 2^e, e >= -64, with max|x| <= 448 * 2^e over the rows that are
stored; where the page holds older tokens it is at least the scale that they have, and they follow when it grows.
"""
from __future__ import annotations

import math

import torch

own = False          # set from outside: False = the plain forms, True = the framework's operators

PAGE = 64
LEAST = -64          # least exponent of a scale
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn


def listed():
    return [
        # four fp32 sequences store their draft trees of 5 tokens behind ragged contexts (one layer, small configuration)
        dict(name="write_tree_4", op="write", n_seqs=4, rows=5, new_lo=3, new_hi=5, hq=8, hkv=2, dim=64, dtype="f32", ctx_lo=400, ctx_hi=520, rot=64, inter=0, norm=1),
        # the prompts of a serving step's arrivals, ~4k tokens, ragged, some behind a cached prefix
        dict(name="write_prompts_4k", op="write", n_seqs=4, rows=0, new_lo=700, new_hi=1347, hq=32, hkv=8, dim=128, dtype="bf16", ctx_lo=0, ctx_hi=100, rot=128, inter=0, norm=1),
        # one fp32 sequence verifies a draft tree of 9 nodes
        dict(name="attend_f32_tree", op="attend", n_seqs=1, new=9, tree=1, hq=8, hkv=2, dim=64, dtype="f32", ctx_lo=701, ctx_hi=701),
        # one long sequence decodes one token
        dict(name="attend_one_16k", op="attend", n_seqs=1, new=1, tree=0, hq=32, hkv=8, dim=128, dtype="bf16", ctx_lo=16384, ctx_hi=16384),
        # a full serving batch, ragged, one token each, seven query heads per key head
        dict(name="attend_batch_256", op="attend", n_seqs=256, new=1, tree=0, hq=28, hkv=4, dim=128, dtype="bf16", ctx_lo=100, ctx_hi=4000),
        # two prompts continue their prefill by 2048 tokens each
        dict(name="attend_chunk_2k", op="attend", n_seqs=2, new=2048, tree=0, hq=32, hkv=8, dim=128, dtype="bf16", ctx_lo=0, ctx_hi=2048),
        # the accepted path of one tree, 16 layers
        dict(name="commit_1", op="commit", n_seqs=1, cands=4, draft=8, layers=16, hkv=8, dim=128, ctx_lo=2048, ctx_hi=2048),
        # a serving step's accepted paths, 4 layers
        dict(name="commit_128", op="commit", n_seqs=128, cands=2, draft=8, layers=4, hkv=4, dim=128, ctx_lo=200, ctx_hi=1024),
        # three more samples of one short prompt, 4 layers of a 4-bit pool
        dict(name="fork_3", op="fork", n_src=1, forks=3, layers=4, hkv=2, dim=64, bits=4, ctx_lo=300, ctx_hi=330, spare=8),
        # eight prompts, seven more samples of each, 16 layers of an 8-bit pool
        dict(name="fork_56", op="fork", n_src=8, forks=7, layers=16, hkv=8, dim=128, bits=8, ctx_lo=100, ctx_hi=1000, spare=70),
        # a few sequences end, the pool of a small model closes up
        dict(name="compact_12", op="compact", n_seqs=12, forks=2, ended=4, layers=2, hkv=2, dim=64, bits=8, ctx_lo=10, ctx_hi=500, spare=20),
        # a third of a serving batch ends, 8 layers
        dict(name="compact_192", op="compact", n_seqs=192, forks=4, ended=64, layers=8, hkv=8, dim=128, bits=8, ctx_lo=100, ctx_hi=600, spare=100),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(["write", "attend", "attend", "attend", "commit", "fork", "compact"])
    dim = rng.choice([64, 128, 128, 256])
    hkv = rng.choice([1, 2, 4, 5, 8])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "write":
        hkv = min(hkv, 4)
        padded = rng.choice([0, 1])
        n = log(1, 300 if padded else 16)
        hi = log(1, 40 if padded else 2000)
        while n * hi > 4000:
            hi = max(1, hi // 2)
        return dict(op=op, n_seqs=n, rows=hi if padded else 0, new_lo=rng.randint(0, hi), new_hi=hi, hq=hkv * rng.choice([2, 5, 7, 8]), hkv=hkv, dim=dim,
                    dtype=dtype, ctx_lo=0, ctx_hi=log(1, 700), rot=rng.choice([dim, dim, dim // 2, 0]), inter=rng.choice([0, 0, 1]), norm=rng.choice([0, 1, 1]))
    if op == "attend":
        hq = hkv * rng.choice([1, 2, 4, 5, 7, 8])
        kind = rng.choice(["one", "tree", "chunk"])
        while True:
            n = log(1, 200 if kind == "one" else 40 if kind == "tree" else 4)
            new = 1 if kind == "one" else rng.randint(2, 65) if kind == "tree" else log(2, 2000)
            hi = log(1, 40000 if n < 4 else 4000)
            keys = hi + new
            if n * keys * hkv * dim <= 3e8 and n * new * keys * hq * dim <= 3.5e10 / (1 if dtype == "bf16" else 8):
                break
        return dict(op=op, n_seqs=n, new=new, tree=int(kind == "tree"), hq=hq, hkv=hkv, dim=dim, dtype=dtype,
                    ctx_lo=rng.choice([0, hi // 2, hi]), ctx_hi=hi)
    if op == "commit":
        while True:
            n, layers, hi = log(1, 200), rng.choice([1, 2, 5, 16]), log(1, 2000)
            if n * (hi + 100) * layers * hkv * dim <= 6e8:
                break
        return dict(op=op, n_seqs=n, cands=rng.choice([1, 2, 4]), draft=rng.randint(1, 12), layers=layers, hkv=hkv, dim=dim,
                    ctx_lo=hi // 2, ctx_hi=hi)
    bits = rng.choice([4, 8])
    while True:
        layers, hi = rng.choice([1, 2, 5, 16]), log(2, 2000)
        n, forks = (log(1, 40), log(1, 12)) if op == "fork" else (log(2, 300), rng.choice([1, 2, 4]))
        if n * (hi + 200 + 64 * forks) * layers * hkv * dim <= 5e8:
            break
    if op == "fork":
        return dict(op=op, n_src=n, forks=forks, layers=layers, hkv=hkv, dim=dim, bits=bits, ctx_lo=0, ctx_hi=hi, spare=rng.choice([0, n * forks // 2, n * forks + 5]))
    return dict(op=op, n_seqs=n, forks=forks, ended=rng.randint(0, n), layers=layers, hkv=hkv, dim=dim, bits=bits, ctx_lo=0, ctx_hi=hi, spare=log(1, 200))


# ---- inputs ------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)


def _lens(g, lo, hi, n):
    """The same lengths, lo to hi, for every seed (outputs have to have their shapes), in an order of the seed's own."""
    x = (lo + (hi - lo) * (torch.arange(n, device="cuda") / (n - 1) if n > 1 else torch.full((1,), 0.5, device="cuda"))).round().to(torch.int32)
    return x[torch.randperm(n, generator=g, device="cuda")]


def page_bytes(dim, bits=8):
    return PAGE * dim + 2 * PAGE * 4 if bits == 4 else 2 * PAGE * dim + 16


def places(dim):
    """[64, D] byte of each token's channel inside the keys, or values: panels of at most 128 channels, in which 16-byte
    chunk c of token t lies at chunk c ^ (t % 8) of the token's 128 bytes (64 channels: c ^ (t / 2 % 4) of its 64)."""
    t, ch = torch.arange(PAGE, device="cuda")[:, None], torch.arange(dim, device="cuda")
    row = min(dim, 128)
    turn = t % 8 if row == 128 else t // 2 % 4
    return ch // row * (PAGE * row) + t * row + ((ch % row // 16) ^ turn) * 16 + ch % 16


def exponent(top):
    """Exponent of the scale for rows whose largest magnitude is `top` (fp32)."""
    m, x = torch.frexp(top)
    e = x - 9 + (m > 0.875).to(x.dtype)                       # 448 = 0.875 * 2^9
    return torch.where(top > 0, e, torch.full_like(e, LEAST)).clamp(min=LEAST)


def pow2(e):
    """2^e in fp32, -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def times2(x, e):
    """x * 2^e, in two steps: e may pass the range of fp32."""
    h = torch.div(e, 2, rounding_mode="floor")
    return x * pow2(h) * pow2(e - h)


def codes(x, e):
    return times2(x, -e).to(F8).view(torch.uint8)


def make_pages(g, n, hkv, dim):
    """A pool in use: keys with a few channels that stand out, values around zero, scales of all sizes."""
    out = torch.zeros((n, hkv, page_bytes(dim)), dtype=torch.uint8, device="cuda")
    lift = torch.randn((hkv, 1, dim), generator=g, device="cuda")
    lift = lift * (lift.abs() > 1.5)
    at = places(dim).reshape(-1)
    for a in range(0, n, 256):
        b = min(n, a + 256)
        size = torch.exp2(2 * torch.rand((2, b - a, hkv, 1, 1), generator=g, device="cuda") - 2)
        for i, x in enumerate((torch.randn((b - a, hkv, PAGE, dim), generator=g, device="cuda") + lift,
                               torch.randn((b - a, hkv, PAGE, dim), generator=g, device="cuda") * 0.7)):
            x = x * size[i]
            e = exponent(x.abs().amax((-2, -1)))
            out[a:b, :, i * PAGE * dim:(i + 1) * PAGE * dim][..., at] = codes(x, e[..., None, None]).flatten(2)
            scales(out, dim)[a:b, :, i] = pow2(e)
    return out


def scales(pages, dim):
    return pages[:, :, 2 * PAGE * dim:].view(torch.float32)


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
    par = torch.full((n, 1 + cands * draft), -1, dtype=torch.int32, device="cuda")
    j = torch.arange(draft, device="cuda", dtype=torch.int32)
    par[:, 1:1 + draft] = j
    used = torch.full((n,), 1 + draft, dtype=torch.int32, device="cuda")
    for _ in range(1, cands):
        at = torch.randint(0, draft, (n, 1), generator=g, device="cuda", dtype=torch.int32)     # depth it leaves at
        node = used[:, None] + j                                                              # its own nodes
        ok = j < draft - at
        col = torch.where(ok, node, torch.zeros_like(node)).long()
        val = torch.where(j == 0, at, node - 1)
        par.scatter_(1, col, torch.where(ok, val, torch.full_like(val, -1)))
        used = used + (draft - at)[:, 0]
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


def pages_of(lens):
    return max(1, int(((lens + PAGE - 1) // PAGE).sum()))


def raw_pool(g, case, pool):
    """Pools of all layers as bytes: the page operators move them as they are."""
    shape = (case["layers"], pool, case["hkv"], page_bytes(case["dim"], case["bits"]))
    return torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)


def prepare(case, seed):
    g, c = _gen(seed), case
    if c["op"] == "write":
        n, hq, hkv, d = c["n_seqs"], c["hq"], c["hkv"], c["dim"]
        dt = DTYPES[c["dtype"]]
        cached, new = _lens(g, c["ctx_lo"], c["ctx_hi"], n), _lens(g, c["new_lo"], c["new_hi"], n)
        kv = cached + new
        offs = torch.cat([new.new_zeros(1), torch.cumsum(new, 0).to(torch.int32)]) if not c["rows"] else torch.arange(n + 1, device="cuda", dtype=torch.int32) * c["rows"]
        total = int(offs[-1])
        width = (c["ctx_hi"] + c["new_hi"] + PAGE - 1) // PAGE
        pool = pages_of(kv)
        table, _, _ = make_table(g, kv, pool, width)
        b = torch.repeat_interleave(torch.arange(n, device="cuda"), offs.diff().long())
        i = torch.arange(total, device="cuda") - offs[b].long()
        pos = torch.where(i < new[b], cached[b] + i, torch.full_like(i, -1)).to(torch.int32)
        qkv = torch.randn((total, (hq + 2 * hkv) * d), generator=g, device="cuda").to(dt)
        q, k, v = qkv[:, :hq * d], qkv[:, hq * d:(hq + hkv) * d], qkv[:, (hq + hkv) * d:]
        q, k, v = q.view(total, hq, d), k.view(total, hkv, d), v.view(total, hkv, d)
        w = [(1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dt) for _ in range(2)] if c["norm"] else [None, None]
        rot = c["rot"]
        ang = torch.arange(c["ctx_hi"] + c["new_hi"] + 1, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(rot // 2, device="cuda", dtype=torch.float64) / max(rot // 2, 1))
        cs = torch.cat([ang.cos(), ang.sin()], 1).float().contiguous() if rot else None
        # the entries to read back: the new ones, and the live older ones of the page that each sequence goes on in
        t = torch.arange(width * PAGE, device="cuda")
        live = (t >= (cached // PAGE * PAGE)[:, None]) & (t < kv[:, None])
        slots = (table.repeat_interleave(PAGE, 1).long() * PAGE + t % PAGE)[live].to(torch.int32)
        return dict(case=c, q=q, k=k, v=v, w=w, cs=cs, pos=pos, table=table, cached=cached, kv=kv, offs=offs, slots=slots,
                    pages=make_pages(g, pool, hkv, d))
    if c["op"] == "attend":
        n, new, hq, hkv, d = c["n_seqs"], c["new"], c["hq"], c["hkv"], c["dim"]
        cached = _ints(g, c["ctx_lo"], c["ctx_hi"], n)
        kv = cached + new
        width = (c["ctx_hi"] + new + PAGE - 1) // PAGE
        pool = pages_of(kv)
        table, need, _ = make_table(g, kv, pool, width)
        pages = make_pages(g, pool, hkv, d)
        # places past a sequence's end hold whatever was there: NaN here
        last = table.gather(1, (need - 1).long()[:, None])[:, 0].long()
        past = torch.arange(PAGE, device="cuda") >= (kv - (need - 1) * PAGE)[:, None]
        at = places(d)
        for i in range(2):
            part = pages[:, :, i * PAGE * d:(i + 1) * PAGE * d]
            old = part[last][..., at]                                              # [n, hkv, 64, D]
            part[last[:, None, None, None], torch.arange(hkv, device="cuda")[:, None, None], at] = old.masked_fill(past[:, None, :, None], 0x7F)
        q = torch.randn((n * new, hq, d), generator=g, device="cuda") * 1.5
        par = make_parents(g, n, new) if c["tree"] else None
        return dict(case=c, q=q.to(DTYPES[c["dtype"]]), pages=pages, table=table, cached=cached, kv=kv, par=par, width=width)
    if c["op"] == "commit":
        n, cap = c["n_seqs"], 1 + c["cands"] * c["draft"]
        cached = _ints(g, c["ctx_lo"], c["ctx_hi"], n)
        par, used = make_cands(g, n, c["cands"], c["draft"])
        kv = cached + used
        width = (c["ctx_hi"] + cap + PAGE - 1) // PAGE
        pool = pages_of(kv)
        table, need, _ = make_table(g, kv, pool, width)
        best = (torch.rand(n, generator=g, device="cuda") * used).to(torch.int32)
        pages = torch.stack([make_pages(g, pool, c["hkv"], c["dim"]) for _ in range(c["layers"])])
        # the entries to read back: the last cached ones and the accepted path, in every layer
        at = cached[:, None] + torch.arange(-3, c["draft"] + 1, device="cuda", dtype=torch.int32)
        live = (at >= 0) & (at < (cached + ancestors(par, c["draft"])[torch.arange(n, device="cuda"), best.long()].sum(1))[:, None])
        slots = table.gather(1, (at.clamp(min=0) // PAGE).long()) * PAGE + at.clamp(min=0) % PAGE
        layer = torch.arange(c["layers"], device="cuda", dtype=torch.int32)[:, None, None] * (pool * PAGE)
        slots = torch.where(live, slots + layer, torch.full_like(slots, -1)).reshape(-1)
        return dict(case=c, pages=pages, table=table, cached=cached, kv=kv, par=par, best=best, slots=slots.to(torch.int32).contiguous(), cap=cap)
    if c["op"] == "fork":
        n, forks = c["n_src"], c["forks"]
        total = n * (1 + forks)
        width = c["ctx_hi"] // PAGE + 2
        cached = torch.zeros(total, dtype=torch.int32, device="cuda")
        cached[:n] = _lens(g, c["ctx_lo"], c["ctx_hi"], n)
        pool = pages_of(cached) + c["spare"]
        table, held, order = make_table(g, cached, pool, width)
        used = int(held.sum())
        free = torch.full((pool,), -1, dtype=torch.int32, device="cuda")
        free[:pool - used] = order[used:]
        # the samples of the prompts, prompt by prompt; some are cut shorter than what the prompt has cached
        src = torch.arange(n, device="cuda", dtype=torch.int32).repeat_interleave(forks)
        dst = (n + torch.randperm(n * forks, generator=g, device="cuda")).to(torch.int32)
        cut = _ints(g, 0, 3, n * forks) == 0
        length = torch.where(cut, (cached[src.long()] * torch.rand(n * forks, generator=g, device="cuda")).to(torch.int32), cached[src.long()])
        book = torch.cat([table.reshape(-1), held, cached, free, free.new_tensor([pool - used]), torch.zeros_like(free)])
        return dict(case=c, book=book, width=width, total=total, pool=pool, src=src, dst=dst, length=length, pages=raw_pool(g, c, pool))
    n, forks = c["n_seqs"], c["forks"]
    width = c["ctx_hi"] // PAGE + 1
    cached = _lens(g, c["ctx_lo"], c["ctx_hi"], n)
    # families of `forks` sequences share the whole pages that the shortest of them has half of
    first = torch.arange(n, device="cuda") // forks * forks
    need = (cached + PAGE - 1) // PAGE
    small = torch.full((n,), 1 << 20, dtype=torch.int32, device="cuda").scatter_reduce(0, first, cached, "amin")[first]
    common = small // 2 // PAGE
    j = torch.arange(width, device="cuda", dtype=torch.int32)
    shared = (j < common[:, None]) & (first != torch.arange(n, device="cuda"))[:, None]
    mine = (j < need[:, None]) & ~shared
    used = int(mine.sum())
    pool = pages_of(cached) + c["spare"]
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    table[mine] = order[:used]
    table = torch.where(shared, table[first], table)
    free = torch.full((pool,), -1, dtype=torch.int32, device="cuda")
    free[:pool - used] = order[used:]
    held_by = torch.zeros(pool, dtype=torch.int32, device="cuda").scatter_add_(0, table[table >= 0].long(), torch.ones_like(table[table >= 0]))
    keep = cached.masked_fill(torch.randperm(n, generator=g, device="cuda") < c["ended"], 0)
    book = torch.cat([table.reshape(-1), need.to(torch.int32), free, free.new_tensor([pool - used]), (held_by - 1).clamp(min=0)])
    return dict(case=c, book=book, width=width, pool=pool, keep=keep, pages=raw_pool(g, c, pool))


# ---- plain forms ---------------------------------------------------------------------------------

def read_plain(pages, slots, dim, dtype):
    """Values at the slots: [n, hkv, D] keys and values, slots of -1 read as zeros."""
    page, off = slots.clamp(min=0).long() // PAGE, slots.clamp(min=0).long() % PAGE
    at = places(dim)[off]                                                          # [n, D]
    out = []
    for i in range(2):
        row = pages[:, :, i * PAGE * dim:(i + 1) * PAGE * dim]
        code = row[page[:, None, None], torch.arange(pages.shape[1], device="cuda")[:, None], at[:, None, :]]
        x = code.view(F8).float() * scales(pages, dim)[page, :, i, None]
        out.append(x.masked_fill((slots < 0)[:, None, None], 0.0).to(dtype))
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


def run_write_plain(s):
    c, pages = s["case"], s["pages"]
    dt, d, rot, n, hkv = DTYPES[c["dtype"]], c["dim"], c["rot"], c["n_seqs"], c["hkv"]
    placed = s["pos"] >= 0
    cs = s["cs"][s["pos"].clamp(min=0).long()] if rot else None
    q = rotate_plain(norm_plain(s["q"], s["w"][0]), cs, rot, c["inter"]).masked_fill(~placed[:, None, None], 0.0).to(dt)
    k = rotate_plain(norm_plain(s["k"], s["w"][1]), cs, rot, c["inter"])
    t = torch.arange(s["q"].shape[0], device="cuda")
    b = (torch.searchsorted(s["offs"], t, right=True, out_int32=True) - 1).clamp(max=n - 1).long()
    at = s["cached"][b].long() + t - s["offs"][b].long()
    # (a row that is not placed goes to a page of its own behind the others)
    extra = pages.shape[0]
    page = torch.where(placed, s["table"][b, (at // PAGE).clamp(max=s["table"].shape[1] - 1)].long(), torch.full_like(at, extra))
    off = at % PAGE
    grid = torch.cat([pages, pages[:1]])
    touched = torch.zeros(extra + 1, dtype=torch.bool, device="cuda").index_fill_(0, page, True)
    # live older places of the pages that sequences go on in
    edge = s["table"].gather(1, (s["cached"] // PAGE).clamp(max=s["table"].shape[1] - 1).long()[:, None])[:, 0].long()
    edge = torch.where(s["cached"] < s["kv"], edge, torch.full_like(edge, extra))
    older = torch.zeros(extra + 1, dtype=torch.long, device="cuda").scatter_(0, edge, (s["cached"] % PAGE).long())
    old_place = torch.arange(PAGE, device="cuda") < older[:, None]                             # [pool + 1, 64]
    where = places(d)
    for i, x in ((0, k), (1, s["v"].float())):
        top = torch.zeros((extra + 1, hkv), device="cuda").scatter_reduce_(0, page[:, None].expand(-1, hkv), x.abs().amax(-1), "amax")
        was = torch.frexp(scales(grid, d)[:, :, i])[1] - 1
        e = torch.where((older > 0)[:, None], torch.maximum(was, exponent(top)), exponent(top))
        e = torch.where(touched[:, None], e, was)
        part = grid[:, :, i * PAGE * d:(i + 1) * PAGE * d]
        code = part[..., where]                                                             # [pool + 1, hkv, 64, D]
        moved = codes(code.view(F8).float(), (e - was)[..., None, None])
        code = torch.where((old_place & touched[:, None])[:, None, :, None], moved, code)
        code[page, :, off] = codes(x, e[page][..., None])
        part[..., where.reshape(-1)] = code.flatten(2)
        scales(grid, d)[:, :, i] = torch.where(touched[:, None], pow2(e), scales(grid, d)[:, :, i])
    pages.copy_(grid[:extra])
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
    ids = s["table"].clamp(min=0).long()
    t = torch.arange(s["width"] * PAGE, device="cuda")
    live = t < s["kv"][:, None]                                             # [n, T]
    where = places(d).reshape(-1)
    kv = []
    for i in range(2):
        x = s["pages"][:, :, i * PAGE * d:(i + 1) * PAGE * d][..., where].view(F8).float() * scales(s["pages"], d)[:, :, i, None]
        x = x.unflatten(2, (PAGE, d))[ids].transpose(1, 2).flatten(2, 3)      # [n, hkv, T, D]
        kv.append(x.masked_fill(~live[:, None, :, None], 0.0))
    k, v = kv
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
    n, cap, d, pool, layers, hkv = c["n_seqs"], s["cap"], c["dim"], s["pages"].shape[1], c["layers"], c["hkv"]
    path = ancestors(s["par"], c["draft"])[torch.arange(n, device="cuda"), s["best"].long()]   # [n, cap]
    rank = torch.cumsum(path, 1) - 1
    node = torch.arange(cap, device="cuda")
    base = s["cached"].long()[:, None]
    seq, pick = path.nonzero(as_tuple=True)                    # the path's nodes, sequence by sequence
    src, dst = (base + node).expand(n, -1)[seq, pick], (base + rank)[seq, pick]
    sp, so = s["table"][seq, src // PAGE].long(), src % PAGE
    dp, do = s["table"][seq, dst // PAGE].long(), dst % PAGE
    moves = src != dst
    touched = torch.zeros(pool + 1, dtype=torch.bool, device="cuda").index_fill_(0, torch.where(moves, dp, torch.full_like(dp, pool)), True)[:pool]
    # what is live in a page: what was cached there, and the path
    table = torch.where(s["table"] < 0, torch.full_like(s["table"], pool), s["table"]).long()
    first = torch.arange(table.shape[1], device="cuda") * PAGE
    older = (s["cached"][:, None] - first).clamp(0, PAGE).long()
    live = torch.arange(PAGE, device="cuda") < torch.zeros(pool + 1, dtype=torch.long, device="cuda").scatter_(0, table.reshape(-1), older.reshape(-1))[:pool, None]
    where, new_len = places(d), (s["cached"] + path.sum(1)).int()
    for one in s["pages"]:
        for i in range(2):
            was = torch.frexp(scales(one, d)[:, :, i])[1] - 1                                 # [pool, hkv]
            top = was.scatter_reduce(0, dp[:, None].expand(-1, hkv), torch.where(moves[:, None], was[sp], was[dp]), "amax")
            part = one[:, :, i * PAGE * d:(i + 1) * PAGE * d]
            code = part[..., where]
            value = code.view(F8).float()
            out = torch.where((live & touched[:, None])[:, None, :, None], codes(value, (top - was)[..., None, None]), code)
            out[dp, :, do] = codes(value[sp, :, so], (top[dp] - was[sp])[..., None])
            part[..., where.reshape(-1)] = out.flatten(2)
            scales(one, d)[:, :, i] = pow2(top)
    k, v = read_plain(s["pages"].flatten(0, 1), s["slots"], d, torch.bfloat16)
    return dict(new_len=new_len, k=k, v=v)


def run_fork_plain(s):
    n, width, pool = s["total"], s["width"], s["pool"]
    table, held, cached, free, count, shares = (t.clone() for t in s["book"].split([n * width, n, n, pool, 1, pool]))
    table = table.view(n, width)
    src, dst, length = s["src"].long(), s["dst"].long(), s["length"].long()
    whole, part = length // PAGE, length % PAGE > 0
    # those with a page begun take one off the stack, fork by fork
    rank = torch.cumsum(part, 0) - 1
    served = ~part | (rank < count)
    take = part & served
    fresh = free[(count - 1 - rank).clamp(min=0).long()]
    j = torch.arange(width, device="cuda")
    share = (j < whole[:, None]) & served[:, None]
    rows = torch.where(share, table[src], torch.full_like(table[src], -1))
    rows = torch.where((j == whole[:, None]) & take[:, None], fresh[:, None], rows)
    begun = table[src, whole.clamp(max=width - 1)]
    table[dst] = rows
    held[dst] = torch.where(served, whole + part, torch.zeros_like(whole)).int()
    cached[dst] = torch.where(served, length, torch.zeros_like(length)).int()
    ones = torch.cat([shares, shares.new_zeros(1)])
    ones.scatter_add_(0, torch.where(share, rows, torch.full_like(rows, pool)).reshape(-1).long(), torch.ones_like(rows).reshape(-1))
    count = count - take.sum().int()
    free = torch.where(torch.arange(pool, device="cuda") < count, free, torch.full_like(free, -1))
    s["pages"][:, fresh[take].long()] = s["pages"][:, begun[take].long()]
    return dict(block_table=table, seq_pages=held, cached_len=cached, free_pages=free, n_free=count, page_shares=ones[:pool], pages=s["pages"])


def run_compact_plain(s):
    c, width, pool = s["case"], s["width"], s["pool"]
    n = c["n_seqs"]
    table, held, free, count, shares = (t.clone() for t in s["book"].split([n * width, n, pool, 1, pool]))
    table = table.view(n, width)
    j, ids = torch.arange(width, device="cuda"), torch.arange(pool, device="cuda")
    # free: pages that lose their last holder go on the stack in the order of their numbers
    need = torch.minimum((s["keep"] + PAGE - 1) // PAGE, held)
    drop = (j >= need[:, None]) & (j < held[:, None])
    to = torch.where(drop, table, torch.full_like(table, pool)).reshape(-1).long()
    left = torch.cat([shares, shares.new_zeros(1)]).scatter_add(0, to, -torch.ones_like(to, dtype=torch.int32))[:pool]
    gone = left < 0
    table = torch.where(drop, torch.full_like(table, -1), table)
    rank = torch.cumsum(gone, 0) - 1
    room = torch.cat([free, free.new_zeros(1)])
    room[torch.where(gone, count + rank, torch.full_like(rank, pool))] = ids.int()
    count, shares = count + gone.sum().int(), left.clamp(min=0)
    # compact: the k-th page in use behind the last place moves to the k-th free one before it
    idle = torch.zeros(pool + 1, dtype=torch.bool, device="cuda")
    idle[torch.where(ids < count, room[:pool].long(), torch.full_like(ids, pool))] = True
    idle = idle[:pool]
    used = pool - count
    far, hole = ~idle & (ids >= used), idle & (ids < used)
    src, dst = far.nonzero()[:, 0], hole.nonzero()[:, 0]
    page_map = torch.where(idle, torch.full_like(ids, -1), ids)
    page_map[src] = dst
    s["pages"][:, dst] = s["pages"][:, src]
    table = torch.where(table >= 0, page_map[table.clamp(min=0).long()].int(), table)
    shares = shares.clone()
    shares[dst] = shares[src]
    shares[src] = 0
    free = torch.where(ids < count, pool - 1 - ids, torch.full_like(ids, -1)).int()
    return dict(block_table=table, seq_pages=need.int(), free_pages=free, n_free=count, page_shares=shares, page_map=page_map.int(),
                n_moved=far.sum().int().reshape(1), pages=s["pages"])


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
    if c["op"] == "write":
        o = ctx.kvb_write(s["pages"], s["q"], s["k"], s["v"], s["table"], s["cached"], s["kv"], s["pos"], None if c["rows"] else s["offs"], c["rows"],
                          s["cs"], q_weight=s["w"][0], k_weight=s["w"][1], interleaved=bool(c["inter"]))
        kv = ctx.kvb_read(s["pages"], s["slots"], c["dim"], DTYPES[c["dtype"]])
        return dict(q=o["q"], k=kv["k"], v=kv["v"])
    if c["op"] == "attend":
        return ctx.kvb_attend(s["q"], s["pages"], s["table"], s["cached"], s["kv"], rows_per_seq=c["new"], node_parent=s["par"])
    if c["op"] == "commit":
        new_len = ctx.kvb_commit(s["pages"], s["table"], s["cached"], s["kv"], s["best"], s["par"])
        kv = ctx.kvb_read(s["pages"].flatten(0, 1), s["slots"], c["dim"], torch.bfloat16)
        return dict(new_len=new_len, k=kv["k"], v=kv["v"])
    width, pool = s["width"], s["pool"]
    if c["op"] == "fork":
        n = s["total"]
        table, held, cached, free, count, shares = s["book"].clone().split([n * width, n, n, pool, 1, pool])
        table = table.view(n, width)
        ctx.kv_fork(s["pages"], s["src"], s["dst"], table, held, cached, free, count, shares, fork_len=s["length"])
        return dict(block_table=table, seq_pages=held, cached_len=cached, free_pages=free, n_free=count, page_shares=shares, pages=s["pages"])
    n = c["n_seqs"]
    table, held, free, count, shares = s["book"].clone().split([n * width, n, pool, 1, pool])
    table = table.view(n, width)
    ctx.kv_free(s["keep"], table, held, free, count, shares)
    o = ctx.kv_compact(s["pages"], table, held, free, count, shares)
    return dict(block_table=table, seq_pages=held, free_pages=free, n_free=count, page_shares=shares, pages=s["pages"], **o)


def run(state):
    if own:
        return run_own(state)
    return {"write": run_write_plain, "attend": run_attend_plain, "commit": run_commit_plain, "fork": run_fork_plain,
            "compact": run_compact_plain}[state["case"]["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    c = case
    size = 4 if c.get("dtype") == "f32" else 2
    if c["op"] == "write":
        new = c["n_seqs"] * (c["new_lo"] + c["new_hi"]) / 2
        rows = c["n_seqs"] * c["rows"] if c["rows"] else new
        d, back = c["dim"], new + c["n_seqs"] * min(31.5, c["ctx_hi"] / 2)          # entries read back
        entry = 2 * c["hkv"] * d
        return dict(bytes=rows * d * size * 2 * c["hq"] + new * (entry * size + entry + 8) + back * entry * (1 + size) + c["n_seqs"] * 12 +
                    c["rot"] * 4 * min(new, c["ctx_hi"] + c["new_hi"]),
                    flops=new * d * 10 * (c["hq"] + 2 * c["hkv"]))
    if c["op"] == "attend":
        ctx = (c["ctx_lo"] + c["ctx_hi"]) / 2
        seen = ctx + (c["new"] + 1) / 2                       # keys a query sees, on average
        n, d = c["n_seqs"], c["dim"]
        return dict(bytes=n * ((ctx + c["new"]) * 2 * c["hkv"] * d + 2 * c["new"] * c["hq"] * d * size),
                    flops=4 * n * c["new"] * seen * c["hq"] * d)
    if c["op"] == "commit":
        n, d = c["n_seqs"] * c["layers"], c["dim"]
        entry = 2 * c["hkv"] * d
        moved = c["draft"] / 4                                # nodes off the first candidate that an average path moves
        return dict(bytes=n * (2 * moved * entry + (c["draft"] + 4) * 3 * entry), flops=0)
    page = c["layers"] * c["hkv"] * page_bytes(c["dim"], c["bits"])
    mean = (c["ctx_lo"] + c["ctx_hi"]) / 2
    if c["op"] == "fork":
        n = c["n_src"] * c["forks"]
        return dict(bytes=2 * n * page + n * (mean / PAGE) * 12, flops=0)
    used = c["n_seqs"] * (mean / PAGE + 0.5) * (1 - 0.4 * (c["forks"] - 1) / c["forks"])        # the shared part is stored once
    kept = used * (1 - c["ended"] / c["n_seqs"])
    moved = kept * (1 - kept / (used + c["spare"]))
    return dict(bytes=2 * moved * page + (used + c["spare"]) * 16 + c["n_seqs"] * (mean / PAGE) * 8, flops=0)


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _entry64(pages, page, off, dim):
    """Keys and values of one token of one page per row, byte by byte from the layout: [n, hkv, D] each."""
    n, hkv, size = pages.shape
    flat, dev = pages.reshape(-1), pages.device
    ch, four = torch.arange(dim, device=dev), torch.arange(4, device=dev)
    row = min(dim, 128)
    head = (page.long()[:, None] * hkv + torch.arange(hkv, device=dev))[..., None] * size      # first byte of each head
    off = off.long()[:, None]
    turn = off % 8 if row == 128 else torch.div(off, 2, rounding_mode="floor") % 4
    byte = torch.div(ch, row, rounding_mode="floor") * PAGE * row + off * row + torch.bitwise_xor(torch.div(ch % row, 16, rounding_mode="floor"), turn) * 16 + ch % 16
    res = []
    for i in range(2):
        b = flat[head + i * PAGE * dim + byte[:, None, :]].to(torch.int64)
        m = flat[head + 2 * PAGE * dim + 4 * i + four].to(torch.int64)
        s = (m[..., 0] + (m[..., 1] << 8) + (m[..., 2] << 16) + (m[..., 3] << 24)).to(torch.int32).view(torch.float32).double()
        low, exp = (b % 8).double(), torch.div(b, 8, rounding_mode="floor") % 16
        x = torch.where(exp > 0, (1 + low / 8) * _two64(exp - 7), low * 2.0 ** -9)
        res.append(torch.where(b >= 128, -x, x) * s[..., None])
    return res


def _two64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _coded64(x, e):
    """What a page of exponent e holds for values x: multiples of an eighth of the power of two below, or of 2^-9."""
    y = x * _two64(-e)
    step = _two64(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return (y / step).round() * step * _two64(e)


def _fits64(top):
    e = torch.arange(LEAST, 128, device=top.device)
    return LEAST + (448 * _two64(e) < top[..., None]).sum(-1)


def _rotated64(x, angle_cos, angle_sin, inter):
    """Each pair as a complex number times cos + i sin."""
    half = angle_cos.shape[-1]
    y = x.clone()
    idx = torch.arange(half, device=x.device)
    ia, ib = (2 * idx, 2 * idx + 1) if inter else (idx, idx + half)
    z = torch.complex(x[..., ia], x[..., ib]) * torch.complex(angle_cos, angle_sin)[:, None]
    y[..., ia], y[..., ib] = z.real, z.imag
    return y


def _scale64(pages, page, dim):
    """Exponents of the keys and values of whole pages: [n, hkv] each."""
    return [torch.frexp(scales(pages, dim)[page][..., i])[1] - 1 for i in range(2)]


def exact(case, seed):
    c = case
    if c["op"] in ("fork", "compact"):
        return None                                            # whole numbers only
    s = prepare(case, seed)
    d = c["dim"]
    if c["op"] == "write":
        rot, new = c["rot"], []
        for x, w in ((s["q"], s["w"][0]), (s["k"], s["w"][1]), (s["v"], None)):
            x = x.double()
            if w is not None:
                x = x * w.double() / (x.square().sum(-1, keepdim=True) / d + 1e-6).sqrt()
            if rot and len(new) < 2:
                cs = s["cs"].double()[s["pos"].clamp(min=0).long()]
                x = _rotated64(x, cs[:, :rot // 2], cs[:, rot // 2:], c["inter"])
            new.append(x)
        new[0][s["pos"] < 0] = 0
        res = [[], []]
        offs, table = s["offs"].tolist(), s["table"].long()
        for b, (ctx, end) in enumerate(zip(s["cached"].tolist(), s["kv"].tolist())):
            if end == ctx:
                continue
            for first in range(ctx // PAGE * PAGE, end, PAGE):
                page, last = table[b, first // PAGE], min(end, first + PAGE)
                old = torch.arange(0, max(0, ctx - first), device="cuda")
                was = _entry64(s["pages"], page.expand(len(old)), old, d)
                lo = offs[b] + max(ctx, first) - ctx
                for i, e0 in enumerate(_scale64(s["pages"], page[None], d)):
                    x = new[1 + i][lo:lo + last - max(ctx, first)]
                    e = _fits64(x.abs().amax((0, 2)))[:, None]
                    if len(old):
                        e = torch.maximum(e, e0[0][:, None])
                    res[i] += [_coded64(was[i], e), _coded64(x, e)]
        return dict(q=new[0], **{name: torch.cat(x) if x else torch.zeros((0, c["hkv"], d), dtype=torch.float64) for name, x in zip("kv", res)})
    if c["op"] == "attend":
        n, new, hq, hkv = c["n_seqs"], c["new"], c["hq"], c["hkv"]
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
            see = see.to(k.device)
            for hh in range(hq):
                g = hh // (hq // hkv)
                w = s["q"][b * new:(b + 1) * new, hh].double() @ k[:, g].T / math.sqrt(d)
                w = w.masked_fill(~see, float("-inf")).softmax(-1)
                out[b * new:(b + 1) * new, hh] = w @ v[:, g]
        return dict(out=out)
    n, span = c["n_seqs"], c["draft"] + 1
    par, best, cached, table = s["par"].tolist(), s["best"].tolist(), s["cached"].tolist(), s["table"].tolist()
    lens, where, pages, live = [], [], [], []       # where an entry of the result comes from; the pages whose scales it is held to
    for b in range(n):
        path, x = [], best[b]
        while x >= 0:
            path.append(x)
            x = par[b][x]
        path.reverse()
        lens.append(cached[b] + len(path))
        took = {}
        for i, x in enumerate(path):
            if x != i:
                took.setdefault((cached[b] + i) // PAGE, set()).add((cached[b] + x) // PAGE)
        for i in range(-3, span):
            p = max(0, cached[b] + i)
            moved = cached[b] + path[i] if 0 <= i < len(path) else p
            where.append(table[b][moved // PAGE] * PAGE + moved % PAGE)
            live.append(0 <= cached[b] + i < lens[b])
            pages.append([table[b][y] for y in {p // PAGE} | took.get(p // PAGE, set())])
    most = max(len(x) for x in pages)
    pages = torch.tensor([x + x[:1] * (most - len(x)) for x in pages], device="cuda").reshape(-1)
    where, live = torch.tensor(where, device="cuda"), torch.tensor(live, device="cuda")[:, None, None]
    got = [[], []]
    for one in s["pages"]:
        value, e = _entry64(one, where // PAGE, where % PAGE, d), _scale64(one, pages, d)
        for i in range(2):
            held = _coded64(value[i], e[i].view(len(where), most, -1).amax(1)[..., None])
            got[i].append(torch.where(live, held, torch.zeros_like(held)))
    return dict(new_len=torch.tensor(lens, dtype=torch.int32), k=torch.cat(got[0]), v=torch.cat(got[1]))
