"""Tree decoding over the 8-bit cache against a plain pass in 64 bits over the tokens that came out: what is cached, and what the model makes
of it.  (The tokens need not be those of decoding one by one: rejected nodes can round what is stored beside them.)"""
import os
import sys

import numpy as np
import pytest
import torch

import kvb_ref as ref

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
U32 = 2.0 ** -24


def heads(model, x, l):
    """Normed and rotated queries and keys, and values, [T, heads, D] each, of layer l's inputs (64 bits); and how far fp32 may be off in keys
    and values: a sum of `hidden` products (hidden + 40 roundings with the norm in front of it), then a head's norm and a pair's rotation."""
    D, Hq, Hk = model.head_dim, model.q_heads, model.kv_heads
    a, w = model.norm(x), model.wqkv[l].double()
    y = (a @ w).view(-1, Hq + 2 * Hk, D)
    off = ((a.abs() @ w.abs()) * (w.shape[0] + 40) * U32).view(-1, Hq + 2 * Hk, D)
    cs = model.cos_sin[:x.shape[0]].double()[:, None]
    cos, sin = cs[..., :D // 2], cs[..., D // 2:]

    def rotated(z, weight):
        z = z * torch.rsqrt(z.pow(2).mean(-1, keepdim=True) + 1e-6) * weight.double()
        p, q = z[..., :D // 2], z[..., D // 2:]
        return torch.cat([p * cos - q * sin, q * cos + p * sin], -1)

    q, k, v = y[:, :Hq], y[:, Hq:Hq + Hk], y[:, Hq + Hk:]
    rms = torch.rsqrt(k.pow(2).mean(-1, keepdim=True) + 1e-6)
    # (the row's own error and its norm's, in both members of a pair; roundings of norm and rotation)
    off_k = (4 * off[:, Hq:Hq + Hk].amax(-1, keepdim=True) * rms + 16 * U32 * k.abs().amax(-1, keepdim=True) * rms) * model.kn[l].abs().max()
    return rotated(q, model.qn[l]), rotated(k, model.kn[l]), v, off_k.expand_as(k), off[:, Hq + Hk:]


def plain(model, tokens, noise=None):
    """Logits of the last of `tokens`, everything in 64 bits.  noise: keys and values are changed by up to half a step of e4m3 (2^-4), those of
    equal tokens alike (as the first layer's values are, whose errors do not average out over a sequence that repeats itself)."""
    x = model.embed[torch.as_tensor(tokens, device=model.embed.device)].double()
    see = torch.ones((len(tokens), len(tokens)), dtype=torch.bool, device=x.device).tril()
    for l in range(model.layers):
        q, k, v, _, _ = heads(model, x, l)
        if noise is not None:
            size, ids = (model.vocab,) + k.shape[1:], torch.as_tensor(tokens, device=x.device)
            k, v = (z * (1 + (2 * torch.rand(size, generator=noise, device=z.device, dtype=torch.float64) - 1) * 2.0 ** -4)[ids] for z in (k, v))
        G = model.q_heads // model.kv_heads
        w = torch.einsum("thd,shd->hts", q, k.repeat_interleave(G, 1)) / model.head_dim ** 0.5
        o = torch.einsum("hts,shd->thd", w.masked_fill(~see, float("-inf")).softmax(-1), v.repeat_interleave(G, 1))
        x = x + o.flatten(1) @ model.wo[l].double()
        x = x + torch.nn.functional.gelu(model.norm(x) @ model.w1[l].double()) @ model.w2[l].double()
    return model.norm(x[-1]) @ model.unembed.double()


@pytest.mark.parametrize("head_dim,q_heads,kv_heads,seed", [(64, 8, 2, 0), (128, 4, 4, 1), (64, 6, 1, 2)])
def test_cached_entries_and_logits(head_dim, q_heads, kv_heads, seed):
    import tree_decoding as ex
    from paper_2505_13204_b200 import binding
    torch.backends.cuda.matmul.allow_tf32 = False
    ctx = binding.Context()
    model = ex.Model(ctx, head_dim=head_dim, q_heads=q_heads, kv_heads=kv_heads, seed=seed)
    prompts = ex.prompts_for(4, model.vocab, seed)
    prompts[0] = prompts[0].repeat(12)                       # one that has whole pages
    n, samples, steps = len(prompts), 2, 16
    fast, cache = ex.decode(ctx, model, prompts, steps, trees=True, bits=8, samples=samples)
    B = n * samples
    assert ctx.poll_status() == 0 and cache.length.tolist() == [len(s) - 1 for s in fast]
    # the first token comes from the prompts' own pass, as it does one by one
    slow, _ = ex.decode(ctx, model, prompts, 1, trees=False, bits=8)
    for b, s in enumerate(fast):
        assert s[:prompts[b % n].numel() + 1] == slow[b % n][:prompts[b % n].numel() + 1]
    # accepted paths move: more tokens than passes
    assert sum(len(s) - prompts[b % n].numel() for b, s in enumerate(fast)) > B * (steps + 1), "some drafts are accepted"
    # what the first layer has cached (it does not depend on the cache): a rounding to e4m3 when it is stored, and one more, of half a step of the
    # subnormals, whenever the page's scale grows; those scales are powers of two, so the last one's step is their sum's bound
    raw = cache.pages[0].cpu().numpy()
    for b, s in enumerate(fast):
        x = model.embed[torch.as_tensor(s[:-1], device=ctx.device)].double()
        _, k, v, off_k, off_v = (y.cpu().numpy() for y in heads(model, x, 0))
        pages = cache.table[b].tolist()
        for t in range(len(s) - 1):
            page = raw[pages[t // ref.PAGE]]
            for h in range(kv_heads):
                for half, want, off in ((0, k[t, h], off_k[t, h]), (1, v[t, h], off_v[t, h])):
                    blk = ref.Block(page[h], half, head_dim)
                    err = np.abs(blk.value(t % ref.PAGE) - want)
                    assert (err <= 2.0 ** -4 * np.abs(want) + 2.0 ** (blk.e - 9) + 1.1 * off).all(), (b, t, h, half)
    # one more token: the logits are as far from the plain pass's as roundings of keys and values by up to half a step make them.  (A rounding is
    # 2^-4 off at most, and less on average than the noise is; the noise is one draw: twice its distance is allowed.)
    one = torch.ones(B, dtype=torch.int32, device=ctx.device)
    more = torch.arange(B, dtype=torch.int32, device=ctx.device) % model.vocab
    got = model(cache, more, cache.plan(one, B, 1), 1).double()
    g = torch.Generator(device=ctx.device).manual_seed(seed)
    want = torch.stack([plain(model, s[:-1] + [int(more[b])]) for b, s in enumerate(fast)])
    noisy = torch.stack([plain(model, s[:-1] + [int(more[b])], g) for b, s in enumerate(fast)])
    here, there = (got - want).pow(2).mean().sqrt().item(), (noisy - want).pow(2).mean().sqrt().item()
    print("logits off by %.4f, noise %.4f, of %.4f" % (here, there, want.std().item()))
    assert here <= 2 * there and ctx.poll_status() == 0
    cache.release()
    ctx.close()
