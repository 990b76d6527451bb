"""The 8-bit cache's calls and the page operators together, as a model uses them: the example's decoding loop."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("head_dim,q_heads,kv_heads,seed", [(64, 8, 2, 0), (128, 4, 4, 1), (64, 6, 1, 2)])
@pytest.mark.parametrize("bits", [4, 8])
def test_samples_of_shared_prompts(head_dim, q_heads, kv_heads, seed, bits):
    """Trees over shared prompts emit what single tokens over prompts of their own do; a prompt's whole pages are stored once; sequences
    that end give back what nobody else holds, and the others go on from pages that have moved."""
    import tree_decoding as ex
    from paper_2505_13204_b200 import binding
    ctx = binding.Context()
    model = ex.Model(ctx, head_dim=head_dim, q_heads=q_heads, kv_heads=kv_heads, seed=seed)
    prompts = ex.prompts_for(5, model.vocab, seed)
    prompts[0] = prompts[0].repeat(12)                       # one that has whole pages
    steps, n = 16, len(prompts)
    fast, cache = ex.decode(ctx, model, prompts, steps, trees=True, bits=bits, samples=3)
    slow, _ = ex.decode(ctx, model, prompts, max(len(s) - prompts[b % n].numel() for b, s in enumerate(fast)) - 1, trees=False, bits=bits)
    new = [len(s) - prompts[b % n].numel() for b, s in enumerate(fast)]
    if bits == 4:   # (entries are rounded one by one: the same whatever is stored with them)
        assert [slow[b % n][:len(f)] for b, f in enumerate(fast)] == fast
        assert sum(new) > 3 * n * (steps + 1), "some drafts are accepted"
    assert all(fast[b] == fast[b % n] for b in range(3 * n))
    assert cache.length.tolist() == [len(s) - 1 for s in fast] and ctx.poll_status() == 0
    held = int(cache.held.sum())
    used = cache.free.numel() - cache.n_free.item()
    whole = sum(p.numel() // ex.PAGE for p in prompts)
    assert whole > 0 and used == held - 2 * whole and int(cache.shares.sum()) == 2 * whole
    # the next token of the sequences that stay, before and after their pages move
    dev = ctx.device
    stay = torch.arange(3 * n, device=dev) % 3 == 1
    cache.end(~stay)
    length, tokens = cache.length.clone(), torch.arange(3 * n, dtype=torch.int32, device=dev)

    def next_token():
        cache.length = length.clone()
        return model(cache, tokens, cache.plan(stay.to(torch.int32), 3 * n, 1), 1)[stay]

    want = next_token()
    assert cache.compact()["n_moved"].item() > 0
    in_use = cache.free.numel() - cache.n_free.item()
    assert sorted(set(cache.table[cache.table >= 0].tolist())) == list(range(in_use))
    assert torch.equal(next_token(), want)
    cache.release()
    assert cache.n_free.item() == cache.free.numel() == len(set(cache.free.tolist()))
    assert (cache.table == binding.NONE).all() and (cache.shares == 0).all() and ctx.poll_status() == 0
