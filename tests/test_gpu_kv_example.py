"""The cache's calls together, as a model uses them: the example's decoding loop."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("head_dim,q_heads,kv_heads,seed", [(64, 8, 2, 0), (128, 4, 4, 1), (64, 6, 1, 2)])
def test_tree_decoding_emits_what_decoding_one_by_one_does(head_dim, q_heads, kv_heads, seed):
    """Strict verification of trees against single tokens: every emitted token is the same, and the
    cache holds as many tokens as the history less the one that is still to be stored."""
    import tree_decoding as ex
    from paper_2505_13204_b200 import binding
    ctx = binding.Context()
    model = ex.Model(ctx, head_dim=head_dim, q_heads=q_heads, kv_heads=kv_heads, seed=seed)
    prompts = ex.prompts_for(5, model.vocab, seed)
    steps = 24
    fast, cache = ex.decode(ctx, model, prompts, steps, trees=True)
    new = [len(s) - p.numel() for s, p in zip(fast, prompts)]
    assert sum(new) > 5 * (steps + 1), "some drafts are accepted"
    assert cache.length.tolist() == [len(s) - 1 for s in fast]
    slow, _ = ex.decode(ctx, model, prompts, max(new) - 1, trees=False)
    assert [s[:len(f)] for s, f in zip(slow, fast)] == fast
    cache.release()
    assert cache.n_free.item() == cache.free.numel() == len(set(cache.free.tolist()))
    assert (cache.table == binding.NONE).all() and ctx.poll_status() == 0
