"""A context whose caches a program appended to and cut: behind a reset and a prompt it decodes as a new one does."""
import pytest

from gpu_util import have_gpu, Pair

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P


def rounds(ctx, prompt, n):
    ctx.prefill(prompt)
    out = []
    for _ in range(n):
        ctx.draft_tree()
        greedy = ctx.verify_tree(None).tolist()
        path, m, tokens = ctx.accept_and_commit()
        out.append((greedy, list(path), m, list(tokens)))
    return out, list(ctx.tokens())


def cut(ctx, which, layer, length, budget):
    """Every second slot of a context's cache goes, and a row is written over."""
    cache = ctx.kv_cache(0, which, layer)
    h, s = cache.heads, cache.slots
    dev = dict(device="cuda")
    weights = (torch.arange(s, **dev) % 2).float().expand(1, h, s).contiguous()
    positions = torch.arange(s, dtype=torch.int32, **dev).expand(1, h, s).contiguous()
    kept, lo = torch.empty(1, h, budget, dtype=torch.int32, **dev), torch.empty(1, dtype=torch.int32, **dev)
    P.kv_evict(cache, weights, positions, torch.tensor([length], dtype=torch.int32, **dev), budget, kept, torch.empty_like(weights), torch.empty_like(positions), lo)
    assert int(lo) == budget and kept[0, 0].tolist() != list(range(budget))
    k = torch.full((1, h, cache.dim), 3.0, dtype=cache.dtype, **dev)
    P.kv_append(cache, k, k, torch.tensor([1], dtype=torch.int32, **dev))
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", ["c0_tiny_f32", "t_mid_bf16"])
def test_a_context_begins_anew_behind_a_reset(name):
    from synth import make_prompt
    pair = Pair(name)
    ctx, prompt = pair.ctx, make_prompt(pair.cfg)
    want, tokens = rounds(ctx, prompt, 3)
    for which, layer in ((-1, 0), (-1, pair.cfg.n_layers - 1), (0, 0)):
        cut(ctx, which, layer, len(prompt) - 1, len(prompt) // 2)
    ctx.reset()
    assert rounds(ctx, prompt, 3) == (want, tokens)
    pair.close()
