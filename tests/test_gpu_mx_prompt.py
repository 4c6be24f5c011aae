"""Prompts of a microscaled context against the oracle with the rounded weights: one pass and several, the token behind them (the oracle's, or the second of
a near-tie), and a round on what they left."""
import numpy as np
import pytest

from gpu_util import have_gpu, prefill_in_step, tol_for

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P
    from synth import make_prompt
    from oracle.tree import Tree
    from test_gpu_mx_context import pair


def verified(ctx, o, tol):
    """A tree over the context's state: logits and features of every row."""
    cfg = o.cfg
    tree = Tree([o.tokens[-1], 5, 9, 11, 3], [-1, 0, 0, 1, 3 if cfg.depth > 2 else 1])      # (no deeper than the context drafts)
    logits, feats = torch.zeros(5, cfg.vocab, device="cuda"), torch.zeros(5, cfg.d_model, device="cuda")
    ctx.verify_tree(P.TreeArrays.from_lists(tree.token, tree.parent), logits_out=logits, feat_out=feats)
    _, ologits, ofeats = o.verify_tree(tree)
    assert np.abs(logits.cpu().numpy() - ologits).max() <= tol
    assert np.abs(feats.cpu().numpy() - ofeats).max() <= tol * max(1.0, np.sqrt((ofeats ** 2).mean(axis=1)).max())


# one row, a pass that is full and one row more, two passes (up to the last length that 16-bit contexts stream too), and three with a last one of one row
@pytest.mark.parametrize("name", ["t_mid_bf16", "t_mid_f16"])
@pytest.mark.parametrize("n", [1, 256, 257, 300, 512, 513, 700])
def test_prompts_of_one_pass_and_several(name, n):
    print(f"mx prompt {name} {n}", flush=True)
    cfg, ctx, o = pair(name, n_layers=2, max_seq=1024)
    tol = tol_for(cfg)
    prefill_in_step(ctx, o, make_prompt(cfg, n=n, seed=n), tol)
    for l in range(cfg.n_layers):
        k, v = ctx.debug_read_kv(-1, l, 0, n)
        assert np.abs(k - o.kv[l][0][:n]).max() <= tol and np.abs(v - o.kv[l][1][:n]).max() <= tol
    verified(ctx, o, tol)
    ctx.close()


# the configurations of test_gpu_mx_context.py's rounds
@pytest.mark.parametrize("name,over", [("t_mid_bf16", dict()), ("t_mid_f16", dict()), ("t_mid_bf16", dict(n_layers=2, d_model=1024, n_q_heads=8, n_kv_heads=2, head_dim=128, d_ffn=1000)),
                                       ("t_mid_f16", dict(n_layers=1, n_specialists=1, d_ffn=40000)), ("t_mid_bf16", dict(depth=2, total_tokens=30))])
def test_the_token_behind_a_prompt(name, over):
    cfg, ctx, o = pair(name, **over)
    first = prefill_in_step(ctx, o, make_prompt(cfg), tol_for(cfg))
    assert ctx.tokens()[-1] == first
    verified(ctx, o, tol_for(cfg))
    ctx.close()


def test_drafted_scores_after_a_prompt_of_several_passes():
    """The specialists' catch-up over the prompt's features, in passes as well: the root's children have the oracle's scores."""
    cfg, ctx, o = pair("t_mid_bf16", n_layers=2, depth=2, total_tokens=30, max_seq=1024)
    prefill_in_step(ctx, o, make_prompt(cfg, n=600, seed=6), tol_for(cfg))
    d, ot = ctx.draft_tree().as_dict(), o.draft_tree()
    mine = {t: s for t, p, s in zip(d["token"], d["parent"], d["score"]) if p == 0}
    theirs = {t: s for t, p, s in zip(ot.token, ot.parent, ot.score) if p == 0}
    common = set(mine) & set(theirs)
    assert len(mine) == len(theirs) and len(common) >= cfg.top_k - 1      # (one place may go to a near-tie)
    for t in common:
        assert abs(mine[t] - theirs[t]) <= 2 * tol_for(cfg), t
    ctx.close()


# QKV, gate and up on either side of the line between two K splits and none (192 tiles of 128 columns), gate and up of 16-bit types beyond it
@pytest.mark.parametrize("name,over", [("t_mid_f16", dict(d_ffn=12288)), ("t_mid_f16", dict(d_ffn=12296)), ("t_mid_bf16", dict(d_model=1024, n_q_heads=192, n_kv_heads=96, head_dim=64, d_ffn=12800)),
                                       ("t_mid_f16", dict(d_model=640, n_q_heads=194, n_kv_heads=97, head_dim=64, d_ffn=1000))])
def test_a_row_has_the_same_bits_where_splits_begin(name, over):
    from test_gpu_mx_context import test_a_row_has_the_same_bits_in_trees_of_any_size as same_bits
    same_bits(name, over)
