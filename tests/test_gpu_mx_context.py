"""A context whose layers' weights are microscaled (poss_load_mx) against the oracle with the rounded weights, and against itself: one row and
a tree's rows, one sequence and a batch."""
import ctypes

import numpy as np
import pytest

from gpu_util import have_gpu, tol_for, tree_from_gpu

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P
    from synth import get_config, make_prompt, make_weights
    from synth.gen import to_float64, to_storage
    from synth.gpu import weights_to_device
    from oracle import mx
    from oracle.model import Weights
    from oracle.poss import PossOracle
    from oracle.tree import Tree
    from test_gpu_paths import one_row_against_tree_rows

MATRICES = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "fc_w")


def rounded(cfg, storage):
    """The weights that the context multiplies with: matrices of the layers through 4 bits (their values are 16-bit numbers), the rest as they are."""
    out = dict(storage)
    for name, w in storage.items():
        if name.split(".")[-1] in MATRICES:
            w64 = to_float64(w, cfg.dtype)
            v = mx.dequantize(*mx.quantize(w64), w64.shape[1])
            out[name] = to_storage(v, cfg.dtype)
            assert np.array_equal(to_float64(out[name], cfg.dtype), v)
    return out


def pair(name, **over):
    cfg = get_config(name, **over)
    storage = make_weights(cfg)
    return cfg, P.Poss(cfg, weights_to_device(cfg, storage), mx=True), PossOracle(Weights(cfg, rounded(cfg, storage)), cfg, act=cfg.dtype)


# widths whose products have one split and several, K that ends inside a k-step (1728) and inside a block's group (1000)
@pytest.mark.parametrize("name,over", [("t_mid_bf16", dict()), ("t_mid_f16", dict()), ("t_mid_bf16", dict(n_layers=2, d_model=1024, n_q_heads=8, n_kv_heads=2, head_dim=128, d_ffn=1000)),
                                       ("t_mid_f16", dict(n_layers=1, n_specialists=1, d_ffn=40000))])
def test_rounds_follow_the_oracle_with_the_rounded_weights(name, over):
    """Prompt, then three rounds in lock-step: logits and features of every tree row, the cache, tokens where the oracle's choice is clear."""
    cfg, ctx, o = pair(name, **over)
    tol = tol_for(cfg)
    prompt = make_prompt(cfg)
    first, want = ctx.prefill(prompt), o.prefill(prompt)
    assert first in (want, o.tokens[-1]) or name.startswith("t_mid")      # (near-ties)
    k, v = ctx.debug_read_kv(-1, cfg.n_layers - 1, 0, len(prompt))
    assert np.abs(k - o.kv[-1][0][:len(prompt)]).max() <= tol and np.abs(v - o.kv[-1][1][:len(prompt)]).max() <= tol
    if first != want:
        pytest.skip("a near-tie behind the prompt: the streams part")
    for rnd in range(3):
        print(f"mx round {name} {over} {rnd}", flush=True)
        tr = ctx.draft_tree()
        otree, d = tree_from_gpu(tr)
        o.draft_tree()
        logits, feats = torch.zeros(tr.n, cfg.vocab, device="cuda"), torch.zeros(tr.n, cfg.d_model, device="cuda")
        g = ctx.verify_tree(None, logits_out=logits, feat_out=feats)[:tr.n]
        og, ologits, ofeats = o.verify_tree(Tree(d["token"], d["parent"]))
        assert np.abs(logits.cpu().numpy() - ologits).max() <= tol
        assert np.abs(feats.cpu().numpy() - ofeats).max() <= tol * max(1.0, np.sqrt((ofeats ** 2).mean(axis=1)).max())
        for i in range(tr.n):
            top2 = np.partition(ologits[i], -2)[-2:]
            assert g[i] == og[i] or top2[1] - top2[0] <= 2 * tol
        path, m, toks = ctx.accept_and_commit()
        o.accept_and_commit(path=path, bonus=toks[-1])
    assert ctx.tokens() == o.tokens
    ctx.close()


def test_drafted_scores_follow_the_oracle():
    """Specialists and fc in 4 bits: the root's children have the oracle's scores."""
    cfg, ctx, o = pair("t_mid_bf16", depth=2, total_tokens=30)
    prompt = make_prompt(cfg)
    first = ctx.prefill(prompt)
    o.prefill(prompt)
    if first != o.tokens[-1]:
        pytest.skip("a near-tie behind the prompt")
    d, ot = ctx.draft_tree().as_dict(), o.draft_tree()
    mine = {t: s for t, p, s in zip(d["token"], d["parent"], d["score"]) if p == 0}
    theirs = {t: s for t, p, s in zip(ot.token, ot.parent, ot.score) if p == 0}
    common = set(mine) & set(theirs)
    assert len(common) >= cfg.top_k - 1                    # (one place may go to a near-tie)
    for t in common:
        assert abs(mine[t] - theirs[t]) <= 2 * tol_for(cfg), t
    ctx.close()


@pytest.mark.parametrize("name,over", [("t_mid_bf16", dict()), ("t_mid_f16", dict()), ("t_mid_bf16", dict(d_model=1024, n_q_heads=8, n_kv_heads=8, head_dim=128, d_ffn=1000)),
                                       ("t_mid_f16", dict(d_model=2048, n_q_heads=16, n_kv_heads=2, d_ffn=8192)), ("t_mid_bf16", dict(d_model=4096, n_q_heads=32, n_kv_heads=8, head_dim=128, d_ffn=14336))])
def test_one_row_has_the_bits_of_a_tree_row(name, over):
    """1, 2, 16 and 17 rows go through different kernels; the sums are the same."""
    cfg = get_config(name, **dict(over, n_layers=2, vocab=1000, max_seq=2048, n_specialists=1))
    from synth.gpu import make_weights_on_device
    ctx = P.Poss(cfg, make_weights_on_device(cfg), mx=True)
    one_row_against_tree_rows(cfg, ctx, (20, 300, 1300))
    ctx.close()


# gate and up of one split with SiLU in the product, in each of its tile shapes, and of several
@pytest.mark.parametrize("name,over", [("t_mid_bf16", dict(d_model=4096, n_q_heads=32, n_kv_heads=8, head_dim=128, d_ffn=14336)), ("t_mid_f16", dict(d_ffn=11000)),
                                       ("t_mid_bf16", dict())])
def test_a_row_has_the_same_bits_in_trees_of_any_size(name, over):
    """(Trees of one group have as many blocks of 64 keys: attention cuts them alike.)"""
    cfg = get_config(name, **dict(over, n_layers=2, vocab=1000, max_seq=512, n_specialists=1, top_k=10, depth=6, total_tokens=120))
    from synth.gpu import make_weights_on_device
    ctx = P.Poss(cfg, make_weights_on_device(cfg), mx=True)
    rs = np.random.RandomState(6)
    prompt, wide = rs.randint(0, 1000, 70).astype(np.int32), [0] + [int(x) for x in rs.permutation(1000)[:120]]
    for group in ((33, 1, 16, 17, 32), (120, 64, 65)):
        got = []
        for rows in group:
            ctx.reset()
            ctx.prefill(prompt)
            logits, feats = torch.zeros(rows, 1000, device="cuda"), torch.zeros(rows, cfg.d_model, device="cuda")
            ctx.verify_tree(P.TreeArrays.from_lists(wide[:rows], [-1] + [0] * (rows - 1)), logits_out=logits, feat_out=feats)
            got.append((logits, feats))
        torch.cuda.synchronize()
        assert torch.isfinite(got[0][0]).all()
        for logits, feats in got[1:]:
            n = logits.shape[0]
            assert torch.equal(feats, got[0][1][:n]) and torch.equal(logits, got[0][0][:n]), n
    ctx.close()


def test_speculation_gives_plain_decodings_tokens():
    """Drafted rounds and root-only rounds (plain decoding) commit the same tokens; injected trees that are accepted as well."""
    cfg = get_config("t_mid_bf16")
    w = weights_to_device(cfg, make_weights(cfg))
    ctx = P.Poss(cfg, w, mx=True)
    prompt = make_prompt(cfg)
    ctx.prefill(prompt)
    while len(ctx.tokens()) < len(prompt) + 20:
        ctx.verify_tree(P.TreeArrays.from_lists([0], [-1]))
        ctx.accept_and_commit()
    plain = ctx.tokens()
    ctx.reset()
    ctx.prefill(prompt)
    for _ in range(6):
        ctx.draft_tree(want_tree=False)
        ctx.verify_tree(want_argmax=False)
        ctx.accept_and_commit()
    got = ctx.tokens()
    n = min(len(plain), len(got))
    assert got[:n] == plain[:n]
    ctx.reset()
    ctx.prefill(prompt)
    chain = plain[len(prompt) + 1:len(prompt) + 6]
    ctx.verify_tree(P.TreeArrays.from_lists([0] + chain, list(range(-1, len(chain)))))
    _, m, toks = ctx.accept_and_commit()
    assert m == len(chain) and toks[:m] == chain
    ctx.close()


def test_a_batch_is_its_sequences_alone():
    cfg = get_config("t_mid_bf16")
    w = weights_to_device(cfg, make_weights(cfg))
    prompts = [make_prompt(cfg, n=n, seed=70 + n) for n in (150, 31, 290)]
    want = []
    ctx = P.Poss(cfg, w, mx=True)
    for p in prompts:
        ctx.reset()
        ctx.prefill(p)
        for _ in range(4):
            ctx.draft_tree(want_tree=False)
            ctx.verify_tree(want_argmax=False)
            ctx.accept_and_commit()
        want.append(ctx.tokens())
    ctx.close()
    ctx = P.Poss(cfg, w, mx=True, batch=3)
    for b, p in enumerate(prompts):
        ctx.prefill(p, seq=b)
    for _ in range(4):
        ctx.draft_tree(want_tree=False)
        ctx.verify_tree(want_argmax=False)
        ctx.accept_and_commit()
    assert [ctx.tokens(b) for b in range(3)] == want
    ctx.close()


def test_two_contexts_of_the_same_weights_side_by_side():
    """A microscaled and an ordinary context over one set of tensors, on streams of their own, each give what they give alone."""
    cfg = get_config("t_mid_f16")
    w = weights_to_device(cfg, make_weights(cfg))
    prompt = make_prompt(cfg)

    def rounds(ctxs):
        for c in ctxs:
            c.reset()
            c.prefill(prompt)
        for _ in range(3):
            for c in ctxs:
                c.draft_tree(want_tree=False)
            for c in ctxs:
                c.verify_tree(want_argmax=False)
            for c in ctxs:
                c.accept_and_commit()
        return [c.tokens() for c in ctxs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    ctxs = [P.Poss(cfg, w, stream=streams[0], mx=True), P.Poss(cfg, w, stream=streams[1])]
    alone = [rounds([c])[0] for c in ctxs]
    assert rounds(ctxs) == alone
    for c in ctxs:
        c.close()


def test_sampling_and_drawn_children_run():
    cfg = get_config("t_mid_bf16")
    ctx = P.Poss(cfg, weights_to_device(cfg, make_weights(cfg)), mx=True)
    rng = np.random.default_rng(3)
    ctx.set_sampling(1.0, rng.random(cfg.depth + 1))
    ctx.set_draft_sampling(rng.random((cfg.depth, cfg.top_k, cfg.top_k)), rng.random((cfg.depth + 1, cfg.top_k + 1)))
    ctx.prefill(make_prompt(cfg))
    for _ in range(2):
        ctx.draft_tree()
        ctx.verify_tree()
        path, m, toks = ctx.accept_and_commit()
        assert len(toks) == m + 1 and all(0 <= t < cfg.vocab for t in toks)
    ctx.close()


def test_refusals():
    lib = P.load_library()
    f32 = P.make_config(get_config("c0_tiny_f32"))
    assert lib.poss_workspace_bytes_mx(ctypes.byref(f32)) == 0
    cfg = get_config("c0_tiny_f32")
    w = weights_to_device(cfg, make_weights(cfg))
    with pytest.raises(P.PossError) as e:
        P.Poss(cfg, w, mx=True)
    assert e.value.code == P.E_INVALID_ARG
    mid = P.make_config(get_config("t_mid_bf16"))
    assert 0 < lib.poss_workspace_bytes_mx(ctypes.byref(mid)) < lib.poss_workspace_bytes(ctypes.byref(mid))
