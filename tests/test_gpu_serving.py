"""The calls over a program's own caches as they are used together: a decoding loop that rotates, appends, attends, weighs and evicts, against float64 step by
step; the same captured into graphs; on streams; over a context's own caches and logits; behind offsets of more than 32 bits."""
import numpy as np
import pytest

from gpu_util import have_gpu, Pair

pytestmark = pytest.mark.gpu

if have_gpu():
    import torch
    import paper_2506_03566_amd as P
    from oracle import serving as o
    TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
    # rotated values and attention: a few half steps of the type, and of float32 sums over some hundred slots
    TOL = {"f32": 2e-5, "bf16": 2.0 ** -7, "f16": 2.0 ** -10}


def f64(t):
    return t.double().cpu().numpy()


class Served:
    """A cache of n sequences with the arrays that a program keeps beside it."""

    def __init__(self, t, n, hq, hkv, dh, slots, page, seed=0, pages=None, first_page=0):
        g = torch.Generator("cuda").manual_seed(seed)
        per = -(-slots // page)
        pages = pages or n * per
        k, v = (torch.empty(pages, hkv, a, b, dtype=TYPES[t], device="cuda") for a, b in ((page, dh), (dh, page)))
        k[first_page:first_page + n * per].normal_(generator=g)
        v[first_page:first_page + n * per].normal_(generator=g)
        table = (first_page + torch.randperm(n * per, generator=g, device="cuda")).int().view(n, per)
        self.cache = P.KvCache(k, v, table)
        s = self.cache.slots
        self.t, self.n, self.hq, self.hkv, self.dh, self.g, self.page = t, n, hq, hkv, dh, g, page
        self.weights, self.other = torch.zeros(n, hkv, s, device="cuda"), torch.zeros(n, hkv, s, device="cuda")
        self.positions, self.positions_other = (torch.full((n, hkv, s), -1, dtype=torch.int32, device="cuda") for _ in range(2))
        self.lengths = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.out = torch.empty(n, hq, dh, dtype=TYPES[t], device="cuda")
        self.lse = torch.empty(n, hq, device="cuda")

    def qkv(self, rows):
        return torch.randn(rows, (self.hq + 2 * self.hkv), self.dh, generator=self.g, device="cuda").to(TYPES[self.t]).split([self.hq, self.hkv, self.hkv], dim=1)

    def slot(self, b, h, s):
        """Key and value of a slot in float64."""
        k, v, table = self.cache.tensors
        pg = int(table[b, s // self.page])
        return f64(k[pg, h, s % self.page]), f64(v[pg, h, :, s % self.page])


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("interleaved,hq,hkv,dh,page", [(False, 8, 2, 64, 32), (True, 3, 3, 128, 64)])
def test_decoding_with_a_budget(t, interleaved, hq, hkv, dh, page):
    """A prompt of each sequence, then token by token: what a step gives and leaves behind is what float64 makes of the slots that are there."""
    print(f"decoding with a budget {t} {hq}/{hkv} heads of {dh}", flush=True)
    n, budget, room = 2, 40, 56
    m = Served(t, n, hq, hkv, dh, 96, page, seed=dh)
    rope = P.Rope(dh, interleaved=interleaved, scaling="linear", factor=2.0)
    w = np.array(rope.frequencies)
    scratch = P.kv_attend_scratch(m.cache, hq, weights=True)
    lens = [45, 3]
    rows = sum(lens)
    seq = torch.tensor([0] * lens[0] + [1] * lens[1], dtype=torch.int32, device="cuda")
    pos = torch.tensor([*range(lens[0]), *range(lens[1])], dtype=torch.int32, device="cuda")
    q, k, v = m.qkv(rows)
    P.kv_append(m.cache, k, v, pos, pos, rope, seq=seq, slot_positions=m.positions)
    keys = o.rotate(f64(k), f64(pos), w, interleaved)
    vals = f64(v)
    # per sequence and head: [position, key, value] of each slot
    slots = [[[(p, keys[b * lens[0] + p, h], vals[b * lens[0] + p, h]) for p in range(lens[b])] for h in range(hkv)] for b in range(n)]
    m.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
    now = list(lens)                                         # the next position of each
    for step in range(30):
        q, k, v = m.qkv(n)
        position = torch.tensor(now, dtype=torch.int32, device="cuda")
        q_out = torch.empty_like(q).contiguous()
        P.kv_append(m.cache, k, v, m.lengths, position, rope, q=q, q_out=q_out, slot_positions=m.positions)
        m.lengths += 1
        before = f64(m.weights)
        P.kv_attend(m.cache, q_out, m.lengths, m.out, lse=m.lse, weights=m.weights, weights_out=m.weights, scratch=scratch, max_len=room + 1)
        kr, qr = o.rotate(f64(k), now, w, interleaved), o.rotate(f64(q), now, w, interleaved)
        assert np.abs(f64(q_out) - qr).max() <= TOL[t] * np.abs(qr).max()
        for b in range(n):
            for h in range(hkv):
                slots[b][h].append((now[b], kr[b, h], f64(v)[b, h]))
            kk, vv = (np.stack([np.stack([s[i] for s in slots[b][h]]) for h in range(hkv)]) for i in (1, 2))
            want, lse, p, s = o.attend(f64(q_out)[b], kk, vv, dh ** -0.5)
            # keys were rounded on the way in: their half steps move a score by 2^-8 (bf16) of sum |q k| at most
            moved = TOL[t] * np.abs(s).max() * 4 + TOL[t]
            assert np.abs(f64(m.out)[b] - want).max() <= moved * np.abs(vv).max() and np.abs(f64(m.lse)[b] - lse).max() <= moved
            got = f64(m.weights)[b] - before[b]
            assert np.abs(got[:, :len(slots[b][0])] - p.reshape(hkv, -1, p.shape[1]).sum(axis=1)).max() <= 2 * moved * hq / hkv + 1e-5
            assert not got[:, len(slots[b][0]):].any()
            assert f64(m.positions)[b, :, :len(slots[b][0])].tolist() == [[s[0] for s in slots[b][h]] for h in range(hkv)]
            now[b] += 1
        if int(m.lengths.max()) >= room:
            weights, positions, lengths = m.weights.cpu().numpy(), m.positions.cpu().numpy(), m.lengths.tolist()
            kept = torch.empty(n, hkv, budget, dtype=torch.int32, device="cuda")
            P.kv_evict(m.cache, m.weights, m.positions, m.lengths.clone(), budget, kept, m.other, m.positions_other, m.lengths, first=2, recent=10)
            for b in range(n):
                for h in range(hkv):
                    stay = o.evict(weights[b, h], positions[b, h], lengths[b], budget, 2, 10)
                    assert kept[b, h, :len(stay)].tolist() == stay
                    slots[b][h] = [slots[b][h][i] for i in stay]
                    assert {0, 1} <= {s[0] for s in slots[b][h]} and set(range(now[b] - 10, now[b])) <= {s[0] for s in slots[b][h]} or len(stay) < budget
            m.weights, m.other, m.positions, m.positions_other = m.other, m.weights, m.positions_other, m.positions
            assert m.lengths.tolist() == [min(x, budget) for x in lengths]
            for b, h, i in ((0, 0, 0), (0, hkv - 1, budget - 1), (0, 0, 20)):
                key, value = m.slot(b, h, i)
                assert np.abs(key - slots[b][h][i][1]).max() <= TOL[t] * 8 and np.array_equal(value, slots[b][h][i][2])
    assert max(now) > room                                   # it did run over


def step_of(m, rope, x, static, scratches):
    """One captured step: append, attend with weights, evict, log-probabilities of the outputs taken as logits."""
    q, k, v = static["qkv"]
    P.kv_append(m.cache, k, v, static["slots"], static["positions"], rope, q=q, q_out=static["q_out"], slot_positions=m.positions)
    P.kv_attend(m.cache, static["q_out"], static["lengths"], m.out, lse=m.lse, weights=m.weights, weights_out=m.other, scratch=scratches[0])
    P.kv_evict(m.cache, m.other, m.positions, static["lengths"], 64, static["kept"], static["weights_out"], m.positions_other, static["lengths_out"], first=1, recent=8)
    P.logprobs(m.out.view(m.n, -1), static["tokens"], n_top=3, temperature=0.9, logp=static["logp"], entropy=static["entropy"], top_ids=static["ids"], top_logp=static["top"], scratch=scratches[1])


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_two_graphs_replayed_with_eager_work_between(t):
    ms, graphs, eager = [], [], []
    for i in range(2):
        def make():
            m = Served(t, 3, 8, 2, 64, 400, 32, seed=20 + i)
            m.weights.uniform_(generator=m.g)
            m.positions.copy_(torch.arange(m.cache.slots, device="cuda").int().expand(3, 2, -1))
            st = dict(qkv=[p.contiguous() for p in m.qkv(3)], q_out=torch.empty(3, 8, 64, dtype=TYPES[t], device="cuda"), lengths=torch.tensor([300, 65, 7 + i], dtype=torch.int32, device="cuda"),
                      slots=torch.tensor([299, 64, 6 + i], dtype=torch.int32, device="cuda"), positions=torch.tensor([299, 64, 6 + i], dtype=torch.int32, device="cuda"),
                      kept=torch.empty(3, 2, 64, dtype=torch.int32, device="cuda"), weights_out=torch.empty_like(m.weights), lengths_out=torch.empty(3, dtype=torch.int32, device="cuda"),
                      tokens=torch.tensor([1, 5, 511], dtype=torch.int32, device="cuda"), logp=torch.empty(3, device="cuda"), entropy=torch.empty(3, device="cuda"),
                      ids=torch.empty(3, 3, dtype=torch.int32, device="cuda"), top=torch.empty(3, 3, device="cuda"))
            return m, st, (P.kv_attend_scratch(m.cache, 8, weights=True), P.logprobs_scratch(3, 512, 3))
        rope = P.Rope(64)

        def outputs(m, st):
            return [x.clone() for x in (st["q_out"], m.out, m.lse, st["kept"], st["weights_out"], st["lengths_out"], m.positions_other, st["logp"], st["entropy"], st["ids"], st["top"], *m.cache.tensors[:2])]
        m, st, sc = make()
        step_of(m, rope, None, st, sc)
        eager.append(outputs(m, st))
        m, st, sc = make()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step_of(m, rope, None, st, sc)
        graphs.append(g)
        ms.append((m, st, outputs, sc, [x.clone() for x in m.cache.tensors[:2]]))
    for turn in range(4):
        for i in (0, 1, 1, 0):
            for x, y in zip(ms[i][0].cache.tensors, ms[i][4]):
                x.copy_(y)                                    # as before the step: it attends to what it then moves
            ms[i][1]["kept"].fill_(-5)
            ms[i][0].out.zero_()
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            for a, b in zip(ms[i][2](*ms[i][:2]), eager[i]):
                assert torch.equal(a, b), turn
        torch.randn(1000, 1000, device="cuda").sum().item()


def test_streams_and_calls_at_once():
    """Two caches served on streams of their own at the same time, and calls on a stream that is not the current one."""
    rope = P.Rope(128)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    ms = [Served("bf16", 4, 8, 8, 128, 3000, 64, seed=40 + i) for i in range(2)]
    inputs = []
    for m in ms:
        m.lengths.copy_(torch.tensor([2999, 1, 0, 1500], dtype=torch.int32))
        inputs.append([p.contiguous() for p in m.qkv(4)])
    x = torch.randn(50, 40000, device="cuda")
    torch.cuda.synchronize()
    want = []
    for m, (q, k, v) in zip(ms, inputs):
        P.kv_attend(m.cache, q, m.lengths, m.out, lse=m.lse)
        want.append((m.out.clone(), m.lse.clone(), P.rotary(q, m.lengths, rope), P.logprobs(x, n_top=4)))
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for m, st, (q, k, v) in zip(ms, (s1, s2), inputs):
            P.kv_attend(m.cache, q, m.lengths, m.out, lse=m.lse, stream=st)
            got.append((m.out, m.lse, P.rotary(q, m.lengths, rope, stream=st), P.logprobs(x, n_top=4, stream=st)))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, r) for p, r in zip(a[:3], b[:3])) and all(torch.equal(p, r) for p, r in zip(a[3][1:], b[3][1:]))


@pytest.mark.parametrize("name,over", [("c0_tiny_f32", {}), ("t_mid_bf16", {}), ("t_mid_bf16", dict(kv_page_order=1, kv_page_tokens=32))])
def test_a_contexts_own_cache_and_logits(name, over):
    """Attention over a context's caches, read through the same pages, and what its logits say of the committed tokens."""
    from synth import make_prompt
    pair = Pair(name, lib_over=over)
    cfg, ctx = pair.cfg, pair.ctx
    prompt = make_prompt(cfg)
    ctx.prefill(prompt)
    t = len(prompt)
    code = {0: "f32", 1: "bf16", 2: "f16"}[cfg.dtype]
    q = torch.randn(1, cfg.n_q_heads, cfg.head_dim, device="cuda").to(TYPES[code])
    out = torch.empty_like(q)
    for which, layer, n in ((-1, 0, t), (-1, cfg.n_layers - 1, t), (0, 0, t - 1), (-1, 0, 1)):
        cache = ctx.kv_cache(0, which, layer)
        assert cache.slots >= t and cache.heads == cfg.n_kv_heads
        wo = torch.zeros(1, cfg.n_kv_heads, cache.slots, device="cuda")
        lse = torch.empty(1, cfg.n_q_heads, device="cuda")
        P.kv_attend(cache, q, torch.tensor([n], dtype=torch.int32, device="cuda"), out, lse=lse, weights_out=wo)
        k, v = ctx.debug_read_kv(which, layer, 0, n)
        want, wl, p, s = o.attend(f64(q)[0], k.astype(np.float64).swapaxes(0, 1), v.astype(np.float64).swapaxes(0, 1), cfg.head_dim ** -0.5)
        tol = TOL[code] if code != "f32" else 1e-5
        assert np.abs(f64(out)[0] - want).max() <= tol * np.abs(v).max() and np.abs(f64(lse)[0] - wl).max() <= 1e-4
        assert np.abs(f64(wo)[0, :, :n] - p.reshape(cfg.n_kv_heads, -1, n).sum(axis=1)).max() <= 1e-4 and not bool(wo[0, :, n:].any())
    tree = ctx.draft_tree()
    logits = torch.zeros(tree.n, cfg.vocab, device="cuda")
    greedy = ctx.verify_tree(None, logits_out=logits)[:tree.n]
    path, m, tokens = ctx.accept_and_commit()
    logp, entropy, ids, top = P.logprobs(logits[path], torch.tensor(tokens, dtype=torch.int32, device="cuda"), n_top=3)
    want, h = o.logprobs(f64(logits)[path])
    assert np.abs(f64(logp) - want[np.arange(len(path)), tokens]).max() < 1e-4 and np.abs(f64(entropy) - h).max() < 1e-4
    assert ids[:, 0].tolist() == tokens == greedy[path].tolist() and torch.equal(top[:, 0], logp)
    for bad in ((1, -1, 0), (-1, -1, 0), (0, -2, 0), (0, cfg.n_specialists, 0), (0, -1, cfg.n_layers), (0, -1, -1)):
        with pytest.raises(P.PossError):
            ctx.kv_cache(*bad)
    pair.close()


def test_each_sequence_of_a_batch_hands_out_its_own_cache():
    """Two sequences with the same prompt, a third with another: the same attention over the first two's caches, not over the third's; both kinds of cache, and with
    layers in 4 bits."""
    from synth import make_prompt
    for mx in (False, True):
        pair = Pair("t_mid_bf16", lib_over=dict(batch=3, **({"mx": True} if mx else {})))
        cfg, ctx = pair.cfg, pair.ctx
        prompt = make_prompt(cfg)
        for b in range(3):
            ctx.prefill(prompt if b < 2 else prompt[::-1].copy() if isinstance(prompt, np.ndarray) else prompt[::-1], seq=b)
        q = torch.randn(1, cfg.n_q_heads, cfg.head_dim, device="cuda").to(torch.bfloat16)
        n = torch.tensor([len(prompt) - 1], dtype=torch.int32, device="cuda")
        for which, layer in ((-1, cfg.n_layers - 1), (0, 0)):
            outs = [P.kv_attend(ctx.kv_cache(b, which, layer), q, n, torch.empty_like(q)) for b in range(3)]
            assert torch.equal(outs[0], outs[1]) and not torch.equal(outs[0], outs[2]) and not bool(outs[2].isnan().any())
        with pytest.raises(P.PossError):
            ctx.kv_cache(3)
        pair.close()


def test_offsets_beyond_32_bits():
    """Pages whose values lie past 2^31 and bytes past 2^33, and rows of logits as far apart."""
    per_page = 8 * 128 * 128
    first = (1 << 31) // per_page + 5
    m = Served("bf16", 1, 8, 8, 128, 640, 128, seed=50, pages=first + 5, first_page=first)
    q, k, v = m.qkv(1)
    rope = P.Rope(128)
    m.lengths.fill_(600)
    pos = torch.tensor([600], dtype=torch.int32, device="cuda")
    q_out = torch.empty(1, 8, 128, dtype=torch.bfloat16, device="cuda")
    P.kv_append(m.cache, k, v, m.lengths, pos, rope, q=q, q_out=q_out)
    key, value = m.slot(0, 7, 600)
    assert np.abs(key - o.rotate(f64(k), [600], np.array(rope.frequencies))[0, 7]).max() <= 2.0 ** -6 and np.array_equal(value, f64(v)[0, 7])
    m.lengths += 1
    wo = torch.zeros(1, 8, m.cache.slots, device="cuda")
    P.kv_attend(m.cache, q_out, m.lengths, m.out, lse=m.lse, weights_out=wo)
    ks, vs, table = m.cache.tensors
    small = [x[first:].cpu().double().numpy() for x in (ks, vs)]
    tab = table[0].cpu().numpy() - first
    want, wl, p, _ = o.attend(f64(q_out)[0], o.gather(small[0], tab, 601, 128), o.gather(small[1], tab, 601, 128, values=True), 128 ** -0.5)
    assert np.abs(f64(m.out)[0] - want).max() <= 2.0 ** -8 * np.abs(small[1]).max() and np.abs(f64(wo)[0, :, :601] - p).max() <= 1e-4
    positions = torch.arange(m.cache.slots, device="cuda").int().expand(1, 8, -1).contiguous()
    kept, lo = torch.empty(1, 8, 300, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    P.kv_evict(m.cache, wo, positions, m.lengths, 300, kept, torch.empty_like(wo), torch.empty_like(positions), lo, recent=1)
    stay = o.evict(wo[0, 3].cpu().numpy(), positions[0, 3].cpu().numpy(), 601, 300, 0, 1)
    assert kept[0, 3].tolist() == stay
    moved = next(i for i in range(300) if stay[i] != i)
    key, value = m.slot(0, 3, moved)
    at = stay[moved]
    assert np.array_equal(key, small[0][tab[at // 128], 3, at % 128]) and np.array_equal(value, small[1][tab[at // 128], 3, :, at % 128])
    del m, ks, vs, small
    buf = torch.empty((1 << 32) + 5000, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, 5000), (1 << 31, 1))
    x.normal_()
    tokens = torch.tensor([7, 4999, 0], dtype=torch.int32, device="cuda")
    logp, entropy, ids, top = P.logprobs(x, tokens, n_top=2)
    want, h = o.logprobs(f64(x))
    assert np.abs(f64(logp) - want[np.arange(3), tokens.tolist()]).max() < 1e-4 and np.abs(f64(entropy) - h).max() < 1e-4 and ids.tolist() == [o.best(r, 2) for r in f64(x)]
    y = buf[5000:].as_strided((2, 2, 64), (1 << 31, 64, 1), 5000)
    z = torch.empty(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    y.normal_()
    P.rotary(y, tokens[:2].contiguous(), P.Rope(64), z)
    assert np.abs(f64(z) - o.rotate(f64(y), [7, 4999], np.array(P.Rope(64).frequencies))).max() <= 2.0 ** -6


def test_rotary_turns_keys_as_a_context_does():
    """Layer 0's keys of a prompt, multiplied here and rotated by the call, are those in the context's cache but for sums in another order."""
    pair = Pair("t_mid_bf16")
    cfg, ctx = pair.cfg, pair.ctx
    from synth import make_prompt
    prompt = make_prompt(cfg)
    ctx.prefill(prompt)
    k, _ = ctx.debug_read_kv(-1, 0, 0, len(prompt))
    w = pair.dev_weights
    h = w["embed"][torch.tensor(prompt, device="cuda").long()].float()
    u = (h * torch.rsqrt(h.pow(2).mean(dim=1, keepdim=True) + cfg.rms_eps) * w["layer0.attn_norm"].float()).to(torch.bfloat16).float()
    x = (u @ w["layer0.wk"].float().t()).view(len(prompt), cfg.n_kv_heads, cfg.head_dim)
    got = P.rotary(x, torch.arange(len(prompt), device="cuda").int(), P.Rope(cfg.head_dim, cfg.rope_theta)).to(torch.bfloat16).float().cpu().numpy()
    differ = got != k
    assert differ.mean() < 0.01 and np.abs(got - k).max() <= 2.0 ** -7 * np.abs(k).max()
    pair.close()
