"""Serving over paged caches of a program's own, as cases that can be timed and compared: rotary positions on the way into the cache,
attention of one new token per sequence, eviction from the cache by accumulated attention weight, and what the Head's logits say of given tokens.

The cache is the library's: keys [page][kv head][slot][dim], values [page][kv head][dim][slot], a page table per sequence.  Five kinds of case:

"append":  new rows' queries rotated, keys rotated and written, values written.
"rotate":  rows rotated and nothing else.
"attend":  softmax(scale q k^T) v of one query row per sequence over its slots, the log of the sum of exponentials and, with `weighed`,
           the weights that each slot has been given so far.
"evict":   every head keeps its `budget` heaviest slots; holes below the budget are filled, in order, with kept slots from above it.
"logprobs": log-probabilities of given tokens, entropy and the best alternatives.

The plain form computes in float32 (angles in float64) with elementary operations and rounds once at the end.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the new token of one sequence: latency is all there is
        dict(name="append_token", kind="append", t="bf16", n_seq=1, rows=1, hq=32, hkv=8, dh=128, page=64, rot=128, inter=False, scaling="none", at=1000),
        # a prompt under frequencies scaled for long contexts
        dict(name="append_prompt", kind="append", t="bf16", n_seq=1, rows=8192, hq=32, hkv=8, dh=128, page=64, rot=128, inter=False, scaling="bands", at=0),
        # float32 heads of odd number, three quarters of each rotated, pairs side by side, positions far out, turned back
        dict(name="rotate_ragged", kind="rotate", t="f32", rows=1001, heads=5, dh=128, rot=96, inter=True, scaling="ramp", far=True, inverse=True),
        # a short sequence's new token
        dict(name="attend_token", kind="attend", t="bf16", n_seq=1, longest=17, spread=False, hq=32, hkv=8, dh=128, page=64, weighed=False),
        # one sequence with a very long cache: split over its length
        dict(name="attend_long", kind="attend", t="bf16", n_seq=1, longest=131072, spread=False, hq=32, hkv=8, dh=128, page=128, weighed=False),
        # a ragged batch, some of it empty or just begun, whose slots are weighed for eviction
        dict(name="attend_batch", kind="attend", t="bf16", n_seq=64, longest=8192, spread=True, hq=32, hkv=8, dh=128, page=64, weighed=True),
        # as many key heads as query heads
        dict(name="attend_heads", kind="attend", t="f16", n_seq=16, longest=2048, spread=True, hq=40, hkv=40, dh=128, page=32, weighed=False),
        # a sequence at its budget: one slot goes
        dict(name="evict_one", kind="evict", t="bf16", n_seq=1, longest=1025, spread=False, budget=1024, hkv=8, dh=128, page=64, first=4, recent=256),
        # a batch cut to half after its prompts
        dict(name="evict_half", kind="evict", t="bf16", n_seq=32, longest=4096, spread=True, budget=2000, hkv=8, dh=128, page=64, first=4, recent=500),
        # one committed token
        dict(name="logprobs_token", kind="logprobs", t="f32", rows=1, vocab=128256, tokens=1, top=5, temperature=1.0),
        # a tree's rows, their candidate children, at a temperature
        dict(name="logprobs_tree", kind="logprobs", t="f32", rows=61, vocab=128256, tokens=10, top=10, temperature=0.7),
        # a prompt's tokens, odd rows
        dict(name="logprobs_prompt", kind="logprobs", t="bf16", rows=4095, vocab=32001, tokens=1, top=1, temperature=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "rotate", "attend", "attend", "evict", "logprobs"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    dh = rng.choice([64, 96, 128, 128, 256])
    page = rng.choice([32, 64, 128])
    hkv = rng.choice([1, 2, 5, 8, 8, 40])
    hq = hkv * (1 if hkv == 40 else rng.choice([1, 2, 4, 7, 8]))
    turned = dict(rot=rng.choice([dh, dh, dh // 2]), inter=rng.random() < 0.4, scaling=rng.choice(["none", "linear", "base", "bands", "ramp"]))
    if kind == "append":
        n_seq = rng.choice([1, 1, rng.randint(2, 100)])
        rows = max(1, min(_log_int(rng, 1, 8192), 8192 * 48 * 128 * 2 // ((hq + 2 * hkv) * dh * SIZE[t])))
        return dict(kind=kind, t=t, n_seq=n_seq, rows=rows, hq=hq, hkv=hkv, dh=dh, page=page, at=rng.randint(0, 3000) if n_seq * hkv * dh < 40000 else 0, **turned)
    if kind == "rotate":
        heads = rng.randint(1, 40)
        rows = max(1, min(_log_int(rng, 1, 8192), 8192 * 40 * 128 * 2 // (heads * dh * SIZE[t])))
        return dict(kind=kind, t=t, rows=rows, heads=heads, dh=dh, far=rng.random() < 0.5, inverse=rng.random() < 0.3, **turned)
    if kind == "attend":
        n_seq = _log_int(rng, 1, 100)
        most = max(1, int(0.5e9) // (n_seq * hkv * dh * 2 * SIZE[t]))
        return dict(kind=kind, t=t, n_seq=n_seq, longest=min(most, _log_int(rng, 1, 131072)), spread=rng.random() < 0.7, hq=hq, hkv=hkv, dh=dh, page=page, weighed=rng.random() < 0.5)
    if kind == "evict":
        n_seq = _log_int(rng, 1, 32)
        longest = min(max(40, int(0.25e9) // (n_seq * hkv * dh * 2 * SIZE[t])), _log_int(rng, 40, 32768))
        budget = max(20, int(longest * rng.uniform(0.2, 1.0)))
        return dict(kind=kind, t=t, n_seq=n_seq, longest=longest, spread=rng.random() < 0.7, budget=budget, hkv=hkv, dh=dh, page=page, first=rng.randint(0, 4), recent=rng.randint(0, budget - 8))
    vocab = _log_int(rng, 1000, 128256)
    rows = max(1, min(_log_int(rng, 1, 4096), 4095 * 32001 * 2 // (vocab * SIZE[t])))
    return dict(kind=kind, t=t, rows=rows, vocab=vocab, tokens=rng.choice([1, 1, 10]), top=rng.choice([0, 1, 5, 10, 20]), temperature=rng.choice([1.0, 0.7, 1.3]))


# ---------------------------------------------------------------- what the program has in hand
THETA, ORIGINAL, FACTOR, LOW, HIGH = 500000.0, 8192, 8.0, 1.0, 4.0


def _frequencies(case):
    """The scaled frequencies of a head's pairs, on the host in 64 bits, and the factor of cosine and sine."""
    r, scaling = case["rot"], case["scaling"]
    theta = THETA * FACTOR ** (r / (r - 2)) if scaling == "base" else THETA
    w = [theta ** (-2.0 * i / r) for i in range(r // 2)]
    if scaling == "linear":
        return [f / FACTOR for f in w], 1.0
    if scaling == "bands":                                 # by how often a pair turns within the original length
        part = [min(1.0, max(0.0, (ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW))) for f in w]
        return [g * f + (1 - g) * f / FACTOR for f, g in zip(w, part)], 1.0
    if scaling == "ramp":                                  # by the pair's index, between those that turn HIGH and LOW times
        def index(turns):
            return r * math.log(ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(theta))
        lo, hi = max(0, math.floor(index(HIGH))), min(r - 1, math.ceil(index(LOW)))
        part = [1 - min(1.0, max(0.0, (i - lo) / max(1e-3, hi - lo))) for i in range(r // 2)]
        return [g * f + (1 - g) * f / FACTOR for f, g in zip(w, part)], 0.1 * math.log(FACTOR) + 1.0
    return w, 1.0


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _lengths(case, g):
    """Slots in use per sequence; in a ragged batch some are empty or hold one token."""
    n, longest = case["n_seq"], case["longest"]
    if not case["spread"]:
        return torch.full((n,), longest, dtype=torch.int32, device="cuda")
    u = torch.rand(n, generator=g, device="cuda")
    lengths = (u * (longest + 1)).int().clamp(max=longest)
    lengths[n // 2] = 0 if case["kind"] == "attend" else 1
    lengths[n // 3] = 1
    lengths[0] = longest
    return lengths


def _pool(case, g, slots):
    """Pages for `slots` slots of every sequence, in any order, and what they hold."""
    n_seq, P = case["n_seq"], case["page"]
    per = -(-slots // P)
    pages = n_seq * per
    table = torch.randperm(pages, generator=g, device="cuda").int().view(n_seq, per)
    t = TYPES[case["t"]]
    k = torch.randn(pages, case["hkv"], P, case["dh"], generator=g, device="cuda", dtype=t)
    v = torch.randn(pages, case["hkv"], case["dh"], P, generator=g, device="cuda", dtype=t)
    return k, v, table


def _positions(case, g):
    rows = case["rows"]
    if case["kind"] == "rotate":
        at = torch.randint(0, 100000 if case["far"] else 4096, (1,), generator=g, device="cuda")
        return (at + torch.arange(rows, device="cuda")).int()
    return (case["at"] + torch.arange(rows, device="cuda") % -(-rows // case["n_seq"])).int()


def prepare(case, seed):
    g, kind, t = _generator(seed), case["kind"], TYPES[case["t"]]
    s = dict(case=case)
    if kind == "logprobs":
        rows, V = case["rows"], case["vocab"]
        x = torch.randn(rows, V, generator=g, device="cuda") * 2.5
        x += torch.randn(V, generator=g, device="cuda")
        x[:, torch.randint(0, V, (V // 50,), generator=g, device="cuda")] = -math.inf      # ids that a grammar forbids
        s["tokens"] = torch.randint(0, V, (rows, case["tokens"]), generator=g, device="cuda").int()
        x[torch.arange(rows, device="cuda"), s["tokens"][:, 0].long()] = torch.rand(rows, generator=g, device="cuda") * 12
        s["x"] = x.to(t)
        if own:
            import paper_2506_03566_amd as P
            s["scratch"] = P.logprobs_scratch(rows, V, case["top"])
        return s
    if kind in ("append", "rotate"):
        rows, dh = case["rows"], case["dh"]
        freq, s["magnitude"] = _frequencies(case)
        s["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
        s["positions"] = _positions(case, g)
        if own:
            import paper_2506_03566_amd as P
            s["rope"] = P.Rope(case["rot"], THETA, interleaved=case["inter"], scaling=case["scaling"], factor=FACTOR, low=LOW, high=HIGH, original=ORIGINAL,
                               magnitude=s["magnitude"])
        if kind == "rotate":
            s["x"] = torch.randn(rows, case["heads"], dh, generator=g, device="cuda").to(t)
            s["out"] = torch.empty_like(s["x"])
            return s
        hq, hkv, n = case["hq"], case["hkv"], case["n_seq"]
        qkv = torch.randn(rows, (hq + 2 * hkv) * dh, generator=g, device="cuda").to(t)       # what the stacked projection gives
        s["q"], s["k_new"], s["v_new"] = (p.view(rows, -1, dh) for p in qkv.split([hq * dh, hkv * dh, hkv * dh], dim=1))
        s["q_out"] = torch.empty(rows, hq, dh, dtype=t, device="cuda")
        s["seq"] = (torch.arange(rows, device="cuda") // -(-rows // n)).int()              # a token of each, or prompts one behind the other
        s["slots"] = s["positions"].clone()
        if rows > 4:
            s["slots"][rows // 2] = -1                     # a row of padding
        s["k"], s["v"], s["table"] = _pool(case, g, case["at"] + -(-rows // n))
    else:
        s["lengths"] = _lengths(case, g)
        s["k"], s["v"], s["table"] = _pool(case, g, case["longest"])
        slots = s["table"].shape[1] * case["page"]
        if kind == "attend":
            n, hq, hkv, dh = case["n_seq"], case["hq"], case["hkv"], case["dh"]
            s["q"] = torch.randn(n, hq, dh, generator=g, device="cuda").mul_(2).to(t)
            s["out"] = torch.empty(n, hq, dh, dtype=t, device="cuda")
            s["lse"] = torch.empty(n, hq, device="cuda")
            if case["weighed"]:
                s["weights"] = torch.rand(n, hkv, slots, generator=g, device="cuda").pow_(6)
                s["weights_out"] = torch.zeros(n, hkv, slots, device="cuda")
        else:
            n, hkv = case["n_seq"], case["hkv"]
            w = (torch.randn(n, hkv, slots, generator=g, device="cuda") * 2).exp_()
            w[torch.rand(n, hkv, slots, generator=g, device="cuda") < 0.1] = 0.0             # never looked at: ties
            s["weights"] = w
            s["positions"] = (torch.arange(slots, device="cuda") + slots // 2).int().expand(n, hkv, slots).contiguous()
            s["positions"][:, :, :case["first"]] = torch.arange(case["first"], device="cuda").int()
            s["kept"] = torch.empty(n, hkv, case["budget"], dtype=torch.int32, device="cuda")
            s["weights_out"], s["positions_out"] = torch.empty_like(w), torch.empty_like(s["positions"])
            s["lengths_out"] = torch.empty_like(s["lengths"])
    if own:
        import paper_2506_03566_amd as P
        s["cache"] = P.KvCache(s["k"], s["v"], s["table"])
        if kind == "attend":
            s["scratch"] = P.kv_attend_scratch(s["cache"], case["hq"], weights=case["weighed"])
    return s


# ---------------------------------------------------------------- the plain forms
def _turned(x, positions, freq, magnitude, rot, inter, inverse=False):
    """x [rows, heads, dh] rotated, in float32."""
    angle = positions.double()[:, None] * freq
    c, s = (angle.cos() * magnitude).float()[:, None], (angle.sin() * magnitude).float()[:, None]
    s = -s if inverse else s
    x = x.float()
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :rot // 2], r[..., rot // 2:])
    a, b = a * c - b * s, b * c + a * s
    r = torch.stack([a, b], dim=-1).flatten(-2) if inter else torch.cat([a, b], dim=-1)
    return torch.cat([r, rest], dim=-1)


def _append(s):
    c, t, P = s["case"], TYPES[s["case"]["t"]], s["case"]["page"]
    turn = (s["positions"], s["freq"], s["magnitude"], c["rot"], c["inter"])
    s["q_out"].copy_(_turned(s["q"], *turn))
    rows = (s["slots"] >= 0).nonzero()[:, 0]
    slot, seq = s["slots"][rows].long(), s["seq"][rows].long()
    page = s["table"][seq, slot // P].long()
    s["k"][page, :, slot % P] = _turned(s["k_new"], *turn).to(t)[rows]
    s["v"][page, :, :, slot % P] = s["v_new"][rows]
    return s["q_out"], s["k"], s["v"]


def _gathered(s):
    """Keys and values [sequence, head, slot, dim] in float32."""
    n, hkv, dh = s["case"]["n_seq"], s["case"]["hkv"], s["case"]["dh"]
    at = s["table"].long()
    k = s["k"][at].float().permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, dh)
    v = s["v"][at].float().permute(0, 2, 1, 4, 3).reshape(n, hkv, -1, dh)
    return k, v


def _attend(s):
    c = s["case"]
    n, hq, hkv, dh = c["n_seq"], c["hq"], c["hkv"], c["dh"]
    k, v = _gathered(s)
    slots = k.shape[2]
    there = (torch.arange(slots, device="cuda") < s["lengths"][:, None])[:, None, None]
    q = s["q"].float().view(n, hkv, hq // hkv, dh) * dh ** -0.5
    score = (q @ k.transpose(2, 3).contiguous()).masked_fill(~there, -math.inf)
    top = score.amax(dim=3, keepdim=True).clamp(min=-1e30)
    e = (score - top).exp()
    total = e.sum(dim=3, keepdim=True)
    p = e / total.clamp(min=1e-30)
    s["out"].copy_((p @ v).view(n, hq, dh))
    s["lse"].copy_((top + total.log()).view(n, hq))
    if not c["weighed"]:
        return s["out"], s["lse"]
    s["weights_out"].copy_(torch.where(there[:, 0], s["weights"] + p.sum(dim=2), s["weights_out"]))
    return s["out"], s["lse"], s["weights_out"]


def _evict(s):
    c, w, pos, P = s["case"], s["weights"], s["positions"], s["case"]["page"]
    slots, budget = w.shape[2], c["budget"]
    i = torch.arange(slots, device="cuda")
    length = s["lengths"].long()[:, None, None]
    there = i < length
    newest = pos.masked_fill(~there, -1 << 31).amax(dim=2, keepdim=True).long()
    always = there & ((pos < c["first"]) | (pos.long() > newest - c["recent"]))
    key = w.masked_fill(always, math.inf).masked_fill(~there, -math.inf)
    order = key.sort(dim=2, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(2, order, i.expand_as(order))
    count = length.clamp(max=budget)
    stays = rank < count
    movers = (~(stays & (i >= count))).to(torch.uint8).sort(dim=2, stable=True).indices      # kept slots above the budget, in order
    hole = ~stays & (i < count)
    source = torch.where(hole, movers.gather(2, (hole.cumsum(dim=2) - 1).clamp(min=0)), i)
    filled = i < count
    s["weights_out"].copy_(torch.where(filled, w.gather(2, source), 0.0))
    s["positions_out"].copy_(torch.where(filled, pos.gather(2, source), -1))
    s["kept"].copy_(torch.nn.functional.pad(torch.where(filled, source, -1), (0, max(0, budget - slots)), value=-1)[:, :, :budget])
    s["lengths_out"].copy_(count.view(-1))
    b, h, to = hole.nonzero(as_tuple=True)
    at = source[b, h, to]
    page, page_to = s["table"][b, at // P].long(), s["table"][b, to // P].long()
    s["k"][page_to, h, to % P] = s["k"][page, h, at % P]
    s["v"][page_to, h, :, to % P] = s["v"][page, h, :, at % P]
    return s["kept"], s["weights_out"], s["positions_out"], s["lengths_out"], s["k"], s["v"]


def _logprobs(s):
    c = s["case"]
    x = s["x"].float()
    z = x / c["temperature"]
    top = z.amax(dim=1, keepdim=True)
    d = z - top
    e = d.exp()
    total = e.sum(dim=1, keepdim=True)
    lse = top + total.log()
    logp = z.gather(1, s["tokens"].long()) - lse
    entropy = (total.log() - torch.where(e > 0, e * d, 0.0).sum(dim=1, keepdim=True) / total)[:, 0]
    ids = x.sort(dim=1, descending=True, stable=True).indices[:, :c["top"]]
    return logp, entropy, ids.int(), z.gather(1, ids) - lse


# ---------------------------------------------------------------- one pass
def run(s):
    c, kind = s["case"], s["case"]["kind"]
    if own:
        import paper_2506_03566_amd as P
        if kind == "append":
            P.kv_append(s["cache"], s["k_new"], s["v_new"], s["slots"], s["positions"], s["rope"], seq=s["seq"], q=s["q"], q_out=s["q_out"])
            return s["q_out"], s["k"], s["v"]
        if kind == "rotate":
            return P.rotary(s["x"], s["positions"], s["rope"], s["out"], inverse=c["inverse"])
        if kind == "attend":
            if not c["weighed"]:
                P.kv_attend(s["cache"], s["q"], s["lengths"], s["out"], lse=s["lse"], scratch=s["scratch"])
                return s["out"], s["lse"]
            P.kv_attend(s["cache"], s["q"], s["lengths"], s["out"], lse=s["lse"], weights=s["weights"], weights_out=s["weights_out"], scratch=s["scratch"])
            return s["out"], s["lse"], s["weights_out"]
        if kind == "evict":
            P.kv_evict(s["cache"], s["weights"], s["positions"], s["lengths"], c["budget"], s["kept"], s["weights_out"], s["positions_out"], s["lengths_out"],
                       first=c["first"], recent=c["recent"])
            return s["kept"], s["weights_out"], s["positions_out"], s["lengths_out"], s["k"], s["v"]
        return P.logprobs(s["x"], s["tokens"], n_top=c["top"], temperature=c["temperature"], scratch=s["scratch"])
    if kind == "rotate":
        return s["out"].copy_(_turned(s["x"], s["positions"], s["freq"], s["magnitude"], c["rot"], c["inter"], c["inverse"]))
    return {"append": _append, "attend": _attend, "evict": _evict, "logprobs": _logprobs}[kind](s)


def work(case):
    kind, e = case["kind"], SIZE[case["t"]]
    if kind == "append":
        values = case["rows"] * (case["hq"] + 2 * case["hkv"]) * case["dh"]
        return {"bytes": 2 * values * e, "flops": 3 * case["rows"] * (case["hq"] + case["hkv"]) * case["rot"]}
    if kind == "rotate":
        values = case["rows"] * case["heads"] * case["dh"]
        return {"bytes": 2 * values * e, "flops": 3 * case["rows"] * case["heads"] * case["rot"]}
    if kind == "logprobs":
        values = case["rows"] * case["vocab"]
        return {"bytes": values * e + case["rows"] * (8 * case["tokens"] + 4 + 8 * case["top"]), "flops": 5 * values}
    n, hkv, dh, longest = case["n_seq"], case["hkv"], case["dh"], case["longest"]
    used = n * longest if not case["spread"] else longest + (n - 1) * longest / 2            # slots in use, about
    if kind == "attend":
        return {"bytes": used * hkv * (2 * dh * e + (8 if case["weighed"] else 0)) + 2 * n * case["hq"] * dh * e, "flops": 4 * used * case["hq"] * dh}
    # of `longest` slots a share of budget / longest stays; as large a share of the holes below the budget is filled from above
    share = min(1.0, case["budget"] / longest)
    moved = n * hkv * case["budget"] * (1 - share) * (0.5 if case["spread"] else 1)
    return {"bytes": used * hkv * 16 + n * hkv * case["budget"] * 4 + moved * 4 * dh * e, "flops": used * hkv}


# ---------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    kind = case["kind"]
    with_own, globals()["own"] = own, False
    try:
        s = prepare(case, seed)
    finally:
        globals()["own"] = with_own
    if kind == "logprobs":
        p = torch.softmax(s["x"].double() / case["temperature"], dim=1)
        logp = p.gather(1, s["tokens"].long()).log()
        return logp, -torch.special.xlogy(p, p).sum(dim=1), None, p.topk(case["top"], dim=1).values.log()

    def turned(x, sign=1):
        w, magnitude = _frequencies(case)
        r, rows = case["rot"], x.shape[0]
        angle = s["positions"].double().view(rows, 1, 1) * torch.tensor(w, dtype=torch.float64, device="cuda") * sign
        by = torch.polar(torch.full_like(angle, magnitude), angle)
        x = x.double().clone()
        first, second = (slice(0, r, 2), slice(1, r, 2)) if case["inter"] else (slice(0, r // 2), slice(r // 2, r))
        z = torch.complex(x[..., first], x[..., second]) * by
        x[..., first], x[..., second] = z.real, z.imag
        return x

    if kind == "rotate":
        return turned(s["x"], -1 if case["inverse"] else 1)
    P = case["page"]
    if kind == "append":
        k, v = s["k"].double(), s["v"].double()
        k_new = turned(s["k_new"])
        slots, seqs, table = s["slots"].tolist(), s["seq"].tolist(), s["table"].tolist()
        rows = [r for r in range(case["rows"]) if slots[r] >= 0]
        page = torch.tensor([table[seqs[r]][slots[r] // P] for r in rows], device="cuda")
        off = torch.tensor([slots[r] % P for r in rows], device="cuda")
        heads = torch.arange(case["hkv"], device="cuda")
        k[page[:, None], heads, off[:, None]] = k_new[rows]
        v[page[:, None], heads, :, off[:, None]] = s["v_new"].double()[rows]
        return turned(s["q"]), k, v
    if kind == "attend":
        n, hq, hkv, dh = case["n_seq"], case["hq"], case["hkv"], case["dh"]
        out, lse = torch.zeros(n, hq, dh, dtype=torch.float64, device="cuda"), torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda")
        weights = s["weights_out"].double() if case["weighed"] else None
        for b, length in enumerate(s["lengths"].tolist()):
            if length == 0:
                continue
            at = s["table"][b].long()
            for h in range(hkv):
                group = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                k = s["k"][at, h].reshape(-1, dh)[:length].double()
                v = s["v"][at, h].transpose(1, 2).reshape(-1, dh)[:length].double()
                score = (s["q"][b, group].double() @ k.t()) / math.sqrt(dh)
                lse[b, group] = torch.logsumexp(score, dim=1)
                p = (score - lse[b, group, None]).exp()
                out[b, group] = p @ v
                if weights is not None:
                    weights[b, h, :length] = s["weights"][b, h, :length].double() + p.sum(dim=0)
        return (out, lse) if weights is None else (out, lse, weights)
    # eviction, head by head; keys and values are moved, not computed, and are held to the plain form's
    if case["n_seq"] * case["hkv"] * case["longest"] > 1 << 21:
        return None
    n, hkv, budget = case["n_seq"], case["hkv"], case["budget"]
    weights = torch.zeros_like(s["weights"], dtype=torch.float64, device="cpu")
    w, pos = s["weights"].cpu().double(), s["positions"].cpu()
    for b, length in enumerate(s["lengths"].tolist()):
        for h in range(hkv):
            values, at = w[b, h, :length].tolist(), pos[b, h, :length].tolist()
            newest = max(at, default=0)
            order = sorted(range(length), key=lambda i: (not (at[i] < case["first"] or at[i] > newest - case["recent"]), 0 if at[i] < case["first"] or at[i] > newest - case["recent"] else -values[i], i))
            keep = set(order[:budget])
            count = min(length, budget)
            above = iter(sorted(i for i in keep if i >= count))
            weights[b, h, :count] = torch.tensor([values[i if i in keep else next(above)] for i in range(count)], dtype=torch.float64)
    return None, weights.cuda(), None, None, None, None
