"""Serving over paged caches of a program's own: argument marshalling for poss_rotary, poss_kv_append, poss_kv_attend, poss_kv_evict and poss_logprobs.

Same names as include/poss.h, which says what each call does.  Tensors of a call are on one GPU; work goes to torch's current stream there
unless a stream is given.  Small calls take a few microseconds: what these functions do for a call is kept short.
"""
import contextlib
import ctypes

from .binding import POSS_OK, PossError, PossKvCache, PossRope, _mx, _mx_call, _mx_empty, _mx_refuse, _mx_type

LOGPROBS_TOP = 32
_AS_IT_IS = contextlib.nullcontext()
_SCALINGS = {"none": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}


def _ints(t, shape, what):
    if t.dtype is not _mx.torch.int32 or t.shape != shape or not t.is_contiguous():
        _mx_refuse("%s: contiguous int32 %s is wanted, got %s %s" % (what, tuple(shape), t.dtype, tuple(t.shape)))
    return t.data_ptr()


def _floats(t, shape, what):
    if t.dtype is not _mx.torch.float32 or t.shape != shape or not t.is_contiguous():
        _mx_refuse("%s: contiguous float32 %s is wanted, got %s %s" % (what, tuple(shape), t.dtype, tuple(t.shape)))
    return t.data_ptr()


def _count(n, what):
    """n, which has to be of 31 bits: what is wider would lose its upper ones on the way."""
    return n if 0 <= n <= 0x7fffffff else _mx_refuse("%s rejected: %d" % (what, n))


def _heads(t, dtype, rows, heads, dim, what):
    """The row distance of [rows, heads, dim] whose heads are contiguous."""
    if t.dtype is not dtype or t.shape != (rows, heads, dim):
        _mx_refuse("%s: %s [%d, %d, %d] is wanted, got %s %s" % (what, dtype, rows, heads, dim, t.dtype, tuple(t.shape)))
    row, head, step = t.stride()
    if (step != 1 and dim > 1) or (head != dim and heads > 1) or (row < heads * dim and rows > 1):
        _mx_refuse("%s: a row's heads must be contiguous, rows must not overlap" % what)
    return row if rows > 1 else heads * dim


class Rope:
    """Rotary positions of a head's first rot_dim values.  scaling: "none", "linear", "base", "bands" or "ramp" (poss_rope_fill has the formulas);
    frequencies: rot_dim / 2 numbers of the caller's own instead."""

    def __init__(self, rot_dim, theta=10000.0, interleaved=False, scaling="none", factor=1.0, low=1.0, high=4.0, original=8192, magnitude=1.0, frequencies=None):
        lib = (_mx if _mx.lib else _mx.open()).lib
        if scaling not in _SCALINGS:
            _mx_refuse("scaling is one of %s" % ", ".join(_SCALINGS))
        self.c = PossRope()
        rc = lib.poss_rope_fill(_count(rot_dim, "rot_dim"), 1 if interleaved else 0, theta, _SCALINGS[scaling], factor, low, high, original, magnitude, ctypes.byref(self.c))
        if rc != POSS_OK:
            raise PossError(rc, lib.poss_last_error(None).decode())
        if frequencies is not None:
            f = [float(x) for x in frequencies]
            if len(f) != rot_dim // 2 or not all(abs(x) < float("inf") for x in f):
                _mx_refuse("frequencies: %d finite numbers are wanted" % (rot_dim // 2))
            self.c.freq[:len(f)] = f
        self.ref = ctypes.byref(self.c)

    @property
    def frequencies(self):
        return list(self.c.freq[:self.c.rot_dim // 2])


def rotary(x, positions, rope, out=None, inverse=False, stream=None):
    """Rows x [rows, heads, dim] rotated to int32 positions [rows], into out (may be x; allocated if not given).  Returns out."""
    t = _mx_type(x.dtype)
    if x.dim() != 3:
        _mx_refuse("x must be [rows, heads, dim]")
    rows, heads, dim = x.shape
    if out is None:
        if stream is None:
            out = _mx.torch.empty_like(x, memory_format=_mx.torch.contiguous_format)
        else:
            with _mx.torch.cuda.stream(stream):
                out = _mx.torch.empty_like(x, memory_format=_mx.torch.contiguous_format)
    if out.dtype is not x.dtype or out.shape != x.shape:
        _mx_refuse("out must be as x")
    xr, xh, xs = x.stride()
    yr, yh, ys = out.stride()
    if dim > 1 and (xs != 1 or ys != 1):
        _mx_refuse("heads must be contiguous")
    if max(rows, heads, dim) > 0x7fffffff or heads == 0 or dim == 0:
        _mx_refuse("shape rejected")
    _mx_call(_mx.lib.poss_rotary, stream, (x, out, positions), t, x.data_ptr(), xr if rows > 1 else 0, xh if heads > 1 else 0, out.data_ptr(), yr if rows > 1 else 0,
             yh if heads > 1 else 0, rows, heads, dim, _ints(positions, (rows,), "positions"), rope.ref, 1 if inverse else 0)
    return out


class KvCache:
    """A paged cache: k [pages, kv_heads, page, dim], v [pages, kv_heads, dim, page] (pages may lie apart), page_table int32 [sequences, pages of each].
    Keeps the tensors; slots: how many a sequence has."""

    def __init__(self, k, v, page_table):
        code = _mx_type(k.dtype)
        if k.dim() != 4 or v.dim() != 4 or page_table.dim() != 2 or v.dtype is not k.dtype or page_table.dtype is not _mx.torch.int32:
            _mx_refuse("k [pages, heads, page, dim], v [pages, heads, dim, page] and an int32 page_table [sequences, pages] are wanted")
        pages, heads, page, dim = k.shape
        if v.shape != (pages, heads, dim, page) or max(pages, heads, page, dim, *page_table.shape) > 0x7fffffff:
            _mx_refuse("v [%d, %d, %d, %d] is wanted, got %s" % (pages, heads, dim, page, tuple(v.shape)))
        if k.stride()[1:] != (page * dim, dim, 1) or v.stride()[1:] != (page * dim, page, 1) or page_table.stride(1) != 1 and page_table.shape[1] > 1:
            _mx_refuse("a page's keys and values and a row of the table must be contiguous")
        n_seq, per = page_table.shape
        whole = heads * page * dim
        self._set(PossKvCache(code, heads, dim, page, pages, n_seq, per, page_table.stride(0) if n_seq > 1 else per, k.stride(0) if pages > 1 else whole,
                              v.stride(0) if pages > 1 else whole, k.data_ptr(), v.data_ptr(), page_table.data_ptr()), k.dtype, (k, v, page_table))
        if len({t.get_device() for t in self.tensors}) != 1 or k.get_device() < 0:
            _mx_refuse("all tensors of a cache must be on one GPU")

    def _set(self, c, dtype, tensors, keep=None):
        self.c, self.dtype, self.tensors, self.keep = c, dtype, tensors, keep
        self.ref = ctypes.byref(c)
        self.n_seq, self.heads, self.dim, self.slots = c.n_seq, c.n_kv_heads, c.head_dim, c.table_pages * c.page_tokens

    @classmethod
    def of_context(cls, ctx, c):
        """What Poss.kv_cache gives: the context's own memory, kept with it."""
        types = {code: t for t, code in (_mx if _mx.lib else _mx.open()).types.items()}
        self = cls.__new__(cls)
        self._set(c, types[c.dtype], (ctx.workspace,), ctx)
        return self


def kv_append(cache, k, v, slots, positions=None, rope=None, seq=None, q=None, q_out=None, slot_positions=None, stream=None):
    """Rows k, v [rows, kv_heads, dim] into slots [rows] of sequences seq [rows] (None: row r is sequence r), keys rotated to positions [rows] by rope;
    q [rows, heads, dim] rotated into q_out (None: into q).  slot_positions: int32 [sequences, kv_heads, slots] that notes the positions.  Returns q_out."""
    if k.dim() != 3 or (q is not None and q.dim() != 3):
        _mx_refuse("k and q must be [rows, heads, dim]")
    rows = k.shape[0]
    if rows > 0x7fffffff:
        _mx_refuse("too many rows")
    kr, vr = _heads(k, cache.dtype, rows, cache.heads, cache.dim, "k"), _heads(v, cache.dtype, rows, cache.heads, cache.dim, "v")
    tensors = [*cache.tensors, k, v, slots]
    hq, qp, qr, op, orow = 0, 0, 0, 0, 0
    if q is not None:
        hq = q.shape[1]
        q_out = q if q_out is None else q_out
        qr, orow = _heads(q, cache.dtype, rows, hq, cache.dim, "q"), _heads(q_out, cache.dtype, rows, hq, cache.dim, "q_out")
        qp, op = q.data_ptr(), q_out.data_ptr()
        tensors += (q, q_out)
    sp = _ints(slots, (rows,), "slots")
    pp = bp = np = 0
    if positions is not None:
        pp = _ints(positions, (rows,), "positions")
        tensors.append(positions)
    if seq is not None:
        bp = _ints(seq, (rows,), "seq")
        tensors.append(seq)
    if slot_positions is not None:
        np = _ints(slot_positions, (cache.n_seq, cache.heads, cache.slots), "slot_positions")
        tensors.append(slot_positions)
    _mx_call(_mx.lib.poss_kv_append, stream, tensors, cache.ref, rope.ref if rope is not None else None, rows, hq, qp, qr, op, orow, k.data_ptr(), kr, v.data_ptr(), vr,
             bp, sp, pp, np)
    return q_out


def kv_attend_scratch(cache, heads, max_len=0, weights=False, stream=None):
    """Scratch for kv_attend of `heads` query heads over this cache, with weights or without."""
    need = _mx.lib.poss_kv_attend_scratch_bytes(cache.ref, _count(heads, "heads"), _count(max_len, "max_len"), 1 if weights else 0)
    if need == 0:
        _mx_refuse("shape rejected")
    return _mx_empty(need, cache.tensors[0].device, stream)


def kv_attend(cache, q, lengths, out, lse=None, weights=None, weights_out=None, scale=None, max_len=0, scratch=None, stream=None):
    """out [sequences, heads, dim] = attention of q over each sequence's first lengths[b] slots; lse float32 [sequences, heads].  weights_out float32
    [sequences, kv_heads, slots] = weights (None: zeros; may be weights_out) + the probabilities, summed over the heads of a key head.  scale: 1 / sqrt(dim) unless given.
    max_len: the most any length is (0: all slots).  scratch: from kv_attend_scratch, not used by another call at the same time; allocated per call if not given."""
    if q.dim() != 3:
        _mx_refuse("q must be [sequences, heads, dim]")
    n, heads = cache.n_seq, q.shape[1]
    qr, orow = _heads(q, cache.dtype, n, heads, cache.dim, "q"), _heads(out, cache.dtype, n, heads, cache.dim, "out")
    tensors = [*cache.tensors, q, out, lengths]
    lp = wp = op = 0
    if lse is not None:
        lp = _floats(lse, (n, heads), "lse")
        tensors.append(lse)
    if weights_out is not None:
        op = _floats(weights_out, (n, cache.heads, cache.slots), "weights_out")
        tensors.append(weights_out)
    if weights is not None:
        wp = _floats(weights, (n, cache.heads, cache.slots), "weights")
        tensors.append(weights)
    if scratch is None:
        scratch = kv_attend_scratch(cache, heads, max_len, weights_out is not None, stream)
    elif not scratch.is_contiguous():
        _mx_refuse("scratch must be contiguous")
    tensors.append(scratch)
    _mx_call(_mx.lib.poss_kv_attend, stream, tensors, cache.ref, heads, q.data_ptr(), qr, out.data_ptr(), orow, _ints(lengths, (n,), "lengths"), _count(max_len, "max_len"),
             cache.dim ** -0.5 if scale is None else scale, lp, wp, op, scratch.data_ptr(), scratch.nbytes)
    return out


def kv_evict(cache, weights, positions, lengths, budget, kept, weights_out, positions_out, lengths_out, first=0, recent=0, stream=None):
    """Cuts every sequence to `budget` slots, each key head for itself (poss_kv_evict).  weights float32 and positions int32 [sequences, kv_heads, slots], lengths
    int32 [sequences]; kept int32 [sequences, kv_heads, budget] and the other outputs are written.  Returns lengths_out."""
    n, h = cache.n_seq, cache.heads
    shape = (n, h, cache.slots)
    if not 0 < budget <= 0x7fffffff or max(first, recent) > 0x7fffffff or min(first, recent) < 0:
        _mx_refuse("budget, first or recent rejected")
    _mx_call(_mx.lib.poss_kv_evict, stream, (*cache.tensors, weights, positions, lengths, kept, weights_out, positions_out, lengths_out), cache.ref,
             _floats(weights, shape, "weights"), _ints(positions, shape, "positions"), _ints(lengths, (n,), "lengths"), budget, first, recent,
             _ints(kept, (n, h, budget), "kept"), _floats(weights_out, shape, "weights_out"), _ints(positions_out, shape, "positions_out"),
             _ints(lengths_out, (n,), "lengths_out"))
    return lengths_out


def logprobs_scratch(rows, vocab, n_top=0, device="cuda", stream=None):
    """Scratch for logprobs of this shape; one that is large enough serves others too."""
    lib = (_mx if _mx.lib else _mx.open()).lib
    need = lib.poss_logprobs_scratch_bytes(_count(rows, "rows"), _count(vocab, "vocab"), _count(n_top, "n_top"))
    if need == 0:
        _mx_refuse("shape rejected")
    return _mx_empty(need, device, stream)


def logprobs(logits, tokens=None, n_top=0, temperature=1.0, logp=None, entropy=None, top_ids=None, top_logp=None, scratch=None, stream=None):
    """(logp, entropy, top_ids, top_logp) of logits [rows, vocab] (float32, bfloat16, float16): log-probabilities of int32 tokens [rows] or [rows, n], float32 of
    that shape (None without tokens), entropy [rows], ids and log-probabilities of the n_top best [rows, n_top].  Outputs are allocated where not given."""
    t = _mx_type(logits.dtype)
    torch = _mx.torch
    if logits.dim() != 2:
        _mx_refuse("logits must be [rows, vocab]")
    rows, vocab = logits.shape
    ld, step = logits.stride()
    if vocab > 0x7fffffff or rows > 0x7fffffff or step != 1 and vocab > 1 or ld < vocab and rows > 1:
        _mx_refuse("logits must have contiguous rows that do not overlap")
    if n_top < 0 or n_top > min(LOGPROBS_TOP, vocab):
        _mx_refuse("n_top must be at most %d and the vocabulary" % LOGPROBS_TOP)
    n_tokens = tp = lp = 0
    tensors = [logits]                                     # (what is allocated here needs no look)
    with torch.cuda.stream(stream) if stream is not None else _AS_IT_IS:
        new, f32 = logits.new_empty, torch.float32
        if tokens is not None:
            n_tokens = 1 if tokens.dim() == 1 else tokens.shape[1] if tokens.dim() == 2 else _mx_refuse("tokens must be [rows] or [rows, n]")
            tp = _ints(tokens, (rows,) if tokens.dim() == 1 else (rows, n_tokens), "tokens")
            tensors.append(tokens)
            if logp is None:
                logp = new(tokens.shape, dtype=f32)
                lp = logp.data_ptr()
            else:
                lp = _floats(logp, tokens.shape, "logp")
                tensors.append(logp)
        if entropy is None:
            entropy = new((rows,), dtype=f32)
            ep = entropy.data_ptr()
        else:
            ep = _floats(entropy, (rows,), "entropy")
            tensors.append(entropy)
        if top_ids is None:
            top_ids = new((rows, n_top), dtype=torch.int32)
            ip = top_ids.data_ptr()
        else:
            ip = _ints(top_ids, (rows, n_top), "top_ids")
            tensors.append(top_ids)
        if top_logp is None:
            top_logp = new((rows, n_top), dtype=f32)
            op = top_logp.data_ptr()
        else:
            op = _floats(top_logp, (rows, n_top), "top_logp")
            tensors.append(top_logp)
    if scratch is None:
        scratch = logprobs_scratch(rows, vocab, n_top, logits.device, stream)
    elif not scratch.is_contiguous():
        _mx_refuse("scratch must be contiguous")
    tensors.append(scratch)
    _mx_call(_mx.lib.poss_logprobs, stream, tensors, t, logits.data_ptr(), ld if rows > 1 else vocab, rows, vocab, temperature, tp, n_tokens,
             lp, ep, n_top, ip, op, scratch.data_ptr(), scratch.nbytes)
    return logp, entropy, top_ids, top_logp
