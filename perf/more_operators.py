"""Operators for several continuations of one observation, as cases that can be timed and compared: each in its plain form and as the
library's call.

A case is a dict of plain values with a "kind":

  decode   one new token per sequence, groups of `width` sequences behind one prefix each: rotation, append to a cache held in 8 bits and
           attention over the group's prefix (such a cache, too) and the sequence's own positions
  prompt   the same for a ragged batch of new rows, causal among the own positions
  beam     the best continuations of `beams` beams over the vocabulary, from logits and the beams' scores
  reorder  the sequences of a cache take over what their parents hold, in place

`own` selects between the two: elementary torch operations in binary32 (binary64 where a border is near), or the library.
"""
import math
import random

import torch

own = False

F16, F32, F64, U8, I8, I32, I64 = torch.float16, torch.float32, torch.float64, torch.uint8, torch.int8, torch.int32, torch.int64
DEV = "cuda"
BASE = 10000.0
BLOCK = 64                       # tokens of a head that share a scale in the cache


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # four action samples of one observation (256 visual and 20 text tokens) in a model of 32 heads, a few tokens in: latency
        dict(name="decode_4_276", kind="decode", groups=1, width=4, heads=32, kv_heads=32, d=128, prefix=276, past=6),
        # a serving batch: four uneven observations, sixteen continuations each, four query heads to a key head
        dict(name="decode_4x16", kind="decode", groups=4, width=16, heads=32, kv_heads=8, d=128, prefix=4000, past=200),
        # many continuations of one very long history
        dict(name="decode_32_100k", kind="decode", groups=1, width=32, heads=32, kv_heads=8, d=128, prefix=100003, past=1000),
        # uneven instructions behind one pruned observation, heads of 64
        dict(name="prompt_8_148", kind="prompt", groups=1, width=8, heads=12, kv_heads=12, d=64, prefix=148, past=0, new=20),
        # three groups of uneven further rows behind uneven own positions, in the middle of blocks
        dict(name="prompt_3x4_ragged", kind="prompt", groups=3, width=4, heads=32, kv_heads=8, d=128, prefix=2000, past=150, new=333),
        # long documents behind a long common one: bound by the matrix cores
        dict(name="prompt_2x2_6000", kind="prompt", groups=2, width=2, heads=32, kv_heads=8, d=128, prefix=6000, past=0, new=900),
        # four beams of one observation over the workload's vocabulary
        dict(name="beam_4_32000", kind="beam", batch=1, beams=4, vocab=32000, k=4, ends=False),
        # an odd vocabulary, some beams finished, twice as many candidates as beams
        dict(name="beam_3x5_odd", kind="beam", batch=3, beams=5, vocab=1003, k=10, ends=True),
        # a serving batch over a large vocabulary, some beams finished
        dict(name="beam_16x8_128k", kind="beam", batch=16, beams=8, vocab=128001, k=16, ends=True),
        # four beams with the tokens of an action each, 32 key heads
        dict(name="reorder_4_short", kind="reorder", groups=1, width=4, kv_heads=32, d=128, past=70),
        # a serving batch of uneven continuations
        dict(name="reorder_8x5_uneven", kind="reorder", groups=8, width=5, kv_heads=8, d=64, past=301),
        # long continuations: bound by memory
        dict(name="reorder_4x16_long", kind="reorder", groups=4, width=16, kv_heads=8, d=128, past=2000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("decode", "prompt", "beam", "reorder"))
    while True:
        if kind == "beam":
            beams = _log(rng, 1, 32)
            c = dict(kind=kind, batch=_log(rng, 1, 64), beams=beams, vocab=_log(rng, 100, 128001), k=min(64, beams * rng.choice((1, 2))),
                     ends=rng.random() < 0.5)
            if c["batch"] * beams * c["vocab"] <= 16 * 8 * 128001:
                return c
            continue
        kv = rng.choice((1, 2, 4, 8, 12, 32))
        c = dict(kind=kind, groups=_log(rng, 1, 16), width=_log(rng, 1, 64), heads=kv * rng.choice((1, 1, 2, 4, 8)), kv_heads=kv,
                 d=rng.choice((64, 128, 128)), prefix=_log(rng, 1, 100000), past=rng.choice((0, _log(rng, 1, 2000))), new=_log(rng, 2, 1000))
        rows, wide = c["groups"] * c["width"], c["heads"] * c["d"]
        if c["heads"] > 64 or rows > 256:
            continue
        if kind == "decode":
            del c["new"]
            if rows * wide * c["prefix"] <= 32 * 32 * 128 * 100003 and c["groups"] * kv * c["prefix"] * c["d"] <= 8 * 100003 * 128 \
                    and rows * kv * c["past"] * c["d"] <= 64 * 8 * 2000 * 128 and rows * c["heads"] * (c["prefix"] + c["past"]) <= 1 << 28:
                return c
        elif kind == "prompt":
            new = rows * c["new"]
            if new <= 20000 and new * wide * (c["prefix"] + c["past"] + c["new"] // 2) <= 4 * 900 * 32 * 128 * 6000 \
                    and rows * kv * c["past"] * c["d"] <= 64 * 8 * 2000 * 128 and new * c["heads"] * (c["prefix"] + c["past"] + c["new"]) <= 1 << 30:
                return c
        else:
            c = {k: c[k] for k in ("kind", "groups", "width", "kv_heads", "d", "past")}
            if c["width"] > 1 and c["past"] > 0 and rows * kv * c["past"] * c["d"] <= 64 * 8 * 2000 * 128:
                return c


# ---------------------------------------------------------------- inputs (made from the seed alone; lengths and parents are the case's)

def _gen(seed, key):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1013 + key)
    return g


def _lengths(count, most, key, least=0):
    """One of `count` has the length `most`, the others lengths between an eighth of it and all of it."""
    rng = random.Random(key)
    n = [max(least, int(round(most * (0.125 + 0.875 * rng.random())))) for _ in range(count)]
    n[0] = most
    return n


def _sizes(case):
    """(prefix lengths of the groups, own lengths and new rows of the sequences)"""
    count = case["groups"] * case["width"]
    return (_lengths(case["groups"], case["prefix"], 1, 1), _lengths(count, case["past"], 2),
            _lengths(count, case["new"], 3, 1) if case["kind"] == "prompt" else [1] * count)


def _parents(case):
    """Parents as a selection leaves them: the leading beams more often, some take over themselves; one in sixteen has none."""
    rng = random.Random(4)
    return [[-1 if rng.random() < 1 / 16 else int(case["width"] * rng.random() ** 1.5) for _ in range(case["width"])] for _ in range(case["groups"])]


def _history(seed, key, batch, kv_heads, d, capacity):
    """Keys (as rotated) and values in half precision: [batch, kv_heads, capacity, d] each.  A few channels of the keys are large."""
    g = _gen(seed, key)
    k, v = (torch.randn((batch, kv_heads, capacity, d), generator=g, device=DEV, dtype=F16) for _ in range(2))
    k[..., :4] *= 3.0
    return k, v


def _capacity(positions):
    return max(1, -(-positions // BLOCK)) * BLOCK


def _attention_inputs(case, seed):
    """Prefix and own keys and values, fused q|k|v rows in half precision."""
    lengths, past, new = _sizes(case)
    longest = max(p + n for p, n in zip(past, new))
    prefix = _history(seed, 1, case["groups"], case["kv_heads"], case["d"], _capacity(max(lengths)))
    mine = _history(seed, 2, case["groups"] * case["width"], case["kv_heads"], case["d"], _capacity(longest))
    rows = torch.randn((sum(new), (case["heads"] + 2 * case["kv_heads"]) * case["d"]), generator=_gen(seed, 3), device=DEV, dtype=F16)
    rows[:, :case["heads"] * case["d"]] *= 1.5
    return prefix, mine, rows


def _beam_inputs(case, seed):
    """Logits with a few leading tokens and a long tail, the beams' scores (sums of logarithms, the best first), which of them have finished."""
    g = _gen(seed, 4)
    shape = (case["batch"] * case["beams"], case["vocab"])
    logits = torch.randn(shape, generator=g, device=DEV) * 2.0
    logits += 4.0 * torch.randn(shape, generator=g, device=DEV).clamp_min(2.0) - 8.0
    r = torch.rand((2, case["batch"], case["beams"]), generator=g, device=DEV)
    done = (r[1] < 0.2).to(I32) if case["ends"] else None
    return logits.to(F16), -(r[0] * 6.0).cumsum(-1), done


# ---------------------------------------------------------------- the cache in plain tensors, in the order of the library's

def _key_codes(codes, d):
    """The keys' codes [batch, heads, blocks, 64 d] as a view [batch, heads, blocks, 64 (4 of 16), d (d / 64, 4, 16)]."""
    return codes.unflatten(-1, (4, d // 64, 4, 16, 16)).permute(0, 1, 2, 3, 6, 4, 5, 7)


def _value_codes(codes, d):
    """The values' codes as a view [batch, heads, blocks, 64 (2, 2, 4, 4), d (d / 16, 16)]."""
    return codes.unflatten(-1, (d // 16, 4, 16, 2, 2, 4)).permute(0, 1, 2, 6, 7, 4, 8, 3, 5)


def _block_codes(x):
    """x [..., 64, d] in half precision -> codes (127 x / amax to the nearest, halfway cases to even), scales binary32 [...]."""
    amax = x.to(F32).abs().amax((-1, -2))
    safe = amax.where(amax > 0, torch.ones_like(amax))
    return torch.round(127.0 * x.to(F32) / safe[..., None, None]).to(I8), amax / 127.0


class _Plain:
    """Codes int8 [batch, heads, blocks, 2, 64 d], scales [batch, heads, blocks, 2], unfinished blocks [batch, heads, 2, 64, d]."""

    def __init__(self, batch, capacity, heads, d):
        blocks = capacity // BLOCK
        self.d, self.capacity = d, capacity
        self.codes = torch.zeros((batch, heads, blocks, 2, BLOCK * d), dtype=I8, device=DEV)
        self.scales = torch.zeros((batch, heads, blocks, 2), dtype=F32, device=DEV)
        self.tail = torch.zeros((batch, heads, 2, BLOCK, d), dtype=F16, device=DEV)

    def view(self, i):
        return (_key_codes, _value_codes)[i](self.codes[:, :, :, i], self.d)

    def fill(self, k, v, lengths):
        for b, length in enumerate(lengths):
            full, rest = length // BLOCK, length % BLOCK
            for i, x in enumerate((k, v)):
                if full:
                    c, self.scales[b, :, :full, i] = _block_codes(x[b, :, :full * BLOCK].unflatten(1, (full, BLOCK)))
                    view = self.view(i)[b, :, :full]
                    view.copy_(c.reshape(view.shape))
                self.tail[b, :, i, :rest] = x[b, :, full * BLOCK:length]
        return self

    def values(self, n):
        """Keys and values of all positions in binary32, zeros where there are none: [batch, heads, capacity, d] each; n: lengths."""
        batch, heads = self.codes.shape[:2]
        position = torch.arange(self.capacity, device=DEV)[None]
        in_tail, none = ((x)[:, None, :, None] for x in (position >= (n // BLOCK * BLOCK)[:, None], position >= n[:, None]))
        row = (position % BLOCK)[:, None, :, None].expand(batch, heads, -1, self.d)
        out = []
        for i in range(2):
            held = self.view(i).to(F32).reshape(batch, heads, -1, BLOCK, self.d) * self.scales[..., i, None, None]
            out.append(torch.where(in_tail, torch.gather(self.tail[:, :, i], 2, row).to(F32), held.flatten(2, 3)).masked_fill(none, 0.0))
        return out

    def append(self, k, v, first, n):
        """Rows k, v [batch, heads, new, d] of positions first[b] ... first[b] + n[b] - 1: blocks from the first row's on are put together
        from the unfinished block and the new rows; finished ones become codes."""
        batch, heads, new, d = k.shape
        touched = (new + 2 * BLOCK - 2) // BLOCK
        slot = torch.arange(touched * BLOCK, device=DEV)
        begin = first // BLOCK * BLOCK
        at = slot[None] + (begin - first)[:, None]                               # row of k, v that belongs in the slot; < 0: is there
        is_new = (at >= 0) & (at < n[:, None])
        index = at.clamp(0, new - 1)[:, None, :, None].expand(batch, heads, -1, d)
        number = (begin // BLOCK)[:, None] + torch.arange(touched, device=DEV)
        end = first + n
        which, j = ((number + 1) * BLOCK <= end[:, None]).nonzero(as_tuple=True)
        last = (end // BLOCK - begin // BLOCK).clamp_max(touched - 1)
        rows = torch.arange(BLOCK, device=DEV)
        pick = last[:, None] * BLOCK + rows[None]
        fresh = torch.gather(is_new, 1, pick) & (rows[None] < (end % BLOCK)[:, None])
        picked = pick[:, None, :, None].expand(batch, heads, BLOCK, d)
        for i, x in enumerate((k, v)):
            have = torch.zeros((batch, heads, touched * BLOCK, d), dtype=F16, device=DEV)
            have[:, :, slot < BLOCK] = self.tail[:, :, i]
            have = torch.where(is_new[:, None, :, None], torch.gather(x, 2, index), have)
            c, sc = _block_codes(have.unflatten(2, (touched, BLOCK)))
            view = self.view(i)
            view[which, :, number[which, j]] = c[which, :, j].reshape(-1, *view.shape[1:2], *view.shape[3:])
            self.scales[which, :, number[which, j], i] = sc[which, :, j]
            self.tail[:, :, i] = torch.where(fresh[:, None, :, None], torch.gather(have, 2, picked), self.tail[:, :, i])


# ---------------------------------------------------------------- the plain forms

def _rotate(x, pos):
    """x [..., d] at positions pos [...] (broadcast over the heads): half-split pairs, angles and products in binary64."""
    half = x.shape[-1] // 2
    a = pos.to(F64).unsqueeze(-1) * BASE ** (-2.0 * torch.arange(half, device=DEV, dtype=F64) / x.shape[-1])
    lo, hi = x[..., :half].to(F64), x[..., half:].to(F64)
    return torch.cat((lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()), -1).to(F32).to(F16)


def _run_attention(s):
    heads, kv, d, groups = s["heads"], s["kv_heads"], s["d"], s["groups"]
    starts, past, length = s["starts"].long(), s["past"].long(), s["length"].long()
    n = starts[1:] - starts[:-1]
    batch, new, mine, prefix = n.numel(), s["max_new"], s["cache"], s["prefix"]
    inside = torch.arange(new, device=DEV)[None] < n[:, None]
    at = (starts[:-1, None] + torch.arange(new, device=DEV)[None]).masked_fill(~inside, 0)
    pos = s["pos"].long()[at][:, None]
    q, k, v = (y.reshape(batch, new, -1, d).transpose(1, 2) for y in s["qkv"][at].split((heads * d, kv * d, kv * d), 2))
    mine.append(_rotate(k, pos), v, past, n)
    q = _rotate(q, pos).to(F32)
    kp, vp = prefix.values(length)
    ko, vo = mine.values(past + n)
    # the group's rows against its prefix, the sequences' against their own positions
    share = batch // groups * (heads // kv) * new
    by_group = q.reshape(groups, batch // groups, kv, -1, d).transpose(1, 2).reshape(groups, kv, share, d)
    sp = (by_group @ kp.transpose(-1, -2)).reshape(groups, kv, batch // groups, -1, prefix.capacity).transpose(1, 2).reshape(batch, heads, new, -1)
    so = (q.reshape(batch, kv, -1, d) @ ko.transpose(-1, -2)).reshape(batch, heads, new, -1)
    hidden = torch.arange(prefix.capacity, device=DEV)[None] >= length[:, None]
    sp = sp.masked_fill(hidden.repeat_interleave(batch // groups, 0)[:, None, None], -math.inf)
    sees = past[:, None] + torch.arange(new, device=DEV)
    so = so.masked_fill((torch.arange(mine.capacity, device=DEV) > sees[:, :, None])[:, None], -math.inf)
    top = torch.maximum(sp.amax(-1, keepdim=True), so.amax(-1, keepdim=True))
    sp, so = (torch.exp((x - top) / math.sqrt(d)) for x in (sp, so))
    total = sp.sum(-1, keepdim=True) + so.sum(-1, keepdim=True)
    sp = sp.reshape(groups, batch // groups, kv, -1, prefix.capacity).transpose(1, 2).reshape(groups, kv, share, -1)
    o = (sp @ vp).reshape(groups, kv, batch // groups, -1, d).transpose(1, 2).reshape(batch, heads, new, d)
    o = (o + (so.reshape(batch, kv, -1, mine.capacity) @ vo).reshape(batch, heads, new, d)) / total
    return o.to(F16).transpose(1, 2).reshape(batch, new, heads * d)[inside], mine.codes, mine.scales, mine.tail


def _run_beam(s):
    logits, k = s["logits"].to(F64), s["k"]
    batch, beams = s["scores"].shape
    vocab = logits.shape[1]
    top = logits.amax(-1, keepdim=True)
    logp = logits - (top + torch.log(torch.exp(logits - top).sum(-1, keepdim=True)))
    total = s["scores"].to(F64)[:, :, None] + logp.reshape(batch, beams, vocab)
    if s["done"] is not None:
        ended = s["done"] != 0
        total = total.masked_fill(ended[:, :, None], -math.inf)
        total[:, :, s["eos"]] = torch.where(ended, s["scores"].to(F64), total[:, :, s["eos"]])
    best = torch.sort(total.flatten(1), dim=-1, descending=True, stable=True)        # equal ones: the lowest beam, then token
    at = best.indices[:, :k]
    parent, token = (at // vocab).to(I32), (at % vocab).to(I32)
    done = (token == s["eos"]).to(I32)
    if s["done"] is not None:
        done |= torch.gather(s["done"], 1, parent.long())
    return parent, token, best.values[:, :k].to(F32), done


def _run_reorder(s):
    """Whole blocks and rows of the unfinished one below the parent's length; everything else stays as it was."""
    c, lengths, width = s["cache"], s["lengths"].long(), s["width"]
    batch, blocks = lengths.numel(), c.codes.shape[2]
    p = s["parents"].long()
    me = torch.arange(batch, device=DEV)
    of = (me // width * width + p.flatten()).where(p.flatten() >= 0, me)
    n = lengths[of]
    full = (torch.arange(blocks, device=DEV)[None] < (n // BLOCK)[:, None])[:, None, :, None]
    rest = (torch.arange(BLOCK, device=DEV)[None] < (n % BLOCK)[:, None])[:, None, None, :, None]
    c.codes.copy_(torch.where(full[..., None], c.codes[of], c.codes))
    c.scales.copy_(torch.where(full, c.scales[of], c.scales))
    c.tail.copy_(torch.where(rest, c.tail[of], c.tail))
    return c.codes, c.scales, c.tail, n.to(I32)


# ---------------------------------------------------------------- states

def _ints(x):
    return torch.tensor(x, dtype=I32, device=DEV)


def _held(k, v, lengths):
    """A cache that holds these keys and values: the library's as a program would have left it (appended at position 0, whose rotation
    changes nothing), or a plain one."""
    batch, kv, capacity, d = k.shape
    if not own:
        return _Plain(batch, capacity, kv, d).fill(k, v, lengths)
    from paper_2509_09090_amd import binding as B
    cache = B.Cache8(batch, capacity, kv, d)
    if max(lengths) > 0:
        n = _ints(lengths)
        inside = torch.arange(capacity, device=DEV)[None] < n[:, None]
        rows = torch.cat([x.transpose(1, 2)[inside].reshape(-1, kv * d) for x in (k, k, v)], 1)
        starts = torch.cat((torch.zeros((1,), dtype=I32, device=DEV), n.cumsum(0).to(I32)))
        B.sqap_cache8_append(rows, starts, torch.zeros((rows.shape[0],), dtype=I32, device=DEV), torch.zeros_like(n), cache, kv, max(lengths))
    return cache


def prepare(case, seed):
    kind = case["kind"]
    if kind == "beam":
        logits, scores, done = _beam_inputs(case, seed)
        s = dict(kind=kind, logits=logits, scores=scores, done=done, eos=2, k=case["k"])
        if own:
            from paper_2509_09090_amd import binding as B
            s["out"] = [torch.empty((case["batch"], case["k"]), dtype=t, device=DEV) for t in (I32, I32, F32, I32)]
            s["ws"] = torch.empty((B.sqap_beam_workspace_bytes(case["batch"], case["beams"], case["vocab"], case["k"]),), dtype=U8, device=DEV)
        return s
    if kind == "reorder":
        lengths = _lengths(case["groups"] * case["width"], case["past"], 2)
        k, v = _history(seed, 2, case["groups"] * case["width"], case["kv_heads"], case["d"], _capacity(max(lengths)))
        return dict(kind=kind, width=case["width"], cache=_held(k, v, lengths), parents=_ints(_parents(case)), lengths=_ints(lengths),
                    longest=max(lengths), after=torch.empty((len(lengths),), dtype=I32, device=DEV))
    lengths, past, new = _sizes(case)
    prefix, mine, rows = _attention_inputs(case, seed)
    starts = [sum(new[:b]) for b in range(len(new) + 1)]
    pos = [lengths[b // case["width"]] + past[b] + j for b in range(len(new)) for j in range(new[b])]
    s = dict(kind=kind, heads=case["heads"], kv_heads=case["kv_heads"], d=case["d"], groups=case["groups"], max_new=max(new), qkv=rows,
             length=_ints(lengths), past=_ints(past), starts=_ints(starts), pos=_ints(pos), prefix=_held(*prefix, lengths), cache=_held(*mine, past))
    if own:
        from paper_2509_09090_amd import binding as B
        s["longest"], s["longest_prefix"] = max(p + n for p, n in zip(past, new)), max(lengths)
        s["o"] = torch.empty((len(pos), case["heads"] * case["d"]), dtype=F16, device=DEV)
        s["q"] = torch.empty_like(s["o"])
        s["ws"] = torch.zeros((B.sqap_cache8_shared_workspace_bytes(len(past), case["groups"], case["heads"], case["kv_heads"], case["d"], len(pos),
                                                                    s["max_new"], s["longest"], s["longest_prefix"]),), dtype=U8, device=DEV)
    return s


def run(s):
    kind = s["kind"]
    if not own:
        return {"decode": _run_attention, "prompt": _run_attention, "beam": _run_beam, "reorder": _run_reorder}[kind](s)
    from paper_2509_09090_amd import binding as B
    if kind == "beam":
        B.sqap_beam_select(s["logits"], s["scores"], s["done"], s["eos"], *s["out"], s["ws"])
        return tuple(s["out"])
    cache = s["cache"]
    if kind == "reorder":
        B.sqap_cache8_reorder(cache, s["parents"], s["lengths"], s["longest"], s["after"])
        return cache.codes, cache.scales, cache.tail, s["after"]
    if kind == "decode":
        B.sqap_cache8_shared_decode_attention(s["qkv"], s["pos"], s["past"], cache, s["prefix"], s["length"], s["heads"], s["o"], s["ws"],
                                              s["longest"], s["longest_prefix"])
    else:
        B.sqap_cache8_append(s["qkv"], s["starts"], s["pos"], s["past"], cache, s["heads"], s["max_new"], Q_out=s["q"])
        B.sqap_cache8_shared_attention(s["q"], s["starts"], s["past"], cache, s["prefix"], s["length"], s["heads"], s["max_new"], s["o"], s["ws"],
                                       s["longest_prefix"])
    return s["o"], cache.codes, cache.scales, cache.tail


def work(case):
    """Bytes: every input read once, every output written once; operations of the products (a multiply-add is two) or, for a selection,
    of the exponentials and comparisons."""
    kind = case["kind"]
    if kind == "beam":
        rows = case["batch"] * case["beams"]
        return {"bytes": rows * (2 * case["vocab"] + 8) + 16 * case["batch"] * case["k"], "flops": 4 * rows * case["vocab"]}
    kv, d = case["kv_heads"], case["d"]

    def held(n):                                                                 # bytes of n positions
        return kv * (n // BLOCK * 2 * (BLOCK * d + 4) + n % BLOCK * 4 * d)
    if kind == "reorder":
        n, moved = _lengths(case["groups"] * case["width"], case["past"], 2), 0
        for g, parents in enumerate(_parents(case)):
            took = [p for i, p in enumerate(parents) if p >= 0 and p != i]
            moved += sum(held(n[g * case["width"] + p]) for p in took) + sum(held(n[g * case["width"] + p]) for p in set(took))
        return {"bytes": moved + 12 * len(n), "flops": 0}
    lengths, past, new = _sizes(case)
    h, rows = case["heads"], sum(new)
    pairs = sum(n * (lengths[b // case["width"]] + past[b] + (n + 1) / 2) for b, n in enumerate(new))
    rows_bytes = rows * d * 2 * (h + 2 * kv) + rows * d * 2 * h + sum(held(p + n) - held(p) for p, n in zip(past, new))
    return {"bytes": sum(map(held, lengths)) + sum(map(held, past)) + rows_bytes, "flops": 4 * pairs * h * d}


# ---------------------------------------------------------------- 64 bits, from the definitions

def _exact_held(x, length):
    """Rows x [heads, length, d] as a cache holds them: whole blocks of 64 in steps of their scale, the rest as they are."""
    x = x.double().clone()
    for begin in range(0, length // BLOCK * BLOCK, BLOCK * 256):
        end = min(begin + BLOCK * 256, length // BLOCK * BLOCK)
        y = x[:, begin:end].reshape(x.shape[0], -1, BLOCK * x.shape[2])
        top = y.abs().max(-1, keepdim=True).values
        x[:, begin:end] = (torch.round(y * 127.0 / top.clamp_min(1e-300)) * (top.float() / 127.0).double()).reshape(x.shape[0], end - begin, -1)
    return x


def _exact_turned(x, pos):
    """x [rows, heads, d] turned by its row's angles, as half-precision values in binary64."""
    d = x.shape[-1]
    z = torch.complex(x[..., : d // 2].double(), x[..., d // 2:].double())
    angle = pos.double()[:, None, None] * torch.exp(-2.0 * torch.arange(d // 2, dtype=F64, device=DEV) / d * math.log(BASE))
    z = z * torch.polar(torch.ones_like(angle), angle)
    return torch.cat((z.real, z.imag), -1).float().half().double()


def exact(case, seed):
    kind = case["kind"]
    if kind == "reorder":
        return None                                                              # copies
    if kind == "beam":
        logits, scores, done = _beam_inputs(case, seed)
        out = []
        for e in range(case["batch"]):
            rows = torch.log_softmax(logits[e * case["beams"]:(e + 1) * case["beams"]].double(), -1) + scores[e].double()[:, None]
            if done is not None:
                rows = torch.cat([scores[e, i].double()[None] if done[e, i] else rows[i] for i in range(case["beams"])])
            out.append(rows.flatten().topk(case["k"]).values)
        return None, None, torch.stack(out), None
    heads, kv, d = case["heads"], case["kv_heads"], case["d"]
    if sum(_sizes(case)[2]) * heads > 1 << 18:
        return None
    lengths, past, new = _sizes(case)
    prefix, mine, rows = _attention_inputs(case, seed)
    out, at = [], 0
    for b, (p, n) in enumerate(zip(past, new)):
        g = b // case["width"]
        if b % case["width"] == 0:
            front = [_exact_held(x[g, :, :lengths[g]], lengths[g]) for x in prefix]
        x = rows[at:at + n].reshape(n, -1, d)
        at += n
        pos = lengths[g] + p + torch.arange(n, device=DEV)
        turned = _exact_turned(x[:, :heads + kv], pos)
        keys = _exact_held(torch.cat((mine[0][b, :, :p].double(), turned[:, heads:].transpose(0, 1)), 1), p + n)
        values = _exact_held(torch.cat((mine[1][b, :, :p].double(), x[:, heads + kv:].double().transpose(0, 1)), 1), p + n)
        hidden = torch.arange(p + n, device=DEV)[None] > p + torch.arange(n, device=DEV)[:, None]
        o = torch.empty((n, heads, d), dtype=F64, device=DEV)
        for h in range(heads):
            j = h * kv // heads
            score = turned[:, h] @ keys[j].T
            score = torch.cat((turned[:, h] @ front[0][j].T, score.masked_fill(hidden, -math.inf)), 1)
            weight = torch.softmax(score * d ** -0.5, -1)
            o[:, h] = weight[:, :lengths[g]] @ front[1][j] + weight[:, lengths[g]:] @ values[j]
        out.append(o.reshape(n, heads * d))
    return torch.cat(out), None, None, None
