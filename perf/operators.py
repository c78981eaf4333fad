"""Operators of a decode loop in few bits, as cases that can be timed and compared: each in its plain form and as the library's call.

A case is a dict of plain values with a "kind":

  mx       activation rows quantized to microscaled 4-bit floating point (32 channels share a power of two) and multiplied with a
           weight held that way
  decode   one new token per sequence: rotation, append to a cache held in 8 bits (64 tokens of a head share a scale; the
           unfinished block stays in half precision) and attention over it
  prefill  a ragged batch of new rows: rotation, append to such a cache, causal attention over what it then holds
  sample   next tokens from logits: temperature, top-k, top-p, min-p, given uniform numbers

`own` selects between the two: elementary torch operations in binary32 (binary64 where a border is near), or the library.
"""
import math

import torch

own = False

F16, F32, F64, U8, I32, I64 = torch.float16, torch.float32, torch.float64, torch.uint8, torch.int32, torch.int64
DEV = "cuda"
BASE = 10000.0
BLOCK = 64                       # tokens of a head that share a scale in the cache
OUTLIER_SCALE, OUTLIER_FRAC = 30.0, 0.01
WEIGHT_STD = 0.02


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # one token through the output projection of a 4096 wide layer: two small launches, latency
        dict(name="mx_1_4096", kind="mx", m=1, n=4096, k=4096, gather=False),
        # the vocabulary head for a decode batch of 8: bound by streaming the weight
        dict(name="mx_head_8", kind="mx", m=8, n=32000, k=4096, gather=False),
        # the rows that survive pruning of one observation, gathered, through gate|up
        dict(name="mx_gate_up_148", kind="mx", m=148, n=22016, k=4096, gather=True),
        # uneven everything: rows, channels that are no multiple of 16, a reduction that is no multiple of 128
        dict(name="mx_ragged_333", kind="mx", m=333, n=1001, k=2848, gather=True),
        # sixteen observations through gate|up: bound by the matrix cores
        dict(name="mx_gate_up_2368", kind="mx", m=2368, n=22016, k=4096, gather=False),
        # one sequence of a 32-head model behind a history of several observations
        dict(name="decode_1_1500", kind="decode", batch=1, heads=32, kv_heads=32, d=128, longest=1500),
        # a serving batch of uneven histories, four query heads to a key head
        dict(name="decode_16_ragged", kind="decode", batch=16, heads=32, kv_heads=8, d=128, longest=8000),
        # one very long history
        dict(name="decode_1_100k", kind="decode", batch=1, heads=32, kv_heads=8, d=128, longest=100003),
        # the first rows of one sequence: half of the visual tokens and the text
        dict(name="prefill_148", kind="prefill", batch=1, heads=32, kv_heads=32, d=128, new=148, past=0),
        # uneven sequences with a history each, appended to in the middle of a block
        dict(name="prefill_3_ragged", kind="prefill", batch=3, heads=32, kv_heads=8, d=128, new=1500, past=2000),
        # one token of the workload's vocabulary, every filter on
        dict(name="sample_1_32000", kind="sample", batch=1, vocab=32000, filters=True),
        # a serving batch over a large vocabulary, parameters per row, some rows greedy or without a filter
        dict(name="sample_64_128k", kind="sample", batch=64, vocab=128001, filters=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("mx", "decode", "prefill", "sample"))
    if kind == "mx":
        while True:
            c = dict(kind=kind, m=_log(rng, 1, 2400), n=_log(rng, 64, 32000), k=32 * _log(rng, 4, 344), gather=rng.random() < 0.3)
            if c["m"] * c["n"] * c["k"] <= 2368 * 22016 * 4096 and c["n"] * c["k"] <= 32000 * 4096:
                return c
    if kind == "decode":
        while True:
            kv = rng.choice((1, 2, 4, 8, 16, 32))
            c = dict(kind=kind, batch=_log(rng, 1, 32), heads=kv * rng.choice((1, 1, 2, 4, 8)), kv_heads=kv, d=rng.choice((64, 128, 128)),
                     longest=_log(rng, 1, 100000))
            if c["heads"] <= 64 and c["batch"] * c["kv_heads"] * c["longest"] * c["d"] <= 8 * 100003 * 128:
                return c
    if kind == "prefill":
        while True:
            kv = rng.choice((1, 2, 4, 8, 16, 32))
            c = dict(kind=kind, batch=_log(rng, 1, 8), heads=kv * rng.choice((1, 1, 2, 4)), kv_heads=kv, d=rng.choice((64, 128)),
                     new=_log(rng, 2, 2000), past=rng.choice((0, _log(rng, 1, 2000))))
            if c["heads"] <= 32 and c["batch"] * c["heads"] * c["new"] * (c["new"] + c["past"]) * c["d"] <= 3 * 32 * 1500 * 3500 * 128 // 2:
                return c
    return dict(kind=kind, batch=_log(rng, 1, 64), vocab=_log(rng, 100, 128001), filters=rng.random() < 0.8)


# ---------------------------------------------------------------- inputs (made from the seed alone)

def _gen(seed, key):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1009 + key)
    return g


def _mx_inputs(case, seed):
    """Activation rows with a few large channels, the rows of them that survive (or None), and a weight, all in half precision."""
    m, n, k = case["m"], case["n"], case["k"]
    g = _gen(seed, 1)
    total = m + m // 2 + 1 if case["gather"] else m
    x = torch.randn((total, k), generator=g, device=DEV)
    x[:, torch.randperm(k, generator=g, device=DEV)[: max(1, int(round(OUTLIER_FRAC * k)))]] *= OUTLIER_SCALE
    rows = torch.randperm(total, generator=g, device=DEV)[:m].sort().values.to(I32) if case["gather"] else None
    return x.to(F16), rows, (torch.randn((n, k), generator=g, device=DEV) * WEIGHT_STD).to(F16)


def _lengths(case, most, key):
    """One sequence has the length `most`, the others lengths between an eighth of it and all of it; they are the case's."""
    g = _gen(key, 2)
    n = (most * (0.125 + 0.875 * torch.rand((case["batch"],), generator=g, device=DEV, dtype=F64))).round().to(I64)
    n[0] = most
    return n


def _history(case, seed, capacity):
    """Keys (as rotated) and values of the positions so far, in half precision: [batch, kv_heads, capacity, d] each.  A few
    channels of the keys are large, as they are in a model."""
    g = _gen(seed, 3)
    shape = (case["batch"], case["kv_heads"], capacity, case["d"])
    k, v = torch.randn(shape, generator=g, device=DEV, dtype=F16), torch.randn(shape, generator=g, device=DEV, dtype=F16)
    k[..., :4] *= 3.0
    return k, v


def _new_rows(case, seed, rows):
    """Fused q|k|v rows in half precision."""
    g = _gen(seed, 4)
    x = torch.randn((rows, (case["heads"] + 2 * case["kv_heads"]) * case["d"]), generator=g, device=DEV, dtype=F16)
    x[:, :case["heads"] * case["d"]] *= 1.5
    return x


def _sample_inputs(case, seed):
    """Logits with a few leading tokens and a long tail, the rows' parameters and their uniform numbers."""
    g = _gen(seed, 5)
    b, v = case["batch"], case["vocab"]
    logits = torch.randn((b, v), generator=g, device=DEV) * 2.0
    logits += 4.0 * torch.randn((b, v), generator=g, device=DEV).clamp_min(2.0) - 8.0
    r = torch.rand((5, b), generator=g, device=DEV)
    u = torch.rand((b,), generator=g, device=DEV)
    temperature = (0.3 + r[0]).where(r[1] > 0.1, torch.zeros_like(u))
    if not case["filters"]:
        return logits.to(F16), temperature, None, None, None, u
    top_k = (1 + (r[2] * min(v, 200)).to(I32)).where(r[3] > 0.2, torch.zeros((b,), dtype=I32, device=DEV))
    top_p = (0.5 + 0.5 * r[4]).where(r[2] > 0.15, torch.ones_like(u))
    min_p = (0.1 * r[3]).where(r[4] > 0.3, torch.zeros_like(u))
    return logits.to(F16), temperature, top_k, top_p, min_p, u


# ---------------------------------------------------------------- the plain forms

_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mx_scale_and_level(x):
    """Blocks of 32 channels: the exponent of the power of two that they share, [..., K / 32], and the signed values of the
    elements in units of it, [..., K / 32, 32]."""
    b = x.to(F32).unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1)
    e = torch.frexp(amax).exponent - 3                       # amax = f 2^E with f in [1/2, 1): floor(log2 amax) = E - 1
    e = e.where(amax > 0, torch.zeros_like(e))
    y = torch.ldexp(b.abs(), -e.unsqueeze(-1))
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    return e, torch.copysign((torch.round(y / step) * step).clamp_max(6.0), b)


def _mx_pack(e, level):
    """The same as codes: two to a byte, the first in the low four bits, and the exponents' bytes."""
    magnitude = torch.bucketize(level.abs(), torch.tensor(_LEVELS, device=DEV)).to(U8)
    code = (magnitude | (torch.signbit(level).to(U8) << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(U8)


def _mx_unpack(code, scale):
    """Values of packed codes, in binary32: [rows, K]."""
    table = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), device=DEV)
    level = torch.stack((table[(code & 15).long()], table[(code >> 4).long()]), -1).flatten(-2)
    return torch.ldexp(level.unflatten(-1, (-1, 32)), scale.to(I32).unsqueeze(-1) - 127).flatten(-2)


def _run_mx(s):
    x = s["x"] if s["rows"] is None else s["x"][s["rows"].long()]
    e, level = _mx_scale_and_level(x)
    return (torch.ldexp(level, e.unsqueeze(-1)).flatten(-2) @ _mx_unpack(s["wq"], s["ws"]).T).to(F16)


def _rotate(x, pos, base=BASE):
    """x [..., d] at positions pos [...] (broadcast over the heads): half-split pairs, angles and products in binary64."""
    half = x.shape[-1] // 2
    a = pos.to(F64).unsqueeze(-1) * base ** (-2.0 * torch.arange(half, device=DEV, dtype=F64) / x.shape[-1])
    lo, hi = x[..., :half].to(F64), x[..., half:].to(F64)
    return torch.cat((lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()), -1).to(F32).to(F16)


def _block_codes(x):
    """x [..., 64, d] in half precision -> codes int8 (127 x / amax to the nearest, halfway cases to even), scales binary32 [...]."""
    amax = x.to(F32).abs().amax((-1, -2))
    safe = amax.where(amax > 0, torch.ones_like(amax))
    return torch.round(127.0 * x.to(F32) / safe[..., None, None]).to(torch.int8), amax / 127.0


def _fill_plain(k, v, n, capacity):
    """A cache of n[b] positions of sequence b in plain tensors: codes [2, batch, kv_heads, blocks, 64, d], scales
    [batch, kv_heads, blocks, 2] of the finished blocks, rows of the unfinished one [batch, kv_heads, 2, 64, d]."""
    batch, heads, _, d = k.shape
    blocks = capacity // BLOCK
    codes = torch.zeros((2, batch, heads, blocks, BLOCK, d), dtype=torch.int8, device=DEV)
    scales = torch.zeros((batch, heads, blocks, 2), dtype=F32, device=DEV)
    tail = torch.zeros((batch, heads, 2, BLOCK, d), dtype=F16, device=DEV)
    for b, length in enumerate(n.tolist()):
        full, rest = length // BLOCK, length % BLOCK
        for i, x in enumerate((k, v)):
            if full:
                codes[i, b, :, :full], scales[b, :, :full, i] = _block_codes(x[b, :, :full * BLOCK].unflatten(1, (full, BLOCK)))
            tail[b, :, i, :rest] = x[b, :, full * BLOCK:length]
    return codes, scales, tail


def _append_plain(s, k, v, first, n):
    """Rows k, v [batch, kv_heads, new, d] of positions first[b] ... first[b] + n[b] - 1: the cache's blocks from the first row's
    on are put together from the unfinished block and the new rows; finished ones become codes."""
    codes, scales, tail = s["codes"], s["scales"], s["tail"]
    batch, heads, new, d = k.shape
    touched = (new + 2 * BLOCK - 2) // BLOCK                                     # blocks that may be touched
    slot = torch.arange(touched * BLOCK, device=DEV)
    begin = first // BLOCK * BLOCK
    at = slot[None] + (begin - first)[:, None]                                   # row of k, v that belongs in the slot; < 0: is there
    is_new = (at >= 0) & (at < n[:, None])
    index = at.clamp(0, new - 1)[:, None, :, None].expand(batch, heads, -1, d)
    old = slot < BLOCK
    blocks = []
    for i, x in enumerate((k, v)):
        have = torch.zeros((batch, heads, touched * BLOCK, d), dtype=F16, device=DEV)
        have[:, :, old] = tail[:, :, i]
        blocks.append(torch.where(is_new[:, None, :, None], torch.gather(x, 2, index), have).unflatten(2, (touched, BLOCK)))
    number = (begin // BLOCK)[:, None] + torch.arange(touched, device=DEV)       # block of the cache
    end = first + n
    done = (number + 1) * BLOCK <= end[:, None]
    which, j = done.nonzero(as_tuple=True)
    for i in range(2):
        c, sc = _block_codes(blocks[i])
        codes[i, which, :, number[which, j]] = c[which, :, j]
        scales[which, :, number[which, j], i] = sc[which, :, j]
    # the unfinished block's rows that are new
    last = (end // BLOCK - begin // BLOCK).clamp_max(touched - 1)
    rows = torch.arange(BLOCK, device=DEV)
    pick = last[:, None] * BLOCK + rows[None]
    fresh = torch.gather(is_new, 1, pick) & (rows[None] < (end % BLOCK)[:, None])
    index = pick[:, None, :, None].expand(batch, heads, BLOCK, d)
    for i in range(2):
        tail[:, :, i] = torch.where(fresh[:, None, :, None], torch.gather(blocks[i].flatten(2, 3), 2, index), tail[:, :, i])


def _attend_plain(s, q, first, end):
    """q [batch, heads, new, d] in half precision, query j of sequence b at position first[b] + j; the cache holds end[b]
    positions.  Returns [batch, heads, new, d] in half precision."""
    codes, scales, tail = s["codes"], s["scales"], s["tail"]
    batch, heads, new, d = q.shape
    kv_heads = codes.shape[2]
    longest = s["capacity"]
    position = torch.arange(longest, device=DEV)
    in_tail = (position[None] >= (end // BLOCK * BLOCK)[:, None])[:, None, :, None]
    row = (position % BLOCK)[None, None, :, None].expand(batch, kv_heads, longest, d)
    kv = []
    for i in range(2):
        held = (codes[i].to(F32) * scales[..., i, None, None]).flatten(2, 3)
        kv.append(torch.where(in_tail, torch.gather(tail[:, :, i], 2, row).to(F32), held))
    q = q.to(F32).reshape(batch, kv_heads, heads // kv_heads * new, d)
    scores = ((q @ kv[0].transpose(-1, -2)) / math.sqrt(d)).reshape(batch, heads, new, longest)
    seen = position[None, None] <= (first[:, None] + torch.arange(new, device=DEV))[:, :, None]
    scores = scores.masked_fill(~seen[:, None], -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    o = p.reshape(batch, kv_heads, -1, longest) @ kv[1].masked_fill((position[None] >= end[:, None])[:, None, :, None], 0.0)
    return (o.reshape(batch, heads, new, d) / p.sum(-1, keepdim=True)).to(F16)


def _run_decode(s):
    heads, kv_heads, d = s["heads"], s["kv_heads"], s["d"]
    batch = s["qkv"].shape[0]
    q, k, v = (x.reshape(batch, -1, 1, d) for x in s["qkv"].split((heads * d, kv_heads * d, kv_heads * d), 1))
    pos = s["pos"][:, None, None]
    past = s["past"].long()
    _append_plain(s, _rotate(k, pos), v, past, torch.ones_like(past))
    o = _attend_plain(s, _rotate(q, pos), past, past + 1)
    return o.reshape(batch, heads * d), s["tail"], s["scales"]


def _run_prefill(s):
    heads, kv_heads, d = s["heads"], s["kv_heads"], s["d"]
    starts, past = s["starts"].long(), s["past"].long()
    n = starts[1:] - starts[:-1]
    batch, new = n.numel(), s["max_new"]
    at = starts[:-1, None] + torch.arange(new, device=DEV)[None]
    inside = torch.arange(new, device=DEV)[None] < n[:, None]
    at = at.where(inside, torch.zeros_like(at))                                 # (rows of a padded batch; those past a sequence are not used)
    x = s["qkv"][at]
    pos = s["pos"].long()[at][:, None]
    q, k, v = (y.reshape(batch, new, -1, d).transpose(1, 2) for y in x.split((heads * d, kv_heads * d, kv_heads * d), 2))
    _append_plain(s, _rotate(k, pos), v, past, n)
    o = _attend_plain(s, _rotate(q, pos), past, past + n)
    return o.transpose(1, 2).reshape(batch, new, heads * d)[inside], s["tail"], s["scales"]


def _run_sample(s):
    logits = s["logits"].to(F64)
    b, v = logits.shape
    t = s["temperature"].to(F64)[:, None]
    greedy = t <= 0
    w = torch.exp((logits - logits.amax(-1, keepdim=True)) / t.where(~greedy, torch.ones_like(t)))
    order = torch.sort(logits, stable=True, dim=-1, descending=True).indices        # equal logits: the lower index first
    w = torch.gather(w, 1, order)
    rank = torch.arange(v, device=DEV)[None]
    keep = (rank == 0) | ~greedy
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        keep &= (rank < k) | (k <= 0)
        keep &= torch.cumsum(w * keep, -1) - w * keep < s["top_p"].to(F64)[:, None] * (w * keep).sum(-1, keepdim=True)
        keep |= rank == 0
        keep &= w >= s["min_p"].to(F64)[:, None] * w[:, :1]
    mass = torch.zeros_like(logits).scatter_(1, order, w * keep)
    total = mass.sum(-1, keepdim=True)
    before = torch.cumsum(mass, -1)
    token = ((before > s["u"].to(F64)[:, None] * total) & (mass > 0)).to(U8).argmax(-1)
    return token.to(I32), (torch.gather(mass, 1, token[:, None]) / total)[:, 0].to(F32)


# ---------------------------------------------------------------- states

def prepare(case, seed):
    kind = case["kind"]
    if kind == "mx":
        x, rows, w = _mx_inputs(case, seed)
        wq, ws = _mx_pack(*_mx_scale_and_level(w))
        s = dict(kind=kind, x=x, rows=rows, wq=wq, ws=ws)
        if own:
            from paper_2509_09090_amd import binding as B
            s["w"] = B.sqap_mx4_weight_pack(wq, ws)
            s["xq"] = torch.empty((case["m"], case["k"] // 2), dtype=U8, device=DEV)
            s["xs"] = torch.empty((case["m"], case["k"] // 32), dtype=U8, device=DEV)
            s["y"] = torch.empty((case["m"], case["n"]), dtype=F16, device=DEV)
        return s
    if kind == "sample":
        logits, temperature, top_k, top_p, min_p, u = _sample_inputs(case, seed)
        return dict(kind=kind, logits=logits, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, u=u,
                    token=torch.empty((case["batch"],), dtype=I32, device=DEV), prob=torch.empty((case["batch"],), dtype=F32, device=DEV))
    batch, heads, kv_heads, d = case["batch"], case["heads"], case["kv_heads"], case["d"]
    if kind == "decode":
        past = _lengths(case, case["longest"], 1)
        n = torch.ones_like(past)
        longest = case["longest"] + 1
    else:
        past = _lengths(case, case["past"], 1)
        n = _lengths(case, case["new"], 2).clamp_min(1)
        longest = case["past"] + case["new"]
    capacity = (longest + BLOCK - 1) // BLOCK * BLOCK
    starts = torch.cat((torch.zeros((1,), dtype=I64, device=DEV), n.cumsum(0)))
    k, v = _history(case, seed, capacity)
    s = dict(kind=kind, heads=heads, kv_heads=kv_heads, d=d, capacity=capacity, past=past.to(I32), starts=starts.to(I32),
             max_new=int(n.max()), qkv=_new_rows(case, seed, int(n.sum())))
    of = torch.repeat_interleave(torch.arange(batch, device=DEV), n)
    s["pos"] = (past[of] + torch.arange(of.numel(), device=DEV) - starts[of]).to(I32)
    if not own:
        s["codes"], s["scales"], s["tail"] = _fill_plain(k, v, past, capacity)
        return s
    from paper_2509_09090_amd import binding as B
    s["cache"] = B.Cache8(batch, capacity, kv_heads, d)
    # the history as a program would have left it there: appended at position 0, whose rotation changes nothing
    inside = torch.arange(capacity, device=DEV)[None] < past[:, None]
    rows = torch.cat([torch.zeros((int(past.sum()), heads * d), dtype=F16, device=DEV)] +
                     [x.transpose(1, 2)[inside].reshape(-1, kv_heads * d) for x in (k, v)], 1)
    at = torch.cat((torch.zeros((1,), dtype=I64, device=DEV), past.cumsum(0))).to(I32)
    B.sqap_cache8_append(rows, at, torch.zeros((rows.shape[0],), dtype=I32, device=DEV), torch.zeros_like(s["past"]), s["cache"], heads,
                         int(past.max()))
    s["o"] = torch.empty((int(n.sum()), heads * d), dtype=F16, device=DEV)
    if kind == "decode":
        s["longest"] = longest
        s["ws"] = torch.zeros((B.sqap_cache8_workspace_bytes(batch, heads, kv_heads, d, longest),), dtype=U8, device=DEV)
    else:
        s["q"] = torch.empty((int(n.sum()), heads * d), dtype=F16, device=DEV)
    return s


def run(s):
    kind = s["kind"]
    if not own:
        return {"mx": _run_mx, "decode": _run_decode, "prefill": _run_prefill, "sample": _run_sample}[kind](s)
    from paper_2509_09090_amd import binding as B
    if kind == "mx":
        B.sqap_mx4_quantize(s["x"], s["rows"], s["xq"], s["xs"])
        B.sqap_mx4_linear(s["xq"], s["xs"], s["w"], s["y"])
        return s["y"]
    if kind == "decode":
        B.sqap_cache8_decode_attention(s["qkv"], s["pos"], s["past"], s["cache"], s["heads"], s["o"], s["ws"], s["longest"])
        return s["o"], s["cache"].tail, s["cache"].scales
    if kind == "prefill":
        B.sqap_cache8_append(s["qkv"], s["starts"], s["pos"], s["past"], s["cache"], s["heads"], s["max_new"], Q_out=s["q"])
        B.sqap_cache8_attention(s["q"], s["starts"], s["past"], s["cache"], s["heads"], s["max_new"], s["o"])
        return s["o"], s["cache"].tail, s["cache"].scales
    B.sqap_sample(s["logits"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["u"], s["token"], s["prob"])
    return s["token"], s["prob"]


def work(case):
    """Bytes: every input read once, every output written once; operations of the products (a multiply-add is two)."""
    kind = case["kind"]
    if kind == "mx":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": 2 * m * k + n * (k // 2 + k // 32) + 2 * m * n, "flops": 2 * m * n * k}
    if kind == "sample":
        return {"bytes": case["batch"] * (2 * case["vocab"] + 28), "flops": 4 * case["batch"] * case["vocab"]}
    h, kv, d, mean = case["heads"], case["kv_heads"], case["d"], 0.5625       # (mean length over the longest, of the others)
    share = (1 + (case["batch"] - 1) * mean) / case["batch"]
    if kind == "decode":
        n = case["batch"] * case["longest"] * share
        return {"bytes": n * kv * 2 * (d + 4 / BLOCK) + case["batch"] * (4 * h + 8 * kv) * d, "flops": 4 * n * h * d}
    new, past = case["batch"] * case["new"] * share, case["past"] * share
    pairs = new * (past + case["new"] * share / 2)
    return {"bytes": new * d * 2 * (h + 2 * kv) + new * d * (2 * h + 2 * kv) + case["batch"] * past * kv * 2 * d, "flops": 4 * pairs * h * d}


# ---------------------------------------------------------------- 64 bits, from the definitions

def _exact_mx_values(x):
    """Nearest element of the eight magnitudes, of two equally near ones that with the even code."""
    b = x.double().reshape(x.shape[0], -1, 32)
    top = b.abs().max(-1, keepdim=True).values
    unit = torch.pow(2.0, torch.floor(torch.log2(top.where(top > 0, torch.ones_like(top)))) - 2.0)
    y = b.abs() / unit
    best, value = torch.full_like(y, math.inf), torch.zeros_like(y)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):                   # even codes first: an odd one has to be nearer
        far = (y - _LEVELS[code]).abs()
        value = torch.where(far < best, torch.full_like(y, _LEVELS[code]), value)
        best = torch.minimum(best, far)
    return (value * unit * b.sign()).reshape(x.shape[0], -1)


def _exact_blocks(x, length):
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
    i = torch.arange(d // 2, dtype=F64, device=DEV)
    angle = pos.double()[:, None, None] * torch.exp(-2.0 * i / d * math.log(BASE))
    z = z * torch.polar(torch.ones_like(angle), angle)
    return torch.cat((z.real, z.imag), -1).float().half().double()


def _exact_attention(case, seed):
    """Attention outputs alone (the cache's rows and scales are copies and single quotients, the same in every precision)."""
    batch, heads, kv_heads, d = case["batch"], case["heads"], case["kv_heads"], case["d"]
    past = _lengths(case, case["longest"] if case["kind"] == "decode" else case["past"], 1)
    n = torch.ones_like(past) if case["kind"] == "decode" else _lengths(case, case["new"], 2).clamp_min(1)
    longest = case["longest"] + 1 if case["kind"] == "decode" else case["past"] + case["new"]
    k, v = _history(case, seed, (longest + BLOCK - 1) // BLOCK * BLOCK)
    qkv = _new_rows(case, seed, int(n.sum()))
    out, at = [], 0
    for b in range(batch):
        p, m = int(past[b]), int(n[b])
        x = qkv[at:at + m].reshape(m, -1, d)
        at += m
        pos = p + torch.arange(m, device=DEV)
        q = _exact_turned(x[:, :heads], pos)
        keys = torch.cat((k[b, :, :p].double(), _exact_turned(x[:, heads:heads + kv_heads], pos).transpose(0, 1)), 1)
        values = torch.cat((v[b, :, :p].double(), x[:, heads + kv_heads:].double().transpose(0, 1)), 1)
        keys, values = _exact_blocks(keys, p + m), _exact_blocks(values, p + m)
        o = torch.empty((m, heads, d), dtype=F64, device=DEV)
        hidden = torch.arange(p + m, device=DEV)[None] > pos[:, None]
        for h in range(heads):
            score = (q[:, h] @ keys[h * kv_heads // heads].T) * d ** -0.5
            o[:, h] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ values[h * kv_heads // heads]
        out.append(o.reshape(m, heads * d))
    return torch.cat(out), None, None


def _exact_sample(case, seed):
    logits, temperature, top_k, top_p, min_p, u = _sample_inputs(case, seed)
    probs = []
    for r in range(case["batch"]):
        x = logits[r].double()
        if float(temperature[r]) <= 0:
            probs.append(1.0)
            continue
        z = torch.softmax(x / float(temperature[r]), 0)
        order = torch.argsort(x, descending=True, stable=True)
        if top_k is not None:
            if int(top_k[r]) > 0:
                order = order[: int(top_k[r])]
            mass = z[order]
            before = torch.cumsum(mass, 0) - mass
            count = max(1, int((before < float(top_p[r]) * float(mass.sum())).sum()))
            order = order[:count]
            order = order[z[order] >= float(min_p[r]) * float(z.max())]
        index = order.sort().values
        mass = z[index]
        run_up = torch.cumsum(mass, 0)
        hit = min(int((run_up <= float(u[r]) * float(mass.sum())).sum()), index.numel() - 1)
        probs.append(float(mass[hit] / mass.sum()))
    return None, torch.tensor(probs, dtype=F64, device=DEV)


def exact(case, seed):
    if case["kind"] == "mx":
        x, rows, w = _mx_inputs(case, seed)
        x = x if rows is None else x[rows.long()]
        return _exact_mx_values(x) @ _exact_mx_values(w).T
    if case["kind"] == "sample":
        return _exact_sample(case, seed)
    return _exact_attention(case, seed)
