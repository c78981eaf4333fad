"""Beam selection and the reordering of a cache in 8 bits, against their definitions (binary64, copies), and their refusals."""
import ctypes

import numpy as np
import pytest

from paper_2509_09090_amd import binding as B
from tests.test_cache8 import _desc

P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4104)


# ---------------------------------------------------------------- refusals (no GPU)

def test_beam_refusals():
    L = B.lib()
    need = B.sqap_beam_workspace_bytes(2, 3, 1000, 6)
    assert need > 0 and B.sqap_beam_workspace_bytes(0, 3, 1000, 6) == 0 and B.sqap_beam_workspace_bytes(2, 0, 1000, 6) == 0
    far = [ctypes.c_void_p(1 << 20 << i) for i in range(5)]
    good = dict(logits=P, ld=1000, batch=2, beams=3, vocab=1000, scores=P, done=None, eos=-1, k=6, parent=far[0], token=far[1], score=far[2],
                done_out=far[3], ws=far[4], bytes=need, stream=None)
    call = lambda **kw: L.sqap_beam_select(*{**good, **kw}.values())                         # noqa: E731
    for bad in (dict(batch=-1), dict(beams=0), dict(vocab=0), dict(k=0), dict(ld=999), dict(logits=None), dict(scores=None), dict(parent=None),
                dict(token=None), dict(score=None), dict(ws=None), dict(bytes=need - 1), dict(ws=ODD), dict(done=P, eos=-1), dict(done=P, eos=1000),
                dict(score=P), dict(score=ctypes.c_void_p(4096 + 20)), dict(done=far[3], eos=1), dict(k=3, score=ctypes.c_void_p(4100))):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(beams=65), dict(k=65), dict(vocab=(1 << 20) + 1, ld=1 << 21), dict(batch=1 << 24)):
        assert call(**bad) == B.EUNSUPPORTED, bad
    assert call(batch=0, logits=None) == B.OK


def test_reorder_refusals():
    L = B.lib()
    far = [ctypes.c_void_p(1 << 20 << i) for i in range(3)]
    good = dict(cache=_desc(), parents=far[0], width=2, lengths=far[1], longest=100, out=far[2], stream=None)
    call = lambda **kw: L.sqap_cache8_reorder(*{**good, **kw}.values())                      # noqa: E731
    for bad in (dict(cache=None), dict(parents=None), dict(lengths=None), dict(width=0), dict(width=-2), dict(width=3), dict(longest=-1),
                dict(out=far[0]), dict(out=ctypes.c_void_p((2 << 20) + 4)), dict(cache=_desc(codes=None)), dict(cache=_desc(capacity=100))):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(width=65, cache=_desc(batch=130)), dict(cache=_desc(head_dim=32)), dict(cache=_desc(tail=4104))):
        assert call(**bad) == B.EUNSUPPORTED, bad
    assert call(cache=_desc(batch=0), parents=None) == B.OK


# ---------------------------------------------------------------- GPU

@pytest.fixture(scope="module")
def G():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from tests import gpu_util
    return gpu_util


# The logarithm of a sum of exponentials: a term's exponent x = (l - max) log2 e is rounded in binary32, the power of two is off by a unit of the
# last place and sums of eight are rounded three times: (|x| + 2 + 3) 2^-24 of the term, where terms with |x| above 40 do not count (2^20 of
# them are less than 2^-20 of the largest, and their own error that share of it).
LSE_OFF = 45 * 2.0 ** -24


def reference(logits, scores, done, eos, k):
    """One batch element -> [(total, parent, token)], best first, those without a probability behind them by beam and token, and totals [beams, vocab]."""
    beams, vocab = logits.shape
    x = logits.astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, x) + 0.0
    total = np.full((beams, vocab), -np.inf)
    for r in range(beams):
        s = float(scores[r])
        if not s > -np.inf:
            continue
        if done is not None and done[r]:
            total[r, eos] = s
            continue
        top = x[r].max()
        if top == -np.inf:
            continue
        d = np.where(x[r] == top, 0.0, -np.inf) if np.isinf(top) else x[r] - top
        total[r] = s + (d - np.log(np.exp(d).sum()))
    order = sorted(((-total[r, t], r, -x[r, t], t) for r in range(beams) for t in np.lexsort((-x[r], -total[r]))[:k] if total[r, t] > -np.inf))[:k]
    rest = [(-np.inf, int(r), int(t)) for r, t in zip(*np.unravel_index(np.flatnonzero(total.ravel() == -np.inf)[:k], total.shape))]
    return ([(-o[0], o[1], o[3]) for o in order] + rest)[:k], total


def select(G, logits, scores, done, eos, k, odd=False, in_place=False):
    import torch
    batch, beams = scores.shape
    dev = lambda a: None if a is None else G.to_dev(a)                # noqa: E731
    x = G.to_dev(logits)
    if odd:                                                           # rows at odd addresses, NaN between them
        wide = torch.full((x.shape[0], x.shape[1] + 3), float("nan"), dtype=torch.float16, device=G.DEV)
        wide[:, 1:-2] = x
        x = wide[:, 1:-2]
    s, d = dev(scores.astype(np.float32)), dev(done)
    parent, token, done_out = (torch.full((batch, k), 77, dtype=torch.int32, device=G.DEV) for _ in range(3))
    score = torch.full((batch, k), 77.0, device=G.DEV)
    if in_place:
        score, done_out = s, d
    ws = torch.full((B.sqap_beam_workspace_bytes(batch, beams, logits.shape[1], k),), 255, dtype=torch.uint8, device=G.DEV)
    B.sqap_beam_select(x, s, d, eos, parent, token, score, done_out, ws)
    return [None if t is None else t.cpu().numpy() for t in (parent, token, score, done_out)]


def check(G, logits, scores, done=None, eos=-1, k=4, **kw):
    """Returns how many elements were compared token by token: those whose totals are further apart than the sums may be off."""
    batch, beams = scores.shape
    got = select(G, logits, scores, done, eos, k, **kw)
    clear = 0
    for b in range(batch):
        want, total = reference(logits[b * beams:(b + 1) * beams], scores[b], None if done is None else done[b], eos, k)
        parent, token, score, done_out = (None if x is None else x[b] for x in got)
        n = len(want)                                                 # (k, or all that there are)
        assert np.all(parent[n:] == -1) and np.all(token[n:] == -1) and np.all(score[n:] == -np.inf)
        assert np.all((parent[:n] >= 0) & (parent[:n] < beams) & (token[:n] >= 0) & (token[:n] < logits.shape[1]))
        assert len(set(zip(parent[:n], token[:n]))) == n
        mine = total[parent[:n], token[:n]]
        if done_out is not None:
            ended = np.array([(done is not None and done[b][p] != 0) or t == eos for p, t in zip(parent[:n], token[:n])], dtype=np.int32)
            assert np.array_equal(done_out[:n], ended) and np.all(done_out[n:] == 0)
        some = sum(w[0] > -np.inf for w in want)
        assert [(int(p), int(t)) for p, t in zip(parent[some:n], token[some:n])] == [w[1:] for w in want[some:]]
        with np.errstate(invalid="ignore"):
            near = (score[:n] == mine) | (np.abs(score[:n] - mine) <= LSE_OFF + 2.0 ** -24 * np.abs(mine))
        assert np.all(near), (b, score[:n], mine)
        if n == 0:
            continue
        ends = np.array([w[0] for w in want])
        with np.errstate(invalid="ignore"):
            assert np.all((mine >= ends - 2 * LSE_OFF) | (mine == ends)), b           # nothing better was left out
        # totals of different beams at the places where their order decides: apart, or the same beam's
        rest = sorted(((-total[r, t], r) for r in range(beams) for t in np.argsort(-total[r], kind="stable")[:k + 1]))[:k + 1]
        with np.errstate(invalid="ignore"):
            apart = all(x[1] == y[1] or y[0] == np.inf or not y[0] - x[0] <= 2 * LSE_OFF for x, y in zip(rest, rest[1:]))
        if apart:
            assert [(int(p), int(t)) for p, t in zip(parent[:n], token[:n])] == [w[1:] for w in want], b
            clear += 1
    return clear


def _logits(rng, rows, vocab, spread=3.0):
    return (rng.standard_normal((rows, vocab)) * spread).astype(np.float16)


def _scores(rng, batch, beams):
    return -np.cumsum(rng.random((batch, beams)) * 2.0, -1).astype(np.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("batch,beams,vocab,k", [(1, 1, 1, 1), (1, 1, 7, 10), (2, 3, 8, 30), (3, 5, 1003, 10), (1, 4, 32000, 4), (2, 3, 2047, 6), (2, 3, 2048, 6),
                                                 (2, 3, 2049, 6), (70, 2, 5001, 4), (3, 32, 4099, 64), (1, 64, 300, 64), (2, 8, 128001, 16), (40, 8, 17001, 8), (2, 31, 427, 62),
                                                 (1, 2, 1 << 20, 64)])
def test_against_the_definition(G, batch, beams, vocab, k):
    rng = np.random.default_rng(batch * 1000 + beams)
    logits, scores = _logits(rng, batch * beams, vocab), _scores(rng, batch, beams)
    done = (rng.random((batch, beams)) < 0.3).astype(np.int32)
    clear = check(G, logits, scores, k=k) + check(G, logits, scores, done, vocab // 2, k, odd=True)
    assert clear >= batch, clear


@pytest.mark.gpu
@pytest.mark.parametrize("beams,vocab,k", [(3, 100, 64), (4, 20000, 8), (64, 8192, 64), (2, 70000, 64)])
def test_equal_logits_go_to_the_lowest(G, beams, vocab, k):
    """All the same, in beams of the same score: the first beam's first tokens.  Then the same few steps in all beams: its lowest tokens, too."""
    logits = np.full((beams, vocab), -0.0, np.float16)
    logits[:, ::2] = 0.0
    scores = np.full((1, beams), -3.0, np.float32)
    parent, token, _, _ = select(G, logits, scores, None, -1, k)
    assert np.all(parent == 0) and np.array_equal(token[0], np.arange(k))
    steps = np.arange(vocab)[::-1] % 50
    logits = np.broadcast_to((-0.5 * steps).astype(np.float16), (beams, vocab)).copy()
    parent, token, _, _ = select(G, logits, scores, None, -1, k)
    want = [(0, t) for t in np.flatnonzero(steps == 0)[:k]] if (steps == 0).sum() >= k else None
    if want is None:
        order = sorted((s, r, t) for r in range(beams) for t, s in enumerate(steps) if s < 40)[:k]
        want = [(r, t) for _, r, t in order]
    assert list(zip(parent[0], token[0])) == want


@pytest.mark.gpu
def test_many_candidates_of_few_threads(G):
    """64 beams of the same order, whose best lie in the first 2048 tokens: more candidates reach the threads' bound than are listed at once."""
    rng = np.random.default_rng(5)
    row = np.full(8192, -8.0, np.float16)
    row[rng.permutation(2048)[:64]] = (-np.arange(64) / 64).astype(np.float16)
    logits = np.broadcast_to(row, (64, 8192)).copy()
    scores = np.zeros((1, 64), np.float32)
    parent, token, _, _ = select(G, logits, scores, None, -1, 64)
    assert np.array_equal(parent[0], np.arange(64)) and np.all(token == int(row.argmax()))


@pytest.mark.gpu
def test_values_that_are_not_finite(G):
    rng = np.random.default_rng(6)
    beams, vocab, k = 6, 5000, 20
    logits, scores = _logits(rng, 2 * beams, vocab), _scores(rng, 2, beams)
    logits[0, ::3] = np.nan
    logits[1, 5:] = -np.inf
    logits[2] = -np.inf
    logits[3] = np.nan
    logits[4, [7, 4000, 4999]] = np.inf
    logits[5, :] = -65504.0
    logits[5, 2500] = 65504.0
    logits[beams, :] = np.nan
    logits[beams, 4321] = -60000.0
    scores[1, 1], scores[1, 2], scores[1, 3] = -np.inf, np.nan, np.inf
    check(G, logits, scores, k=k)
    check(G, logits, scores, done=np.ones((2, beams), np.int32), eos=0, k=k)
    scores[:] = -np.inf
    check(G, logits, scores, k=k)


@pytest.mark.gpu
def test_scores_beyond_the_logits_steps(G):
    """Sums so large that the logits' differences are lost in them: still by logit, then token."""
    logits = np.array([[0.5, 1.0, 0.75, 1.0], [2.0, 0.0, 2.0, 0.0]], np.float16)
    parent, token, score, _ = select(G, logits, np.full((1, 2), -1e30, np.float32), None, -1, 6)
    assert list(zip(parent[0], token[0])) == [(0, 1), (0, 3), (0, 2), (0, 0), (1, 0), (1, 2)]
    assert np.all(score == np.float32(-1e30))


@pytest.mark.gpu
def test_in_place_and_replayed(G):
    """Outputs over the inputs; a captured call with other inputs, several times, among eager work."""
    import torch
    rng = np.random.default_rng(7)
    batch, beams, vocab = 3, 4, 9001
    logits, scores = _logits(rng, batch * beams, vocab), _scores(rng, batch, beams)
    done = (rng.random((batch, beams)) < 0.3).astype(np.int32)
    apart = select(G, logits, scores, done, 3, beams)
    for x, y in zip(apart, select(G, logits, scores, done, 3, beams, in_place=True)):
        assert np.array_equal(x, y)
    x, s, d = (G.to_dev(a) for a in (logits, scores, done))
    out = [torch.zeros((batch, beams), dtype=t, device=G.DEV) for t in (torch.int32, torch.int32, torch.float32, torch.int32)]
    ws = torch.zeros((B.sqap_beam_workspace_bytes(batch, beams, vocab, beams),), dtype=torch.uint8, device=G.DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.sqap_beam_select(x, s, d, 3, *out, ws)
    for i in range(4):
        logits, scores = _logits(rng, batch * beams, vocab), _scores(rng, batch, beams)
        x.copy_(G.to_dev(logits))
        s.copy_(G.to_dev(scores))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, select(G, logits, scores, done, 3, beams)):
            assert np.array_equal(got.cpu().numpy(), want), i


def _moved(codes, scales, tail, parents, lengths, width, capacity):
    want = [x.copy() for x in (codes, scales, tail)]
    after = lengths.copy()
    for i, p in enumerate(parents.ravel()):
        if not 0 <= p < width:
            continue
        of = i // width * width + p
        after[i] = lengths[of]
        n = int(lengths[of])
        if of == i or not 0 < n <= capacity:
            continue
        want[0][i, :, :n // 64], want[1][i, :, :n // 64] = codes[of, :, :n // 64], scales[of, :, :n // 64]
        want[2][i, :, :, :n % 64] = tail[of, :, :, :n % 64]
    return want, after


@pytest.mark.gpu
@pytest.mark.parametrize("groups,width,kv,d,capacity,longest", [(1, 1, 1, 64, 64, 64), (2, 2, 3, 64, 192, 192), (3, 4, 2, 128, 320, 320), (2, 5, 1, 64, 128, 0),
                                                                (1, 8, 2, 128, 256, 100000), (2, 16, 1, 64, 384, 70), (1, 17, 2, 64, 128, 128),
                                                                (2, 33, 1, 128, 192, 192), (1, 64, 2, 64, 128, 128)])
def test_reorder(G, groups, width, kv, d, capacity, longest):
    """Cycles, one for all, its own parents, none; lengths at the ends of blocks, 0, none (padded) and beyond the capacity; `longest` too small, too large."""
    import torch
    rng = np.random.default_rng(width)
    batch = groups * width
    for kind in ("mixed", "cycle", "one", "all edges"):
        cache = B.Cache8(batch, capacity, kv, d, device=G.DEV)
        held = [rng.integers(-128, 128, cache.codes.shape).astype(np.int8), rng.integers(0, 1 << 32, cache.scales.shape, dtype=np.uint32),
                rng.integers(0, 1 << 16, cache.tail.shape).astype(np.uint16)]
        cache.codes.copy_(G.to_dev(held[0]))
        cache.scales.view(torch.int32).copy_(G.to_dev(held[1].view(np.int32)))
        cache.tail.view(torch.int16).copy_(G.to_dev(held[2].view(np.int16)))
        lengths = rng.integers(0, capacity + 1, batch).astype(np.int32)
        parents = rng.integers(-1, width + 1, (groups, width)).astype(np.int32)
        if kind == "cycle":
            parents = np.tile(np.roll(np.arange(width), 1), (groups, 1)).astype(np.int32)
        elif kind == "one":
            parents[:] = width - 1
        elif kind == "all edges":
            lengths = np.resize(np.array([0, 1, 63, 64, 65, -1, capacity, capacity + 1, 127, capacity - 1], np.int32), batch)
        want, after = _moved(*held, parents, lengths, width, capacity)
        out = torch.full((batch,), 55, dtype=torch.int32, device=G.DEV)
        B.sqap_cache8_reorder(cache, G.to_dev(parents), G.to_dev(lengths), longest, out if kind != "one" else None)
        assert np.array_equal(cache.codes.cpu().numpy(), want[0])
        assert np.array_equal(cache.scales.view(torch.int32).cpu().numpy().view(np.uint32), want[1])
        assert np.array_equal(cache.tail.view(torch.int16).cpu().numpy().view(np.uint16), want[2])
        if kind != "one":
            assert np.array_equal(out.cpu().numpy(), after)


@pytest.mark.gpu
@pytest.mark.parametrize("beams,vocab,k", [(1, 100, 2), (2, 3, 6), (2, 3, 10), (4, 64, 64), (1, 1, 3), (64, 70, 64)])
def test_fewer_than_asked_for(G, beams, vocab, k):
    """Beams that have finished, beams without a score, logits without a probability: what is left follows by beam and token."""
    rng = np.random.default_rng(beams + k)
    logits, scores = _logits(rng, 5 * beams, vocab), _scores(rng, 5, beams)
    done = np.ones((5, beams), np.int32)
    done[1, ::2] = 0
    done[2:] = 0
    scores[1, ::2] = -np.inf
    scores[2] = -np.inf
    logits[3 * beams:4 * beams, 1:] = -np.inf
    logits[4 * beams:] = np.nan
    check(G, logits, scores, done, eos=vocab - 1, k=k)
    check(G, logits, scores, done, eos=0, k=k, odd=True)


@pytest.mark.gpu
def test_reorder_with_a_length_that_no_cache_has(G):
    """`longest` decides how the work is split: one far beyond the capacity costs what the capacity does, not a launch for all those blocks."""
    import torch
    groups, width, kv, d, capacity = 16, 2, 32, 64, 192
    rng = np.random.default_rng(9)
    cache = B.Cache8(groups * width, capacity, kv, d, device=G.DEV)
    held = [rng.integers(-128, 128, cache.codes.shape).astype(np.int8), rng.integers(0, 1 << 32, cache.scales.shape, dtype=np.uint32),
            rng.integers(0, 1 << 16, cache.tail.shape).astype(np.uint16)]
    views = (cache.codes, cache.scales.view(torch.int32), cache.tail.view(torch.int16))
    lengths = np.resize(np.array([190, 70, 64], np.int32), groups * width)
    parents = np.tile(np.array([1, 0], np.int32), (groups, 1))
    want, _ = _moved(*held, parents, lengths, width, capacity)
    ms = {}
    for longest in (capacity, 2 ** 31 - 1, capacity, 2 ** 31 - 1):
        for x, y in zip(views, held):
            x.copy_(G.to_dev(y.view(np.int32) if y.dtype == np.uint32 else y.view(np.int16) if y.dtype == np.uint16 else y))
        p, n = G.to_dev(parents), G.to_dev(lengths)
        torch.cuda.synchronize()
        start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        B.sqap_cache8_reorder(cache, p, n, longest)
        stop.record()
        torch.cuda.synchronize()
        ms[longest] = start.elapsed_time(stop)
        for x, y in zip(views, want):
            assert np.array_equal(x.cpu().numpy().view(y.dtype), y), longest
    assert ms[2 ** 31 - 1] < 20 * ms[capacity] + 1.0, ms


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [5000, 128001, 1 << 20])
@pytest.mark.parametrize("below", [1.0, 3.75, 11.0, 13.875])
def test_sums_of_flat_tails(G, vocab, below):
    """All tokens but one as far below the largest: every term's exponent is rounded alike, so that nothing cancels.  Rising tails, too, whose sums are brought
    below a larger logit again and again."""
    logits = np.full((3, vocab), -below, np.float16)
    logits[0, vocab // 3] = 0.0
    logits[1] = (np.arange(vocab) // 256 % 64 * (below / 64) - below).astype(np.float16)
    logits[2] += np.float16(1000.0)
    logits[2, 1] = 1000.0
    scores = np.array([[-0.25, -20.0, -1.5]], np.float32)
    parent, token, score, _ = select(G, logits, scores, None, -1, 3)
    for r in range(3):                                                # (each beam by itself, so that all of them come out)
        check(G, logits[r:r + 1], scores[:, r:r + 1], k=4)
    x = logits.astype(np.float64)
    total = scores[0][:, None] + x - (np.log(np.exp(x - x.max(1, keepdims=True)).sum(1, keepdims=True)) + x.max(1, keepdims=True))
    mine = total[parent[0], token[0]]
    assert np.all(np.abs(score[0] - mine) <= LSE_OFF + 2.0 ** -24 * np.abs(mine))
