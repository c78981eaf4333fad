"""Attention of sequences that share prefixes in a cache of 8 bits, against the definition in 64 bits, and its refusals."""
import ctypes

import numpy as np
import pytest

from paper_2509_09090_amd import binding as B
from tests import lowbit_ref as R
from tests.test_cache8 import BASE, ODD, P, Model, _desc

KEPT = 16384                                                          # bytes of a workspace that are left alone


def _front(**kw):
    """A cache of prefixes."""
    return _desc(**{**dict(codes=8192, scales=8192, tail=8192), **kw})


# ---------------------------------------------------------------- refusals (no GPU)

def test_prompt_refusals():
    L = B.lib()
    need = B.sqap_cache8_shared_workspace_bytes(4, 2, 4, 2, 64, 3, 2, 1, 5000)
    assert B.sqap_cache8_shared_workspace_bytes(4, 2, 4, 2, 64, 3, 2, 1, 500) == 0
    assert need > KEPT and all(B.sqap_cache8_shared_workspace_bytes(*bad) == 0 for bad in (
        (0, 1, 4, 2, 64, 3, 2, 1, 5), (4, 3, 4, 2, 64, 3, 2, 1, 5), (4, 0, 4, 2, 64, 3, 2, 1, 5), (4, 2, 5, 2, 64, 3, 2, 1, 5), (4, 2, 4, 2, 64, 0, 2, 1, 5),
        (4, 2, 4, 2, 64, 3, 0, 1, 5), (4, 2, 4, 2, 64, 3, 2, 0, 5), (4, 2, 4, 2, 64, 3, 2, 1, -1)))
    good = dict(Q=P, ldq=256, starts=P, past=P, rows=3, max_new=2, H=4, cache=_desc(batch=4), prefix=_front(capacity=512), length=P, longest_prefix=5000,
                O=P, ldo=256, ws=P, bytes=need, stream=None)
    call = lambda **kw: L.sqap_cache8_shared_attention(*{**good, **kw}.values())             # noqa: E731
    for bad in (dict(rows=-1), dict(max_new=-1), dict(H=5), dict(cache=None), dict(prefix=None), dict(Q=None), dict(starts=None), dict(past=None), dict(length=None),
                dict(O=None), dict(ldq=255), dict(ldo=8), dict(ws=None), dict(bytes=need - 1), dict(ws=ODD), dict(longest_prefix=-1), dict(cache=_desc(batch=3)),
                dict(prefix=_front(batch=0)), dict(prefix=_front(kv_heads=4)), dict(prefix=_front(kv_heads=1)), dict(prefix=_front(head_dim=128)),
                dict(prefix=_front(codes=None)), dict(prefix=_front(capacity=70)), dict(prefix=_front(codes=4096)), dict(prefix=_front(scales=4096)),
                dict(prefix=_front(tail=4096))):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(Q=ODD), dict(O=ODD), dict(ldo=260), dict(cache=_desc(batch=4096)), dict(prefix=_front(tail=4104)), dict(cache=_desc(head_dim=96)),
                dict(rows=2 ** 31 - 1, max_new=2 ** 30)):
        assert call(**bad) == B.EUNSUPPORTED, bad
    assert call(rows=0, Q=None) == B.OK and call(cache=_desc(batch=0), starts=None) == B.OK


@pytest.mark.parametrize("case", [(4, 2, 32, 8, 128, 300, 100000, 1, 100), (4, 4, 32, 8, 64, 700, 20000, 1, 5000), (8, 2, 12, 12, 64, 8, 40, 1, 6000), (1, 1, 64, 64, 128, 1, 9, 1, 20000),
                                  (4, 1, 4, 2, 64, 30, 2 ** 31 - 1, 1, 500)])
def test_workspace_of_prompts_that_announce_more_rows_than_there_are(case):
    """No sequence has more rows than there are: the call asks for no more, and no less."""
    L = B.lib()
    need = B.sqap_cache8_shared_workspace_bytes(*case)
    batch, groups, H, kv, d, rows, max_new, _, longest_prefix = case
    assert need == B.sqap_cache8_shared_workspace_bytes(batch, groups, H, kv, d, rows, rows, 1, longest_prefix)
    call = lambda n, most: L.sqap_cache8_shared_attention(P, H * d, P, P, rows, most, H, _desc(batch=batch, kv_heads=kv, head_dim=d),       # noqa: E731
                                                          _front(batch=groups, kv_heads=kv, head_dim=d), P, longest_prefix, P, H * d, P, n, None)
    if need:
        assert call(need - 1, max_new) == B.EINVAL


def test_decode_refusals():
    L = B.lib()
    need = B.sqap_cache8_shared_workspace_bytes(4, 2, 4, 2, 64, 4, 1, 100, 500)
    good = dict(QKV=P, ld=512, pos=P, past=P, H=4, base=BASE, cache=_desc(batch=4), prefix=_front(capacity=512), length=P, longest=100, longest_prefix=500, O=P,
                ldo=256, ws=P, bytes=need, stream=None)
    call = lambda **kw: L.sqap_cache8_shared_decode_attention(*{**good, **kw}.values())      # noqa: E731
    for bad in (dict(H=3), dict(base=ctypes.c_double(0.0)), dict(cache=None), dict(prefix=None), dict(length=None), dict(longest=0), dict(longest_prefix=-1),
                dict(QKV=None), dict(pos=None), dict(past=None), dict(O=None), dict(ld=504), dict(ldo=248), dict(ws=None), dict(bytes=need - 1), dict(ws=ODD),
                dict(cache=_desc(batch=5)), dict(prefix=_front(kv_heads=1)), dict(prefix=_front(head_dim=128))):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(QKV=ODD), dict(O=ODD), dict(cache=_desc(batch=4096)), dict(prefix=_front(codes=4104)),
                dict(H=1 << 18, cache=_desc(batch=4000, kv_heads=1 << 14), prefix=_front(kv_heads=1 << 14), ld=1 << 26, ldo=1 << 26)):
        assert call(**bad) == B.EUNSUPPORTED, bad
    assert call(cache=_desc(batch=0), pos=None) == B.OK


# ---------------------------------------------------------------- GPU

@pytest.fixture(scope="module")
def G():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from tests import gpu_util
    return gpu_util


class Shared:
    """Groups of sequences behind a prefix each, on the host next to the device's caches."""

    def __init__(self, G, groups, width, H, kv, d, lengths, capacity=256, seed=0, prefix_rows=None):
        import torch
        self.t, self.G, self.H, self.kv, self.d, self.width = torch, G, H, kv, d, width
        self.lengths = np.asarray(lengths, dtype=np.int32)
        self.prefix = Model(G, groups, H, kv, d, max(1, int(self.lengths.max())), seed)
        if self.lengths.sum():
            self.prefix.append(list(self.lengths), x=prefix_rows, attend=False)
        self.own = Model(G, groups * width, H, kv, d, capacity, seed + 1)
        self.device_lengths = G.to_dev(self.lengths)

    def workspace(self, rows, max_new, longest, longest_prefix):
        n = B.sqap_cache8_shared_workspace_bytes(len(self.own.past), len(self.lengths), self.H, self.kv, self.d, rows, max_new, longest, longest_prefix)
        return self.t.full((n,), 255, dtype=self.t.uint8, device=self.G.DEV)                 # any contents: NaN

    def positions(self, counts):
        return np.concatenate([self.lengths[b // self.width] + self.own.past[b] + np.arange(n) for b, n in enumerate(counts)]).astype(np.int32)

    def check(self, o, y, counts, skip=()):
        at, group = 0, self.H // self.kv
        for b, n in enumerate(counts):
            rows, at = slice(at, at + n), at + n
            if n == 0 or b in skip:
                continue
            g, sees = b // self.width, self.lengths[b // self.width] + self.own.past[b] + np.arange(n)
            for h in range(self.kv):
                k, v = (np.concatenate([R.held(x[:, h]), R.held(z[:, h])]) for x, z in ((self.prefix.k[g], self.own.k[b]), (self.prefix.v[g], self.own.v[b])))
                for head in range(h * group, (h + 1) * group):
                    got = o[rows, head * self.d:(head + 1) * self.d].astype(np.float64)
                    with np.errstate(invalid="ignore"):
                        want, mass, off = R.attend(y[rows, head].astype(np.float64), k, v, sees)
                    assert np.array_equal(np.isnan(got), np.isnan(want)), (b, head)
                    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), (b, head)
                    fine = np.isfinite(want)
                    v_top = np.abs(v[np.isfinite(v)]).max() if np.isfinite(v).any() else 0.0
                    far = np.abs(np.where(fine, got - np.where(fine, want, 0.0), 0.0))
                    limit = R.attention_bound(np.where(fine, want, 0.0), mass, np.where(np.isfinite(off), off, 0.0), k.shape[0], v_top, False)
                    assert np.all((far <= limit) | ~fine), (b, head, float(np.nanmax(far / limit)))

    def prompt(self, counts, x=None, most=None, longest_prefix=None, padding=3, in_place=False):
        t, G = self.t, self.G
        total = int(sum(counts))
        before = self.own.past.copy()
        y = self.own.append(counts, x=x, pos=self.positions(counts), attend=False)
        starts = G.to_dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
        q = t.full((total + padding, self.H * self.d + 8), float("nan"), dtype=t.float16, device=G.DEV)
        q[:total, :-8] = G.to_dev(np.ascontiguousarray(y[:, :self.H]).reshape(total, -1))
        o = t.full((total + padding, self.H * self.d), 9.0, dtype=t.float16, device=G.DEV)
        if in_place:
            q[total:] = 9.0
            o = q[:, :-8]
        most = int(max(counts)) if most is None else most
        longest_prefix = int(self.lengths.max()) if longest_prefix is None else longest_prefix
        ws = self.workspace(total + padding, most, 1, longest_prefix)
        B.sqap_cache8_shared_attention(q[:, :-8], starts, G.to_dev(before), self.own.cache, self.prefix.cache, self.device_lengths, self.H, most, o, ws, longest_prefix)
        after, self.own.past = self.own.past, before
        self.check(o[:total].cpu().numpy(), y, counts)
        self.own.past = after
        assert bool((o[total:] == 9).all()) and bool((ws[:KEPT] == 255).all())

    def decode(self, x=None, longest=None, longest_prefix=None):
        t, G = self.t, self.G
        batch = len(self.own.past)
        x = self.own.rows(batch) if x is None else x
        pos = self.positions([1] * batch)
        y = self.own.turned(x, pos)
        o = t.full((batch, self.H * self.d + 16), 9.0, dtype=t.float16, device=G.DEV)
        longest = int(self.own.past.max()) + 1 if longest is None else longest
        longest_prefix = int(self.lengths.max()) if longest_prefix is None else longest_prefix
        ws = self.workspace(batch, 1, longest, longest_prefix)
        B.sqap_cache8_shared_decode_attention(G.to_dev(x.reshape(batch, -1)), G.to_dev(pos), G.to_dev(self.own.past), self.own.cache, self.prefix.cache,
                                              self.device_lengths, self.H, o[:, :-16], ws, longest, longest_prefix)
        self.own.note([1] * batch, y)
        self.check(o[:, :-16].cpu().numpy(), y, [1] * batch)
        assert bool((o[:, -16:] == 9).all()) and bool((ws[:KEPT] == 255).all())
        self.own.past += 1
        return o


# groups, width, heads, key heads, head size, prefixes: pairs of a group and key head below, at and above 16, 64, 128; more than 16 heads to a key head
SHAPES = [(1, 1, 1, 1, 64, [1]), (1, 4, 4, 4, 128, [276]), (2, 3, 4, 2, 64, [64, 63]), (3, 2, 8, 1, 128, [0, 65, 200]), (2, 8, 8, 4, 128, [700, 130]),
          (1, 17, 4, 4, 64, [128]), (1, 16, 8, 2, 64, [1000]), (1, 13, 10, 2, 128, [333]), (2, 33, 4, 1, 64, [90, 5000]), (1, 5, 32, 1, 128, [191]),
          (1, 40, 4, 1, 128, [2500]), (1, 1, 20, 1, 64, [4097]), (2, 64, 4, 2, 64, [300, 70])]


@pytest.mark.gpu
@pytest.mark.parametrize("groups,width,H,kv,d,lengths", SHAPES)
def test_single_rows(G, groups, width, H, kv, d, lengths):
    """Own positions 0, in a block, across its end; then a longer history of uneven sequences; hints too small and too large."""
    s = Shared(G, groups, width, H, kv, d, lengths, seed=width)
    s.decode()
    s.own.append(list(s.own.rng.integers(0, 64, groups * width)), attend=False)
    s.decode(longest=1, longest_prefix=0)
    s.own.append([int(n) for n in 63 - s.own.past % 64], attend=False)
    s.decode(longest=100000, longest_prefix=100000)                   # every sequence finishes a block
    s.decode()
    s.own.check_contents()


@pytest.mark.gpu
@pytest.mark.parametrize("groups,width,H,kv,d,lengths", SHAPES)
def test_prompts(G, groups, width, H, kv, d, lengths):
    """Rows of many lengths, none at all, behind own positions or at the start; announcements larger than needed."""
    s = Shared(G, groups, width, H, kv, d, lengths, capacity=448, seed=width + 100)
    batch = groups * width
    s.prompt([1 + (5 * b) % 7 for b in range(batch)], in_place=True)
    s.prompt([int(n) for n in s.own.rng.integers(0, 80, batch)], most=100, longest_prefix=0)
    s.prompt([130 if b == batch - 1 else b % 3 for b in range(batch)], longest_prefix=100000, padding=0, in_place=True)
    s.own.check_contents()


@pytest.mark.gpu
@pytest.mark.parametrize("H,kv,d", [(16, 4, 64), (16, 4, 128), (4, 4, 128), (20, 5, 64)])
def test_prompts_of_many_sequences(G, H, kv, d):
    """More tiles than the device holds at once: in one pass and in parts; prefixes that end a block, in one or are empty; up to four own blocks."""
    s = Shared(G, 4, 40, H, kv, d, [70, 0, 128, 191], capacity=256, seed=H + d)
    counts = lambda: [int(n) for n in s.own.rng.integers(0, 8, 160)]                         # noqa: E731
    s.prompt(counts(), most=7)
    s.own.append([int(n) for n in s.own.rng.integers(0, 150, 160)], attend=False)
    s.prompt(counts(), most=8, in_place=True)
    s.prompt(counts(), most=8, longest_prefix=100000, padding=0)
    s.own.append([int(n) for n in 63 - s.own.past % 64], attend=False)
    s.prompt([2 + b % 3 for b in range(160)], longest_prefix=100000, in_place=True)          # every sequence finishes a block
    s.own.check_contents()


@pytest.mark.gpu
def test_many_own_blocks(G):
    """Own histories that are split over workgroups, too."""
    s = Shared(G, 1, 2, 8, 2, 64, [300], capacity=4096, seed=3)
    s.own.append([3000, 1999], attend=False)
    s.decode()
    s.prompt([40, 7])


@pytest.mark.gpu
@pytest.mark.parametrize("hint", [None, 100000])                  # (in one pass, and in parts)
@pytest.mark.parametrize("width", [2, 40, 140])
def test_infinite_values_and_keys(G, width, hint):
    """Infinities and NaN among values and keys of the unfinished blocks of a prefix and of own positions, a prefix block without scale, scores that
    are minus infinity over a whole prefix."""
    H, kv, d, lengths = 4, 2, 64, [70, 130, 1]
    rows = np.random.default_rng(8).standard_normal((201, H + 2 * kv, d)).astype(np.float16)
    rows[66, H + kv, 3] = np.inf
    rows[69, H + kv, 3], rows[69, H + kv + 1, 7] = -np.inf, np.nan
    rows[80, H + 1, 5] = np.inf                                       # a whole block of keys of the second prefix
    s = Shared(G, 3, width, H, kv, d, lengths, seed=4, prefix_rows=rows)
    s.prefix.cache.tail[2, :, 0, 0, 5] = -float("inf")                # a prefix of one position: scores of minus infinity, or plus
    s.prefix.k[2][0, :, 5] = -np.inf
    x = s.own.rows(3 * width)
    x[0, H + kv, 9] = np.inf
    x[2 * width, H + kv + 1, 2] = -np.inf
    s.decode(x)
    s.decode()
    x = s.own.rows(6 * width)
    x[1, H + kv, 40] = np.inf                                         # seen by the rows behind it alone
    s.prompt([2] * (3 * width), x=x, longest_prefix=hint)


@pytest.mark.gpu
@pytest.mark.parametrize("width", [2, 40, 80])
@pytest.mark.parametrize("decode,hint", [(True, 100), (False, 100), (False, 100000)])
def test_what_does_not_fit(G, width, decode, hint):
    """Padded sequences keep their outputs; sequences without room, rows or prefix lengths that cannot be give NaN, and nothing reaches the others."""
    t, H, kv, d, groups = __import__("torch"), 4, 2, 64, 4
    s = Shared(G, groups, width, H, kv, d, [100, 5, 64, 70], capacity=128, seed=5)
    batch = groups * width
    s.own.append([60] * batch, attend=False)
    past = s.own.past.copy()
    past[1], past[width] = -1, 128                                    # padded; no room
    lengths = G.to_dev(np.array([100, 5, -1, 129], np.int32))         # (room for two blocks)
    n = 1 if decode else 2
    counts = [n] * batch
    x = s.own.rows(n * batch)
    pos = np.concatenate([s.lengths[b // width] + past[b] + np.arange(n) for b in range(batch)]).astype(np.int32)
    o = t.full((n * batch, H * d), 9.0, dtype=t.float16, device=G.DEV)
    ws = s.workspace(n * batch, n, 128, hint)
    if decode:
        B.sqap_cache8_shared_decode_attention(G.to_dev(x.reshape(batch, -1)), G.to_dev(pos), G.to_dev(past), s.own.cache, s.prefix.cache, lengths, H, o, ws, 128, hint)
        y = s.own.turned(x, pos)
    else:
        starts = G.to_dev(np.arange(batch + 1, dtype=np.int32) * n)
        q = t.full_like(o, 9.0)
        B.sqap_cache8_append(G.to_dev(x.reshape(n * batch, -1)), starts, G.to_dev(pos), G.to_dev(past), s.own.cache, H, n, Q_out=q)
        B.sqap_cache8_shared_attention(q, starts, G.to_dev(past), s.own.cache, s.prefix.cache, lengths, H, n, o, ws, hint)
        y = s.own.turned(x, pos)
    s.own.note(counts, y)
    got = o.cpu().numpy()
    bad = {1, width} | set(range(2 * width, batch))
    s.check(got, y, counts, skip=bad)
    assert np.all(got[n:2 * n] == 9) and np.all(np.isnan(got[n * width:n * width + n])) and np.all(np.isnan(got[2 * width * n:]))


@pytest.mark.gpu
@pytest.mark.parametrize("hint", [70, 100000])
def test_rows_that_are_not_announced(G, hint):
    """More rows than announced: NaN for that sequence; more than all of a group's together: for the group.  Starts out of order: skipped."""
    t, H, kv, d, width = __import__("torch"), 2, 1, 64, 3
    s = Shared(G, 2, width, H, kv, d, [70, 20], seed=6)
    counts = [1, 5, 1, 2, 2, 2]
    before = s.own.past.copy()
    y = s.own.append(counts, pos=s.positions(counts), attend=False)
    s.own.past = before
    q = G.to_dev(np.ascontiguousarray(y[:, :H]).reshape(13, -1))
    for most, starts, bad, left in ((3, [0, 1, 6, 7, 9, 11, 13], range(1, 6), ()), (2, [0, 1, 6, 7, 9, 11, 13], range(7), ()), (0, [0, 1, 6, 7, 9, 11, 13], range(13), ()),
                                    (5, [0, 1, 6, 7, 9, 40, 13], (), range(9, 13)), (5, [0, 1, -6, 7, 9, 11, 13], (), range(1, 7))):
        o = t.full((13, H * d), 9.0, dtype=t.float16, device=G.DEV)
        B.sqap_cache8_shared_attention(q, G.to_dev(np.array(starts, np.int32)), G.to_dev(before), s.own.cache, s.prefix.cache, s.device_lengths, H, most, o,
                                       s.workspace(13, max(most, 1), 1, hint), hint)
        got = o.cpu().numpy()
        bad, left = list(bad), list(left)
        assert np.all(np.isnan(got[bad])) and np.all(got[left] == 9), (most, starts)
        at = np.concatenate([[0], np.cumsum(counts)])
        s.check(got, y, counts, skip={b for b in range(6) for r in range(at[b], at[b + 1]) if r in bad or r in left})


@pytest.mark.gpu
@pytest.mark.parametrize("width", [3, 40])
def test_replayed_with_other_lengths(G, width):
    """A captured decode call, replayed with other rows, positions, lengths; on a workspace that a call with counters uses in between."""
    t, H, kv, d = __import__("torch"), 8, 2, 64
    s = Shared(G, 2, width, H, kv, d, [200, 900], seed=7)
    batch = 2 * width
    n = max(B.sqap_cache8_shared_workspace_bytes(batch, 2, H, kv, d, batch, 1, 256, 900), B.sqap_cache8_workspace_bytes(2, H, kv, d, 900))
    ws = t.zeros((n,), dtype=t.uint8, device=G.DEV)
    rows, pos = t.zeros((batch, (H + 2 * kv) * d), dtype=t.float16, device=G.DEV), t.zeros((batch,), dtype=t.int32, device=G.DEV)
    past, o = t.zeros((batch,), dtype=t.int32, device=G.DEV), t.zeros((batch, H * d), dtype=t.float16, device=G.DEV)
    graph = t.cuda.CUDAGraph()
    t.cuda.synchronize()
    with t.cuda.graph(graph):
        B.sqap_cache8_shared_decode_attention(rows, pos, past, s.own.cache, s.prefix.cache, s.device_lengths, H, o, ws, 256, 900)
    for i in range(4):
        s.own.append(list(s.own.rng.integers(0, 50, batch)), attend=False)
        x, at = s.own.rows(batch), s.positions([1] * batch)
        rows.copy_(G.to_dev(x.reshape(batch, -1)))
        pos.copy_(G.to_dev(at))
        past.copy_(G.to_dev(s.own.past))
        graph.replay()
        t.cuda.synchronize()
        y = s.own.turned(x, at)
        s.own.note([1] * batch, y)
        s.check(o.cpu().numpy(), y, [1] * batch)
        s.own.past += 1
        other, out = B.Cache8(2, 900, kv, d, device=G.DEV), t.zeros((2, H * d), dtype=t.float16, device=G.DEV)
        B.sqap_cache8_decode_attention(rows[:2], pos[:2], t.full((2,), 800, dtype=t.int32, device=G.DEV), other, H, out, ws, 900)
        assert int(ws[:KEPT].max()) == 0


# ---- prompts long enough to be worked out together with their prefixes (three quarters of a tile of 128 pairs to a sequence, on average)

@pytest.mark.gpu
@pytest.mark.parametrize("groups,width,H,kv,d,lengths,calls", [
    (1, 1, 4, 2, 64, [100], [[300], [2]]),
    (1, 2, 2, 2, 128, [0], [[96, 200], [130, 64]]),
    (2, 3, 8, 2, 128, [700, 130], [[200, 33, 0, 129, 64, 301], [64, 0, 31, 127, 1, 64]]),
    (3, 1, 6, 1, 64, [64, 0, 191], [[65, 100, 16], [1, 63, 128]]),
    (1, 1, 4, 4, 128, [6000], [[130], [97]]),
    (1, 3, 32, 1, 64, [3001], [[5, 40, 3], [9, 1, 2]]),
    (1, 2, 20, 1, 128, [333], [[100, 77]]),
    (4, 4, 4, 4, 64, [1, 2, 65, 900], [[100 + 10 * b for b in range(16)]]),
    # (those above are less than 64 tiles, most of them)
    (1, 1, 32, 4, 64, [100], [[300], [260]]),
    (1, 2, 32, 2, 128, [0], [[96, 200], [150, 130]]),
    (2, 3, 32, 4, 128, [700, 130], [[200, 33, 0, 129, 64, 301], [64, 0, 31, 127, 1, 64]]),
    (3, 1, 48, 8, 64, [64, 0, 191], [[65, 100, 16], [1, 63, 128]]),
    (1, 1, 64, 64, 128, [6000], [[130], [128]]),
    (1, 3, 64, 1, 64, [3001], [[60, 70, 3], [9, 118, 2]]),
    (1, 2, 40, 2, 128, [333], [[130, 77], [205, 1]]),
])
def test_long_prompts(G, groups, width, H, kv, d, lengths, calls):
    s = Shared(G, groups, width, H, kv, d, lengths, capacity=640, seed=groups + 50)
    for counts in calls:
        s.prompt(counts, longest_prefix=0 if counts == calls[-1] else None, in_place=counts == calls[-1])
    s.own.check_contents()


@pytest.mark.gpu
def test_long_prompts_of_many_sequences(G):
    """A whole thousand sequences in four groups, some without rows; one more than are worked out that way."""
    for batch in (1024, 1028):
        s = Shared(G, 4, batch // 4, 8, 1, 64, [70, 5, 0, 128], capacity=64, seed=60)
        s.prompt([int(n) for n in s.own.rng.integers(8, 20, batch - 3)] + [0, 30, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("H", [4, 32])
def test_long_prompts_with_infinite_values(G, H):
    """As test_infinite_values_and_keys: in unfinished blocks of a prefix and of own positions, a block of keys without scale, scores of minus
    infinity over a whole prefix."""
    kv, d, lengths = 2, 64, [70, 130, 1]
    rows = np.random.default_rng(8).standard_normal((201, H + 2 * kv, d)).astype(np.float16)
    rows[66, H + kv, 3] = np.inf
    rows[69, H + kv, 3], rows[69, H + kv + 1, 7] = -np.inf, np.nan
    rows[80, H + 1, 5] = np.inf
    s = Shared(G, 3, 1, H, kv, d, lengths, capacity=512, seed=61, prefix_rows=rows)
    s.prefix.cache.tail[2, :, 0, 0, 5] = -float("inf")
    s.prefix.k[2][0, :, 5] = -np.inf
    x = s.own.rows(330)
    x[100, H + kv, 9] = np.inf                                        # (of 110 rows the last 46 are unfinished)
    x[150, H + kv + 1, 2] = -np.inf                                   # in a block that is finished
    x[329, H + kv + 1, 2] = np.nan
    s.prompt([110, 110, 110], x=x)


@pytest.mark.gpu
@pytest.mark.parametrize("H", [4, 16])
def test_long_prompts_that_do_not_fit(G, H):
    """NaN where there is no room, more rows than announced, more in a group than announced together or a length that cannot be; padded ones left alone."""
    t, kv, d, width = __import__("torch"), 1, 64, 2
    s = Shared(G, 5, width, H, kv, d, [70, 20, 64, 9, 30], capacity=192, seed=62)
    counts = [60, 40, 50, 45, 33, 70, 64, 64, 30, 90]
    before = s.own.past.copy()
    y = s.own.append(counts, pos=s.positions(counts), attend=False)
    s.own.past = before
    total = sum(counts)
    q = G.to_dev(np.ascontiguousarray(y[:, :H]).reshape(total, -1))
    at = np.concatenate([[0], np.cumsum(counts)])
    starts = at.astype(np.int32)
    for most, lengths, past, starts_, bad, left in (
            (100, [70, 20, 64, 9, 30], {1: -1, 3: 160}, None, {3}, {1}),
            (100, [70, -1, 64, 1000, 30], {}, None, {2, 3, 6, 7}, set()),
            (69, [70, 20, 64, 9, 30], {}, None, {5, 9}, set()),
            (59, [70, 20, 64, 9, 30], {}, None, {0, 5, 6, 7, 8, 9}, set()),
            (100, [70, 20, 64, 9, 30], {}, {3: 700}, set(), {2, 3}),
            (100, [70, 20, 64, 9, 30], {}, {4: -5}, {5}, {2, 3, 4})):
        p = before.copy()
        for b, n in past.items():
            p[b] = n
        st = starts.copy()
        for b, n in (starts_ or {}).items():
            st[b] = n
        o = t.full((total, H * d), 9.0, dtype=t.float16, device=G.DEV)
        B.sqap_cache8_shared_attention(q, G.to_dev(st), G.to_dev(p), s.own.cache, s.prefix.cache, G.to_dev(np.array(lengths, np.int32)), H, most, o,
                                       s.workspace(total, most, 1, 70), 70)
        got = o.cpu().numpy()
        for b in range(10):
            part = got[at[b]:at[b + 1]]
            if b in bad:
                assert np.all(np.isnan(part)), (most, b)
            elif b in left:
                assert np.all(part == 9), (most, b)
        s.check(got, y, counts, skip=bad | left)


@pytest.mark.gpu
@pytest.mark.parametrize("H", [4, 32])
def test_long_prompts_replayed(G, H):
    """A captured prompt call, replayed with other rows and lengths."""
    t, kv, d, total = __import__("torch"), 2, 128, 300
    s = Shared(G, 2, 2, H, kv, d, [500, 64], capacity=1024, seed=63)
    q, o = (t.zeros((total, H * d), dtype=t.float16, device=G.DEV) for _ in range(2))
    starts, past = t.zeros((5,), dtype=t.int32, device=G.DEV), t.zeros((4,), dtype=t.int32, device=G.DEV)
    ws = s.workspace(total, 200, 1, 500)
    graph = t.cuda.CUDAGraph()
    t.cuda.synchronize()
    with t.cuda.graph(graph):
        B.sqap_cache8_shared_attention(q, starts, past, s.own.cache, s.prefix.cache, s.device_lengths, H, 200, o, ws, 500)
    for counts in ([100, 60, 70, 50], [200, 0, 1, 99], [3, 2, 1, 140]):
        before, n = s.own.past.copy(), sum(counts)
        y = s.own.append(counts, pos=s.positions(counts), attend=False)
        q[:n] = G.to_dev(np.ascontiguousarray(y[:, :H]).reshape(n, -1))
        starts.copy_(G.to_dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)))
        past.copy_(G.to_dev(before))
        o.fill_(9.0)
        graph.replay()
        t.cuda.synchronize()
        after, s.own.past = s.own.past, before
        s.check(o.cpu().numpy(), y, counts)
        s.own.past = after
        assert bool((o[n:] == 9).all())


# ---- streams

@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 150])
def test_calls_on_streams_of_their_own(G, rows):
    """Calls over the same caches on two streams at once, each with a workspace of its own, give what one after the other gives, bit for bit."""
    t, H, kv, d, batch = __import__("torch"), 32, 4, 64, 6
    s = Shared(G, 2, 3, H, kv, d, [900, 3333], capacity=256, seed=80)
    counts = [rows] * batch
    before = s.own.past.copy()
    y = s.own.append(counts, pos=s.positions(counts), attend=False)
    after, s.own.past = s.own.past, before
    q = G.to_dev(np.ascontiguousarray(y[:, :H]).reshape(rows * batch, -1))
    starts, past = G.to_dev(np.arange(batch + 1, dtype=np.int32) * rows), G.to_dev(before)

    def call(o, ws, longest_prefix):
        B.sqap_cache8_shared_attention(q, starts, past, s.own.cache, s.prefix.cache, s.device_lengths, H, rows, o, ws, longest_prefix)

    outputs = []
    for longest_prefix in (3333, 100000):
        o, ws = t.full((rows * batch, H * d), 9.0, dtype=t.float16, device=G.DEV), s.workspace(rows * batch, rows, 1, longest_prefix)
        call(o, ws, longest_prefix)
        s.check(o.cpu().numpy(), y, counts)
        outputs.append((longest_prefix, o, t.full_like(o, 9.0), ws))
    streams = [t.cuda.Stream(), t.cuda.Stream()]
    t.cuda.synchronize()
    for _ in range(5):
        for stream, (longest_prefix, _, o, ws) in zip(streams, outputs):
            with t.cuda.stream(stream):
                o.fill_(9.0)
                call(o, ws, longest_prefix)
    t.cuda.synchronize()
    assert all(t.equal(x, o) for _, x, o, _ in outputs)
    s.own.past = after
