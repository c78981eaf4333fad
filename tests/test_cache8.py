"""The key/value cache in 8 bits: what it holds, attention of many rows and of one row per sequence, against the definitions in 64 bits."""
import ctypes

import numpy as np
import pytest

from paper_2509_09090_amd import binding as B
from tests import lowbit_ref as R


# ---------------------------------------------------------------- refusals (no GPU)

def _desc(**kw):
    c = B.Cache8Desc(4096, 4096, 4096, 2, 128, 2, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4104)
BASE = ctypes.c_double(1e4)


def test_append_refusals():
    L = B.lib()
    good = dict(QKV=P, ld=512, starts=P, pos=P, past=P, rows=3, max_new=2, H=4, base=BASE, cache=_desc(), Q_out=P, ldq=256, stream=None)
    call = lambda **kw: L.sqap_cache8_append(*{**good, **kw}.values())                       # noqa: E731
    for bad in (dict(rows=-1), dict(max_new=-1), dict(H=0), dict(H=3), dict(base=ctypes.c_double(0.0)), dict(cache=None), dict(QKV=None),
                dict(starts=None), dict(pos=None), dict(past=None), dict(ld=504), dict(ldq=248), dict(cache=_desc(batch=-1)),
                dict(cache=_desc(capacity=0)), dict(cache=_desc(capacity=100)), dict(cache=_desc(kv_heads=0)), dict(cache=_desc(codes=None)),
                dict(cache=_desc(scales=None)), dict(cache=_desc(tail=None))):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(QKV=ODD), dict(ld=516), dict(Q_out=ODD), dict(ldq=260), dict(cache=_desc(head_dim=32)), dict(cache=_desc(codes=4104)),
                dict(cache=_desc(tail=4104)), dict(cache=_desc(scales=4098)), dict(cache=_desc(batch=70000))):
        assert call(**bad) == B.EUNSUPPORTED, bad
    assert call(rows=0, QKV=None) == B.OK
    assert call(max_new=0) == B.OK
    assert call(cache=_desc(batch=0)) == B.OK


def test_attention_refusals():
    L = B.lib()
    good = dict(Q=P, ldq=256, starts=P, past=P, rows=3, max_new=2, H=4, cache=_desc(), O=P, ldo=256, stream=None)
    call = lambda **kw: L.sqap_cache8_attention(*{**good, **kw}.values())                    # noqa: E731
    for bad in (dict(rows=-1), dict(max_new=-1), dict(H=-4), dict(H=5), dict(cache=None), dict(Q=None), dict(starts=None), dict(past=None),
                dict(O=None), dict(ldq=255), dict(ldo=8), dict(cache=_desc(capacity=65))):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(Q=ODD), dict(O=ODD), dict(ldo=260), dict(cache=_desc(head_dim=96)), dict(rows=2 ** 30, max_new=2 ** 30),
                dict(rows=2 ** 30 - 64, max_new=2 ** 30 - 64, cache=_desc(batch=65535))):
        assert call(**bad) == B.EUNSUPPORTED, bad
    assert call(rows=0) == B.OK


def test_decode_and_read_refusals():
    L = B.lib()
    need = B.sqap_cache8_workspace_bytes(2, 4, 2, 64, 4096)
    assert need > 0 and B.sqap_cache8_workspace_bytes(2, 4, 2, 64, 256) == 0
    assert B.sqap_cache8_workspace_bytes(0, 4, 2, 64, 4096) == 0 and B.sqap_cache8_workspace_bytes(2, 5, 2, 64, 4096) == 0
    good = dict(QKV=P, ld=512, pos=P, past=P, H=4, base=BASE, cache=_desc(capacity=4096), longest=4096, O=P, ldo=256, ws=P, bytes=need, stream=None)
    call = lambda **kw: L.sqap_cache8_decode_attention(*{**good, **kw}.values())             # noqa: E731
    for bad in (dict(H=3), dict(base=ctypes.c_double(-1.0)), dict(cache=None), dict(longest=0), dict(QKV=None), dict(pos=None), dict(past=None),
                dict(O=None), dict(ld=504), dict(ldo=248), dict(ws=None), dict(bytes=need - 1), dict(ws=ODD)):
        assert call(**bad) == B.EINVAL, bad
    assert b"" != L.sqap_last_error()
    for bad in (dict(QKV=ODD), dict(O=ODD), dict(cache=_desc(head_dim=256)), dict(H=2 * 16 * 65536, ld=1 << 40, ldo=1 << 40)):
        assert call(**bad) == B.EUNSUPPORTED, bad
    read = dict(cache=_desc(), lengths=P, first=0, count=4, out=P, ld=256, stream=None)
    call = lambda **kw: L.sqap_cache8_read(*{**read, **kw}.values())                         # noqa: E731
    for bad in (dict(cache=None), dict(lengths=None), dict(first=-1), dict(count=-1), dict(out=None), dict(ld=248), dict(first=2 ** 31 - 1)):
        assert call(**bad) == B.EINVAL, bad
    assert call(out=ODD) == B.EUNSUPPORTED
    assert call(count=0) == B.OK


# ---------------------------------------------------------------- GPU

@pytest.fixture(scope="module")
def G():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from tests import gpu_util
    return gpu_util


class Model:
    """A batch of sequences on the host next to the cache on the device.  The rotation's bits are those of sqap_rope."""
    most = 0                                                              # rows that are announced at least

    def __init__(self, G, batch, H, kv, d, capacity, seed=0):
        import torch
        self.t, self.G, self.H, self.kv, self.d = torch, G, H, kv, d
        self.rng = np.random.default_rng(seed)
        self.cache = B.Cache8(batch, capacity, kv, d, device=G.DEV)
        for x in (self.cache.codes, self.cache.scales, self.cache.tail):                     # needs no initialisation
            x.view(torch.uint8).fill_(0xFF)
        self.k = [np.zeros((0, kv, d), np.float16) for _ in range(batch)]
        self.v = [np.zeros((0, kv, d), np.float16) for _ in range(batch)]
        self.past = np.zeros(batch, dtype=np.int32)

    def rows(self, n, k_size=1.0, v_size=1.0):
        w = self.rng.standard_normal((n, self.H + 2 * self.kv, self.d))
        w[:, self.H:self.H + self.kv] *= k_size
        w[:, self.H + self.kv:] *= v_size
        return w.astype(np.float16)

    def turned(self, x, pos):
        """q|k|v rows [n, heads, d] -> the same with q and k rotated (host array of the device's bits)."""
        n = x.shape[0]
        flat = self.G.to_dev(x.reshape(n, -1))
        if n:
            B.sqap_rope(flat[:, :(self.H + self.kv) * self.d], self.G.to_dev(np.asarray(pos, dtype=np.int32)), self.H + self.kv, self.d)
        got = flat.cpu().numpy().reshape(x.shape)
        want = R.turn(x[:, :self.H + self.kv], pos) if n else x[:, :self.H + self.kv]
        with np.errstate(invalid="ignore"):
            near = np.abs(got[:, :self.H + self.kv].astype(np.float64) - want.astype(np.float64)) <= 2.0 ** -10 * np.abs(want.astype(np.float64)) + 2.0 ** -24
        assert np.all(near | ~np.isfinite(want))
        return got

    def note(self, counts, turned):
        at = 0
        for b, n in enumerate(counts):
            self.k[b] = np.concatenate([self.k[b], turned[at:at + n, self.H:self.H + self.kv]])
            self.v[b] = np.concatenate([self.v[b], turned[at:at + n, self.H + self.kv:]])
            at += n

    def append(self, counts, x=None, pos=None, attend=True):
        """Appends counts[b] rows to each sequence; returns outputs and what they should be near."""
        t, G = self.t, self.G
        total = int(sum(counts))
        x = self.rows(total) if x is None else x
        pos = np.concatenate([self.past[b] + np.arange(n) for b, n in enumerate(counts)]) if pos is None else pos
        y = self.turned(x, pos)
        starts = G.to_dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
        past = G.to_dev(self.past)
        most = max(self.most, int(max(counts)) if len(counts) else 0)
        padded = max(total, self.most)                                    # (rows behind the last sequence)
        q = t.full((padded, self.H * self.d), 9.0, dtype=t.float16, device=G.DEV)
        o = t.full((padded, self.H * self.d), 9.0, dtype=t.float16, device=G.DEV)
        rows = t.full((padded, (self.H + 2 * self.kv) * self.d), float("nan"), dtype=t.float16, device=G.DEV)
        rows[:total] = G.to_dev(x.reshape(total, -1))
        at = t.zeros(padded, dtype=t.int32, device=G.DEV)
        at[:total] = G.to_dev(np.asarray(pos, dtype=np.int32))
        before = rows.clone()
        B.sqap_cache8_append(rows, starts, at, past, self.cache, self.H, most, Q_out=q)
        assert t.equal(rows.view(t.int16), before.view(t.int16))
        assert np.array_equal(q[:total].cpu().numpy().view(np.uint16), y[:, :self.H].reshape(total, -1).view(np.uint16))
        self.note(counts, y)
        if attend:
            B.sqap_cache8_attention(q, starts, past, self.cache, self.H, most, o)
            self.check(o[:total].cpu().numpy(), y, counts, True)
            assert bool((o[total:] == 9).all())
        assert bool((q[total:] == 9).all())
        self.past = (self.past + np.asarray(counts)).astype(np.int32)
        return y

    def check(self, o, y, counts, single_half):
        at, group = 0, self.H // self.kv
        for b, n in enumerate(counts):
            if n == 0:
                continue
            sees = self.past[b] + np.arange(n)
            for h in range(self.kv):
                k, v = R.held(self.k[b][:, h]), R.held(self.v[b][:, h])
                for j in range(group):
                    head = h * group + j
                    got = o[at:at + n, head * self.d:(head + 1) * self.d].astype(np.float64)
                    with np.errstate(invalid="ignore"):
                        want, mass, off = R.attend(y[at:at + n, head].astype(np.float64), k, v, sees)
                    assert np.array_equal(np.isnan(got), np.isnan(want)), (b, head)
                    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), (b, head)
                    fine = np.isfinite(want)
                    v_top = np.abs(v[np.isfinite(v)]).max() if np.isfinite(v).any() else 0.0
                    far = np.abs(np.where(fine, got - np.where(fine, want, 0.0), 0.0))
                    limit = R.attention_bound(np.where(fine, want, 0.0), mass, np.where(np.isfinite(off), off, 0.0), k.shape[0], v_top, single_half)
                    assert np.all((far <= limit) | ~fine), (b, head, float(np.nanmax(far / limit)))
            at += n

    def decode(self, x=None, longest=None, workspace=None, active=None):
        t, G = self.t, self.G
        batch = len(self.past)
        x = self.rows(batch) if x is None else x
        y = self.turned(x, self.past)
        o = t.full((batch, self.H * self.d), 9.0, dtype=t.float16, device=G.DEV)
        longest = int(self.past.max()) + 1 if longest is None else longest
        ws = t.zeros((B.sqap_cache8_workspace_bytes(batch, self.H, self.kv, self.d, longest),), dtype=t.uint8, device=G.DEV) if workspace is None else workspace
        B.sqap_cache8_decode_attention(G.to_dev(x.reshape(batch, -1)), G.to_dev(self.past), G.to_dev(self.past), self.cache, self.H, o, ws, longest)
        ones = [1] * batch
        self.note(ones, y)
        self.check(o.cpu().numpy(), y, ones, False)
        if ws.numel():
            assert int(ws[:4 * batch * self.H].max()) == 0, "a counter was not put back"
        self.past += 1
        return o

    def check_contents(self):
        t, G = self.t, self.G
        batch, most = len(self.past), int(self.past.max()) + 3
        out = t.full((batch * most, 2 * self.kv * self.d + 8), 5.0, dtype=t.float16, device=G.DEV)
        B.sqap_cache8_read(self.cache, G.to_dev(self.past), 0, most, out[:, :2 * self.kv * self.d])
        got = out.cpu().numpy()
        assert np.all(got[:, -8:] == 5.0)
        got = got[:, :-8].reshape(batch, most, 2, self.kv, self.d)
        for b, n in enumerate(self.past):
            for which, x in enumerate((self.k[b], self.v[b])):
                for h in range(self.kv):
                    want = R.held(x[:, h])
                    full = n // 64 * 64
                    want[:full] = np.float32(want[:full])           # code times scale in binary32
                    assert np.array_equal(got[b, :n, which, h], want.astype(np.float16), equal_nan=True), (b, which, h)
            assert not got[b, n:].any()

    def state(self):
        """The parts of the buffers that hold something."""
        parts = []
        for b, n in enumerate(self.past):
            parts += [self.cache.codes[b, :, :n // 64], self.cache.scales[b, :, :n // 64], self.cache.tail[b, :, :, :n % 64]]
        return [p.clone().cpu() for p in parts]


@pytest.fixture(params=["few", "many"])
def announced(request, monkeypatch):
    """With many rows announced attention goes by tiles of 128 rows, with few by tiles of 16; what comes out is the same."""
    monkeypatch.setattr(Model, "most", 0 if request.param == "few" else 128 * 97)


CASES = [  # H, kv, d, then rows per sequence of one call after the other
    (1, 1, 64, [[1]]),
    (2, 2, 128, [[5], [1], [70]]),
    (4, 1, 64, [[64, 1], [63, 64], [2, 0], [1, 200]]),
    (8, 2, 128, [[129, 60, 3], [1, 4, 62], [0, 64, 190]]),
    (6, 2, 64, [[300], [33]]),
    (32, 1, 128, [[10, 65], [120, 1]]),
    (20, 1, 64, [[7, 7], [121, 1]]),
    (3, 3, 128, [[513, 200], [100, 512]]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(CASES)))
def test_prompts(G, case, announced):
    H, kv, d, calls = CASES[case]
    m = Model(G, len(calls[0]), H, kv, d, 64 * 18, seed=case)
    for counts in calls:
        m.append(counts)
    m.check_contents()


@pytest.mark.gpu
@pytest.mark.parametrize("H,kv,d", [(1, 1, 128), (4, 4, 64), (4, 2, 128), (6, 2, 64), (8, 1, 64), (16, 1, 128), (20, 1, 128), (33, 1, 64)])
@pytest.mark.parametrize("past", [[0, 1], [62, 63, 64], [65, 0, 127], [500, 255, 256], [3000, 17, 191]])
def test_single_rows(G, H, kv, d, past):
    m = Model(G, len(past), H, kv, d, 64 * 48, seed=H * d + past[0])
    m.append(past, attend=False)
    m.decode()
    m.decode(longest=64)                                                  # how the work is split is not what it gives
    m.decode(longest=100000)
    m.check_contents()


@pytest.mark.gpu
def test_contents_do_not_depend_on_the_calls(G, announced):
    H, kv, d = 4, 2, 128
    x = np.random.default_rng(3).standard_normal((150, H + 2 * kv, d)).astype(np.float16)
    states = []
    for split in ([150], [64, 86], [1, 62, 1, 1, 85], [100, 28, 22], [149, 1]):
        m = Model(G, 1, H, kv, d, 192)
        at = 0
        for n in split:
            if n == 1:
                m.decode(x[at:at + 1])
            else:
                m.append([n], x[at:at + n], attend=False)
            at += n
        states.append(m.state())
    m = Model(G, 1, H, kv, d, 192)
    for i in range(150):
        m.decode(x[i:i + 1])
    states.append(m.state())
    for s in states[1:]:
        assert all(a.numpy().tobytes() == b.numpy().tobytes() for a, b in zip(states[0], s))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_sizes_that_differ_between_blocks(G, d, announced):
    """Values of blocks between 2^-10 and 2^10, zeros, keys so large that one position takes it all, and halfway quotients."""
    m = Model(G, 1, 4, 2, d, 64 * 12, seed=9)
    for k_size, v_size in ((1, 1), (1, 2.0 ** 10), (1, 2.0 ** -10), (20, 2.0 ** -10), (1, 2.0 ** 4), (0, 1), (1, 0), (30, 1)):
        x = m.rows(64, k_size, v_size)
        m.append([64], x)
    x = m.rows(64)
    x[:, m.H:] = (np.round(x[:, m.H:].astype(np.float64) * 40) / 128).astype(np.float16)
    x[0, m.H:, 0] = np.float16(127 / 64)                                  # 127 x / amax = 64 x: halfway at odd multiples of 1/128
    m.append([64], x, pos=np.zeros(64))
    m.decode(m.rows(1, 1, 2.0 ** 8))
    m.decode(m.rows(1, 40, 2.0 ** -8))
    m.check_contents()


@pytest.mark.gpu
def test_zero_values_give_zero(G, announced):
    m = Model(G, 1, 2, 1, 64, 256)
    m.append([100], m.rows(100, 1, 0))
    o = m.decode(m.rows(1, 1, 0))
    assert not o.cpu().numpy().any()


@pytest.mark.gpu
def test_values_that_are_not_finite(G, announced):
    """In the tail they reach the rows that see them; in a finished block, that head's rows that see any of it."""
    for d, where in ((64, "k"), (128, "v"), (64, "v"), (128, "k")):
        m = Model(G, 2, 4, 2, d, 64 * 6, seed=d)
        x = m.rows(150 + 70)
        lane = m.H + (m.kv if where == "v" else 0)
        x[100, lane, 3] = np.inf                                          # sequence 0, position 100: block 1, finished
        x[148, lane + 1, 5] = -np.inf                                     # position 148: the tail
        x[150 + 66, lane + 1, d - 1] = np.nan                             # sequence 1, position 66: the tail
        x[150 + 67, lane + 1, d - 1] = np.inf
        m.append([150, 70], x)
        y = m.rows(2)
        m.decode(y)
        m.append([50, 3])                                                 # (its block is finished: NaN as a whole)
        m.decode()
        m.check_contents()


@pytest.mark.gpu
def test_queries_that_are_not_finite_stay_alone(G, announced):
    m = Model(G, 1, 4, 2, 64, 256)
    x = m.rows(90)
    x[40, 1, 7] = np.nan
    x[41, 2, 7] = np.inf
    m.append([90], x)


@pytest.mark.gpu
@pytest.mark.parametrize("max_new", [1, 20, 700])
def test_more_rows_than_announced(G, max_new):
    """All outputs of such a sequence are NaN, however many; its neighbour's are what they should be."""
    import torch
    H, kv, d = 4, 2, 64
    m = Model(G, 2, H, kv, d, 1024, seed=3)
    dev = lambda a: G.to_dev(np.asarray(a, dtype=np.int32))               # noqa: E731
    n, few = 900, min(max_new, 30)
    x = m.rows(n + few)
    starts, past, pos = dev([0, n, n + few]), dev([0, 0]), dev(np.concatenate([np.arange(n), np.arange(few)]))
    q, o = (torch.full((n + few, H * d), 9.0, dtype=torch.float16, device=G.DEV) for _ in range(2))
    B.sqap_cache8_append(G.to_dev(x.reshape(n + few, -1)), starts, pos, past, m.cache, H, max_new, Q_out=q)
    B.sqap_cache8_attention(q, starts, past, m.cache, H, max_new, o)
    got = o.cpu().numpy()
    assert np.isnan(got[:n]).all() and np.isfinite(got[n:]).all()
    y = m.turned(x[n:], np.arange(few))
    m.note([0, few], y)
    m.check(got[n:], y, [0, few], True)


@pytest.mark.gpu
def test_skipped_sequences_and_rows_beside(G):
    import torch
    H, kv, d = 4, 2, 64
    m = Model(G, 4, H, kv, d, 128, seed=2)
    m.append([100, 30, 128, 64])
    before = [t.clone() for t in (m.cache.codes, m.cache.scales, m.cache.tail)]
    dev = lambda a: G.to_dev(np.asarray(a, dtype=np.int32))               # noqa: E731
    x = G.to_dev(m.rows(60).reshape(60, -1))
    o = torch.full((60, H * d), 9.0, dtype=torch.float16, device=G.DEV)
    q = torch.full_like(o, 9.0)
    # sequence 0: 29 rows do not fit; 1: a padded entry; 2: no rows; 3: more rows than max_new
    starts, past, pos = dev([3, 32, 36, 36, 57]), dev([100, -1, 128, 64]), dev(np.zeros(60))
    B.sqap_cache8_append(x, starts, pos, past, m.cache, H, 20 + 9, Q_out=q)
    B.sqap_cache8_attention(x[:, :H * d], starts, past, m.cache, H, 20, o)
    got = o.cpu().numpy()
    assert np.all(got[:3] == 9) and np.all(got[32:36] == 9) and np.all(got[57:] == 9)
    assert np.isnan(got[3:32]).all() and np.isnan(got[36:57]).all()
    for t, u in zip(before[:2], (m.cache.codes, m.cache.scales)):
        assert torch.equal(t[:3].view(torch.uint8), u[:3].view(torch.uint8))
    assert torch.equal(before[2][:3].view(torch.uint8), m.cache.tail[:3].view(torch.uint8))
    qn = q.cpu().numpy()
    assert np.all(qn[:36] == 9) and np.all(qn[57:] == 9) and np.all(qn[36:57] != 9)        # (21 rows are within that call's max_new)
    # starts out of order or beyond the rows
    for bad in ([0, 5, 3, 3, 3], [-2, 0, 0, 0, 0], [0, 0, 0, 0, 61]):
        keep = [t.clone() for t in (m.cache.codes, m.cache.scales, m.cache.tail)]
        o.fill_(9.0)
        B.sqap_cache8_append(x, dev(bad), pos, dev([128, 0, 0, 0] if bad[1] == 5 else [0, 0, 0, 0]), m.cache, H, 60)
        B.sqap_cache8_attention(x[:, :H * d], dev(bad), dev([-1, 0, 0, 0]), m.cache, H, 60, o)
        assert bool((o == 9.0).all())
        for t, u in zip(keep, (m.cache.codes, m.cache.scales, m.cache.tail)):
            assert torch.equal(t.view(torch.uint8), u.view(torch.uint8))
    # single rows: full, padded
    o.fill_(9.0)
    ws = torch.zeros((max(16, B.sqap_cache8_workspace_bytes(4, H, kv, d, 128)),), dtype=torch.uint8, device=G.DEV)
    B.sqap_cache8_decode_attention(x[:4], dev([0] * 4), dev([128, -1, 10 ** 9, -5]), m.cache, H, o[:4], ws, 128)
    got = o.cpu().numpy()
    assert np.isnan(got[0]).all() and np.all(got[1] == 9) and np.isnan(got[2]).all() and np.all(got[3:] == 9)
    for t, u in zip(keep, (m.cache.codes, m.cache.scales, m.cache.tail)):
        assert torch.equal(t.view(torch.uint8), u.view(torch.uint8))


@pytest.mark.gpu
def test_pitches_and_queries_in_place(G):
    import torch
    H, kv, d, n = 4, 2, 128, 75
    m = Model(G, 1, H, kv, d, 256, seed=4)
    x = m.rows(n)
    y = m.turned(x, np.arange(n))
    wide = torch.full((n, (H + 2 * kv) * d + 40), 3.0, dtype=torch.float16, device=G.DEV)
    rows = wide[:, 8:8 + (H + 2 * kv) * d]
    rows.copy_(G.to_dev(x.reshape(n, -1)))
    starts, past, pos = (G.to_dev(np.asarray(a, dtype=np.int32)) for a in ([0, n], [0], np.arange(n)))
    B.sqap_cache8_append(rows, starts, pos, past, m.cache, H, n, Q_out=rows[:, :H * d])
    out = torch.full((n, H * d + 16), 3.0, dtype=torch.float16, device=G.DEV)
    B.sqap_cache8_attention(rows[:, :H * d], starts, past, m.cache, H, n, out[:, :H * d])
    got = wide.cpu().numpy()
    assert np.all(got[:, :8] == 3) and np.all(got[:, -32:] == 3)
    assert np.array_equal(got[:, 8:8 + H * d].view(np.uint16), y[:, :H].reshape(n, -1).view(np.uint16))
    assert np.array_equal(got[:, 8 + H * d:-32].view(np.uint16), x[:, H:].reshape(n, -1).view(np.uint16))
    m.note([n], y)
    m.check(out.cpu().numpy()[:, :H * d], y, [n], True)
    assert bool((out[:, H * d:] == 3).all())


@pytest.mark.gpu
@pytest.mark.parametrize("H,kv,n,behind", [(4, 2, 75, 0), (8, 8, 300, 100), (32, 32, 500, 0)])
def test_outputs_over_the_queries(G, H, kv, n, behind):
    import torch
    m = Model(G, 1, H, kv, 64, 64 * 9, seed=n)
    if behind:
        m.append([behind])
    x = G.to_dev(m.rows(n).reshape(n, -1))
    starts, past, pos = (G.to_dev(np.asarray(a, dtype=np.int32)) for a in ([0, n], [behind], behind + np.arange(n)))
    B.sqap_cache8_append(x, starts, pos, past, m.cache, H, n, Q_out=x[:, :H * 64])
    apart = torch.empty((n, H * 64), dtype=torch.float16, device=G.DEV)
    B.sqap_cache8_attention(x[:, :H * 64], starts, past, m.cache, H, n, apart)
    B.sqap_cache8_attention(x[:, :H * 64], starts, past, m.cache, H, n, x[:, :H * 64])
    assert torch.equal(x[:, :H * 64], apart) and bool(torch.isfinite(apart).all())


@pytest.mark.gpu
def test_one_workspace_for_calls_of_all_sizes(G):
    """Calls of other batches, heads and lengths follow each other on one workspace, zeroed once: the sums of a small batch stay away from the
    counters of a large one."""
    import torch
    models = [Model(G, batch, H, kv, d, 64 * 48, seed=batch) for batch, H, kv, d in ((1, 8, 8, 128), (16, 32, 4, 64), (3, 4, 1, 128), (5, 40, 1, 64))]
    for m in models:
        m.append([2000 + 40 * b for b in range(len(m.past))], attend=False)
    size = max(B.sqap_cache8_workspace_bytes(len(m.past), m.H, m.kv, m.d, 64 * 40) for m in models)
    ws = torch.full((size,), 0xA5, dtype=torch.uint8, device=G.DEV)
    ws[:16384] = 0
    for m in models + models[::-1]:
        assert B.sqap_cache8_workspace_bytes(len(m.past), m.H, m.kv, m.d, 64 * 40) > 16384
        m.decode(longest=64 * 40, workspace=ws)
    assert int(ws[:16384].max()) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("base", [1e-3, 0.5, 1.0, 1e6])
def test_far_positions_and_other_bases(G, base):
    """Queries and keys turned as by sqap_rope, up to the last position that 32 bits hold and beyond 2^31 turns."""
    import torch
    H, kv, d, n = 2, 1, 64, 256
    rng = np.random.default_rng(int(base * 1000) % 97)
    x = G.to_dev(rng.standard_normal((n, (H + 2 * kv) * d)).astype(np.float16))
    pos = rng.integers(0, 2 ** 31, n)
    pos[:4] = 2 ** 31 - 1, 0, 1, 2 ** 31 - 2
    pos = G.to_dev(pos.astype(np.int32))
    want = x.clone()
    B.sqap_rope(want[:, :(H + kv) * d], pos, H + kv, d, base)
    cache, q = B.Cache8(1, 320, kv, d, device=G.DEV), torch.empty((n, H * d), dtype=torch.float16, device=G.DEV)
    one = lambda *a: G.to_dev(np.asarray(a, dtype=np.int32))              # noqa: E731
    B.sqap_cache8_append(x, one(0, n), pos, one(0), cache, H, n, Q_out=q, base=base)
    assert torch.equal(q, want[:, :H * d])
    k = want[:, H * d:(H + 1) * d].cpu().numpy()
    out = torch.empty((n, 2 * d), dtype=torch.float16, device=G.DEV)
    B.sqap_cache8_read(cache, one(n), 0, n, out)
    assert np.array_equal(out[:, :d].cpu().numpy(), np.float32(R.held(k)).astype(np.float16))
    o, ws = torch.empty((1, H * d), dtype=torch.float16, device=G.DEV), torch.zeros(0, dtype=torch.uint8, device=G.DEV)
    B.sqap_cache8_decode_attention(x[5:6], pos[:1], one(n), cache, H, o, ws, n + 1, base=base)
    row = x[5:6].clone()
    B.sqap_rope(row[:, :(H + kv) * d], pos[:1], H + kv, d, base)
    assert torch.equal(cache.tail[0, 0, 0, 0], row[0, H * d:(H + 1) * d])


@pytest.mark.gpu
def test_replayed_with_growing_lengths(G):
    """A captured single-row step is replayed with the lengths that the device holds; eager steps of another cache between."""
    import torch
    H, kv, d, batch = 8, 2, 64, 3
    a, b = Model(G, batch, H, kv, d, 2048, seed=6), Model(G, batch, H, kv, d, 2048, seed=6)
    for m in (a, b):
        m.append([1000, 61, 0], attend=False)
    longest = 1100
    ws = [torch.zeros((B.sqap_cache8_workspace_bytes(batch, H, kv, d, longest),), dtype=torch.uint8, device=G.DEV) for _ in range(2)]
    x = torch.empty((batch, (H + 2 * kv) * d), dtype=torch.float16, device=G.DEV)
    past = G.to_dev(a.past)
    o = torch.empty((batch, H * d), dtype=torch.float16, device=G.DEV)
    new = [a.rows(batch) for _ in range(5)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    x.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.sqap_cache8_decode_attention(x, past, past, a.cache, H, o, ws[0], longest)
        past.add_(1)
    for i in range(5):
        x.copy_(G.to_dev(new[i].reshape(batch, -1)))
        graph.replay()
        want = b.decode(new[i], longest=longest, workspace=ws[1])
        torch.cuda.synchronize()
        assert torch.equal(o, want)
    assert all(p.numpy().tobytes() == q.numpy().tobytes() for p, q in zip(
        b.state(), (setattr(a, "past", b.past), a.state())[1]))


@pytest.mark.gpu
def test_offsets_beyond_32_bits(G):
    """A cache whose codes take more than 4 GiB: rows appended at its end come back and are attended to."""
    import torch
    H = kv = 1
    d, n = 128, (1 << 24) + 192                                           # 4.3 GB of codes, 64 rows to a block
    m = Model.__new__(Model)
    m.t, m.G, m.H, m.kv, m.d, m.rng = torch, G, H, kv, d, np.random.default_rng(1)
    m.cache = B.Cache8(1, n, kv, d, device=G.DEV)
    m.past = np.array([n - 128], dtype=np.int32)
    x = m.rows(127)
    pos = np.arange(127)
    y = m.turned(x, pos)
    starts = G.to_dev(np.array([0, 127], dtype=np.int32))
    past = G.to_dev(m.past)
    B.sqap_cache8_append(G.to_dev(x.reshape(127, -1)), starts, G.to_dev(pos.astype(np.int32)), past, m.cache, H, 127)
    out = torch.empty((127, 2 * d), dtype=torch.float16, device=G.DEV)
    B.sqap_cache8_read(m.cache, past + 127, n - 128, 127, out)
    want = np.concatenate([R.held(y[:, 1])[:, None], R.held(y[:, 2])[:, None]], 1)
    want[:64] = np.float32(want[:64])
    assert np.array_equal(out.cpu().numpy().reshape(127, 2, d), want.astype(np.float16))
    # a query far along the first keys' direction: the rest, all zeros, has no weight
    q = (y[:64, 1].astype(np.float64).mean(0) * 400).astype(np.float16)
    row = np.concatenate([q, np.zeros(2 * d, np.float16)]).reshape(1, -1)
    o = torch.empty((1, d), dtype=torch.float16, device=G.DEV)
    ws = torch.zeros((B.sqap_cache8_workspace_bytes(1, 1, 1, d, n),), dtype=torch.uint8, device=G.DEV)
    B.sqap_cache8_decode_attention(G.to_dev(row), G.to_dev(np.zeros(1, np.int32)), past + 127, m.cache, H, o, ws, n)
    k, v = R.held(np.concatenate([y[:, 1], np.zeros((1, d), np.float16)])), R.held(np.concatenate([y[:, 2], np.zeros((1, d), np.float16)]))
    s = k @ q.astype(np.float64) / np.sqrt(d)
    p = np.exp(s - s.max())
    assert p.sum() > 1e6 * (n - 128) * np.exp(-s.max())
    want, mass, off = R.attend(q.astype(np.float64)[None], k, v, [127])
    got = o.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - want) <= R.HALF_STEP * np.abs(want) + R.HALF_TINY + (2 * off + 2.0 ** -18 + 1e-6) * mass), np.abs(got - want).max()
