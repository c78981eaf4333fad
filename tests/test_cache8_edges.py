"""The 8-bit cache where a call's parts meet: probabilities far below the largest, keys that are not finite behind a tile's first rows, shares
of a single row's positions that have nothing to add, and calls that announce no rows."""
import numpy as np
import pytest

from paper_2509_09090_amd import binding as B
from tests import lowbit_ref as R
from tests.test_cache8 import G, Model, announced                                            # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


class Pairs(Model):
    """Probabilities of prompts enter the second product as two halves, as those of single rows do."""

    def check(self, o, y, counts, single_half):
        super().check(o, y, counts, False)


@pytest.mark.parametrize("H,kv,d,calls", [(1, 1, 64, [[3], [20]]), (4, 1, 128, [[70, 9], [5, 60]]), (6, 3, 64, [[200], [129]]), (8, 8, 128, [[40, 100]])])
def test_prompts_keep_probabilities_in_binary32(G, announced, H, kv, d, calls):              # noqa: F811
    """Keys so small that the scores' own error is far below half a step of a half."""
    m = Pairs(G, len(calls[0]), H, kv, d, 64 * 8, seed=H)
    for counts in calls:
        m.append(counts, m.rows(sum(counts), 2.0 ** -6))


def _spread(rows):
    """One head of 64: position 0 has the score 16 * 9.375 / 8 = 18.75 and values of zero, all others the score 0 and ones."""
    x = np.zeros((rows, 3, 64), np.float16)
    x[:, 0, 0] = 16
    x[0, 1, 0] = 9.375
    x[1:, 2] = 1
    return x


def _check_spread(got, sees):
    """Outputs are t / (1 + t), t = sees * exp(-18.75) = sees * 2^-27.05.  The exponential's argument is off by its roundings in binary32 (27.05 in
    units of ln 2: 2^-20 each, a few of them), the scale of the first block's keys and values by two more; what a probability loses below the
    smallest half that it enters with is 2^-34 of the largest; one rounding to half."""
    t = sees * np.exp(-18.75)
    want = t / (1 + t)
    limit = R.HALF_STEP * want + R.HALF_TINY + 2.0 ** -16 * want + sees * 2.0 ** -34
    assert np.all(np.abs(got.astype(np.float64) - want[:, None]) <= limit[:, None]), (got[-1, :3], want[-1])


def test_many_small_probabilities_add_up_in_prompts(G, announced):                          # noqa: F811
    import torch
    n = 4100
    x, most = _spread(n), max(n, Model.most)
    dev = lambda a: G.to_dev(np.asarray(a, dtype=np.int32))                                   # noqa: E731
    cache, starts, past = B.Cache8(1, n, 1, 64, device=G.DEV), dev([0, n]), dev([0])
    q, o = (torch.zeros((most, 64), dtype=torch.float16, device=G.DEV) for _ in range(2))
    rows = torch.zeros((most, 192), dtype=torch.float16, device=G.DEV)
    rows[:n] = G.to_dev(x.reshape(n, -1))
    B.sqap_cache8_append(rows, starts, torch.zeros(most, dtype=torch.int32, device=G.DEV), past, cache, 1, most, Q_out=q)
    B.sqap_cache8_attention(q, starts, past, cache, 1, most, o)
    _check_spread(o[:n].cpu().numpy(), np.arange(n))


@pytest.mark.parametrize("longest", [64, 4101, 100000])
def test_many_small_probabilities_add_up_in_single_rows(G, longest):                        # noqa: F811
    import torch
    n = 4100
    dev = lambda a: G.to_dev(np.asarray(a, dtype=np.int32))                                   # noqa: E731
    cache = B.Cache8(1, n + 1, 1, 64, device=G.DEV)
    rows = G.to_dev(_spread(n).reshape(n, -1))
    B.sqap_cache8_append(rows, dev([0, n]), dev(np.zeros(n)), dev([0]), cache, 1, n)
    o = torch.zeros((1, 64), dtype=torch.float16, device=G.DEV)
    ws = torch.zeros((B.sqap_cache8_workspace_bytes(1, 1, 1, 64, longest),), dtype=torch.uint8, device=G.DEV)
    B.sqap_cache8_decode_attention(rows[n - 1:], dev([0]), dev([n]), cache, 1, o, ws, longest)
    _check_spread(o.cpu().numpy(), np.array([n]))


@pytest.mark.parametrize("H,kv,d,past,n,bad", [(1, 1, 64, 10, 118, 100), (1, 1, 128, 50, 80, 70), (4, 2, 64, 40, 160, 150), (3, 1, 128, 77, 200, 255),
                                               (2, 2, 64, 1, 140, 64), (8, 1, 64, 61, 70, 127)])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_keys_that_are_not_finite_leave_the_rows_before_their_block(G, announced, H, kv, d, past, n, bad, value):       # noqa: F811
    """The history ends where neither a wavefront's rows nor a tile's end with a block, so that rows which see nothing of the block with the bad
    key stand beside rows that do."""
    m = Model(G, 2, H, kv, d, 64 * 6, seed=past)
    m.append([past, 3])
    x = m.rows(n + 2)
    x[bad - past, H + kv - 1, 5] = value
    m.append([n, 2], x)
    m.check_contents()


@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_bad_key_seen_by_a_bad_query_alone(G, announced, value):                             # noqa: F811
    """Of 32 (and of 16) rows the last alone sees the block, and its query has no score that is a number."""
    m = Model(G, 1, 1, 1, 64, 64 * 4, seed=8)
    m.append([1])
    x = m.rows(140)
    x[99, 1, 5] = np.nan
    x[63, 0] = value
    m.append([140], x)


@pytest.mark.parametrize("longest", [64, 1025, 100000])
@pytest.mark.parametrize("H,kv,d", [(4, 4, 64), (20, 1, 64), (8, 2, 128)])
def test_last_share_without_a_score(G, H, kv, d, longest):                                   # noqa: F811
    """The new row opens a block, and its key is infinite: heads whose score is minus infinity see the others as if it were not there, the rest
    are NaN; how many shares there are makes no difference."""
    m = Model(G, 1, H, kv, d, 64 * 20, seed=H)
    m.append([1024], attend=False)
    x = m.rows(1)
    i = d // 2 - 1                                                        # a slow pair: turned by less than an eighth
    x[0, H:H + kv, i] = np.inf
    x[0, H:H + kv, i + d // 2] = 0
    x[0, :H, i] = x[0, :H, i + d // 2] = -2
    x[0, 1, i] = x[0, 1, i + d // 2] = 2
    o = m.decode(x, longest=longest).cpu().numpy().reshape(H, d)
    assert np.isnan(o[1]).all() and np.isfinite(np.delete(o, 1, 0)).all()


@pytest.mark.parametrize("longest", [64, 1041, 100000])
def test_infinite_value_in_a_share_without_weight(G, longest):                               # noqa: F811
    """An infinite value reaches the rows that see it however small its probability, in whichever share it lies."""
    m = Model(G, 1, 4, 4, 64, 64 * 20, seed=2)
    m.append([1024], attend=False)
    x = m.rows(1)
    x[0, 4:8] = -30 * x[0, :4]                                            # scores around -240
    x[0, 8, 3], x[0, 9, 4], x[0, 10, 5] = np.inf, -np.inf, np.nan
    o = m.decode(x, longest=longest).cpu().numpy().reshape(4, 64)
    assert o[0, 3] == np.inf and o[1, 4] == -np.inf and np.isnan(o[2, 5]) and np.isfinite(o).sum() == 4 * 64 - 3


def test_no_rows_announced(G):                                                               # noqa: F811
    """Sequences of more rows than announced have outputs of NaN, also where none are announced."""
    import torch
    m = Model(G, 3, 4, 2, 64, 128, seed=1)
    dev = lambda a: G.to_dev(np.asarray(a, dtype=np.int32))                                   # noqa: E731
    x = G.to_dev(m.rows(40).reshape(40, -1))
    o = torch.full((40, 256), 9.0, dtype=torch.float16, device=G.DEV)
    keep = m.cache.tail.clone()
    starts, past = dev([2, 33, 33, 38]), dev([0, 0, -1])
    B.sqap_cache8_append(x, starts, dev(np.arange(40)), past, m.cache, 4, 0)
    B.sqap_cache8_attention(x[:, :256], starts, past, m.cache, 4, 0, o)
    got = o.cpu().numpy()
    assert np.isnan(got[2:33]).all() and np.all(got[:2] == 9) and np.all(got[33:] == 9)
    assert torch.equal(keep.view(torch.uint8), m.cache.tail.view(torch.uint8))


LARGE = [(2.0 ** e, sign) for e in (10, 19, 21, 24.5, 25.5, 26.5, 27.5, 28.5, 29.4) for sign in (1, -1)]


def _level(n, score, sign, rng):
    """One head of 64 whose scores are all the same, near sign * score in units of ln 2, and values that all blocks have the same largest of."""
    x = np.zeros((n, 3, 64), np.float16)
    each = np.sqrt(score * np.log(2) * 8)
    x[:, 0, 0], x[:, 1, 0] = each, sign * each
    x[:, 2] = rng.uniform(-1, 1, (n, 64))
    x[:, 2, 0] = 1
    return x


@pytest.mark.parametrize("score,sign", LARGE)
def test_level_scores_of_any_size_in_prompts(G, announced, score, sign):                     # noqa: F811
    """Scores so large that a unit of their last place is more than a probability's exponent: where all are alike the outputs are means all the same."""
    import torch
    n, rng = 300, np.random.default_rng(int(score) % 1009)
    x, most = _level(n, score, sign, rng), max(n, Model.most)
    dev = lambda a: G.to_dev(np.asarray(a, dtype=np.int32))                                   # noqa: E731
    cache, starts, past = B.Cache8(1, n, 1, 64, device=G.DEV), dev([0, n]), dev([0])
    q, o = (torch.zeros((most, 64), dtype=torch.float16, device=G.DEV) for _ in range(2))
    rows = torch.zeros((most, 192), dtype=torch.float16, device=G.DEV)
    rows[:n] = G.to_dev(x.reshape(n, -1))
    B.sqap_cache8_append(rows, starts, torch.zeros(most, dtype=torch.int32, device=G.DEV), past, cache, 1, most, Q_out=q)
    B.sqap_cache8_attention(q, starts, past, cache, 1, most, o)
    got, v = o[:n].cpu().numpy().astype(np.float64), R.held(x[:, 2])
    _check_means(got, np.cumsum(v, 0) / np.arange(1, n + 1)[:, None], np.cumsum(np.abs(v), 0) / np.arange(1, n + 1)[:, None], score)


def _check_means(got, want, mass, score):
    """The unfinished block's keys are not what the finished ones' codes stand for to the last place of binary32: that parts their weights by up to 2^-22
    of the score (codes times scale, the product, its scale).  Where this is no longer small, outputs are some mean of the values, and exact for ones."""
    off = 2.0 ** -22 * score
    assert np.isfinite(got).all()
    if off < 0.01:
        assert np.all(np.abs(got - want) <= R.HALF_STEP * np.abs(want) + R.HALF_TINY + (2.0 ** -18 + 2 * off) * mass)
    assert np.all(np.abs(got) <= 1 + R.HALF_STEP) and np.all(np.abs(got[:, 0] - 1) <= R.HALF_STEP)


@pytest.mark.parametrize("longest", [64, 1025])
@pytest.mark.parametrize("score,sign", LARGE)
def test_level_scores_of_any_size_in_single_rows(G, score, sign, longest):                   # noqa: F811
    import torch
    n, rng = 1000, np.random.default_rng(int(score) % 1009)
    dev = lambda a: G.to_dev(np.asarray(a, dtype=np.int32))                                   # noqa: E731
    cache, x = B.Cache8(1, n + 1, 1, 64, device=G.DEV), _level(n + 1, score, sign, rng)
    rows = G.to_dev(x.reshape(n + 1, -1))
    B.sqap_cache8_append(rows[:n], dev([0, n]), dev(np.zeros(n)), dev([0]), cache, 1, n)
    o = torch.zeros((1, 64), dtype=torch.float16, device=G.DEV)
    ws = torch.zeros((B.sqap_cache8_workspace_bytes(1, 1, 1, 64, longest),), dtype=torch.uint8, device=G.DEV)
    B.sqap_cache8_decode_attention(rows[n:], dev([0]), dev([n]), cache, 1, o, ws, longest)
    v = R.held(x[:, 2])
    _check_means(o.cpu().numpy().astype(np.float64), v.mean(0)[None], np.abs(v).mean(0)[None], score)
