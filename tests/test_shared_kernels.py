"""Attention of prompts behind shared prefixes, by the kernels that a call reaches: what a call asks for as workspace tells them apart, and each test says
which it is about.  longest_prefix is a hint that steers the choice and nothing else."""
import numpy as np
import pytest

from paper_2509_09090_amd import binding as B
from tests.test_cache8 import BASE, P, _desc
from tests.test_shared import Shared

ALONE, TOGETHER, PARTS = "tiles of 16 by themselves", "blocks of all tiles dealt out", "prefix and own positions in parts"
FAR = 100000                                                          # a hint


def kernels(batch, groups, H, kv, d, rows, most, longest_prefix):
    """Nothing is asked for by the first, a size without rows in it by the second."""
    need = lambda n: B.sqap_cache8_shared_workspace_bytes(batch, groups, H, kv, d, n, most, 1, longest_prefix)        # noqa: E731
    return ALONE if need(rows) == 0 else TOGETHER if need(rows) == need(rows + 1) else PARTS


@pytest.fixture(scope="module")
def G():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from tests import gpu_util
    return gpu_util


# groups of three, few of them: own positions by tiles of 16 with eight wavefronts; more: by tiles of 128; many: by tiles of 16 with two
@pytest.mark.gpu
@pytest.mark.parametrize("groups,hint,by", [(2, 70, ALONE), (2, FAR, PARTS), (34, FAR, PARTS), (171, FAR, PARTS)])
def test_rows_of_another_group(G, groups, hint, by):
    """Starts that lead a sequence to rows of another group: it is skipped, and those rows are their own sequence's."""
    import torch
    H, kv, d, width = 2, 1, 64, 3
    s = Shared(G, groups, width, H, kv, d, [70, 20] + [9] * (groups - 2), seed=6)
    counts = [1, 5, 1, 2, 2, 2] + [1] * (3 * groups - 6)
    total, at = sum(counts), np.concatenate([[0], np.cumsum(counts)])
    assert kernels(3 * groups, groups, H, kv, d, total, 5, hint) == by
    before = s.own.past.copy()
    y = s.own.append(counts, pos=s.positions(counts), attend=False)
    s.own.past = before
    q = G.to_dev(np.ascontiguousarray(y[:, :H]).reshape(total, -1))
    # sequence 4 at rows 2 and 3, which are sequence 1's; at 9 .. 13, the last of them the next group's where there is one; sequence 0 beyond its group
    for starts, skipped in (({4: 2, 5: 4}, {3, 4, 5}), ({5: 14}, {4, 5}), ({1: 9}, {0, 1})):
        st = at.astype(np.int32)
        for b, row in starts.items():
            st[b] = row
        o = torch.full((total, H * d), 9.0, dtype=torch.float16, device=G.DEV)
        B.sqap_cache8_shared_attention(q, G.to_dev(st), G.to_dev(before), s.own.cache, s.prefix.cache, s.device_lengths, H, 5, o, s.workspace(total, 5, 1, hint), hint)
        got = o.cpu().numpy()
        s.check(got, y, counts, skip=skipped)
        assert all(np.all(got[at[b]:at[b + 1]] == 9) for b in skipped), starts


@pytest.mark.parametrize("rows,most,longest_prefix,none", [(20, 1, 500, True), (8, 1, 500, False), (8, 2, 500, True), (20, 1, FAR, False), (20, 0, FAR, True)])
def test_workspace_of_a_row_each(rows, most, longest_prefix, none):
    """Prompts of one row to a sequence ask for what longer ones of as little work do; a row for each of the eight sequences may be single rows', too."""
    assert (B.sqap_cache8_shared_workspace_bytes(8, 2, 32, 32, 128, rows, most, 1, longest_prefix) == 0) == none


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [[1] * 8, [1, 0, 1, 1, 0, 1, 1, 1]])
@pytest.mark.parametrize("padding", [0, 3])
def test_prompts_of_a_row_each(G, counts, padding):
    """Without a workspace; and the same with no rows announced: NaN for those there are."""
    import torch
    H, kv, d = 4, 2, 64
    s = Shared(G, 2, 4, H, kv, d, [130, 70], seed=90)
    s.own.append([9 * b for b in range(8)], attend=False)
    before, total = s.own.past.copy(), sum(counts)
    y = s.own.append(counts, pos=s.positions(counts), attend=False)
    s.own.past = before
    starts = G.to_dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
    q = torch.zeros((total + padding, H * d), dtype=torch.float16, device=G.DEV)
    q[:total] = G.to_dev(np.ascontiguousarray(y[:, :H]).reshape(total, -1))
    for most, hint in ((1, 130), (0, 130), (0, FAR)):
        o = torch.full_like(q, 9.0)
        B.sqap_cache8_shared_attention(q, starts, G.to_dev(before), s.own.cache, s.prefix.cache, s.device_lengths, H, most, o, None, hint)
        got = o.cpu().numpy()
        assert np.all(got[total:] == 9)
        if most:
            s.check(got[:total], y, counts)
        else:
            assert np.all(np.isnan(got[:total]))


PREFIX, CACHE = dict(batch=2, capacity=1024, kv_heads=2, head_dim=64), dict(batch=4, capacity=320, kv_heads=2, head_dim=64)


def _sizes(batch, capacity, kv_heads, head_dim):
    blocks = batch * kv_heads * (capacity // 64)
    return dict(codes=blocks * 128 * head_dim, scales=8 * blocks, tail=batch * kv_heads * 256 * head_dim)


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("mine", ("codes", "scales", "tail"))
@pytest.mark.parametrize("front", ("codes", "scales", "tail"))
def test_a_prefix_over_the_sequences(decode, mine, front):
    """One of the buffers over another's beginning or end (no GPU: all of these are refused)."""
    L, far = B.lib(), {x: (i + 1) << 24 for i, x in enumerate(("codes", "scales", "tail"))}
    cache = _desc(**CACHE, **far)
    size, over = _sizes(**PREFIX)[front], _sizes(**CACHE)[mine]
    for at in (far[mine], far[mine] + over - 16, far[mine] - size + 16):
        prefix = _desc(**PREFIX, **{**{x: y << 4 for x, y in far.items()}, front: at})
        need = B.sqap_cache8_shared_workspace_bytes(4, 2, 4, 2, 64, 4, 1, 320, 1000)
        if decode:
            status = L.sqap_cache8_shared_decode_attention(P, 512, P, P, 4, BASE, cache, prefix, P, 320, 1000, P, 256, P, need, None)
        else:
            status = L.sqap_cache8_shared_attention(P, 256, P, P, 4, 1, 4, cache, prefix, P, 1000, P, 256, P, need, None)
        assert status == B.EINVAL, at


@pytest.mark.gpu
def test_a_prefix_beside_the_sequences(G):
    """Prefixes and sequences in one allocation, end to end."""
    import torch
    s = Shared(G, 2, 2, 4, 2, 64, [130, 70], capacity=192, seed=91)
    for name in ("codes", "scales", "tail"):
        of = [getattr(x.cache, name) for x in (s.own, s.prefix)]
        both = torch.cat([x.flatten() for x in of])
        for model, x, part in zip((s.own, s.prefix), of, both.split([x.numel() for x in of])):
            setattr(model.cache, name, part.view(x.shape))
            setattr(model.cache._desc, name, part.data_ptr())
    s.prompt([5, 0, 70, 1])
    s.decode()
    s.own.check_contents()


# ---- blocks of all tiles dealt out over the device: tiles that are finished in one workgroup's range, that are cut, that have no rows

def _dealt(s, counts, hint=FAR, padding=3, most=None):
    rows, batch, groups = int(sum(counts)) + padding, len(s.own.past), len(s.lengths)
    return kernels(batch, groups, s.H, s.kv, s.d, rows, max(counts) if most is None else most, hint) == TOGETHER


@pytest.mark.gpu
@pytest.mark.parametrize("groups,width,H,kv,d,lengths,calls", [
    (1, 1, 64, 4, 64, [100], [[300], [140]]),
    (1, 2, 64, 2, 128, [0], [[96, 200], [130, 64]]),
    (2, 3, 32, 4, 128, [700, 130], [[200, 33, 0, 129, 64, 301], [64, 0, 31, 127, 1, 64]]),
    (3, 1, 48, 8, 64, [64, 0, 191], [[65, 100, 16], [1, 63, 128]]),
    (1, 1, 64, 64, 128, [6000], [[130], [128]]),
    (1, 3, 64, 1, 64, [3001], [[60, 70, 3], [9, 118, 2]]),
    (1, 2, 40, 2, 128, [333], [[130, 77], [205, 1]]),
    (1, 2, 64, 8, 64, [70], [[500, 600], [130, 25]]),                 # 552 tiles of 9 to 12 blocks: whole ones to a workgroup
    (2, 1, 32, 1, 128, [1, 64], [[700, 640], [1, 270]]),
])
def test_dealt_out(G, groups, width, H, kv, d, lengths, calls):
    """Outputs beside the queries and over them; behind own positions."""
    s = Shared(G, groups, width, H, kv, d, lengths, capacity=960, seed=groups + 150)
    for counts, in_place in zip(calls, (False, True)):
        assert _dealt(s, counts)
        s.prompt(counts, longest_prefix=FAR, in_place=in_place)
    s.own.check_contents()


@pytest.mark.gpu
@pytest.mark.parametrize("H,n", [(32, 110), (64, 470)])               # (mostly cut tiles; mostly whole ones)
def test_dealt_out_with_infinite_values(G, H, n):
    """Infinities and NaN in unfinished blocks of a prefix and of own positions, a prefix block of keys and a block of own values without a scale, scores
    of minus infinity over a whole prefix."""
    kv, d, lengths = 2, 64, [70, 130, 1]
    rows = np.random.default_rng(8).standard_normal((201, H + 2 * kv, d)).astype(np.float16)
    rows[66, H + kv, 3] = np.inf
    rows[69, H + kv, 3], rows[69, H + kv + 1, 7] = -np.inf, np.nan
    rows[80, H + 1, 5] = np.inf
    s = Shared(G, 3, 1, H, kv, d, lengths, capacity=512, seed=161, prefix_rows=rows)
    s.prefix.cache.tail[2, :, 0, 0, 5] = -float("inf")
    s.prefix.k[2][0, :, 5] = -np.inf
    x = s.own.rows(3 * n)
    x[n - 10, H + kv, 9] = np.inf                                     # (unfinished: seen by the rows behind it alone)
    x[n + 40, H + kv + 1, 2] = -np.inf                                # in a block that is finished
    x[3 * n - 1, H + kv + 1, 2] = np.nan
    assert n % 64 >= 10 and _dealt(s, [n] * 3)
    s.prompt([n] * 3, x=x, longest_prefix=FAR, in_place=H == 32)


@pytest.mark.gpu
def test_dealt_out_that_does_not_fit(G):
    """NaN where there is no room, more rows than announced, more in a group than announced together or a length that cannot be; padded ones, and those
    whose starts lead elsewhere, left alone."""
    import torch
    H, kv, d, width = 16, 1, 64, 2
    good = [70, 20, 64, 9, 30]
    s = Shared(G, 5, width, H, kv, d, good, capacity=192, seed=162)
    counts = [60, 40, 50, 45, 33, 70, 64, 64, 30, 90]
    before = s.own.past.copy()
    y = s.own.append(counts, pos=s.positions(counts), attend=False)
    s.own.past = before
    total, at = sum(counts), np.concatenate([[0], np.cumsum(counts)])
    q = G.to_dev(np.ascontiguousarray(y[:, :H]).reshape(total, -1))
    for most, lengths, past, starts, bad, left in (
            (100, good, {1: -1, 3: 160}, {}, {3}, {1}),
            (100, [70, -1, 64, 1000, 30], {}, {}, {2, 3, 6, 7}, set()),
            (69, good, {}, {}, {5, 9}, set()),
            (59, good, {}, {}, {0, 5, 6, 7, 8, 9}, set()),
            (100, good, {}, {3: 700}, set(), {2, 3}),
            (100, good, {}, {4: -5}, {5}, {2, 3, 4}),
            (110, good, {}, {1: 105}, set(), {0, 1}),                 # rows 100 .. 104 are the next group's
            (110, good, {}, {9: 420}, set(), {8, 9})):                # rows 420 .. 425 are the group's before
        p, st = before.copy(), at.astype(np.int32)
        for b, n in past.items():
            p[b] = n
        for b, n in starts.items():
            st[b] = n
        assert _dealt(s, counts, padding=0, most=most)
        o = torch.full((total, H * d), 9.0, dtype=torch.float16, device=G.DEV)
        B.sqap_cache8_shared_attention(q, G.to_dev(st), G.to_dev(p), s.own.cache, s.prefix.cache, G.to_dev(np.array(lengths, np.int32)), H, most, o,
                                       s.workspace(total, most, 1, FAR), FAR)
        got = o.cpu().numpy()
        for b in range(10):
            part = got[at[b]:at[b + 1]]
            assert np.all(np.isnan(part)) if b in bad else np.all(part == 9) if b in left else True, (most, starts, b)
        s.check(got, y, counts, skip=bad | left)


@pytest.mark.gpu
def test_dealt_out_and_replayed(G):
    """A captured prompt call, replayed with other rows and lengths, with eager work between the replays."""
    import torch
    H, kv, d, total = 32, 2, 128, 300
    s = Shared(G, 2, 2, H, kv, d, [500, 64], capacity=1024, seed=163)
    q, o = (torch.zeros((total, H * d), dtype=torch.float16, device=G.DEV) for _ in range(2))
    starts, past = torch.zeros((5,), dtype=torch.int32, device=G.DEV), torch.zeros((4,), dtype=torch.int32, device=G.DEV)
    ws = s.workspace(total, 200, 1, FAR)
    assert _dealt(s, [total], padding=0, most=200)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.sqap_cache8_shared_attention(q, starts, past, s.own.cache, s.prefix.cache, s.device_lengths, H, 200, o, ws, FAR)
    for counts in ([100, 60, 70, 50], [200, 0, 1, 99], [3, 2, 1, 140], [0, 0, 0, 5]):
        before, n = s.own.past.copy(), sum(counts)
        y = s.own.append(counts, pos=s.positions(counts), attend=False)
        q[:n] = G.to_dev(np.ascontiguousarray(y[:, :H]).reshape(n, -1))
        starts.copy_(G.to_dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)))
        past.copy_(G.to_dev(before))
        o.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        after, s.own.past = s.own.past, before
        s.check(o.cpu().numpy(), y, counts)
        s.own.past = after
        assert bool((o[n:] == 9).all())
