"""Calls of the operators in few bits whose rows or positions are more than one launch takes (2^32 threads), and operands of different sizes."""
import ctypes

import numpy as np
import pytest

from paper_2509_09090_amd import binding as B
from tests import lowbit_ref as R
from tests.test_calls import recorded                                                        # noqa: F401  (a fixture)
from tests.test_cache8 import G                                                              # noqa: F401  (a fixture)


@pytest.mark.parametrize("codes,scales", [(16, 2), (64, 2), (32, 1), (32, 4), (16, 1)])
def test_product_of_other_channels_is_refused(recorded, codes, scales):                       # noqa: F811
    """Codes or scales that are not of the weight's 64 channels do not reach the library, which would read past them."""
    import torch
    calls, _ = recorded
    xq, xs = torch.zeros((3, codes), dtype=torch.uint8), torch.zeros((3, scales), dtype=torch.uint8)
    with pytest.raises(ValueError, match="channels"):
        B.sqap_mx4_linear(xq, xs, B.Mx4Weight(None, 5, 64), torch.zeros((3, 5), dtype=torch.float16))
    assert not calls


def test_longest_of_any_size():
    """A caller that knows no bound may name the largest number: as many shares, and the same workspace, as for any long cache."""
    for sizes in ((1, 32, 8, 128), (3, 8, 8, 64), (16, 40, 2, 64)):
        need = [B.sqap_cache8_workspace_bytes(*sizes, longest) for longest in (1 << 20, 2 ** 31 - 64, 2 ** 31 - 63, 2 ** 31 - 1)]
        assert need[0] > 0 and need == need[:1] * 4


def test_attention_of_too_many_tiles_is_refused():
    """2^24 tiles of 128 pairs, counted as if every sequence had as many rows as announced."""
    p = ctypes.c_void_p(4096)
    for batch, kv, H, max_new in ((2, 2, 4, 1 << 28), (512, 32, 32, 1 << 17), (65535, 1, 1, (1 << 15) + 1)):
        cache = B.Cache8Desc(4096, 4096, 4096, batch, 1 << 20, kv, 64)
        assert B.lib().sqap_cache8_attention(p, H * 64, p, p, 1 << 30, max_new, H, ctypes.byref(cache), p, H * 64, None) == B.EUNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("gathered", [False, True])
def test_quantizer_of_many_short_rows(G, gathered):                                          # noqa: F811
    import torch
    m, n = (1 << 24) + 5, 1009
    rng = np.random.default_rng(1)
    some = (rng.standard_normal((n, 32)) * np.exp(rng.uniform(-6, 6, (n, 1)))).astype(np.float16)
    at = torch.arange(m, device=G.DEV) % n
    x = G.to_dev(some)
    q = torch.full((m + 1, 16), 0x5A, dtype=torch.uint8, device=G.DEV)
    s = torch.full((m + 1, 1), 0x5A, dtype=torch.uint8, device=G.DEV)
    if gathered:
        B.sqap_mx4_quantize(x, at.to(torch.int32), q[:m], s[:m])
    else:
        B.sqap_mx4_quantize(x[at], None, q[:m], s[:m])
    code, scale = R.mx4_quantize(some)
    assert torch.equal(q[:m], G.to_dev(R.pack4(code))[at]) and torch.equal(s[:m], G.to_dev(scale)[at])
    assert bool((q[m] == 0x5A).all()) and bool((s[m] == 0x5A).all())


@pytest.mark.gpu
def test_reading_back_many_positions(G):                                                     # noqa: F811
    import torch
    d, n, count = 64, 100, (1 << 24) + 3
    cache = B.Cache8(2, 128, 1, d, device=G.DEV)
    x = G.to_dev(np.random.default_rng(2).standard_normal((2 * n, 3 * d)).astype(np.float16))
    one = lambda a: G.to_dev(np.asarray(a, dtype=np.int32))                                   # noqa: E731
    B.sqap_cache8_append(x, one([0, n, 2 * n]), one(np.zeros(2 * n)), one([0, 0]), cache, 1, n)
    few, many = (torch.full((2 * c, 2 * d), 5.0, dtype=torch.float16, device=G.DEV) for c in (n + 1, count))
    lengths = one([n, n - 30])
    B.sqap_cache8_read(cache, lengths, 0, n + 1, few)
    B.sqap_cache8_read(cache, lengths, 0, count, many)
    assert bool(few[:n].any()) and not bool(few[n].any())
    for b in range(2):
        part = many[b * count:(b + 1) * count]
        assert torch.equal(part[:n + 1], few[b * (n + 1):(b + 1) * (n + 1)]) and not bool(part[n + 1:].view(torch.int16).any())


@pytest.mark.gpu
def test_sampling_of_many_rows(G):                                                           # noqa: F811
    import torch
    b = (1 << 22) + 3
    gen = torch.Generator(device=G.DEV)
    gen.manual_seed(3)
    logits = torch.randn((b, 3), generator=gen, device=G.DEV).half()
    u, t = torch.rand(b, generator=gen, device=G.DEV), 0.5 + torch.rand(b, generator=gen, device=G.DEV)
    k = torch.randint(1, 4, (b,), generator=gen, device=G.DEV, dtype=torch.int32)
    p, m = 0.5 + torch.rand(b, generator=gen, device=G.DEV), 0.2 * torch.rand(b, generator=gen, device=G.DEV)
    token, prob = torch.full((b + 1,), -9, dtype=torch.int32, device=G.DEV), torch.full((b + 1,), -9.0, device=G.DEV)
    B.sqap_sample(logits, t, k, p, m, u, token[:b], prob[:b])
    for first in (0, b // 2 + 1, b - 300):
        rows = slice(first, first + 300)
        few, chance = torch.empty(300, dtype=torch.int32, device=G.DEV), torch.empty(300, device=G.DEV)
        B.sqap_sample(logits[rows], t[rows], k[rows], p[rows], m[rows], u[rows], few, chance)
        assert torch.equal(few, token[rows]) and torch.equal(chance, prob[rows])
    assert int(token[:b].min()) >= 0 and int(token[b]) == -9 and float(prob[b]) == -9.0
