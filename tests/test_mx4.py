"""Microscaled 4-bit floating point: quantizer, packed weight and product against the definitions in 64 bits."""
import ctypes

import numpy as np
import pytest

from paper_2509_09090_amd import binding as B
from tests import lowbit_ref as R


# ---------------------------------------------------------------- refusals (no GPU)

def test_quantize_refusals():
    L, p = B.lib(), ctypes.c_void_p(4096)
    good = dict(X=p, ldx=64, rows=None, M=2, K=64, Xq=p, Xs=p, stream=None)
    call = lambda **kw: L.sqap_mx4_quantize(*{**good, **kw}.values())            # noqa: E731
    assert call(M=-1) == B.EINVAL
    assert call(K=0) == B.EINVAL
    assert call(ldx=63) == B.EINVAL
    for name in ("X", "Xq", "Xs"):
        assert call(**{name: None}) == B.EINVAL
    assert call(K=48) == B.EUNSUPPORTED
    assert call(K=(1 << 20) + 32, ldx=1 << 21) == B.EUNSUPPORTED
    assert call(ldx=68) == B.EUNSUPPORTED
    assert call(X=ctypes.c_void_p(4098)) == B.EUNSUPPORTED
    assert call(Xq=ctypes.c_void_p(4098)) == B.EUNSUPPORTED
    assert call(M=2 ** 31 - 1, K=4096, ldx=4096) == B.EUNSUPPORTED
    assert call(M=0, X=None, Xq=None, Xs=None) == B.OK


def test_weight_and_linear_refusals():
    L, p, h = B.lib(), ctypes.c_void_p(4096), ctypes.c_void_p(1)
    good = dict(Wq=p, Ws=p, N=4, K=32, out=ctypes.byref(h), stream=None)
    call = lambda **kw: L.sqap_mx4_weight_pack(*{**good, **kw}.values())         # noqa: E731
    assert call(N=0) == B.EINVAL and h.value is None
    assert call(K=-32) == B.EINVAL
    assert call(Wq=None) == B.EINVAL
    assert call(Ws=None) == B.EINVAL
    assert call(out=None) == B.EINVAL
    assert call(K=40) == B.EUNSUPPORTED
    assert call(N=(1 << 24) + 1) == B.EUNSUPPORTED
    assert call(Wq=ctypes.c_void_p(4104)) == B.EUNSUPPORTED
    assert L.sqap_mx4_weight_free(None) == B.OK
    junk = ctypes.cast((ctypes.c_uint32 * 64)(), ctypes.c_void_p)
    assert L.sqap_mx4_weight_free(junk) == B.EINVAL
    assert L.sqap_mx4_weight_info(junk, None, None, None) == B.EINVAL
    assert L.sqap_mx4_linear(p, p, 1, junk, p, 32, None) == B.EINVAL
    assert L.sqap_mx4_linear(p, p, 1, None, p, 32, None) == B.EINVAL
    assert b"handle" in L.sqap_last_error()


# ---------------------------------------------------------------- GPU

@pytest.fixture(scope="module")
def G():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from tests import gpu_util
    return gpu_util


def _quantize(G, x, rows=None):
    import torch
    xd = G.to_dev(x)
    m = x.shape[0] if rows is None else len(rows)
    q = torch.full((m, x.shape[1] // 2), 0x5A, dtype=torch.uint8, device=G.DEV)
    s = torch.full((m, x.shape[1] // 32), 0x5A, dtype=torch.uint8, device=G.DEV)
    B.sqap_mx4_quantize(xd, None if rows is None else G.to_dev(np.asarray(rows, dtype=np.int32)), q, s)
    return q, s


def _halves(bits):
    return np.asarray(bits, dtype=np.uint16).view(np.float16)


@pytest.mark.gpu
def test_quantizer_on_every_half(G):
    """Every half with a block of its own, next to values of its size, halfway cases among them, zeros and signs."""
    rng = np.random.default_rng(1)
    x = np.zeros((65536, 32), dtype=np.float16)
    x[:, 0] = _halves(np.arange(65536))
    with np.errstate(all="ignore"):
        share = rng.integers(-32, 33, (65536, 30)) / 32.0
        x[:, 1:31] = np.where(np.isfinite(x[:, :1]), x[:, :1].astype(np.float64) * share, 0.0).astype(np.float16)
    code, scale = R.mx4_quantize(x)
    q, s = _quantize(G, x.reshape(4096, 512))
    assert np.array_equal(s.cpu().numpy().reshape(-1), scale.reshape(-1))
    assert np.array_equal(R.unpack4(q.cpu().numpy()).reshape(-1), code.reshape(-1))


@pytest.mark.gpu
@pytest.mark.parametrize("m,k", [(1, 32), (3, 96), (1, 4096), (37, 2048), (5, 2080), (2, 11008)])
def test_quantizer_rows_and_pitches(G, m, k):
    rng = np.random.default_rng(m * k)
    wide = (rng.standard_normal((m + 9, k + 24)) * np.exp(rng.uniform(-12, 8, (m + 9, 1)))).astype(np.float16)
    wide[0, 5] = np.inf
    wide[1, :64] = 0.0
    rows = rng.integers(0, m + 9, m)
    rows[0] = 0
    import torch
    xd = G.to_dev(wide)[:, 8:8 + k]                                      # 16-byte aligned, pitch above K
    q = torch.zeros((m, k // 2), dtype=torch.uint8, device=G.DEV)
    s = torch.zeros((m, k // 32), dtype=torch.uint8, device=G.DEV)
    B.sqap_mx4_quantize(xd, G.to_dev(rows.astype(np.int32)), q, s)
    code, scale = R.mx4_quantize(wide[rows, 8:8 + k])
    assert np.array_equal(s.cpu().numpy(), scale)
    assert np.array_equal(R.unpack4(q.cpu().numpy()), code)


def _random_operand(rng, rows, k, spread=6):
    return rng.integers(0, 16, (rows, k)).astype(np.uint8), rng.integers(127 - spread, 127 + spread + 1, (rows, k // 32)).astype(np.uint8)


def _check_product(got, x, w):
    """A product is exact; a sum of K of them in binary32, in any order and with up to one rounding or truncation per term of a block
    sum and per block, is off by at most (K / 32 + 8) 2^-23 times the sum of magnitudes; then one rounding to half."""
    want, mass = x @ w.T, np.abs(x) @ np.abs(w).T
    assert np.all(np.abs(want) < 60000)
    far = np.abs(got.astype(np.float64) - want)
    assert np.all(far <= R.HALF_STEP * np.abs(want) + R.HALF_TINY + (x.shape[1] / 32 + 8) * 2.0 ** -23 * mass), float(far.max())


# every kernel, tiles that end inside rows, channels and K, single rows and channels
@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 1, 32), (1, 16, 64), (2, 17, 128), (1, 300, 11008), (8, 64, 96), (15, 65, 160), (16, 130, 1056), (5, 1001, 4096),
                                   (17, 64, 32), (33, 63, 288), (64, 257, 512), (65, 66, 544), (160, 100, 2848), (161, 65, 256), (333, 1001, 2848),
                                   (512, 64, 128), (513, 3, 96), (515, 300, 416), (768, 513, 1024), (1030, 256, 224)])
def test_product(G, m, n, k):
    import torch
    rng = np.random.default_rng(m * 7919 + n * 31 + k)
    (xc, xs), (wc, ws) = _random_operand(rng, m, k), _random_operand(rng, n, k, 3)
    xs = np.where(xs > 130, 130, xs).astype(np.uint8)
    ws = (ws - 4).astype(np.uint8)
    w = B.sqap_mx4_weight_pack(G.to_dev(R.pack4(wc)), G.to_dev(ws))
    assert (w.N, w.K) == (n, k) and w.device_bytes > n * k // 2
    out = torch.full((m + 2, n + 7), 7.0, dtype=torch.float16, device=G.DEV)
    y = out[1:m + 1, 3:3 + n]                                            # any alignment, any pitch
    B.sqap_mx4_linear(G.to_dev(R.pack4(xc)), G.to_dev(xs), w, y)
    got = out.cpu().numpy()
    w.free()
    _check_product(got[1:m + 1, 3:3 + n], R.mx4_values(xc, xs), R.mx4_values(wc, ws))
    got[1:m + 1, 3:3 + n] = 7.0
    assert np.all(got == 7.0), "something beside the outputs was written"


# enough outputs for the tiles, with one stage of K to many, odd and even numbers of them, whole and ragged
@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(100, 20011, 96), (33, 24500, 256), (130, 17000, 1312), (700, 5003, 352), (161, 9000, 768), (90, 26001, 2080),
                                   (1100, 10001, 544), (2050, 5200, 32), (1290, 8200, 1280), (515, 16500, 1024), (60, 20011, 800), (150, 20011, 800),
                                   (160, 24000, 96), (148, 22016, 1056), (200, 12300, 32)])
def test_product_of_many_outputs(G, m, n, k):
    test_product(G, m, n, k)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(60, 20011), (100, 20011), (150, 20011), (700, 5003), (1100, 10001)])
def test_tiles_keep_values_that_are_not_finite_in_their_row(G, m, n):
    test_values_that_are_not_finite_stay_in_their_row(G, m, n)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [3, 40, 100, 700])
def test_values_that_are_not_finite_stay_in_their_row(G, m, n=70):
    import torch
    rng = np.random.default_rng(m)
    k = 352
    (xc, xs), (wc, ws) = _random_operand(rng, m, k), _random_operand(rng, n, k)
    xs[m // 2, k // 32 - 1] = 255
    xs[0, 0] = 255
    ws[5, 3] = 255
    w = B.sqap_mx4_weight_pack(G.to_dev(R.pack4(wc)), G.to_dev(ws))
    y = torch.empty((m, n), dtype=torch.float16, device=G.DEV)
    B.sqap_mx4_linear(G.to_dev(R.pack4(xc)), G.to_dev(xs), w, y)
    got, want = y.cpu().numpy(), R.mx4_values(xc, xs) @ R.mx4_values(wc, ws).T
    w.free()
    assert np.array_equal(np.isnan(got), np.isnan(want))


@pytest.mark.gpu
def test_extreme_scales(G):
    """Scales at both ends of the byte, whose products leave and enter the range of a half."""
    import torch
    k = 256
    xc, wc = np.full((4, k), 2, dtype=np.uint8), np.full((3, k), 2, dtype=np.uint8)                 # ones
    xs, ws = np.full((4, k // 32), 127, dtype=np.uint8), np.full((3, k // 32), 127, dtype=np.uint8)
    xs[0], ws[0] = 0, 254                               # 2^-127 x 2^127
    xs[1], xs[2], xs[3] = 254, 135, 100                 # overflow, 65536 -> infinity, 2^-19 exact
    xc[3, 32:] = 0
    w = B.sqap_mx4_weight_pack(G.to_dev(R.pack4(wc)), G.to_dev(ws))
    y = torch.empty((4, 3), dtype=torch.float16, device=G.DEV)
    B.sqap_mx4_linear(G.to_dev(R.pack4(xc)), G.to_dev(xs), w, y)
    with np.errstate(over="ignore"):
        want = (R.mx4_values(xc, xs) @ R.mx4_values(wc, ws).T).astype(np.float16)
    assert np.array_equal(y.cpu().numpy(), want)


@pytest.mark.gpu
def test_empty_and_repeated_calls_and_streams(G):
    import torch
    rng = np.random.default_rng(5)
    m, n, k = 300, 200, 1056
    x = rng.standard_normal((m, k)).astype(np.float16)
    wv = (rng.standard_normal((n, k)) * 0.1).astype(np.float16)
    w = B.sqap_mx4_weight_pack(*_quantize(G, wv))
    q, s = _quantize(G, x)
    y = torch.empty((m, n), dtype=torch.float16, device=G.DEV)
    B.sqap_mx4_linear(q[:0], s[:0], w, y[:0])
    B.sqap_mx4_quantize(G.to_dev(x)[:0], None, q[:0], s[:0])
    B.sqap_mx4_linear(q, s, w, y)
    first = y.clone()
    # a captured quantizer and product, replayed with eager work between
    xd = G.to_dev(x)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    y2 = torch.empty_like(y)
    with torch.cuda.graph(graph, stream=side):
        B.sqap_mx4_quantize(xd, None, q, s)
        B.sqap_mx4_linear(q, s, w, y2)
    for _ in range(3):
        y2.fill_(float("nan"))
        q.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y2, first)
        B.sqap_mx4_linear(q, s, w, y)
        assert torch.equal(y, first)
    with torch.cuda.stream(side):
        y.fill_(0)
        B.sqap_mx4_linear(q, s, w, y)
    side.synchronize()
    assert torch.equal(y, first)
    (xc, xs), (wc, ws) = R.mx4_quantize(x), R.mx4_quantize(wv)
    _check_product(first.cpu().numpy(), R.mx4_values(xc, xs), R.mx4_values(wc, ws))
    w.free()
