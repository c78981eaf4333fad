"""Layer buffers, caches and heads of different widths: refused before anything is launched.  No GPU."""
import pytest
import torch

from paper_2509_09090_amd import binding as B, decoder


class Reached(Exception):
    pass


def _layer(monkeypatch, cache, kv_width, head_dim=32):
    """One layer of two heads of 32 over `cache`, up to its first call of the library."""
    def reached(*args, **kw):
        raise Reached
    monkeypatch.setattr(B, "sqap_rmsnorm_quantize_act", reached)
    mx = B.Mx4Weight(None, 1, 32)
    buf = decoder.LayerBuffers(2, 64, 96, device="cpu", kv_width=kv_width, mx4=True, cache8_workspace=0)
    x, pos = torch.zeros(2, 64, dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    decoder.layer_forward(decoder.LayerWeights(mx, mx, mx, mx, x, x), buf, x, None, pos, 2, 64 // head_dim, head_dim, x, x, kv=cache, past=pos, longest=1)


@pytest.mark.parametrize("kv_heads,cache_dim,kv_width,head_dim", [(1, 32, 64, 32), (2, 32, 32, 32), (1, 64, 32, 32), (1, 64, 64, 32), (None, None, 32, 32)])
def test_widths_that_do_not_go_together(monkeypatch, kv_heads, cache_dim, kv_width, head_dim):
    """Keys of another width than the buffers' rows, heads of another size than the cache's, narrow rows without a cache that shares heads."""
    cache = None if kv_heads is None else B.Cache8(2, 64, kv_heads, cache_dim, device="cpu")
    with pytest.raises(ValueError, match="columns"):
        _layer(monkeypatch, cache, kv_width, head_dim)


@pytest.mark.parametrize("kv_heads,kv_width", [(1, 32), (2, 64), (2, None), (None, None), (None, 64)])
def test_widths_that_do(monkeypatch, kv_heads, kv_width):
    with pytest.raises(Reached):
        _layer(monkeypatch, None if kv_heads is None else B.Cache8(2, 64, kv_heads, 32, device="cpu"), kv_width)
