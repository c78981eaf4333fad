"""The operators in few bits together, as a decoder over them runs: layers of microscaled weights and 8-bit caches, the vocabulary head and
sampling, call by call against the definitions in 64 bits on what the call was given, and as a captured step against the eager one.
And their argument marshalling."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2509_09090_amd import binding as B, decoder
from tests import lowbit_ref as R

from tests.test_calls import recorded                              # noqa: F401  (a fixture)
from tests.test_mx4 import _check_product


# ---------------------------------------------------------------- no GPU

def test_arguments_reach_the_library(recorded):                    # noqa: F811
    calls, _ = recorded
    half = lambda *s: torch.zeros(s, dtype=torch.float16)            # noqa: E731
    x, wide = half(6, 64), half(6, 200)[:, :64]
    u8, s8, i32, f32, ws = (torch.zeros(s, dtype=t) for s, t in (((6, 32), torch.uint8), ((6, 2), torch.uint8), ((4,), torch.int32),
                                                               ((6,), torch.float32), ((24,), torch.float32)))
    cache = B.Cache8(3, 100, 2, 64, device="cpu")
    assert (cache.capacity, cache.codes.shape[2]) == (128, 2)
    p = lambda t: t.data_ptr()                                       # noqa: E731
    desc = ctypes.addressof(cache._desc)
    at = lambda a: ctypes.cast(a, ctypes.c_void_p).value             # noqa: E731

    def expect(name, *args):
        got_name, got = calls.pop()
        assert not calls and got_name == name
        assert tuple(at(a) if isinstance(a, ctypes.POINTER(B.Cache8Desc)) else a for a in got) == args

    B.sqap_mx4_quantize(wide, i32, u8, s8)
    expect("sqap_mx4_quantize", p(wide), 200, p(i32), 4, 64, p(u8), p(s8), 0x77)
    B.sqap_mx4_quantize(wide, None, u8, s8, stream=3)
    expect("sqap_mx4_quantize", p(wide), 200, None, 6, 64, p(u8), p(s8), 3)
    w = B.Mx4Weight(None, 5, 64)
    B.sqap_mx4_linear(u8, s8, w, wide)
    expect("sqap_mx4_linear", p(u8), p(s8), 6, None, p(wide), 200, 0x77)
    B.sqap_cache8_append(wide, i32, f32, ws, cache, 8, 5, base=500.5)
    expect("sqap_cache8_append", p(wide), 200, p(i32), p(f32), p(ws), 6, 5, 8, 500.5, desc, None, 0, 0x77)
    B.sqap_cache8_append(wide, i32, f32, ws, cache, 8, 5, Q_out=x)
    expect("sqap_cache8_append", p(wide), 200, p(i32), p(f32), p(ws), 6, 5, 8, 10000.0, desc, p(x), 64, 0x77)
    B.sqap_cache8_attention(wide, i32, f32, cache, 8, 5, x, stream=7)
    expect("sqap_cache8_attention", p(wide), 200, p(i32), p(f32), 6, 5, 8, desc, p(x), 64, 7)
    B.sqap_cache8_decode_attention(wide, i32, f32, cache, 8, x, ws, 77)
    expect("sqap_cache8_decode_attention", p(wide), 200, p(i32), p(f32), 8, 10000.0, desc, 77, p(x), 64, p(ws), 96, 0x77)
    B.sqap_sample(wide, f32, i32, None, ws, f32, i32)
    expect("sqap_sample", p(wide), 200, 6, 64, p(f32), p(i32), None, p(ws), p(f32), p(i32), None, 0x77)
    B.sqap_sample(wide, None, None, f32, None, f32, i32, ws, stream=2)
    expect("sqap_sample", p(wide), 200, 6, 64, None, None, p(f32), None, p(f32), p(i32), p(ws), 2)
    with pytest.raises(ValueError):
        B.sqap_sample(half(2, 3, 8), None, None, None, None, f32, i32)
    with pytest.raises(IndexError):
        B.sqap_mx4_quantize(half(6), None, u8, s8)
    with pytest.raises(TypeError):
        B.sqap_cache8_attention(wide, i32, f32, cache, 8.5, 5, x)


def test_layer_refusals():
    mx, plain = B.Mx4Weight(None, 1, 32), B.Weight(None, 1, 1)
    buf = decoder.LayerBuffers(2, 64, 96, device="cpu", kv_width=32, mx4=True)
    assert buf.qkv.shape == (2, 128) and buf.hs.shape == (2, 3)
    x, pos = torch.zeros(2, 64, dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    layer = lambda w, **kw: decoder.layer_forward(decoder.LayerWeights(w, w, w, w, x, x), buf, x, None, pos, 2, 2, 32, x, x, **kw)      # noqa: E731
    cache = B.Cache8(2, 64, 1, 32, device="cpu")
    for w, kw in ((mx, dict(rotate=True)), (mx, dict(fold_quantizer=True)), (plain, dict(fold_quantizer=True, kv=cache))):
        with pytest.raises(ValueError):
            layer(w, **kw)
    other = B.Cache8(3, 64, 1, 32, device="cpu")
    with pytest.raises(ValueError):
        decoder._cache8_attention(buf, buf.qkv, buf.attn, pos, 2, 2, other, pos, None, 0, 1, None)
    with pytest.raises(ValueError):
        decoder._cache8_attention(buf, buf.qkv, buf.attn, pos[:1], 2, 2, cache, pos, None, 0, 1, None)


# ---------------------------------------------------------------- GPU

HIDDEN, H, KV, D, FFN, VOCAB, LAYERS, BATCH, LONGEST = 256, 4, 2, 64, 352, 1003, 2, 3, 192


@pytest.fixture(scope="module")
def G():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from tests import gpu_util
    return gpu_util


class Net:
    """A small decoder: embeddings, layers, final norm, head.  `mx4`: weights in microscaled floating point, or else in W4A4."""

    def __init__(self, G, mx4=True, seed=0):
        rng = np.random.default_rng(seed)
        self.G, self.mx4, self.held = G, mx4, {}
        dev = lambda a: G.to_dev(a.astype(np.float16))              # noqa: E731
        gain = lambda: dev(1 + 0.1 * rng.standard_normal(HIDDEN))   # noqa: E731
        self.table = dev(rng.standard_normal((VOCAB, HIDDEN)))
        self.weights = [decoder.LayerWeights(*(self.pack(rng, n, k) for n, k in (((H + 2 * KV) * D, HIDDEN), (HIDDEN, HIDDEN), (2 * FFN, HIDDEN), (HIDDEN, FFN))),
                                             gain(), gain()) for _ in range(LAYERS)]
        self.gamma, self.head = gain(), self.pack(rng, VOCAB, HIDDEN, mx4=True)
        ws = B.sqap_cache8_workspace_bytes(BATCH, H, KV, D, LONGEST)
        self.buf = decoder.LayerBuffers(256, HIDDEN, FFN, device=G.DEV, kv_width=KV * D, mx4=mx4, cache8_workspace=ws)
        e = lambda *s, t=torch.float16: torch.empty(s, dtype=t, device=G.DEV)        # noqa: E731
        self.x, self.d, self.y, self.logits = e(256, HIDDEN), e(256, HIDDEN), e(BATCH, HIDDEN), e(BATCH, VOCAB)
        self.xq, self.xs = e(BATCH, HIDDEN // 2, t=torch.uint8), e(BATCH, HIDDEN // 32, t=torch.uint8)

    def pack(self, rng, n, k, mx4=None):
        G = self.G
        w = G.to_dev((rng.standard_normal((n, k)) * 3 / np.sqrt(k)).astype(np.float16))
        if self.mx4 if mx4 is None else mx4:
            q, s = torch.empty((n, k // 2), dtype=torch.uint8, device=G.DEV), torch.empty((n, k // 32), dtype=torch.uint8, device=G.DEV)
            B.sqap_mx4_quantize(w, None, q, s)
            packed = B.sqap_mx4_weight_pack(q, s)
            self.held[packed.handle.value] = R.mx4_values(R.unpack4(q.cpu().numpy()), s.cpu().numpy())
            return packed
        q, s = torch.empty((n, k // 2), dtype=torch.uint8, device=G.DEV), torch.empty((n,), dtype=torch.float16, device=G.DEV)
        B.sqap_quantize_weight(w, q, s)
        return B.sqap_weight_pack(q, s)

    def caches(self):
        return [B.Cache8(BATCH, LONGEST, KV, D, device=self.G.DEV) for _ in range(LAYERS)]

    def forward(self, tokens, pos, caches, past, last_rows, starts=None, max_new=0):
        """tokens [M] -> logits of rows last_rows (None: all)."""
        m = pos.numel()
        x, d = self.x[:m], self.d[:m]
        for i, (w, kv) in enumerate(zip(self.weights, caches)):
            decoder.layer_forward(w, self.buf, self.table if i == 0 else x, None if i == 0 else d, pos, BATCH, H, D, x, d,
                                  rows=tokens if i == 0 else None, kv=kv, past=past, starts=starts, max_new=max_new, longest=LONGEST)
        if last_rows is None:
            B.sqap_rmsnorm_quantize_act(x, None, self.gamma, 1e-5, None, None, delta=d, y_out=self.y)
        else:
            B.sqap_rmsnorm_quantize_act(x[last_rows].contiguous(), None, self.gamma, 1e-5, None, None, delta=d[last_rows].contiguous(), y_out=self.y)
        B.sqap_mx4_quantize(self.y, None, self.xq, self.xs)
        B.sqap_mx4_linear(self.xq, self.xs, self.head, self.logits)
        return self.logits

    def free(self):
        for w in self.weights:
            w.free()
        self.head.free()


def _prompt(G, rng, counts):
    tokens = rng.integers(0, VOCAB, sum(counts)).astype(np.int32)
    pos = np.concatenate([np.arange(n) for n in counts]).astype(np.int32)
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    return G.to_dev(tokens), G.to_dev(pos), G.to_dev(starts), G.to_dev((starts[1:] - 1).astype(np.int64))


PARAMETERS = (np.array([0.0, 0.9, 1.3], np.float32), np.array([0, 40, 0], np.int32), np.array([1.0, 0.9, 0.8], np.float32),
              np.array([0.0, 0.0, 0.05], np.float32))


class Checked:
    """Stands before the binding's functions and checks each call's outputs against the definition on the inputs that it was given."""

    def __init__(self, net, monkeypatch):
        self.net, self.count, self.open = net, {}, 0
        self.keys, self.pending = {}, {}
        for name in ("sqap_mx4_quantize", "sqap_mx4_linear", "sqap_cache8_append", "sqap_cache8_attention", "sqap_cache8_decode_attention", "sqap_sample"):
            monkeypatch.setattr(B, name, self.around(name, getattr(B, name)))

    def around(self, name, call):
        def run(*args, **kw):
            keep = [a.clone() if isinstance(a, torch.Tensor) else a for a in args]
            call(*args, **kw)
            getattr(self, name[5:])(keep, args, kw)
            self.count[name] = self.count.get(name, 0) + 1
        return run

    def mx4_quantize(self, was, now, kw):
        x = was[0].cpu().numpy()
        code, scale = R.mx4_quantize(x if was[1] is None else x[was[1].cpu().numpy()])
        assert np.array_equal(R.unpack4(now[2].cpu().numpy()), code) and np.array_equal(now[3].cpu().numpy(), scale)

    def mx4_linear(self, was, now, kw):
        x = R.mx4_values(R.unpack4(was[0].cpu().numpy()), was[1].cpu().numpy())
        _check_product(now[3].cpu().numpy(), x, self.net.held[was[2].handle.value])

    def turned(self, qkv, pos):
        y = qkv.clone()
        B.sqap_rope(y[:, :(H + KV) * D], pos, H + KV, D)
        return y.cpu().numpy().reshape(-1, H + 2 * KV, D)

    def note(self, cache, y, past, starts):
        held = self.keys.setdefault(id(cache), [(np.zeros((0, KV, D), np.float16),) * 2] * BATCH)
        for b in range(BATCH):
            new = y[starts[b]:starts[b + 1]]
            k, v = (np.concatenate([old[:past[b]], part]) for old, part in zip(held[b], (new[:, H:H + KV], new[:, H + KV:])))
            held[b] = (k, v)

    def attended(self, cache, y, o, past, starts, single_half):
        o = o.cpu().numpy()
        for b in range(BATCH):
            rows = slice(starts[b], starts[b + 1])
            sees = past[b] + np.arange(starts[b + 1] - starts[b])
            for h in range(H):
                k, v = (R.held(part[:, h * KV // H]) for part in self.keys[id(cache)][b])
                want, mass, off = R.attend(y[rows, h].astype(np.float64), k, v, sees)
                far = np.abs(o[rows, h * D:(h + 1) * D].astype(np.float64) - want)
                assert np.all(far <= R.attention_bound(want, mass, off, k.shape[0], np.abs(v).max(), single_half)), (b, h)

    def cache8_append(self, was, now, kw):
        qkv, starts, pos, past, cache = was[:5]
        y = self.turned(qkv, pos)
        assert np.array_equal(kw["Q_out"].cpu().numpy().view(np.uint16), y[:, :H].reshape(-1, H * D).view(np.uint16))
        self.note(cache, y, past.cpu().numpy(), starts.cpu().numpy())

    def cache8_attention(self, was, now, kw):
        q, starts, past, cache = was[:4]
        self.attended(cache, q.cpu().numpy().reshape(-1, H, D), now[6], past.cpu().numpy(), starts.cpu().numpy(), True)

    def cache8_decode_attention(self, was, now, kw):
        qkv, pos, past, cache = was[:4]
        y, starts = self.turned(qkv, pos), np.arange(BATCH + 1)
        self.note(cache, y, past.cpu().numpy(), starts)
        self.attended(cache, y, now[5], past.cpu().numpy(), starts, False)

    def sample(self, was, now, kw):
        logits, t, k, p, m, u = (a.cpu().numpy() for a in was[:6])
        for b in range(BATCH):
            token, prob, near = R.sample(logits[b], *(float(a[b]) for a in (t,)), int(k[b]), float(p[b]), float(m[b]), float(u[b]))
            if near <= 2.0 ** -28:
                self.open += 1
                continue
            assert int(now[6][b]) == token and abs(float(now[7][b]) - prob) <= 2.0 ** -23 * prob + 2.0 ** -40


@pytest.mark.gpu
@pytest.mark.parametrize("mx4", [True, False])
def test_prompts_and_steps_call_by_call(G, monkeypatch, mx4):
    """Prompts of three lengths, more rows behind them, then single rows across the end of a block."""
    rng = np.random.default_rng(3)
    net = Net(G, mx4)
    caches, seen = net.caches(), Checked(net, monkeypatch)
    t, k, p, m = (G.to_dev(a) for a in PARAMETERS)
    token, prob = torch.empty(BATCH, dtype=torch.int32, device=G.DEV), torch.empty(BATCH, device=G.DEV)
    past = torch.zeros(BATCH, dtype=torch.int32, device=G.DEV)
    for counts in ([70, 62, 1], [3, 0, 64]):
        tokens, pos, starts, last = _prompt(G, rng, counts)
        pos += past.repeat_interleave(torch.tensor(counts, device=G.DEV))
        logits = net.forward(tokens, pos, caches, past, last.clamp_min(0), starts, max(counts))
        past += torch.tensor(counts, dtype=torch.int32, device=G.DEV)
    steps = 4
    for _ in range(steps):
        B.sqap_sample(logits, t, k, p, m, G.to_dev(rng.random(BATCH).astype(np.float32)), token, prob)
        logits = net.forward(token.clone(), past.clone(), caches, past, None)
        past += 1
    assert torch.isfinite(logits).all() and seen.open <= 1
    n = 4 * LAYERS if mx4 else 0
    assert seen.count == {"sqap_mx4_quantize": (n + 1) * (steps + 2), "sqap_mx4_linear": (n + 1) * (steps + 2), "sqap_cache8_append": 2 * LAYERS,
                          "sqap_cache8_attention": 2 * LAYERS, "sqap_cache8_decode_attention": LAYERS * steps, "sqap_sample": steps}
    net.free()


@pytest.mark.gpu
def test_captured_step_gives_the_eager_tokens(G):
    """One step of the whole decoder, the draw and the advance of the lengths in a graph: replayed it draws what the eager step draws, and
    leaves the caches bit for bit as that does; eager work of its own lies between the replays."""
    rng = np.random.default_rng(4)
    net = Net(G, seed=1)
    t, k, p, m = (G.to_dev(a) for a in PARAMETERS)
    counts = [60, 1, 126]
    tokens, pos, starts, last = _prompt(G, rng, counts)
    zero = torch.zeros(BATCH, dtype=torch.int32, device=G.DEV)
    first = torch.tensor(counts, dtype=torch.int32, device=G.DEV)
    steps = 10
    uniforms = G.to_dev(rng.random((steps, BATCH)).astype(np.float32))

    def begin():
        caches, past, u = net.caches(), first.clone(), uniforms[0].clone()
        net.forward(tokens, pos, caches, zero, last, starts, max(counts))
        token = torch.zeros(BATCH, dtype=torch.int32, device=G.DEV)
        return caches, past, u, token

    def step(caches, past, u, token):
        B.sqap_sample(net.logits, t, k, p, m, u, token)
        net.forward(token, past, caches, past, None)
        past.add_(1)

    runs = []
    for captured in (False, True):
        state = begin()
        caches, past, u, token = state
        if captured:
            graph, side, logits = torch.cuda.CUDAGraph(), torch.cuda.Stream(), net.logits.clone()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=side):
                step(*state)
            net.logits.copy_(logits)
        drawn = []
        for i in range(steps):
            u.copy_(uniforms[i])
            if captured:
                graph.replay()
                torch.cuda.synchronize()
                (net.table.float() @ net.table[:64].float().T).sum().item()
            else:
                step(*state)
            drawn.append(token.clone())
        runs.append((torch.stack(drawn), past, [[x[b, :, :n] for c in caches for b, n in enumerate((past // 64).tolist()) for x in (c.codes, c.scales)] +
                                                [c.tail[b, :, :, :n] for c in caches for b, n in enumerate((past % 64).tolist())]][0]))
    (a, past_a, held_a), (b, past_b, held_b) = runs
    assert torch.equal(a, b) and torch.equal(past_a, past_b) and past_a.tolist() == [c + steps for c in counts]
    assert int(a.min()) >= 0 and len({tuple(r) for r in a.tolist()}) > 1
    for x, y in zip(held_a, held_b):
        assert torch.equal(x, y)
    net.free()
