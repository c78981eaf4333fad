"""Attention behind shared prefixes, beam selection and reordering together, as a decoder that searches runs them: call by call against the definitions
on what each call was given, and as a captured step against the eager one.  And their argument marshalling."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2509_09090_amd import binding as B, decoder
from tests import lowbit_ref as R
from tests.test_beam import reference
from tests.test_calls import recorded                              # noqa: F401  (a fixture)


# ---------------------------------------------------------------- no GPU

def test_arguments_reach_the_library(recorded):                    # noqa: F811
    calls, _ = recorded
    half = lambda *s: torch.zeros(s, dtype=torch.float16)            # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)               # noqa: E731
    x, wide, ws = half(6, 64), half(6, 200)[:, :64], torch.zeros(24, dtype=torch.float32)
    pos, past, starts, length = i32(6), i32(6), i32(7), i32(2)
    cache, prefix = B.Cache8(6, 100, 2, 64, device="cpu"), B.Cache8(2, 300, 2, 64, device="cpu")
    p = lambda t: t.data_ptr()                                       # noqa: E731
    at = lambda a: ctypes.cast(a, ctypes.c_void_p).value             # noqa: E731

    def expect(name, *args):
        got_name, got = calls.pop()
        assert not calls and got_name == name
        assert tuple(at(a) if isinstance(a, ctypes.POINTER(B.Cache8Desc)) else a for a in got) == args

    own, front = ctypes.addressof(cache._desc), ctypes.addressof(prefix._desc)
    B.sqap_cache8_shared_attention(wide, starts, past, cache, prefix, length, 8, 5, x, ws, 77)
    expect("sqap_cache8_shared_attention", p(wide), 200, p(starts), p(past), 6, 5, 8, own, front, p(length), 77, p(x), 64, p(ws), 96, 0x77)
    B.sqap_cache8_shared_decode_attention(wide, pos, past, cache, prefix, length, 8, x, ws, 9, 77, base=500.5, stream=3)
    expect("sqap_cache8_shared_decode_attention", p(wide), 200, p(pos), p(past), 8, 500.5, own, front, p(length), 9, 77, p(x), 64, p(ws), 96, 3)
    parents = i32(2, 3)
    B.sqap_cache8_reorder(cache, parents, past, 50)
    expect("sqap_cache8_reorder", own, p(parents), 3, p(past), 50, None, 0x77)
    B.sqap_cache8_reorder(cache, parents, past, 50, pos, stream=4)
    expect("sqap_cache8_reorder", own, p(parents), 3, p(past), 50, p(pos), 4)
    scores, out, tokens = torch.zeros(2, 3), i32(2, 4), i32(2, 4)
    B.sqap_beam_select(wide, scores, None, -1, out, tokens, ws, None, ws)
    expect("sqap_beam_select", p(wide), 200, 2, 3, 64, p(scores), None, -1, 4, p(out), p(tokens), p(ws), None, p(ws), 96, 0x77)
    B.sqap_beam_select(wide, scores, parents, 7, out, tokens, ws, i32(1), ws, stream=5)
    assert calls.pop()[1][6:8] == (p(parents), 7)
    for wrong in (lambda: B.sqap_cache8_reorder(cache, i32(2, 2), past, 50), lambda: B.sqap_cache8_reorder(cache, i32(6), past, 50),
                  lambda: B.sqap_beam_select(half(5, 64), scores, None, -1, out, tokens, ws, None, ws),
                  lambda: B.sqap_beam_select(wide, scores, None, -1, i32(3, 4), tokens, ws, None, ws),
                  lambda: B.sqap_beam_select(wide, torch.zeros(6), None, -1, out, tokens, ws, None, ws)):
        with pytest.raises(ValueError):
            wrong()
    assert not calls


def test_a_prefix_wants_a_cache_in_8_bits():
    mx = B.Mx4Weight(None, 1, 32)
    buf = decoder.LayerBuffers(2, 64, 96, device="cpu", mx4=True)
    x, pos = torch.zeros(2, 64, dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        decoder.layer_forward(decoder.LayerWeights(mx, mx, mx, mx, x, x), buf, x, None, pos, 2, 2, 32, x, x, prefix=B.Cache8(1, 64, 1, 64, device="cpu"))


# ---------------------------------------------------------------- GPU

HIDDEN, H, KV, D, FFN, VOCAB, LAYERS, GROUPS, WIDTH, OWN, LONGEST, EOS = 256, 4, 2, 64, 352, 1003, 2, 2, 3, 128, 192, 5
BATCH = GROUPS * WIDTH


@pytest.fixture(scope="module")
def G():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from tests import gpu_util
    return gpu_util


class Net:
    """A small decoder over microscaled weights, with observations in caches of prefixes and beams in caches of their own."""

    def __init__(self, G, seed=0):
        rng = np.random.default_rng(seed)
        self.G = G
        dev = lambda a: G.to_dev(a.astype(np.float16))              # noqa: E731
        gain = lambda: dev(1 + 0.1 * rng.standard_normal(HIDDEN))   # noqa: E731
        self.table = dev(rng.standard_normal((VOCAB, HIDDEN)))
        self.weights = [decoder.LayerWeights(*(self.pack(rng, n, k) for n, k in (((H + 2 * KV) * D, HIDDEN), (HIDDEN, HIDDEN), (2 * FFN, HIDDEN), (HIDDEN, FFN))),
                                             gain(), gain()) for _ in range(LAYERS)]
        self.gamma, self.head = gain(), self.pack(rng, VOCAB, HIDDEN)
        ws = max(B.sqap_cache8_shared_workspace_bytes(BATCH, GROUPS, H, KV, D, rows, new, OWN, LONGEST) for rows, new in ((BATCH, 1), (40, 9)))
        self.buf = decoder.LayerBuffers(256, HIDDEN, FFN, device=G.DEV, kv_width=KV * D, mx4=True, cache8_workspace=ws)
        e = lambda *s, t=torch.float16: torch.empty(s, dtype=t, device=G.DEV)        # noqa: E731
        self.x, self.d, self.y, self.logits = e(256, HIDDEN), e(256, HIDDEN), e(BATCH, HIDDEN), e(BATCH, VOCAB)
        self.xq, self.xs = e(BATCH, HIDDEN // 2, t=torch.uint8), e(BATCH, HIDDEN // 32, t=torch.uint8)
        self.prefixes = [B.Cache8(GROUPS, LONGEST, KV, D, device=G.DEV) for _ in range(LAYERS)]
        self.caches = [B.Cache8(BATCH, OWN, KV, D, device=G.DEV) for _ in range(LAYERS)]
        self.select_ws = e(B.sqap_beam_workspace_bytes(GROUPS, WIDTH, VOCAB, WIDTH), t=torch.uint8)
        self.length = torch.tensor([150, 64], dtype=torch.int32, device=G.DEV)

    def pack(self, rng, n, k):
        w = self.G.to_dev((rng.standard_normal((n, k)) * 3 / np.sqrt(k)).astype(np.float16))
        q, s = torch.empty((n, k // 2), dtype=torch.uint8, device=self.G.DEV), torch.empty((n, k // 32), dtype=torch.uint8, device=self.G.DEV)
        B.sqap_mx4_quantize(w, None, q, s)
        return B.sqap_mx4_weight_pack(q, s)

    def forward(self, tokens, pos, batch, caches, last_rows=None, **kw):
        m = pos.numel()
        x, d = self.x[:m], self.d[:m]
        prefixes = self.prefixes if caches is not self.prefixes else [None] * LAYERS
        for i, (w, kv, front) in enumerate(zip(self.weights, caches, prefixes)):
            more = {} if front is None else dict(prefix=front, prefix_len=self.length, longest_prefix=150)
            decoder.layer_forward(w, self.buf, self.table if i == 0 else x, None if i == 0 else d, pos, batch, H, D, x, d,
                                  rows=tokens if i == 0 else None, kv=kv, **kw, **more)
        if caches is self.prefixes:
            return
        if last_rows is not None:
            x, d = x[last_rows].contiguous(), d[last_rows].contiguous()
        B.sqap_rmsnorm_quantize_act(x, None, self.gamma, 1e-5, None, None, delta=d, y_out=self.y)
        B.sqap_mx4_quantize(self.y, None, self.xq, self.xs)
        B.sqap_mx4_linear(self.xq, self.xs, self.head, self.logits)

    def observe(self, rng):
        """The observations into the prefixes, then a few words of its own to every beam."""
        G, n = self.G, self.length.tolist()
        ints = lambda a: G.to_dev(np.asarray(a, dtype=np.int32))     # noqa: E731
        self.forward(ints(rng.integers(0, VOCAB, sum(n))), ints(np.concatenate([np.arange(x) for x in n])), GROUPS, self.prefixes,
                     past=torch.zeros(GROUPS, dtype=torch.int32, device=G.DEV), starts=ints([0, n[0], sum(n)]), max_new=max(n))
        counts = [3, 9, 1, 5, 2, 8]
        at = np.concatenate([[0], np.cumsum(counts)])
        self.forward(ints(rng.integers(0, VOCAB, at[-1])), ints(np.concatenate([n[b // WIDTH] + np.arange(c) for b, c in enumerate(counts)])), BATCH, self.caches,
                     last_rows=G.to_dev((at[1:] - 1).astype(np.int64)), past=torch.zeros(BATCH, dtype=torch.int32, device=G.DEV), starts=ints(at),
                     max_new=max(counts))
        self.past = ints(counts)
        self.scores = torch.zeros((GROUPS, WIDTH), device=G.DEV)
        self.scores[:, 1:] -= 0.5
        self.done = torch.zeros((GROUPS, WIDTH), dtype=torch.int32, device=G.DEV)
        self.parents, self.tokens = (torch.zeros((GROUPS, WIDTH), dtype=torch.int32, device=G.DEV) for _ in range(2))
        self.after = torch.zeros_like(self.past)
        self.pos = torch.zeros_like(self.past)

    def step(self):
        """Choose, take over, go on with the chosen tokens."""
        B.sqap_beam_select(self.logits, self.scores, self.done, EOS, self.parents, self.tokens, self.scores, self.done, self.select_ws)
        for kv in self.caches:
            B.sqap_cache8_reorder(kv, self.parents, self.past, OWN, self.after)
        self.past.copy_(self.after)
        torch.add(self.past, self.length.repeat_interleave(WIDTH, output_size=BATCH), out=self.pos)
        self.forward(self.tokens.view(-1), self.pos, BATCH, self.caches, past=self.past, longest=OWN)
        self.past.add_(1)

    def free(self):
        for w in self.weights:
            w.free()
        self.head.free()


class Checked:
    """Stands before the binding's functions and checks each call's outputs against the definition on the inputs that it was given."""

    def __init__(self, monkeypatch):
        self.held, self.count = {}, {}
        for name in ("append", "attention", "shared_attention", "shared_decode_attention", "reorder"):
            monkeypatch.setattr(B, "sqap_cache8_" + name, self.around(name, getattr(B, "sqap_cache8_" + name)))
        monkeypatch.setattr(B, "sqap_beam_select", self.around("select", B.sqap_beam_select))

    def around(self, name, call):
        def run(*args, **kw):
            keep = [a.clone() if isinstance(a, torch.Tensor) else a for a in args]
            call(*args, **kw)
            getattr(self, name)(keep, args, kw)
            self.count[name] = self.count.get(name, 0) + 1
        return run

    def rows_of(self, cache):
        return self.held.setdefault(id(cache), [(np.zeros((0, KV, D), np.float16),) * 2] * cache.batch)

    def turned(self, qkv, pos):
        y = qkv.clone()
        B.sqap_rope(y[:, :(H + KV) * D], pos, H + KV, D)
        return y.cpu().numpy().reshape(-1, H + 2 * KV, D)

    def note(self, cache, y, past, starts):
        held = self.rows_of(cache)
        for b in range(cache.batch):
            new = y[starts[b]:starts[b + 1]]
            held[b] = tuple(np.concatenate([old[:past[b]], part]) for old, part in zip(held[b], (new[:, H:H + KV], new[:, H + KV:])))

    def append(self, was, now, kw):
        y = self.turned(was[0], was[2])
        self.note(was[4], y, was[3].cpu().numpy(), was[1].cpu().numpy())

    def attended(self, q, o, cache, past, starts, prefix=None):
        o = o.cpu().numpy()
        for b in range(cache.batch):
            rows = slice(starts[b], starts[b + 1])
            front = self.rows_of(prefix)[b // (cache.batch // prefix.batch)] if prefix is not None else None
            n = 0 if front is None else front[0].shape[0]
            sees = n + past[b] + np.arange(starts[b + 1] - starts[b])
            for h in range(H):
                k, v = (R.held(x[:, h * KV // H]) for x in self.rows_of(cache)[b])
                if front is not None:
                    k, v = (np.concatenate([R.held(x[:, h * KV // H]), y]) for x, y in zip(front, (k, v)))
                want, mass, off = R.attend(q[rows, h].astype(np.float64), k, v, sees)
                far = np.abs(o[rows, h * D:(h + 1) * D].astype(np.float64) - want)
                assert np.all(far <= R.attention_bound(want, mass, off, k.shape[0], np.abs(v).max(), False)), (b, h)

    def attention(self, was, now, kw):
        self.attended(was[0].cpu().numpy().reshape(-1, H, D), now[6], was[3], was[2].cpu().numpy(), was[1].cpu().numpy())

    def shared_attention(self, was, now, kw):
        self.attended(was[0].cpu().numpy().reshape(-1, H, D), now[8], was[3], was[2].cpu().numpy(), was[1].cpu().numpy(), was[4])

    def shared_decode_attention(self, was, now, kw):
        y, starts, past = self.turned(was[0], was[1]), np.arange(BATCH + 1), was[2].cpu().numpy()
        self.note(was[3], y, past, starts)
        self.attended(y, now[7], was[3], past, starts, was[4])

    def reorder(self, was, now, kw):
        held = self.rows_of(was[0])
        parents, lengths = was[1].cpu().numpy().ravel(), was[2].cpu().numpy()
        of = [b // WIDTH * WIDTH + p for b, p in enumerate(parents)]
        assert np.array_equal(now[4].cpu().numpy(), lengths[of])
        held[:] = [tuple(x[:lengths[p]] for x in held[p]) for p in of]

    def select(self, was, now, kw):
        logits, scores, done = (x.cpu().numpy() for x in was[:3])
        for b in range(GROUPS):
            want, total = reference(logits[b * WIDTH:(b + 1) * WIDTH], scores[b], done[b], EOS, WIDTH)
            parent, token, score = (now[i][b].cpu().numpy() for i in (4, 5, 6))
            assert np.allclose(score, [w[0] for w in want], rtol=2.0 ** -23, atol=2.0 ** -17)
            assert np.allclose(total[parent, token], [w[0] for w in want], rtol=0, atol=2.0 ** -17)
            assert [int(x) for x in now[7][b]] == [int(done[b][p] != 0 or t == EOS) for p, t in zip(parent, token)]


@pytest.mark.gpu
def test_search_call_by_call(G, monkeypatch):
    """Two observations of their own lengths, three beams each with words of their own, then steps across the end of a block."""
    rng = np.random.default_rng(3)
    net, seen = Net(G), Checked(monkeypatch)
    net.observe(rng)
    net.past_start = net.past.clone()
    steps = 6
    for i in range(steps):
        if i == 3:                                                    # (far enough for the sequences to finish a block)
            n = 52
            ints = lambda a: G.to_dev(np.asarray(a, dtype=np.int32))  # noqa: E731
            counts = [n - 2 * b for b in range(BATCH)]
            at = np.concatenate([[0], np.cumsum(counts)])
            small, net.buf.cache8_ws = net.buf.cache8_ws, torch.zeros(B.sqap_cache8_shared_workspace_bytes(BATCH, GROUPS, H, KV, D, int(at[-1]), n, OWN, LONGEST),
                                                                      dtype=torch.uint8, device=G.DEV)
            buf, net.buf = net.buf, decoder.LayerBuffers(512, HIDDEN, FFN, device=G.DEV, kv_width=KV * D, mx4=True, cache8_workspace=net.buf.cache8_ws.numel())
            x, d, net.x, net.d = net.x, net.d, *(torch.empty((512, HIDDEN), dtype=torch.float16, device=G.DEV) for _ in range(2))
            past, length = net.past.cpu().numpy(), net.length.cpu().numpy()
            net.forward(ints(rng.integers(0, VOCAB, at[-1])), ints(np.concatenate([length[b // WIDTH] + past[b] + np.arange(c) for b, c in enumerate(counts)])), BATCH,
                        net.caches, last_rows=G.to_dev((at[1:] - 1).astype(np.int64)), past=net.past, starts=ints(at), max_new=n)
            net.past += ints(counts)
            net.buf, net.x, net.d = buf, x, d
            net.buf.cache8_ws = small
        net.step()
    assert torch.isfinite(net.logits).all() and int(net.past.max()) > 64
    assert seen.count == {"append": 3 * LAYERS, "attention": LAYERS, "shared_attention": 2 * LAYERS, "shared_decode_attention": steps * LAYERS,
                          "reorder": steps * LAYERS, "select": steps}
    net.free()


@pytest.mark.gpu
def test_captured_search_gives_the_eager_one(G):
    """A step of the search in a graph, replayed with eager work between: the same parents, tokens and scores, the same caches."""
    runs = []
    for captured in (False, True):
        net = Net(G, seed=1)
        net.observe(np.random.default_rng(4))
        if captured:
            state = [x.clone() for x in (net.logits, net.scores, net.done, net.past)]
            caches = [[x.clone() for x in (c.codes, c.scales, c.tail)] for c in net.caches]
            graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=side):
                net.step()
            for x, y in zip((net.logits, net.scores, net.done, net.past), state):
                x.copy_(y)
            for c, kept in zip(net.caches, caches):
                for x, y in zip((c.codes, c.scales, c.tail), kept):
                    x.copy_(y)
        chosen = []
        for _ in range(70):
            if captured:
                graph.replay()
                torch.cuda.synchronize()
                (net.table.float() @ net.table[:64].float().T).sum().item()
            else:
                net.step()
            chosen.append(torch.cat([net.parents.double(), net.tokens.double(), net.scores.double(), net.done.double()]))
        held = [x for c in net.caches for b, n in enumerate(net.past.tolist()) for x in (c.codes[b, :, :n // 64], c.scales[b, :, :n // 64], c.tail[b, :, :, :n % 64])]
        runs.append((torch.stack(chosen), net.past.clone(), [x.clone() for x in held]))
        net.free()
    (a, past_a, held_a), (b, past_b, held_b) = runs
    assert torch.equal(a, b) and torch.equal(past_a, past_b)
    assert len({tuple(r.flatten().tolist()) for r in a[:, :GROUPS]}) > 1        # parents change
    for x, y in zip(held_a, held_b):
        assert torch.equal(x, y)
