"""Beam selection: where its outputs and its workspace may lie, and where not (no GPU)."""
import ctypes

import pytest

from paper_2509_09090_amd import binding as B

BATCH, BEAMS, VOCAB = 3, 4, 1000
BYTES = dict(logits=2 * BATCH * BEAMS * VOCAB, scores=4 * BATCH * BEAMS, done=4 * BATCH * BEAMS)
OUTPUTS = ("parent", "token", "score", "done_out")


def _call(k, **at):
    """Every buffer by itself, but those of `at`."""
    need = B.sqap_beam_workspace_bytes(BATCH, BEAMS, VOCAB, k)
    names = ("logits", "scores", "done", "parent", "token", "score", "done_out", "ws")
    p = {name: (i + 1) << 20 for i, name in enumerate(names)}
    p.update(at)
    v = {name: ctypes.c_void_p(x) for name, x in p.items()}
    return B.lib().sqap_beam_select(v["logits"], VOCAB, BATCH, BEAMS, VOCAB, v["scores"], v["done"], 1, k, v["parent"], v["token"], v["score"], v["done_out"], v["ws"],
                                    need, None)


@pytest.mark.parametrize("k", [BEAMS, 6])
@pytest.mark.parametrize("name", ("logits", "scores", "done"))
@pytest.mark.parametrize("out", OUTPUTS + ("ws",))
def test_over_an_input(k, name, out):
    base = (("logits", "scores", "done").index(name) + 1) << 20
    need = B.sqap_beam_workspace_bytes(BATCH, BEAMS, VOCAB, k)
    size = need if out == "ws" else 4 * BATCH * k
    in_place = k == BEAMS and (out, name) in (("score", "scores"), ("done_out", "done"))
    step = 16 if out == "ws" else 4
    for at in (base, base + (BYTES[name] - 1) // step * step, base - (size - 1) // step * step):
        if in_place and at == base:
            continue                                                  # (that may be)
        assert _call(k, **{out: at}) == B.EINVAL, (out, name, at - base)
        assert b" lie over " in B.lib().sqap_last_error()


@pytest.mark.parametrize("k", [BEAMS, 6])
def test_over_one_another(k):
    for i, one in enumerate(OUTPUTS + ("ws",)):
        for other in (OUTPUTS + ("ws",))[:i]:
            at = (OUTPUTS.index(other) + 4) << 20
            assert _call(k, **{one: at}) == B.EINVAL, (one, other)
            assert b" lie over " in B.lib().sqap_last_error()
