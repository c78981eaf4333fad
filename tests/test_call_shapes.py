"""Calls over shared prefixes, of beam selection and of reordering: tensors that are shorter than what a call reads or writes, or not in one piece, are
refused before the library is called (no GPU)."""
import pytest
import torch

from paper_2509_09090_amd import binding as B
from tests.test_calls import Sub, recorded                            # noqa: F401  (a fixture)


class OnDevice(torch.Tensor):
    """A host tensor that says it is on the device."""
    is_cuda = True


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


def half(*s):
    return torch.zeros(s, dtype=torch.float16)


def _calls():
    cache, prefix, ws = B.Cache8(6, 100, 2, 64, device="cpu"), B.Cache8(2, 300, 2, 64, device="cpu"), torch.zeros(24)
    prompt = dict(Q=half(9, 256), starts=i32(7), past=i32(6), cache=cache, prefix=prefix, prefix_len=i32(2), H=4, max_new=5, O=half(9, 256), workspace=ws, longest_prefix=77)
    decode = dict(QKV=half(6, 512), pos=i32(6), past=i32(6), cache=cache, prefix=prefix, prefix_len=i32(2), H=4, O=half(6, 256), workspace=ws, longest=9,
                  longest_prefix=77)
    reorder = dict(cache=cache, parents=i32(2, 3), lengths=i32(6), longest=50, lengths_out=i32(6))
    select = dict(logits=half(6, 64), scores=torch.zeros(2, 3), done=i32(2, 3), eos=1, parent_out=i32(2, 4), token_out=i32(2, 4), score_out=torch.zeros(2, 4),
                  done_out=i32(2, 4).as_subclass(OnDevice), workspace=ws)
    return {f: (getattr(B, f), k) for f, k in (("sqap_cache8_shared_attention", prompt), ("sqap_cache8_shared_decode_attention", decode),
                                                ("sqap_cache8_reorder", reorder), ("sqap_beam_select", select))}


def _strided(t):
    wide = torch.zeros((*t.shape, 2), dtype=t.dtype)
    return wide[..., 0]


SHORT = [("sqap_cache8_shared_attention", name) for name in ("starts", "past", "prefix_len", "O")] + \
        [("sqap_cache8_shared_decode_attention", name) for name in ("QKV", "pos", "past", "prefix_len", "O")] + \
        [("sqap_cache8_reorder", name) for name in ("parents", "lengths", "lengths_out")] + \
        [("sqap_beam_select", name) for name in ("logits", "scores", "done", "parent_out", "token_out", "score_out", "done_out")]


@pytest.mark.parametrize("function,name", SHORT)
@pytest.mark.parametrize("kind", [torch.Tensor, Sub])
def test_too_short_or_in_pieces(recorded, function, name, kind):     # noqa: F811
    calls, _ = recorded
    call, arguments = _calls()[function]
    call(**arguments)
    assert [c[0] for c in calls] == [function]
    calls.clear()
    t = arguments[name]
    if type(t) is OnDevice:
        kind, t = OnDevice, t.as_subclass(torch.Tensor)
    bad = [t[:-1].contiguous()]
    if t.dtype != torch.float16:                                      # (rows of halves have a pitch)
        bad += [_strided(t), t[:1].expand(t.shape)]
        if t.dim() == 2:
            bad.append(t[:, :-1])
    if t.dtype == torch.int32:
        bad.append(t.to(torch.int16))
    for x in bad:
        if name == "parent_out" and x.dim() == 2 and x.is_contiguous() and x.dtype == torch.int32 and x.shape[0] == 2:
            continue                                                  # (fewer outputs)
        with pytest.raises(ValueError):
            call(**{**arguments, name: x if kind is torch.Tensor else x.as_subclass(kind)})
    assert not calls


@pytest.mark.parametrize("function", ["sqap_cache8_shared_attention", "sqap_cache8_shared_decode_attention", "sqap_cache8_reorder", "sqap_beam_select"])
def test_longer_ones_and_none(recorded, function):                    # noqa: F811
    """Longer arrays, workspaces of none and outputs that are not asked for are passed on; a workspace in pieces is not."""
    calls, _ = recorded
    call, arguments = _calls()[function]
    more = {n: torch.cat([t, t]) for n, t in arguments.items() if n in ("starts", "past", "pos", "prefix_len", "lengths", "token_out", "score_out")}
    call(**{**arguments, **more})
    none = {n: None for n in ("workspace", "lengths_out", "done", "done_out") if n in arguments}
    call(**{**arguments, **none})
    assert len(calls) == 2
    if "workspace" in arguments:
        with pytest.raises(ValueError):
            call(**{**arguments, "workspace": torch.zeros(1).expand(24)})
    assert len(calls) == 2
