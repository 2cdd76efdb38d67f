"""Tensors with fewer elements than a call would touch are refused before anything is launched; so are rules that live on no device of the call."""
import pytest
import torch

from test_rotary import mv  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def _ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


def _refused(call, good, short, match="fewer elements"):
    """call(**good) passes; with any one of ``short`` cut by one element (of its flat form) it does not."""
    call(**good)
    for name in short:
        cut = good[name].flatten()[:-1].clone()
        with pytest.raises(ValueError, match=match if isinstance(match, str) else match[name]):
            call(**dict(good, **{name: cut}))


def test_rotary_tensors(mv):
    batch, rows, heads, d = 3, 5, 2, 64
    x = torch.randn((batch, rows, heads, d), device="cuda").to(torch.bfloat16)
    out = torch.empty_like(x)
    desc = mv.rope_desc(batch, rows, heads, 0, d, axis_pairs=[10, 12, 10])
    turns = mv.massv_rope_frequencies(d)
    call = lambda **kw: mv.massv_rotary(desc, kw.pop("turns"), x, None, out, None, **kw)
    _refused(call, dict(turns=turns, positions=_ints(batch, rows, 3)), ("turns", "positions"), dict(turns="rot_dim / 2", positions="positions has fewer elements"))
    _refused(call, dict(turns=turns, seq_lens=_ints(batch), pos_delta=_ints(batch)), ("turns", "seq_lens", "pos_delta"),
             dict(turns="rot_dim / 2", seq_lens="seq_lens has fewer", pos_delta="pos_delta has fewer"))
    with pytest.raises(ValueError, match="rot_dim / 2"):                    # another model's
        call(turns=mv.massv_rope_frequencies(2 * d), seq_lens=_ints(batch))
    call(turns=turns, seq_lens=_ints(batch + 2), pos_delta=_ints(batch + 1))          # a buffer for more sequences
