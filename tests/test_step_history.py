"""A verify step under rules records its tokens in the history that the rules read, wherever the caller keeps it."""
import pytest
import torch

import test_step_operators_gpu as steps


class _Rules:
    def __init__(self, *history):
        self.history = history


def test_where_a_step_records(monkeypatch):
    """The history of the rules, unless the inputs name another one; none where there is none."""
    import __graft_entry__ as entry
    entry.build()
    import paper_2505_10526_b200 as pkg
    from paper_2505_10526_b200 import step as module
    calls = []
    monkeypatch.setattr(module.mv, "massv_history_add", lambda vocab, tokens, lens, bits, counts, status: calls.append((bits, counts)))
    s = object.__new__(pkg.VerifyStep)
    s.vocab, s.out_tokens, s.accept_len, s.dev_status = 64, None, None, None
    bits, counts, other_bits, other_counts = (torch.zeros(4, dtype=torch.int32) for _ in range(4))
    for w, want in ((dict(rules=_Rules(bits, counts)), (bits, counts)), (dict(rules=_Rules(None, None)), None), (dict(rules=None), None), (dict(rules=object()), None),
                    (dict(rules=_Rules(bits, counts), output_bits=bits), (bits, counts)), (dict(rules=_Rules(bits, counts), output_bits=bits, counts=counts), (bits, counts)),
                    (dict(rules=_Rules(bits, counts), output_bits=other_bits), (other_bits, None)), (dict(rules=_Rules(bits, counts), output_bits=other_bits, counts=other_counts), (other_bits, other_counts)),
                    (dict(rules=None, output_bits=other_bits), (other_bits, None))):
        calls.clear()
        s.record(w)
        assert len(calls) == (want is not None)
        if want is not None:
            assert calls[0][0] is want[0] and calls[0][1] is want[1]


@pytest.mark.gpu
@pytest.mark.parametrize("T", [0.0, 0.8])
@pytest.mark.parametrize("named", [(), ("output_bits",)])
def test_a_history_that_only_the_rules_hold(T, named):
    """With `rules` alone in the inputs every step still follows the tokens of the steps before it."""
    mv, step, w, s, turns, rot, g = steps._setup(T, 14)
    torch.manual_seed(3)
    for _ in range(3):
        steps._new_block(w, s, g)
        exp = steps._expected(w, s, T, turns, rot)
        before = {n: w[n].clone() for n in ("seq_lens", "counts")}
        step.run({n: v for n, v in w.items() if n not in ("output_bits", "counts") or n in named})
        steps._check(mv, step, w, s, exp, before)
