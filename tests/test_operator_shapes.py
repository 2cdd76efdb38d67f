"""Tensors with fewer elements than a call would touch are refused before anything is launched; so are rules that live on no device of the call."""
import pytest
import torch

import test_attn_shared as attn
import test_logit_rules as rules_of
from test_rotary import mv  # noqa: F401  (a fixture)


def _ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


def _refused(call, good, short, match="fewer elements"):
    """call(**good) passes; with any one of ``short`` cut by one element (of its flat form) it does not."""
    call(**good)
    for name in short:
        cut = good[name].flatten()[:-1].clone()
        with pytest.raises(ValueError, match=match if isinstance(match, str) else match[name]):
            call(**dict(good, **{name: cut}))


@pytest.mark.gpu
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


# ---------------------------------------------------------------- rules
def _needs(batch, gamma, vocab):
    words = (vocab + 31) // 32
    return dict(allowed=batch * (gamma + 1) * words, bias_start=batch + 1, prompt_bits=batch * words, output_bits=batch * words, counts=batch * vocab, repetition=batch, frequency=batch, presence=batch)


@pytest.mark.parametrize("batch,gamma,vocab", [(1, 0, 1), (3, 2, 100), (2, 7, 4104)])
def test_rules_are_held_against_the_call(mv, batch, gamma, vocab):
    """Without a GPU: the lengths that logit_rules notes are looked at ahead of every other tensor."""
    z = torch.zeros((batch, gamma + 1, vocab))
    needs = _needs(batch, gamma, vocab)
    calls = [lambda r: mv.massv_logits_apply(gamma, r, z, z)]
    if vocab % 8 == 0:
        desc = mv.accept_desc(batch, gamma, 64, vocab, 1.0)
        calls.append(lambda r: mv.massv_accept_logits(desc, r, z, z, None, None, None, None, None, None))
    for call in calls:
        rules = mv.logit_rules()
        assert isinstance(rules, mv.LogitRules) and list(rules.sizes) == [-1] * 10 and rules.device == -1
        rules.sizes[:] = [needs.get(n, 0) for n in rules_of.NAMES]
        with pytest.raises(ValueError, match="CUDA device"):               # past the rules, at the first tensor
            call(rules)
        for i, name in enumerate(rules_of.NAMES):
            if name in needs:
                rules.sizes[i] -= 1
                with pytest.raises(ValueError, match=f"rules' {name} has fewer"):
                    call(rules)
                rules.sizes[i] += 1
        with pytest.raises(ValueError, match="CUDA device"):               # bare addresses: the caller's word
            call(mv.LogitRules())


@pytest.mark.gpu
def test_rules_of_another_batch_or_vocabulary(mv):
    batch, gamma, vocab = 4, 2, 1000
    s = rules_of._make(batch, gamma, vocab, rules_of.ALL, 5)
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")

    def apply(z, rules=rules_of._rules(mv, s), drafts=True):
        mv.massv_logits_apply(gamma, rules, z, torch.empty_like(z), s["draft_tokens"] if drafts else None, status)
    apply(s["logits"])
    apply(s["logits"][:2].contiguous())                                     # the first sequences of them
    for z in (torch.zeros((batch + 1, gamma + 1, vocab), device="cuda"), torch.zeros((batch, gamma + 1, vocab + 1), device="cuda")):
        with pytest.raises(ValueError, match="rules'"):
            apply(z, drafts=False)
    for name in _needs(batch, gamma, vocab):
        tensors = {n: s[n] for n in rules_of.NAMES}
        tensors[name] = tensors[name].flatten()[:-1].clone()
        with pytest.raises(ValueError, match=f"rules' {name} has fewer"):
            apply(s["logits"], mv.logit_rules(**tensors))
    assert int(status.item()) == 0
    rules = rules_of._rules(mv, s)
    assert rules.device == torch.cuda.current_device()
    rules.device += 1                                                       # as tensors of another device would note
    with pytest.raises(ValueError, match="current device"):
        apply(s["logits"], rules)


# ---------------------------------------------------------------- the other tensors
@pytest.mark.gpu
def test_shared_attention_tensors(mv):
    w = attn._make([3, 2], [256, 130], [10, 4], 2, 8, 2, 64, 1)
    batch, rows, hq, d = w["q"].shape
    desc = mv.attn_desc(batch, rows - 1, hq, 2, d, w["page_table"].shape[1], w["k_pages"].shape[0])
    ws = mv.alloc_workspace(mv.massv_verify_attn_shared_workspace_size(desc, 2), "cuda")
    names = ("q", "k_new", "v_new", "k_pages", "v_pages", "page_table", "seq_lens", "out", "out_f32", "lse", "dev_status")
    good = {n: w[n] for n in names[:7]}
    good.update(out=torch.empty_like(w["q"]), out_f32=torch.empty(w["q"].shape, device="cuda"), lse=torch.empty((batch, rows, hq), device="cuda"), dev_status=_ints(1))
    _refused(lambda **kw: mv.massv_verify_attn_shared(desc, w["start"], w["shared"], workspace=ws, **kw), good, names, {n: f"{n} has fewer elements" for n in names})
    assert int(good["dev_status"].item()) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("T", [0.0, 1.0])
def test_acceptance_tensors(mv, T):
    batch, gamma, vocab = 3, 2, 2048
    s = rules_of._make(batch, gamma, vocab, ("history",), 5)
    desc, rules = mv.accept_desc(batch, gamma, 64, vocab, T), rules_of._rules(mv, s)
    ws = mv.alloc_workspace(mv.massv_accept_logits_workspace_size(desc), "cuda")
    good = dict(logits=s["logits"], logits_out=torch.empty_like(s["logits"]), draft_tokens=s["draft_tokens"], draft_probs=torch.softmax(s["logits"][:, :gamma], -1).contiguous(),
                u_accept=torch.rand((batch, gamma), device="cuda"), u_sample=torch.rand((batch, gamma + 1), device="cuda"), out_tokens=_ints(batch, gamma + 1), accept_len=_ints(batch),
                probs_out=torch.empty_like(s["logits"]), dev_status=_ints(1))
    names = list(good)
    if T == 0:
        good["probs_out"] = None
        names = [n for n in names if n not in ("probs_out", "draft_probs", "u_accept", "u_sample")]          # (not read)
        for n in ("draft_probs", "u_accept", "u_sample"):
            good[n] = good[n].flatten()[:1].clone()
    _refused(lambda **kw: mv.massv_accept_logits(desc, rules, workspace=ws, **kw), good, names, {n: f"{n} has fewer elements" for n in names})
    mv.massv_accept_logits(desc, None, workspace=ws, **dict(good, logits_out=good["logits_out"].flatten()[:4]))       # without rules nothing is written there
    assert int(good["dev_status"].item()) == 0


@pytest.mark.gpu
def test_apply_and_history_tensors(mv):
    batch, gamma, vocab, n = 3, 2, 1001, 4
    s = rules_of._make(batch, gamma, vocab, ("history",), 5)
    out = torch.empty_like(s["logits"])
    apply = lambda **kw: mv.massv_logits_apply(gamma, rules_of._rules(mv, s), s["logits"], out, **kw)
    _refused(apply, dict(draft_tokens=s["draft_tokens"], dev_status=_ints(1)), ("draft_tokens", "dev_status"), dict(draft_tokens="draft_tokens has fewer", dev_status="dev_status has fewer"))
    add = lambda **kw: mv.massv_history_add(vocab, _ints(batch, n), **kw)
    good = dict(lens=_ints(batch), bits=_ints(batch, 32), counts=_ints(batch, vocab), dev_status=_ints(1))
    _refused(add, good, list(good), {name: f"{name} has fewer elements" for name in good})
    with pytest.raises(OverflowError):
        mv.massv_history_add(2 ** 32 + vocab, _ints(batch, n), None, good["bits"])
