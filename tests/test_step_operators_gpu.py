"""Rotary positions, attention over a shared prefix, rules on logits and their history as one verify step, several steps in a row, against the same in 64 bits; eager
and as a replayed graph."""
import math

import numpy as np
import pytest
import torch

import oracle
import test_attn_shared as attn
import test_logit_rules as rules_of
from parity_util import compare_accept

pytestmark = pytest.mark.gpu


def _turn(x, lens, turns, rot):
    """Half layout, in 64 bits, rounded to bf16 as the step's buffers are."""
    rows = x.shape[1]
    pos = lens.long()[:, None] + torch.arange(rows, device="cuda")
    angle = (pos[..., None] * turns).double() * (2 * math.pi / 2.0 ** 64)
    c, s = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]
    y, n = x.double().clone(), rot // 2
    a, b = x[..., :n].double(), x[..., n:rot].double()
    y[..., :n], y[..., n:rot] = a * c - b * s, a * s + b * c
    return y


def _setup(T, seed):
    import paper_2505_10526_b200 as pkg
    mv = pkg.binding
    sizes, shared, tails, gamma, hq, hkv, d, vocab, hidden, rot = [3, 2], [400, 260], [30, 5, 90], 3, 8, 2, 64, 1032, 128, 32
    batch, rows = sum(sizes), gamma + 1
    w = attn._make(sizes, shared, tails, gamma, hq, hkv, d, seed)
    # room for a few more blocks behind every sequence
    pages, extra = w["k_pages"].shape[0], 3
    spare = torch.randn((batch * extra, hkv, 16, d), device="cuda").to(torch.bfloat16)
    w["k_pages"], w["v_pages"] = (torch.cat((w[n], spare)).contiguous() for n in ("k_pages", "v_pages"))
    table = torch.cat((w["page_table"], torch.full((batch, extra), -1, dtype=torch.int32, device="cuda")), 1).contiguous()
    for b in range(batch):
        used = (int(w["seq_lens"][b]) + rows + 15) // 16
        table[b, used:used + extra] = torch.arange(pages + extra * b, pages + extra * (b + 1), dtype=torch.int32)
    w["page_table"] = table
    s = rules_of._make(batch, gamma, vocab, rules_of.ALL, seed, 0.6)
    s["mask"][..., 5] = True
    s["allowed"] = rules_of._pack(s["mask"])
    s["counts"] = torch.where(s["c"] > 0, s["c"], torch.zeros_like(s["c"])).to(torch.int32)
    g = torch.Generator(device="cuda").manual_seed(seed)
    w.update(group_start=w["start"], shared_lens=w["shared"], lm_head=(torch.randn((vocab, hidden), device="cuda", generator=g) * 0.3).to(torch.bfloat16),
             hidden=torch.randn((batch, rows, hidden), device="cuda", generator=g).to(torch.bfloat16), rules=rules_of._rules(mv, s),
             output_bits=s["output_bits"], counts=s["counts"], pos_delta=-torch.arange(batch, dtype=torch.int32, device="cuda"))
    for n, shape in (("draft_probs", (batch, gamma, vocab)), ("u_accept", (batch, gamma)), ("u_sample", (batch, rows))):
        w[n] = torch.zeros(shape, device="cuda")
    w["draft_tokens"] = s["draft_tokens"]
    turns = mv.massv_rope_frequencies(rot, 1e4)
    step = pkg.VerifyStep(batch, gamma, hq, hkv, d, hidden, vocab, T, table.shape[1], w["k_pages"].shape[0], want_attn_f32=True, rope=dict(rot_dim=rot, turns=turns), n_groups=2, rules=True)
    return mv, step, w, s, turns, rot, g


def _new_block(w, s, g):
    for n in ("q", "k_new", "v_new", "hidden"):
        w[n].copy_(torch.randn(w[n].shape, device="cuda", generator=g).to(torch.bfloat16))
    w["u_accept"].copy_(torch.rand(w["u_accept"].shape, device="cuda", generator=g)); w["u_sample"].copy_(torch.rand(w["u_sample"].shape, device="cuda", generator=g))


def _expected(w, s, T, turns, rot):
    """What the step should leave, from its inputs as they are now."""
    batch, rows, vocab = s["logits"].shape
    gamma = rows - 1
    q, k = (_turn(w[n], w["seq_lens"] + w["pos_delta"], turns, rot) for n in ("q", "k_new"))
    z = (w["hidden"].double().view(-1, w["hidden"].shape[-1]) @ w["lm_head"].double().T).view(batch, rows, vocab)
    s["logits"] = z.float()
    s["c"] = w["counts"].long().clone()
    # drafts and the drafter's distribution follow the target's under the rules, row after row
    for j in range(gamma):
        p = torch.softmax(rules_of._want(s)[0][:, j] / (T or 1.0), -1)
        q_j = 0.7 * p + 0.3 * torch.roll(p, 1, -1)
        w["draft_probs"][:, j] = q_j.float()
        w["draft_tokens"][:, j] = (torch.multinomial(q_j, 1)[:, 0] if T else p.argmax(-1)).to(torch.int32)
    want, _ = rules_of._want(s)
    flat = np.ascontiguousarray(want.view(batch * rows, vocab).cpu().numpy())
    p = np.ascontiguousarray(torch.softmax(want / T, -1).view(batch * rows, vocab).cpu().numpy()) if T else None
    ref = oracle.accept(T, np.where(np.isinf(flat), -1e300, flat), p, w["draft_tokens"].cpu().numpy(), w["draft_probs"].cpu().numpy(), w["u_accept"].cpu().numpy(), w["u_sample"].cpu().numpy())
    return q, k, want, ref


def _check(mv, step, w, s, exp, before):
    q, k, want, ref = exp
    assert int(step.dev_status.item()) == 0
    for got, x in ((step.q_turned, q), (step.k_turned, k)):
        assert bool(((got.double() - x).abs() <= x.abs() * 2.0 ** -8 + 1e-5).all())
    turned = dict(w, q=step.q_turned, k_new=step.k_turned, seq_lens=before["seq_lens"])
    attn._check(turned, step.attn_out, step.attn_out_f32, step.lse)
    # logits: products of 128 bf16 pairs summed in fp32 (2^-24 each of sums below 100), then five roundings; penalties divide by 0.5 at least
    assert bool(((step.logits.double() - want).abs()[torch.isfinite(want)] <= 2e-3).all()) and torch.equal(torch.isinf(step.logits), torch.isinf(want))
    stats = compare_accept(ref, step.out_tokens.cpu().numpy(), step.accept_len.cpu().numpy(), step.gamma)
    assert stats["hard"] == 0, stats
    assert torch.equal(w["seq_lens"], before["seq_lens"] + step.accept_len)
    counts = before["counts"].clone()
    for b in range(step.B):
        for t in step.out_tokens[b, :int(step.accept_len[b])].tolist():
            counts[b, t] += 1
    assert torch.equal(w["counts"], counts) and torch.equal(w["output_bits"], rules_of._pack(counts > 0))


@pytest.mark.parametrize("T", [0.0, 0.8])
def test_steps_in_a_row(T):
    mv, step, w, s, turns, rot, g = _setup(T, 11)
    torch.manual_seed(1)
    for _ in range(4):
        _new_block(w, s, g)
        exp = _expected(w, s, T, turns, rot)
        before = {n: w[n].clone() for n in ("seq_lens", "counts")}
        step.run(w)
        _check(mv, step, w, s, exp, before)


@pytest.mark.parametrize("T", [0.0, 0.8])
def test_steps_as_a_graph(T):
    mv, step, w, s, turns, rot, g = _setup(T, 12)
    torch.manual_seed(2)
    graph = torch.cuda.CUDAGraph()
    keep = {n: w[n].clone() for n in ("seq_lens", "counts", "output_bits")}
    with torch.cuda.graph(graph):
        step.run(w)
    for n, v in keep.items():
        assert torch.equal(w[n], v)
    for _ in range(3):
        _new_block(w, s, g)
        exp = _expected(w, s, T, turns, rot)
        before = {n: w[n].clone() for n in ("seq_lens", "counts")}
        graph.replay()
        _check(mv, step, w, s, exp, before)


def test_a_rollback_keeps_lengths_and_history():
    mv, step, w, s, turns, rot, g = _setup(0.0, 13)
    _new_block(w, s, g)
    _expected(w, s, 0.0, turns, rot)
    before = {n: w[n].clone() for n in ("seq_lens", "counts", "output_bits")}
    step.run(w, commit=False)
    step.commit(w["seq_lens"], rollback=True)
    for n, v in before.items():
        assert torch.equal(w[n], v)


def test_rules_ahead_of_a_nucleus_draw():
    """A drafter's row: the rules, then massv_sample_top_p over what they leave; only allowed tokens are drawn, and the masses are those of the logits under the rules."""
    import paper_2505_10526_b200 as pkg
    mv = pkg.binding
    s = rules_of._make(9, 0, 5003, rules_of.ALL, 3, 0.05)
    want = rules_of._want(s)[0].view(9, 5003)   # before the rules go over the same memory
    z = s["logits"].view(9, 5003)
    mv.massv_logits_apply(0, rules_of._rules(mv, s), z, z)
    tokens, probs = torch.zeros((9,), dtype=torch.int32, device="cuda"), torch.empty_like(z)
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    mv.massv_sample_top_p(z, torch.rand((9,), device="cuda"), tokens, 0.9, 1.0, probs, status)
    assert int(status.item()) == 0 and bool(s["mask"][torch.arange(9), 0, tokens.long()].all())
    assert float((probs.double() - torch.softmax(want / 0.9, -1)).abs().max()) < 1e-5
