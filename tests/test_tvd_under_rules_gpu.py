"""Total variation behind an acceptance under rules, from the statistics that call leaves: against 64 bits, in workspaces of exactly the size and larger."""
import pytest
import torch

import test_logit_rules as rules_of
from test_logit_rules import mv  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("spare", [0, 1 << 22])
@pytest.mark.parametrize("which", [None, rules_of.ALL])
@pytest.mark.parametrize("batch,gamma,vocab", [(3, 2, 1024), (4, 5, 10248), (2, 3, 152064), (60, 3, 50264)])
def test_after_an_acceptance_under_rules(mv, batch, gamma, vocab, which, spare):
    T = 0.9
    s = rules_of._make(batch, gamma, vocab, which or (), vocab + gamma)
    desc = mv.accept_desc(batch, gamma, 64, vocab, T)
    g = torch.Generator(device="cuda").manual_seed(vocab)
    q = torch.softmax(4.0 * torch.randn((batch, gamma, vocab), generator=g, device="cuda"), dim=-1).contiguous()
    # (a larger buffer, such as one that massv_accept uses as well)
    ws = mv.alloc_workspace(mv.massv_accept_logits_workspace_size(desc) + spare, "cuda").fill_(0xff)
    out = torch.empty_like(s["logits"]) if which else s["logits"]
    tokens, lens, status = torch.zeros((batch, gamma + 1), dtype=torch.int32, device="cuda"), torch.zeros((batch,), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
    mv.massv_accept_logits(desc, rules_of._rules(mv, s) if which else None, s["logits"], out if which else None, s["draft_tokens"], q, torch.rand((batch, gamma), device="cuda"),
                           torch.rand((batch, gamma + 1), device="cuda"), tokens, lens, None, ws, status)
    tvd, acc = torch.full((2, batch, gamma), -7.0, device="cuda")
    mv.massv_tvd_after_accept(desc, out, q, ws, tvd, acc, mv.alloc_workspace(mv.massv_tvd_workspace_size(desc), "cuda"), status)
    assert int(status.item()) == 0
    p, q64 = torch.softmax(out[:, :gamma].double() / T, -1), q.double()
    want_tvd, want_acc = 0.5 * (p - q64).abs().sum(-1), torch.minimum(p, q64).sum(-1)
    # a row's sum: fp32 within a slice of 1,024 (exponentials 2^-22 of themselves, their arguments below 60 off by 2^-24 of them, eight roundings of the
    # partial sums), 1e-5 of the total at most
    assert float((tvd.double() - want_tvd).abs().max()) < 1e-5 and float((acc.double() - want_acc).abs().max()) < 1e-5
