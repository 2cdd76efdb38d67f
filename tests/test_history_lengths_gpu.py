"""Lengths outside [0, n_max] are reported by massv_history_add for every n_max, none included, and add no token beyond the array."""
import pytest
import torch

from test_logit_rules import mv  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch", [1, 3, 700])
@pytest.mark.parametrize("n", [0, 1, 5])
def test_lengths_out_of_range(mv, batch, n):
    vocab = 40
    tokens = torch.full((batch, n), 7, dtype=torch.int32, device="cuda")
    for at, length in ((None, 0), (batch - 1, n + 1), (0, -1), (batch // 2, 2 ** 31 - 1), (batch - 1, -2 ** 31)):
        bits, counts = torch.zeros((batch, 2), dtype=torch.int32, device="cuda"), torch.zeros((batch, vocab), dtype=torch.int32, device="cuda")
        lens, status = torch.full((batch,), n, dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
        want = torch.full((batch,), n, device="cuda")
        if at is not None:
            lens[at] = length
            want[at] = min(max(length, 0), n)
        mv.massv_history_add(vocab, tokens, lens, bits, counts, status)
        assert int(status.item()) == (0 if at is None else -1)
        assert torch.equal(counts.sum(1), want) and torch.equal(counts[:, 7].long(), want) and torch.equal(bits[:, 0], (want > 0).int() * 128) and int(bits[:, 1].sum()) == 0
