"""Committed lengths just below 2^31, where the block's end would overflow: skipped and reported like any other length without room, by every attention
kernel; nothing of the other sequences changes."""
import pytest
import torch

import test_attn_shared as attn
from test_attn_shared import mv  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def _split(mv, w, kernel, chunk, window):
    batch, rows, hq, d = w["q"].shape
    desc = mv.attn_desc(batch, rows - 1, hq, w["k_new"].shape[2], d, w["page_table"].shape[1], w["k_pages"].shape[0], window=window, kv_chunk=chunk, kernel=kernel)
    ws = mv.alloc_workspace(mv.massv_verify_attn_workspace_size(desc), "cuda").fill_(0xff)
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    out, out32, lse = torch.full_like(w["q"], 3.0), torch.full(w["q"].shape, 3.0, device="cuda"), torch.full(w["q"].shape[:3], 3.0, device="cuda")
    mv.massv_verify_attn(desc, w["q"], w["k_new"], w["v_new"], w["k_pages"], w["v_pages"], w["page_table"], w["seq_lens"], out, out32, lse, ws, status)
    return out, out32, lse, int(status.item())


@pytest.mark.parametrize("short_by", [0, 1, 3])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_lengths_near_two_to_the_31(mv, d, short_by):
    gamma = 3                                                       # rows: 4, so that each of these lengths overflows with its block
    w = attn._make([5, 4], [512, 384], [9, 30, 200], gamma, 8, 2, d, d)
    calls = [lambda: attn._run(mv, w)] + [lambda k=k, c=c, n=n: _split(mv, w, k, c, n) for k, c, n in ((0, 0, 0), (1, 0, 0), (1, 256, 0), (2, 0, 0), (2, 256, 0), (0, 0, 100), (1, 256, 100))]
    for call in calls:
        for b in (0, 7):
            w["seq_lens"][b] = -1
        want = call()
        for b in (0, 7):
            w["seq_lens"][b] = 2 ** 31 - 1 - short_by
        got = call()
        assert want[3] == got[3] == -3
        for b in (0, 7):
            assert bool((got[0][b] == 3).all())
        for x, y in zip(got[:3], want[:3]):
            assert torch.equal(torch.nan_to_num(x, nan=7.0), torch.nan_to_num(y, nan=7.0))
