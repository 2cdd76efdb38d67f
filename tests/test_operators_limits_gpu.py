"""The largest and the smallest that massv_rotary, massv_verify_attn_shared and the calls under logit rules take: offsets past 32 bits, the most sequences and
groups, one prefix cut over all SMs, workspaces of exactly the size asked for, two streams at once, and the build that checks its own indices."""
import os
import subprocess
import sys

import pytest
import torch

import test_attn_shared as attn
import test_logit_rules as rules_of
from test_attn_shared import mv  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,sizes,shared,gamma,hq,hkv", [(64, [2], 30000, 0, 1, 1), (128, [3], 20000, 7, 8, 1), (256, [2], 12345, 7, 8, 1), (128, [64], 128, 7, 16, 2), (64, [1], 5000, 3, 4, 4)])
def test_workspace_of_exactly_the_size(mv, d, sizes, shared, gamma, hq, hkv):
    """One prefix over all SMs, one block of it, none: nothing behind the workspace is written, and the result is right."""
    w = attn._make(sizes, [shared], [7, 130], gamma, hq, hkv, d, 5)
    desc = mv.attn_desc(sum(sizes), gamma, hq, hkv, d, w["page_table"].shape[1], w["k_pages"].shape[0])
    n = mv.massv_verify_attn_shared_workspace_size(desc, 1)
    big = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    out, out32, lse, status = attn._run(mv, w, ws=big[:n])
    assert status == 0 and bool((big[n:] == 0x5a).all())
    attn._check(w, out, out32, lse)


def test_the_most_sequences(mv):
    """2,048 sequences in 256 groups of 8, on two streams at once with a workspace each."""
    w = attn._make([8] * 256, [128 + 16 * (i % 4) for i in range(256)], [0, 1, 30], 0, 2, 1, 64, 6)
    desc = mv.attn_desc(2048, 0, 2, 1, 64, w["page_table"].shape[1], w["k_pages"].shape[0])
    side = torch.cuda.Stream()
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    ws = [mv.alloc_workspace(mv.massv_verify_attn_shared_workspace_size(desc, 256), "cuda") for _ in range(2)]
    outs = [(torch.empty_like(w["q"]), torch.empty(w["q"].shape, device="cuda"), torch.empty(w["q"].shape[:3], device="cuda")) for _ in range(2)]
    side.wait_stream(torch.cuda.current_stream())
    for i, stream in enumerate((torch.cuda.current_stream(), side)):
        with torch.cuda.stream(stream):
            for _ in range(3):
                mv.massv_verify_attn_shared(desc, w["start"], w["shared"], w["q"], w["k_new"], w["v_new"], w["k_pages"], w["v_pages"], w["page_table"], w["seq_lens"], *outs[i], ws[i], status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and all(torch.equal(a, b) for a, b in zip(*outs))
    attn._check(w, *outs[0])


@pytest.mark.parametrize("d", [64, 256])
def test_pages_past_32_bits(mv, d):
    """The pages in use lie behind 2^31 elements of a pool."""
    w = attn._make([3, 2], [384, 200], [10, 100], 2, 4, 2, d, 7)
    shift = 2 ** 31 // (2 * 16 * d) + 3
    for n in ("k_pages", "v_pages"):
        pool = torch.empty((shift + w[n].shape[0], 2, 16, d), dtype=torch.bfloat16, device="cuda")
        pool[shift:] = w[n]
        w[n] = pool
    w["page_table"] = torch.where(w["page_table"] >= 0, w["page_table"] + shift, w["page_table"])
    out, out32, lse, status = attn._run(mv, w)
    assert status == 0
    attn._check(w, out, out32, lse)


@pytest.mark.parametrize("half", [True, False])
def test_tokens_past_32_bits(mv, half):
    """Slices of a projection whose last tokens lie behind 2^31 elements."""
    tokens, stride, heads, d = 70000, 31000, 3, 64
    x = torch.empty((1, tokens, stride), dtype=torch.bfloat16, device="cuda")
    x[:, -50:] = torch.randn((1, 50, stride), device="cuda").to(torch.bfloat16)
    x[:, :50] = x[:, -50:]
    turns = mv.massv_rope_frequencies(d)
    desc = mv.rope_desc(1, tokens, heads, 0, d, layout=mv.ROPE_HALF if half else mv.ROPE_INTERLEAVED)
    q = x.view(1, tokens, stride)[..., :heads * d].unflatten(-1, (heads, d))
    out = torch.empty((1, tokens, heads, d), dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda") % (tokens - 50)       # the last 50 stand where the first 50 do
    mv.massv_rotary(desc, turns, q, None, out, None, positions=pos)
    assert torch.equal(out[:, -50:], out[:, :50]) and bool(out[:, 1:50].ne(q[:, 1:50]).any())


def test_logits_past_32_bits(mv):
    """The last row of 1,025 of 2^21 logits, in place: what its sequence's rules say, the row ahead of it untouched."""
    batch, vocab = 1025, 2 ** 21
    z = torch.empty((batch, vocab), device="cuda")
    z[-2:] = torch.randn((2, vocab), device="cuda")
    keep = z[-2:].clone()
    bits = torch.zeros((batch, vocab // 32), dtype=torch.int32, device="cuda")
    bits[-1, -1] = -2 ** 31                                                     # the last token of the last row
    counts = torch.zeros((batch, vocab), dtype=torch.int32, device="cuda")
    mv.massv_history_add(vocab, torch.full((batch, 1), -1, dtype=torch.int32, device="cuda").index_fill_(0, torch.tensor([batch - 1], device="cuda"), vocab - 1),
                         torch.zeros((batch,), dtype=torch.int32, device="cuda").index_fill_(0, torch.tensor([batch - 1], device="cuda"), 1), bits, counts)
    presence = torch.full((batch,), 0.5, device="cuda")
    mv.massv_logits_apply(0, mv.logit_rules(output_bits=bits, counts=counts, presence=presence), z, z)
    keep[-1, -1] -= 0.5
    assert int(counts[-1, -1]) == 1 and int(counts[-1].sum()) == 1 and torch.equal(z[-2:], keep)


def test_the_most_rows_of_the_smallest_vocabulary(mv):
    s = rules_of._make(65535, 0, 3, ("allowed", "history"), 8)
    z = s["logits"].view(65535, 3)
    want, size = rules_of._want(s)
    mv.massv_logits_apply(0, rules_of._rules(mv, s), z, z)
    want, ok = want.view(65535, 3), s["mask"].view(65535, 3)
    assert bool(torch.isneginf(z[~ok]).all()) and bool(((z.double() - want).abs()[ok] <= 5 * 2.0 ** -24 * 80).all())      # values below 80 ever: |z| < 40 times 2


def test_accept_workspace_of_exactly_the_size(mv):
    batch, gamma, vocab = 9, 4, 5000
    s = rules_of._make(batch, gamma, vocab, rules_of.ALL, 9)
    s["mask"][..., 1] = True
    s["allowed"] = rules_of._pack(s["mask"])
    desc = mv.accept_desc(batch, gamma, 64, vocab, 0.8)
    n = mv.massv_accept_logits_workspace_size(desc)
    big = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    tokens, lens, status = torch.zeros((batch, gamma + 1), dtype=torch.int32, device="cuda"), torch.zeros((batch,), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
    q = torch.softmax(torch.randn((batch, gamma, vocab), device="cuda"), -1)
    mv.massv_accept_logits(desc, rules_of._rules(mv, s), s["logits"], torch.empty_like(s["logits"]), s["draft_tokens"], q, torch.rand((batch, gamma), device="cuda"),
                           torch.rand((batch, gamma + 1), device="cuda"), tokens, lens, None, big[:n], status)
    assert int(status.item()) == 0 and bool((big[n:] == 0x5a).all()) and int(lens.min()) >= 1


@pytest.mark.parametrize("T", [0.0, 1.0])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_accept_with_logits_that_are_no_numbers(mv, T, value):
    """A row of nothing but NaN (or, at T > 0, one with an infinite logit) under no mask: reported, tokens inside the vocabulary, the others served as without it."""
    batch, gamma, vocab = 3, 1, 3000
    s = rules_of._make(batch, gamma, vocab, ("history",), 10)
    desc = mv.accept_desc(batch, gamma, 64, vocab, T)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.softmax(torch.randn((batch, gamma, vocab), device="cuda", generator=g), -1)
    u, v = torch.rand((batch, gamma), device="cuda", generator=g), torch.rand((batch, gamma + 1), device="cuda", generator=g)

    def call(z):
        tokens, lens, status = torch.zeros((batch, gamma + 1), dtype=torch.int32, device="cuda"), torch.zeros((batch,), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
        ws = mv.alloc_workspace(mv.massv_accept_logits_workspace_size(desc), "cuda")
        mv.massv_accept_logits(desc, rules_of._rules(mv, s), z, torch.empty_like(z), s["draft_tokens"], q if T else None, u if T else None, v if T else None, tokens, lens, None, ws, status)
        return tokens, lens, int(status.item())
    tokens, lens, status = call(s["logits"])
    z = s["logits"].clone()
    if value != value:
        z[1] = value
    else:
        z[1, 0, 5] = value
    bad_tokens, bad_lens, bad_status = call(z)
    assert status == 0 and (bad_status == -1 or (T == 0 and value == float("inf")))
    assert int(bad_lens.min()) >= 1 and int(bad_lens.max()) <= gamma + 1 and all(0 <= int(bad_tokens[1, i]) < vocab for i in range(int(bad_lens[1])))
    for b in (0, 2):
        assert torch.equal(tokens[b], bad_tokens[b]) and int(lens[b]) == int(bad_lens[b])


def test_the_build_that_checks_its_indices():
    here = os.path.dirname(os.path.abspath(__file__))
    files = [os.path.join(here, f) for f in ("test_attn_shared.py", "test_rotary.py", "test_logit_rules.py")]
    run = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "-k", "64_bits or without_room or none or under_rules or history", *files],
                         env=dict(os.environ, MASSV_DEBUG="1"), capture_output=True, text=True, timeout=500, cwd=os.path.dirname(here))
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-500:]
