"""Rules on logits, alone and inside the acceptance, and the history they read: against 64 bits and the oracle; what is refused."""
import ctypes
import math

import numpy as np
import pytest
import torch

import __graft_entry__ as entry
import oracle
from parity_util import compare_accept

NAMES = ("allowed", "bias_start", "bias_tokens", "bias_values", "prompt_bits", "output_bits", "counts", "repetition", "frequency", "presence")


@pytest.fixture(scope="module")
def mv():
    entry.build()
    import paper_2505_10526_b200 as pkg
    return pkg.binding


def test_refusals(mv):
    lib, a = mv._lib, 0x1000                          # an aligned address, never dereferenced
    R = mv.LogitRules

    def apply(batch=1, gamma=0, vocab=100, rules=R(), z=a, out=a, drafts=None):
        return lib.massv_logits_apply(batch, gamma, vocab, ctypes.byref(rules) if rules is not None else None, z, out, drafts, None, None)
    assert apply(batch=0) == -1 and apply(gamma=-1) == -1 and apply(vocab=0) == -1 and apply(rules=None) == -1 and apply(z=None) == -1 and apply(out=None) == -1
    assert apply(z=a + 4) == -1 and apply(out=a + 8) == -1
    assert apply(batch=65536) == -2 and apply(gamma=8) == -2 and apply(vocab=(1 << 21) + 1) == -2
    for bad in (R(bias_start=a, n_bias=3, bias_tokens=a), R(bias_start=a, n_bias=-1), R(bias_start=a, n_bias=1, bias_values=a), R(output_bits=a), R(counts=a)):
        assert apply(rules=bad) == -1

    def accept(desc, rules=None, z=a, out=None, drafts=a, q=a, ua=a, us=a, tokens=a, lens=a, probs=None, ws=a * 16, n=1 << 40):
        return lib.massv_accept_logits(ctypes.byref(desc), ctypes.byref(rules) if rules is not None else None, z, out, drafts, q, ua, us, tokens, lens, probs, ws, n, None, None)
    t0, t1 = mv.accept_desc(2, 3, 0, 1024, 0.0), mv.accept_desc(2, 3, 0, 1024, 1.0)
    assert mv.massv_accept_logits_workspace_size(t0) > 0 and mv.massv_accept_logits_workspace_size(t1) > 0            # (`hidden` is not read)
    for bad in (mv.accept_desc(2, 8, 64, 1024, 0.0), mv.accept_desc(2, 3, 64, 1023, 0.0), mv.accept_desc(200, 3, 64, 1024, 0.0)):
        assert mv.massv_accept_logits_workspace_size(bad) == 0 and accept(bad) == -2
    assert accept(mv.accept_desc(2, 3, 0, 1024, -1.0)) == -1
    assert accept(t0, z=None) == -1 and accept(t0, drafts=None) == -1 and accept(t0, tokens=None) == -1 and accept(t0, lens=None) == -1 and accept(t0, probs=a) == -1
    assert accept(t1, q=None) == -1 and accept(t1, ua=None) == -1 and accept(t1, us=None) == -1 and accept(t1, rules=R()) == -1        # rules at T > 0 need logits_out
    assert accept(t0, rules=R(counts=a)) == -1 and accept(t1, z=a + 4) == -1 and accept(t1, out=a + 4) == -1
    assert accept(t0, ws=None) == -4 and accept(t0, ws=a + 16) == -4 and accept(t1, n=64) == -4

    add = lib.massv_history_add
    assert add(0, 10, a, 1, None, a, None, None, None) == -1 and add(1, 0, a, 1, None, a, None, None, None) == -1 and add(1, 10, None, 1, None, a, None, None, None) == -1
    assert add(1, 10, a, -1, None, a, None, None, None) == -1 and add(1, 10, a, 1, None, None, None, None, None) == -1
    assert add(1 << 20, 10, a, 1 << 20, None, a, None, None, None) == -2
    assert add(3, 10, None, 0, None, a, None, None, None) == 0                                                       # no tokens: nothing to launch

    f = torch.zeros((1, 64))
    with pytest.raises(ValueError, match="CUDA device"):
        mv.massv_logits_apply(0, mv.logit_rules(), f, f)
    with pytest.raises(ValueError, match="batch, gamma"):
        mv.massv_logits_apply(2, mv.logit_rules(), f, f)
    with pytest.raises(TypeError):
        mv.massv_logits_apply(0, t0, f, f)
    with pytest.raises(ValueError):
        mv.logit_rules(bias_tokens=torch.zeros(3, dtype=torch.int32))


# ---------------------------------------------------------------- on the GPU
def _pack(bits):
    w = torch.nn.functional.pad(bits, (0, -bits.shape[-1] % 32)).unflatten(-1, (-1, 32)).long()
    words = (w << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _make(batch, gamma, vocab, which, seed, density=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, dev = gamma + 1, "cuda"
    rand = lambda *shape: torch.rand(shape, device=dev, generator=g)
    ints = lambda hi, *shape: torch.randint(0, hi, shape, device=dev, generator=g)
    s = dict.fromkeys(NAMES)
    s["logits"] = torch.randn((batch, rows, vocab), device=dev, generator=g) * 5
    s["draft_tokens"] = ints(vocab, batch, gamma).to(torch.int32)
    s["mask"] = torch.ones((batch, rows, vocab), dtype=torch.bool, device=dev)
    if "allowed" in which:
        s["mask"] = rand(batch, rows, vocab) < density
        s["allowed"] = _pack(s["mask"])
    s["bias"] = torch.zeros((batch, vocab), dtype=torch.float64, device=dev)
    if "bias" in which:
        n = [min(vocab, 5 * b + 2) if b % 3 != 1 else 0 for b in range(batch)]       # some sequences have none
        s["bias_start"] = torch.tensor([0] + list(np.cumsum(n)), dtype=torch.int32, device=dev)
        total = sum(n)
        s["bias_tokens"] = ints(vocab, total).to(torch.int32)
        s["bias_values"] = torch.randn((total,), device=dev, generator=g) * 4
        for b in range(batch):
            for k in range(int(s["bias_start"][b]), int(s["bias_start"][b + 1])):    # in order: the last entry of a token counts
                s["bias"][b, int(s["bias_tokens"][k])] = float(s["bias_values"][k])
    s["prompt"] = rand(batch, vocab) < 0.05
    s["c"] = torch.where(rand(batch, vocab) < 0.05, 1 + ints(9, batch, vocab), 0)
    if "history" in which:
        s["prompt_bits"], s["output_bits"], s["counts"] = _pack(s["prompt"]), _pack(s["c"] > 0), s["c"].to(torch.int32)
        # what is read only where the bit is set
        s["counts"] = torch.where(s["c"] > 0, s["counts"], torch.full_like(s["counts"], 1000))
    else:
        s["prompt"], s["c"] = torch.zeros_like(s["prompt"]), torch.zeros_like(s["c"])
    for name in ("repetition", "frequency", "presence"):
        if name in which or "history" in which:
            s[name] = 0.5 + rand(batch)
    return s


def _want(s, drafts=True):
    """64-bit logits under the rules, and a bound on the fp32 evaluation's error: five roundings at most, each of half a step of the
    largest value that the chain can hold."""
    z = s["logits"].double()
    batch, rows, vocab = z.shape
    c = s["c"][:, None].expand(batch, rows, vocab).clone().double()
    if drafts:
        for j in range(1, rows):
            for i in range(j):
                for b in range(batch):
                    t = int(s["draft_tokens"][b, i])
                    if 0 <= t < vocab:
                        c[b, j, t] += 1
    z = z + s["bias"][:, None]
    one, zero = torch.ones(batch, device="cuda"), torch.zeros(batch, device="cuda")
    r, f, p = (x.double()[:, None, None] for x in (s["repetition"] if s["repetition"] is not None else one, s["frequency"] if s["frequency"] is not None else zero,
                                                   s["presence"] if s["presence"] is not None else zero))
    size = (s["logits"].abs().double() + s["bias"].abs()[:, None]) * torch.maximum(r, 1 / r) + f * c + p
    z = torch.where(s["prompt"][:, None] | (c > 0), torch.where(z > 0, z / r, z * r), z)
    z = z - f * c - p * (c > 0)
    return z.masked_fill(~s["mask"], -math.inf), 5 * 2.0 ** -24 * size


def _rules(mv, s):
    return mv.logit_rules(**{n: s[n] for n in NAMES})


ALL = ("allowed", "bias", "history")


def _near(got, want, bound):
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and bool((got[inf] < 0).all())
    assert bool(((got.double() - want).abs() <= bound)[~inf].all())


@pytest.mark.gpu
@pytest.mark.parametrize("batch,gamma,vocab", [(1, 0, 1), (1, 0, 31), (2, 1, 33), (3, 2, 1000), (1, 5, 1024), (2, 7, 1025), (5, 4, 2051), (3, 0, 4097), (2, 3, 9000), (70, 0, 5003), (1, 1, 152064)])
@pytest.mark.parametrize("which", [ALL, ("allowed",), ("bias",), ("history",), ("repetition", "presence"), ()])
def test_apply(mv, batch, gamma, vocab, which):
    s = _make(batch, gamma, vocab, which, batch + vocab)
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    # the output between margins, which stay; rows in between are all written
    big = torch.full((s["logits"].numel() + 1024,), float("nan"), device="cuda")
    out = big[512:512 + s["logits"].numel()].view_as(s["logits"])
    before = s["logits"].clone()
    mv.massv_logits_apply(gamma, _rules(mv, s), s["logits"], out, s["draft_tokens"], status)
    # (without counts, drafts of the block are still history)
    want, bound = _want(s, drafts="history" in which or "repetition" in which)
    assert int(status.item()) == 0
    _near(out, want, bound)
    assert torch.equal(s["logits"], before) and bool(torch.isnan(big[:512]).all()) and bool(torch.isnan(big[-512:]).all())
    mv.massv_logits_apply(gamma, _rules(mv, s), s["logits"], s["logits"], s["draft_tokens"], status)           # in place
    assert torch.equal(s["logits"], out)


@pytest.mark.gpu
def test_what_is_masked_may_be_anything(mv):
    """NaN, infinities and the type's lowest value: in masked places they are -inf, elsewhere they stay; a row may be left empty."""
    batch, gamma, vocab = 2, 1, 1031
    s = _make(batch, gamma, vocab, ("allowed",), 3)
    z = s["logits"]
    z[0, 0, ::3] = float("nan"); z[0, 1, ::5] = float("inf"); z[1, 0, ::2] = torch.finfo(torch.float32).min; z[1, 0, 1::2] = -float("inf")
    s["mask"][1, 1] = False
    s["allowed"] = _pack(s["mask"])
    out = torch.empty_like(z)
    mv.massv_logits_apply(gamma, _rules(mv, s), z, out, s["draft_tokens"])
    want = torch.where(s["mask"], z, torch.full_like(z, -math.inf))
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(out.nan_to_num(nan=0.5), want.nan_to_num(nan=0.5))
    assert bool((out[1, 1] == -math.inf).all())


@pytest.mark.gpu
def test_entries_that_are_wrong_are_reported_and_ignored(mv):
    batch, gamma, vocab = 3, 2, 2000
    s = _make(batch, gamma, vocab, ALL, 8)

    def status_of(**change):
        t = dict(s, **change)
        status, out = torch.zeros((1,), dtype=torch.int32, device="cuda"), torch.empty_like(s["logits"])
        mv.massv_logits_apply(gamma, _rules(mv, t), s["logits"], out, t["draft_tokens"], status)
        return int(status.item()), out
    ok, base = status_of()
    assert ok == 0
    tokens, values, start = s["bias_tokens"].clone(), s["bias_values"], s["bias_start"].clone()
    for bad in (-1, vocab, 2 ** 31 - 1, -2 ** 31):
        wrong = tokens.clone()
        wrong[0] = bad
        rc, out = status_of(bias_tokens=wrong)
        assert rc == -1 and torch.equal(out[1:], base[1:])
        keep = [k for k in range(len(tokens)) if k != 0]
        without = status_of(bias_tokens=tokens[keep].contiguous(), bias_values=values[keep].contiguous(), bias_start=(start - (start > 0).int()).contiguous())
        assert without[0] == 0 and torch.equal(out, without[1])
    wrong = start.clone()
    wrong[batch] = len(tokens) + 50                                # past the end of the arrays: what there is counts
    rc, out = status_of(bias_start=wrong)
    assert rc == -1 and torch.equal(out, base)
    wrong = start.clone()
    wrong[1] = -7
    assert status_of(bias_start=wrong)[0] == -1
    for bad in (0.0, -1.0, float("nan")):
        rep = s["repetition"].clone()
        rep[1] = bad
        rc, out = status_of(repetition=rep)
        rep[1] = 1.0
        assert rc == -1 and torch.equal(out, status_of(repetition=rep)[1])
    drafts = s["draft_tokens"].clone()
    drafts[0, 0] = -1; drafts[1, 1] = vocab
    rc, out = status_of(draft_tokens=drafts)
    want, bound = _want(dict(s, draft_tokens=drafts))
    assert rc == 0
    _near(out, want, bound)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [0.0, 0.7, 1.0])
@pytest.mark.parametrize("batch,gamma,vocab,density", [(1, 0, 8, 0.5), (1, 5, 1024, 0.5), (4, 3, 1032, 0.02), (7, 7, 4104, 0.3), (64, 7, 2048, 0.1), (3, 2, 40000, 0.9), (40, 1, 152064, 0.05)])
def test_accept_under_rules(mv, T, batch, gamma, vocab, density):
    s = _make(batch, gamma, vocab, ALL, vocab + batch, density)
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = gamma + 1
    s["mask"][..., 3] = True
    s["allowed"] = _pack(s["mask"])
    sampling = T > 0
    # drafts that follow the distribution under the rules, which follows the drafts ahead: row after row
    q = torch.zeros((batch, gamma, vocab), device="cuda")
    for j in range(gamma):
        z = _want(s)[0][:, j] + torch.randn((batch, vocab), device="cuda", generator=g) * 0.5
        q[:, j] = torch.softmax(z / (T or 1.0), -1).float()
        s["draft_tokens"][:, j] = (torch.multinomial(q[:, j], 1, generator=g)[:, 0] if sampling else z.argmax(-1)).to(torch.int32)
    ua, us = torch.rand((batch, gamma), device="cuda", generator=g), torch.rand((batch, rows), device="cuda", generator=g)
    desc = mv.accept_desc(batch, gamma, 0, vocab, T)
    ws = mv.alloc_workspace(mv.massv_accept_logits_workspace_size(desc), "cuda").fill_(0xff)
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    tokens, lens = torch.full((batch, rows), -9, dtype=torch.int32, device="cuda"), torch.zeros((batch,), dtype=torch.int32, device="cuda")
    out = torch.full_like(s["logits"], float("nan"))
    probs = torch.full_like(s["logits"], float("nan")) if sampling else None
    rest = (s["draft_tokens"], q if sampling else None, ua if sampling else None, us if sampling else None, tokens, lens)
    mv.massv_accept_logits(desc, _rules(mv, s), s["logits"], out, *rest, probs, ws, status)
    assert int(status.item()) == 0
    want, bound = _want(s)
    _near(out, want, bound)
    z = np.ascontiguousarray(want.cpu().numpy().reshape(batch * rows, vocab))
    p = np.ascontiguousarray(torch.softmax(want / T, -1).cpu().numpy().reshape(batch * rows, vocab)) if sampling else None
    ref = oracle.accept(T, np.where(np.isinf(z), -1e300, z), p, s["draft_tokens"].cpu().numpy(), q.cpu().numpy() if sampling else None, ua.cpu().numpy() if sampling else None,
                        us.cpu().numpy() if sampling else None)
    stats = compare_accept(ref, tokens.cpu().numpy(), lens.cpu().numpy(), gamma)
    assert stats["hard"] == 0, stats
    if sampling:
        # exponents up to |z| / T off by 2^-22 relative, plus the logits' own error over T
        assert float((probs.double().cpu() - torch.from_numpy(p).view(batch, rows, vocab)).abs().max()) < 1e-4
    # the same call twice, and from logits that the rules have been applied to: bit for bit
    first = tokens.clone(), lens.clone()
    plain = (mv.accept_desc(batch, gamma, 0, vocab, T), None, out, None) + rest
    mv.massv_accept_logits(*plain, None, ws, status)
    assert torch.equal(tokens, first[0]) and torch.equal(lens, first[1])
    mv.massv_accept_logits(desc, _rules(mv, s), s["logits"], s["logits"] if sampling else None, *rest, None, ws, status)
    assert torch.equal(tokens, first[0]) and torch.equal(lens, first[1]) and (not sampling or torch.equal(s["logits"], out))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [0.0, 1.0])
def test_a_row_that_the_rules_leave_empty(mv, T):
    """Token 0 and MASSV_ERR_INVALID_ARG for the sequence that stops there; the others are served."""
    batch, gamma, vocab = 3, 2, 1040
    s = _make(batch, gamma, vocab, ("allowed",), 4, 0.9)
    s["mask"][1] = False
    s["allowed"] = _pack(s["mask"])
    q = torch.full((batch, gamma, vocab), 1.0 / vocab, device="cuda")
    us = torch.full((batch, gamma + 1), 0.3, device="cuda")
    desc = mv.accept_desc(batch, gamma, 0, vocab, T)
    ws = mv.alloc_workspace(mv.massv_accept_logits_workspace_size(desc), "cuda")
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    tokens, lens = torch.zeros((batch, gamma + 1), dtype=torch.int32, device="cuda"), torch.zeros((batch,), dtype=torch.int32, device="cuda")
    mv.massv_accept_logits(desc, _rules(mv, s), s["logits"], s["logits"], s["draft_tokens"], q if T else None, us[:, :gamma].contiguous() if T else None, us if T else None, tokens, lens,
                           None, ws, status)
    assert int(status.item()) == -1 and int(lens[1]) == 1 and tokens[1].tolist() == [0, -1, -1]
    for b in (0, 2):
        n = int(lens[b])
        assert 1 <= n <= gamma + 1 and bool(s["mask"][b, n - 1, int(tokens[b, n - 1])])


@pytest.mark.gpu
@pytest.mark.parametrize("batch,vocab,n", [(1, 1, 1), (2, 33, 7), (5, 1000, 300), (3, 152064, 5000), (64, 4097, 8), (1, 40, 0)])
def test_history(mv, batch, vocab, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    words = (vocab + 31) // 32
    bits, counts = torch.zeros((batch, words), dtype=torch.int32, device="cuda"), torch.zeros((batch, vocab), dtype=torch.int32, device="cuda")
    prompt = torch.zeros_like(bits)
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    want = torch.zeros((batch, vocab), dtype=torch.long)
    for step in range(3):
        tokens = torch.randint(0, vocab, (batch, n), device="cuda", generator=g).to(torch.int32)
        lens = torch.randint(0, n + 1, (batch,), device="cuda", generator=g).to(torch.int32) if step else None
        if lens is not None and n:
            tokens[torch.arange(n, device="cuda")[None] >= lens[:, None]] = -1                # padding is not looked at
        mv.massv_history_add(vocab, tokens, lens, bits, counts, status)
        mv.massv_history_add(vocab, tokens, lens, prompt, None, status)
        for b in range(batch):
            want[b] += torch.bincount(tokens[b, :n if lens is None else int(lens[b])].cpu().long(), minlength=vocab)
    assert int(status.item()) == 0
    assert torch.equal(counts.cpu().long(), want) and torch.equal(bits, _pack(want.cuda() > 0)) and torch.equal(prompt, bits)
    if n:
        tokens[0, 0] = vocab
        before = counts.clone()
        mv.massv_history_add(vocab, tokens[:1, :1].contiguous(), None, bits[:1], counts[:1], status)
        assert int(status.item()) == -1 and torch.equal(counts, before)
        status.zero_()
        tokens.clamp_(0, vocab - 1)
        mv.massv_history_add(vocab, tokens, torch.full((batch,), n + 3, dtype=torch.int32, device="cuda"), bits, counts, status)      # taken as n
        assert int(status.item()) == -1 and int((counts - before).sum()) == batch * n
        before = counts.clone()
        status.zero_()
        mv.massv_history_add(vocab, tokens, torch.full((batch,), -2, dtype=torch.int32, device="cuda"), bits, counts, status)         # taken as 0
        assert int(status.item()) == -1 and torch.equal(counts, before)


@pytest.mark.gpu
def test_captured_and_on_another_stream(mv):
    batch, gamma, vocab = 4, 3, 5000
    s = _make(batch, gamma, vocab, ALL, 2)
    rules, out, status = _rules(mv, s), torch.empty_like(s["logits"]), torch.zeros((1,), dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mv.massv_logits_apply(gamma, rules, s["logits"], out, s["draft_tokens"], status)
    for seed in (5, 6):                                            # other logits, drafts and masks in the same buffers
        t = _make(batch, gamma, vocab, ALL, seed)
        for name in ("logits", "draft_tokens", "allowed", "counts", "output_bits", "prompt_bits", "bias_values", "bias_tokens", "repetition", "frequency", "presence"):
            s[name].copy_(t[name])
        graph.replay()
        _near(out, *_want(dict(t)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = torch.empty_like(out)
        mv.massv_logits_apply(gamma, rules, s["logits"], other, s["draft_tokens"], status)
    side.synchronize()
    assert torch.equal(other, out) and int(status.item()) == 0
