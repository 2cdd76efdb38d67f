"""Rotary positions: the frequencies against their formulas in many digits, the turned queries and keys against 64 bits, what is refused."""
import ctypes
import math
from decimal import Decimal, getcontext

import pytest
import torch

import __graft_entry__ as entry

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


@pytest.fixture(scope="module")
def mv():
    entry.build()
    import paper_2505_10526_b200 as pkg
    return pkg.binding


def _frequencies(rot, base, kind="none", factor=1.0, ctx=0.0, slow=1.0, fast=32.0):
    """Radians per position, in 60 digits."""
    getcontext().prec = 60
    b = Decimal(base)
    if kind == "base":
        b = b * (Decimal(factor).ln() * rot / (rot - 2)).exp()
    index = lambda t: Decimal(rot) * (Decimal(ctx) / (2 * PI * Decimal(t))).ln() / (2 * b.ln())
    if kind == "pairs":
        clamp = lambda x: max(0, min(rot - 1, x))
        lo, hi = clamp(math.floor(index(fast))), clamp(math.ceil(index(slow)))
    out = []
    for i in range(rot // 2):
        f = (-b.ln() * 2 * i / rot).exp()
        if kind == "linear":
            f /= Decimal(factor)
        if kind in ("turns", "pairs"):
            if kind == "turns":
                w = (Decimal(ctx) * f / (2 * PI) - Decimal(slow)) / (Decimal(fast) - Decimal(slow))
            else:
                w = 1 - Decimal(i - lo) / Decimal(hi - lo) if hi > lo else Decimal(int(i <= lo))
            w = max(Decimal(0), min(Decimal(1), w))
            f = f * (w + (1 - w) / Decimal(factor))
        out.append(f)
    return out


@pytest.mark.parametrize("rot,base,kw", [
    (2, 10000.0, {}), (64, 10000.0, {}), (128, 1e6, {}), (106, 500000.0, {}), (256, 1e4, dict(kind="linear", factor=8.0)), (128, 1e4, dict(kind="base", factor=4.0)),
    (128, 5e5, dict(kind="turns", factor=8.0, ctx=8192.0, slow=1.0, fast=4.0)), (128, 1e6, dict(kind="pairs", factor=4.0, ctx=32768.0)),
    (64, 1e4, dict(kind="pairs", factor=40.0, ctx=4096.0)), (8, 1e4, dict(kind="pairs", factor=2.0, ctx=16.0, slow=1.0, fast=2.0)), (128, 1e4, dict(kind="turns", factor=1.0, ctx=100.0))])
def test_frequencies(mv, rot, base, kw):
    kinds = dict(linear=mv.ROPE_SCALE_LINEAR, base=mv.ROPE_SCALE_BASE, turns=mv.ROPE_SCALE_TURNS, pairs=mv.ROPE_SCALE_PAIRS, none=mv.ROPE_SCALE_NONE)
    got = mv.massv_rope_frequencies(rot, base, kind=kinds[kw.get("kind", "none")], factor=kw.get("factor", 1.0), original_context=kw.get("ctx", 0.0),
                                    slow=kw.get("slow", 1.0), fast=kw.get("fast", 32.0), device="cpu").tolist()
    for t, f in zip(got, _frequencies(rot, base, **kw)):
        want = f / (2 * PI) % 1 * (1 << 64)
        # formed in 64-bit significands: a dozen roundings of 2^-64 relative to a value below 2^64 / 6, and one to an integer
        assert abs(Decimal(t % (1 << 64)) - want) <= 16


def test_given_frequencies_wrap(mv):
    turns = mv.massv_rope_frequencies(8, kind=mv.ROPE_SCALE_GIVEN, inv_freq=[0.0, 2 * math.pi * 0.25, -2 * math.pi * 0.25, 2 * math.pi * 3.5], device="cpu").tolist()
    want = [0.0, 0.25, 0.75, 0.5]
    for t, w in zip(turns, want):
        off = (t / 2 ** 64 - w + 0.5) % 1 - 0.5
        assert abs(off) < 1e-15                       # 2 pi in 53 bits times 3.5, over 2 pi


def test_refusals(mv):
    def freq(rot, base=1e4, **kw):
        with pytest.raises(mv.MassvError) as e:
            mv.massv_rope_frequencies(rot, base, device="cpu", **kw)
        return e.value.status
    assert freq(0) == -1 and freq(7) == -1 and freq(258) == -2
    assert freq(64, 1.0) == -1 and freq(64, math.inf) == -1 and freq(64, math.nan) == -1
    assert freq(64, kind=9) == -2 and freq(64, kind=mv.ROPE_SCALE_GIVEN) == -1 and freq(2, kind=mv.ROPE_SCALE_BASE, factor=2.0) == -2
    assert freq(64, kind=mv.ROPE_SCALE_LINEAR, factor=0.5) == -1 and freq(64, kind=mv.ROPE_SCALE_TURNS, factor=2.0) == -1
    assert freq(64, kind=mv.ROPE_SCALE_PAIRS, factor=2.0, original_context=4096, slow=32.0, fast=1.0) == -1
    assert freq(4, kind=mv.ROPE_SCALE_GIVEN, inv_freq=[1.0, math.inf]) == -1
    with pytest.raises(ValueError):
        mv.massv_rope_frequencies(8, kind=mv.ROPE_SCALE_GIVEN, inv_freq=[1.0], device="cpu")

    lib, a = mv._lib, 0x1000                           # aligned addresses, never dereferenced

    def call(d, q=a, qs=None, k=a, ks=None, pos=None, lens=a, delta=None, qo=a, qos=None, ko=a, kos=None, turns=a):
        w, v = d.n_q_heads * d.head_dim, d.n_kv_heads * d.head_dim
        return lib.massv_rotary(ctypes.byref(d), turns, q, w if qs is None else qs, k, v if ks is None else ks, pos, lens, delta, qo, w if qos is None else qos, ko,
                                v if kos is None else kos, None)
    ok = (1, 2, 4, 2, 64)
    d = mv.rope_desc(*ok)
    assert call(d, q=None) == -1 and call(d, ko=None) == -1 and call(d, turns=None) == -1 and call(d, q=a + 8) == -1
    assert call(d, pos=a) == -1 and call(d, lens=None) == -1 and call(d, pos=a, lens=None, delta=a) == -1
    assert call(d, qs=4 * 64 - 8) == -1 and call(d, qs=4 * 64 + 4) == -1 and call(d, qs=512) == -1      # short, not in groups of eight, in place with another stride
    assert call(mv.rope_desc(0, 2, 4, 2, 64)) == -1 and call(mv.rope_desc(1, 2, 0, 0, 64)) == -1 and call(mv.rope_desc(1, 2, 4, 2, 64, magnitude=math.inf)) == -1
    assert call(mv.rope_desc(1, 2, 4, 2, 64, axis_pairs=[16, 8])) == -1 and call(mv.rope_desc(1, 2, 4, 2, 64, axis_pairs=[40, -8])) == -1
    for bad in (mv.rope_desc(1, 2, 4, 2, 60), mv.rope_desc(1, 2, 4, 2, 264), mv.rope_desc(1, 2, 4, 2, 64, rot_dim=66), mv.rope_desc(1, 2, 4, 2, 64, rot_dim=7),
                mv.rope_desc(1, 2, 4, 2, 64, layout=2), mv.rope_desc(1 << 20, 1 << 12, 4, 2, 64)):
        assert call(bad) == -2
    bf = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA device"):
        mv.massv_rotary(d, torch.zeros(32, dtype=torch.int64), bf, bf[:, :2], bf, bf[:, :2])


# ---------------------------------------------------------------- on the GPU
def _want(x, angle, rot, half, magnitude):
    """64-bit result, and the sum of the magnitudes of the two products behind each element."""
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    n = rot // 2
    at = (slice(0, n), slice(n, rot)) if half else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = (x[..., s].double() for s in at)
    c, s = (f(angle)[:, None] * magnitude for f in (torch.cos, torch.sin))
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    size[..., at[0]] = size[..., at[1]] = (a.abs() + b.abs()) * abs(magnitude)
    return y, size


def _check(got, x, angle, rot, half, magnitude):
    want, size = _want(x, angle, rot, half, magnitude)
    # sine, cosine, their factor and the two products each off by 2^-22 of the products at most, one rounding to bf16 of 2^-8
    assert bool(((got.double() - want).abs() <= want.abs() * 2.0 ** -8 + size * 2.0 ** -20).all())
    assert torch.equal(got[..., rot:], x[..., rot:])


@pytest.mark.gpu
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("batch,rows,hq,hkv,d,rot", [
    (1, 1, 1, 1, 8, 2), (1, 6, 28, 4, 128, 128), (3, 5, 7, 1, 64, 64), (2, 3, 16, 8, 256, 64), (5, 8, 4, 2, 96, 48), (2, 7, 3, 3, 40, 36), (1, 9, 5, 1, 128, 106),
    (4, 1, 12, 2, 128, 34), (1, 1301, 9, 3, 128, 128), (3, 500, 2, 1, 72, 72), (1, 4099, 1, 0, 256, 254), (2, 2, 0, 3, 64, 32)])
def test_against_64_bits(mv, half, batch, rows, hq, hkv, d, rot):
    g = torch.Generator(device="cuda").manual_seed(batch * rows + d + rot)
    n = batch * rows
    q, k = (torch.randn((batch, rows, h, d), dtype=torch.bfloat16, device="cuda", generator=g) if h else None for h in (hq, hkv))
    lens = torch.randint(0, 1 << 30, (batch,), device="cuda", generator=g).to(torch.int32)      # positions up to 10^9
    lens[0] = 0
    delta = -torch.randint(0, 5000, (batch,), device="cuda", generator=g).to(torch.int32)       # negative positions too
    turns = mv.massv_rope_frequencies(rot, 1e6)
    magnitude = 1.25 if rot % 4 else 1.0
    desc = mv.rope_desc(batch, rows, hq, hkv, d, rot, layout=mv.ROPE_HALF if half else mv.ROPE_INTERLEAVED, magnitude=magnitude)
    # the angle from the fixed-point frequency in whole numbers: exact modulo a turn
    pos = (lens.long() + delta)[:, None] + torch.arange(rows, device="cuda")
    phase = pos.reshape(n, 1) * turns                                             # int64 wraps modulo 2^64
    angle = phase.double() * (2 * math.pi / 2.0 ** 64)
    out = [torch.full_like(x, float("nan")) if x is not None else None for x in (q, k)]
    mv.massv_rotary(desc, turns, q, k, out[0], out[1], seq_lens=lens, pos_delta=delta)
    for x, y in zip((q, k), out):
        if x is not None:
            _check(y.view(n, -1, d), x.view(n, -1, d), angle, rot, half, magnitude)
    # in place, from explicit positions
    same = [x.clone() if x is not None else None for x in (q, k)]
    mv.massv_rotary(desc, turns, same[0], same[1], same[0], same[1], positions=pos.to(torch.int32).reshape(n, 1).contiguous())
    for x, y in zip(same, out):
        assert x is None or torch.equal(x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("pairs,d", [([16, 24, 24], 128), ([0, 5, 8], 32), ([9, 1], 24), ([32, 0, 0], 64)])
def test_axes_of_a_fused_projection(mv, half, pairs, d):
    """Slices of [tokens, (q + 2 kv) heads * d], three position components, tokens around the bounds of a CTA's share."""
    hq, hkv, rot = 6, 2, 2 * sum(pairs)
    g = torch.Generator(device="cuda").manual_seed(d)
    for n in (1, 3, 1183, 1184, 1187):
        qkv = torch.randn((n, (hq + 2 * hkv) * d), dtype=torch.bfloat16, device="cuda", generator=g)
        before = qkv.clone()
        q, k = qkv[:, :hq * d].unflatten(-1, (hq, d)), qkv[:, hq * d:(hq + hkv) * d].unflatten(-1, (hkv, d))
        pos = torch.randint(-100, 40000, (n, len(pairs)), device="cuda", generator=g).to(torch.int32)
        turns = mv.massv_rope_frequencies(rot, 1e4, kind=mv.ROPE_SCALE_TURNS, factor=4.0, original_context=4096, slow=1.0, fast=32.0)
        axis = torch.repeat_interleave(torch.arange(len(pairs), device="cuda"), torch.tensor(pairs, device="cuda"))
        angle = (pos.long()[:, axis] * turns).double() * (2 * math.pi / 2.0 ** 64)
        desc = mv.rope_desc(1, n, hq, hkv, d, rot, layout=mv.ROPE_HALF if half else mv.ROPE_INTERLEAVED, axis_pairs=pairs)
        qo, ko = torch.full((n, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full((n, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        mv.massv_rotary(desc, turns, q, k, qo, ko, positions=pos)
        assert torch.equal(qkv, before)
        _check(qo, q, angle, rot, half, 1.0)
        _check(ko, k, angle, rot, half, 1.0)
        mv.massv_rotary(desc, turns, q, k, q, k, positions=pos)                    # in place, inside the fused tensor
        assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, (hq + hkv) * d:], before[:, (hq + hkv) * d:])


@pytest.mark.gpu
@pytest.mark.parametrize("half", [True, False])
def test_backward_is_the_gradient(mv, half):
    """The gradient of sum(w * rotary(x)), from the formula and from differences (the map is linear: exact up to rounding)."""
    n, h, d, rot, m = 7, 3, 32, 20, 1.5
    g = torch.Generator(device="cuda").manual_seed(5)
    w = torch.randn((n, h, d), dtype=torch.bfloat16, device="cuda", generator=g)
    pos = torch.randint(0, 4000, (n, 1), device="cuda", generator=g).to(torch.int32)
    turns = mv.massv_rope_frequencies(rot, 1e4)
    lay = mv.ROPE_HALF if half else mv.ROPE_INTERLEAVED
    grad = torch.empty_like(w)
    mv.massv_rotary(mv.rope_desc(1, n, h, 0, d, rot, layout=lay, magnitude=m, backward=True), turns, w, None, grad, None, positions=pos)
    angle = (pos.long() * turns).double() * (2 * math.pi / 2.0 ** 64)
    _check(grad, w, -angle, rot, half, m)
    fwd = mv.rope_desc(1, n, h, 0, d, rot, layout=lay, magnitude=m)
    for e in range(d):
        x = torch.zeros_like(w)
        x[..., e] = 1.0
        y = torch.empty_like(x)
        mv.massv_rotary(fwd, turns, x, None, y, None, positions=pos)
        slope = (w.double() * y.double()).sum(-1)
        # y's two non-zero elements are rounded to bf16 (2^-8 each), so is the gradient
        bound = (w.double() * y.double()).abs().sum(-1) * 2.0 ** -8 + grad[..., e].double().abs() * 2.0 ** -8 + 1e-5
        assert bool(((slope - grad[..., e].double()).abs() <= bound).all())


@pytest.mark.gpu
def test_values_that_are_not_numbers_stay_where_they_are(mv):
    """A NaN or an infinity reaches its pair and nothing else: not the other pairs, not the elements behind rot_dim."""
    n, h, d, rot = 4, 2, 32, 12
    for lay in (mv.ROPE_HALF, mv.ROPE_INTERLEAVED):
        x = torch.ones((n, h, d), dtype=torch.bfloat16, device="cuda")
        x[1, 0, 3] = float("nan"); x[2, 1, 13] = float("inf"); x[3, 0, 12] = float("nan")
        y = torch.empty_like(x)
        mv.massv_rotary(mv.rope_desc(1, n, h, 0, d, rot, layout=lay), mv.massv_rope_frequencies(rot, 1e4), x, None, y, None, seq_lens=torch.zeros(1, dtype=torch.int32, device="cuda"))
        partner = 9 if lay == mv.ROPE_HALF else 2
        bad = ~torch.isfinite(y)
        want = torch.zeros_like(bad)
        want[1, 0, 3] = want[1, 0, partner] = want[2, 1, 13] = want[3, 0, 12] = True
        assert torch.equal(bad, want)


@pytest.mark.gpu
def test_bytes_around_the_outputs_and_the_streams(mv):
    """Nothing outside the outputs is written; the call goes to the current stream and can be captured."""
    n, h, d = 5, 3, 40
    big = torch.full((n * h * d + 512,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big[256:256 + n * h * d].view(n, h, d)
    x = torch.randn((n, h, d), device="cuda").to(torch.bfloat16)
    lens = torch.tensor([11], dtype=torch.int32, device="cuda")
    desc, turns = mv.rope_desc(1, n, h, 0, d, 40), mv.massv_rope_frequencies(40, 1e4)
    mv.massv_rotary(desc, turns, x, None, out, None, seq_lens=lens)
    want = out.clone()
    assert bool((big[:256] == 7).all()) and bool((big[-256:] == 7).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = torch.empty_like(x)
        mv.massv_rotary(desc, turns, x, None, other, None, seq_lens=lens)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mv.massv_rotary(desc, turns, x, None, other, None, seq_lens=lens)
    lens.fill_(12)
    graph.replay()
    lens_out = torch.empty_like(x)
    mv.massv_rotary(desc, turns, x, None, lens_out, None, seq_lens=lens)
    torch.cuda.synchronize()
    assert torch.equal(other, lens_out) and not torch.equal(other, want)
    with pytest.raises(ValueError, match="as many as"):
        mv.massv_rotary(desc, turns, x[:4], None, out, None, seq_lens=lens)
    with pytest.raises(ValueError, match="contiguous"):
        mv.massv_rotary(desc, turns, x.transpose(0, 1).contiguous().transpose(0, 1), None, out, None, seq_lens=lens)
