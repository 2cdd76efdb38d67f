"""Verify attention over a shared prefix: against attention in 64 bits on the same bf16 values, and what is refused."""
import ctypes
import math

import pytest
import torch

import __graft_entry__ as entry


@pytest.fixture(scope="module")
def mv():
    entry.build()
    import paper_2505_10526_b200 as pkg
    return pkg.binding


def test_refusals(mv):
    lib, a = mv._lib, 0x1000
    d = mv.attn_desc(4, 3, 8, 2, 64, 20, 100)

    def call(desc, n_groups=1, start=a, shared=a, q=a, ws=a, n=1 << 50):
        return lib.massv_verify_attn_shared(ctypes.byref(desc), n_groups, start, shared, q, a, a, a, a, a, a, a, None, None, ws, n, None, None)
    assert call(d, n_groups=0) == -1 and call(d, start=None) == -1 and call(d, shared=None) == -1 and call(d, q=None) == -1 and call(d, q=a + 8) == -1
    assert call(d, n_groups=257) == -2 and call(mv.attn_desc(4, 3, 8, 2, 64, 20, 100, window=64)) == -2 and call(mv.attn_desc(4, 3, 8, 2, 80, 20, 100)) == -2
    assert call(mv.attn_desc(4, 9, 8, 2, 64, 20, 100)) == -2 and call(mv.attn_desc(4, 3, 8, 3, 64, 20, 100)) == -2
    assert call(d, ws=None) == -4 and call(d, ws=a + 16) == -4 and call(d, n=1000) == -4
    size = mv.massv_verify_attn_shared_workspace_size
    assert size(d, 1) > 0 and size(mv.attn_desc(2049, 3, 8, 2, 64, 20, 100), 1) == 0 and size(d, 0) == 0 and size(d, 257) == 0 and size(mv.attn_desc(4, 3, 8, 2, 64, 20, 100, window=1), 1) == 0
    i, b = torch.zeros(2, dtype=torch.int32), torch.zeros(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA device"):
        mv.massv_verify_attn_shared(d, i, i[:1], b, b, b, b, b, i, i, b)
    with pytest.raises(TypeError):
        mv.massv_verify_attn_shared(mv.accept_desc(1, 1, 64, 64, 1.0), i, i[:1], b, b, b, b, b, i, i, b)


@pytest.mark.parametrize("kw", [dict(window=64, n_groups=1), dict(n_groups=257), dict(n_groups=-1)])
def test_a_step_that_cannot_share_is_refused(mv, kw):
    import paper_2505_10526_b200 as pkg
    with pytest.raises(ValueError, match="share a prefix"):
        pkg.VerifyStep(4, 3, 8, 2, 64, 64, 64, 0.0, 20, 100, device="cpu", **kw)


# ---------------------------------------------------------------- on the GPU
def _make(sizes, shared, tails, gamma, hq, hkv, d, seed, slope=0.0, extra_pages=1):
    """Groups of sizes[g] sequences whose page tables agree on the whole pages of shared[g] positions; tails: positions behind them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    batch, rows = sum(sizes), gamma + 1
    group = [i for i, n in enumerate(sizes) for _ in range(n)]
    lens = [shared[group[b]] + tails[b % len(tails)] for b in range(batch)]
    per_seq = max((n + rows + 15) // 16 for n in lens) + extra_pages
    own = [max(0, (lens[b] + rows + 15) // 16 - shared[group[b]] // 16) for b in range(batch)]
    n_pages = sum(s // 16 for s in shared) + sum(own) + 2
    ids = torch.randperm(n_pages, generator=g, device="cuda").tolist()
    table = torch.full((batch, per_seq), -1, dtype=torch.int32)           # entries that no position needs are not looked at
    at, prefix = 0, []
    for s in shared:
        prefix.append(ids[at:at + s // 16])
        at += s // 16
    for b in range(batch):
        mine = prefix[group[b]] + ids[at:at + own[b]]
        at += own[b]
        table[b, :len(mine)] = torch.tensor(mine, dtype=torch.int32)
    bf = dict(dtype=torch.bfloat16, device="cuda", generator=g)
    w = dict(q=torch.randn((batch, rows, hq, d), **bf), k_new=torch.randn((batch, rows, hkv, d), **bf), v_new=torch.randn((batch, rows, hkv, d), **bf),
             k_pages=torch.randn((n_pages, hkv, 16, d), **bf), v_pages=torch.randn((n_pages, hkv, 16, d), **bf), page_table=table.cuda(),
             seq_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), shared=torch.tensor(shared, dtype=torch.int32, device="cuda"),
             start=torch.tensor([sum(sizes[:i]) for i in range(len(sizes) + 1)], dtype=torch.int32, device="cuda"))
    for spare in ids[at:]:                                                # pages of nobody hold what poisons a product with weight zero
        w["k_pages"][spare] = float("nan"); w["v_pages"][spare] = float("nan")
    if slope:                                                             # scores whose maxima keep rising along the context
        for b in range(batch):
            for i, page in enumerate(table[b].tolist()):
                if page >= 0:
                    w["k_pages"][page] = (torch.randn((hkv, 16, d), **bf).float() * (1 + slope * i)).to(torch.bfloat16)
    return w


def _reference(w, b):
    """Rows of sequence b in 64 bits, and the weighted magnitudes that bound the rounding of the weights."""
    rows, hq, d = w["q"].shape[1:]
    hkv, n = w["k_new"].shape[2], int(w["seq_lens"][b])
    G = hq // hkv
    pages = w["page_table"][b, :(n + 15) // 16].long()
    k, v = (torch.cat([w[p][pages].transpose(0, 1).reshape(hkv, -1, d)[:, :n], w[x][b].transpose(0, 1)], dim=1).double() for p, x in (("k_pages", "k_new"), ("v_pages", "v_new")))
    s = w["q"][b].double().view(rows, hkv, G, d).permute(1, 0, 2, 3).reshape(hkv, rows * G, d) @ k.transpose(1, 2) / math.sqrt(d)
    pos, row = torch.arange(n + rows, device="cuda"), n + torch.arange(rows, device="cuda").repeat_interleave(G)
    s.masked_fill_((pos[None] > row[:, None])[None], -math.inf)
    a = torch.softmax(s, -1)
    back = lambda x: x.view(hkv, rows, G, -1).permute(1, 0, 2, 3).reshape(rows, hq, -1)
    return back(a @ v), back(a @ v.abs()), back(torch.logsumexp(s, -1, keepdim=True))[..., 0], float(s[torch.isfinite(s)].abs().max())


def _run(mv, w, n_pages=None, f32=True, ws=None):
    batch, rows, hq, d = w["q"].shape
    desc = mv.attn_desc(batch, rows - 1, hq, w["k_new"].shape[2], d, w["page_table"].shape[1], w["k_pages"].shape[0])
    if ws is None:
        ws = mv.alloc_workspace(mv.massv_verify_attn_shared_workspace_size(desc, w["shared"].numel()), "cuda").fill_(0xff)
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    big = torch.full((w["q"].numel() + 512,), 3.0, dtype=torch.bfloat16, device="cuda")
    out = big[256:-256].view_as(w["q"])
    out32 = torch.full(out.shape, float("nan"), device="cuda") if f32 else None
    lse = torch.full(out.shape[:3], float("nan"), device="cuda") if f32 else None
    mv.massv_verify_attn_shared(desc, w["start"], w["shared"], w["q"], w["k_new"], w["v_new"], w["k_pages"], w["v_pages"], w["page_table"], w["seq_lens"], out, out32, lse, ws, status)
    assert bool((big[:256] == 3).all()) and bool((big[-256:] == 3).all())
    return out, out32, lse, int(status.item())


def _check(w, out, out32, lse, skipped=()):
    for b in range(w["q"].shape[0]):
        if b in skipped:
            continue
        want, size, want_lse, top = _reference(w, b)
        # weights rounded to bf16 by 2^-8 at most; the scores' fp32 sums of d products move a weight by top * 2^-20, its exponential
        # and the sums by 2^-20; the bf16 output another 2^-8 of itself
        bound = size * (2.0 ** -8 + 2.0 ** -20 * (2 + 2 * top))
        assert bool(((out32.double()[b] - want).abs() <= bound).all()), b
        assert bool(((out.double()[b] - want).abs() <= bound * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8).all()), b
        assert float((lse.double()[b] - want_lse).abs().max()) <= 2.0 ** -20 * (4 + 3 * top), b
        n = int(w["seq_lens"][b])
        for j in range(w["q"].shape[1]):                                   # the block's rows are in their slots
            page, at = int(w["page_table"][b, (n + j) // 16]), (n + j) % 16
            assert torch.equal(w["k_pages"][page, :, at], w["k_new"][b, j]) and torch.equal(w["v_pages"][page, :, at], w["v_new"][b, j])


CASES = [
    # sizes, shared positions, tails, gamma, query heads, KV heads
    ([2], [128], [0, 1], 0, 1, 1), ([2], [127], [3], 2, 4, 1), ([3], [128], [0], 5, 7, 1), ([4], [256 + 17], [0, 40, 15, 16], 5, 28, 4), ([2], [1000], [5, 300], 7, 8, 8),
    ([1, 2, 3], [300, 129, 640], [10, 0, 63, 64], 3, 12, 4), ([5, 0, 4], [512, 900, 2000], [33, 1], 2, 10, 2), ([9], [4096], [100, 7, 0], 5, 9, 1), ([7], [700], [1], 0, 64, 1),
    ([16], [1536], [20, 200], 0, 32, 2), ([33], [384], [5, 70, 128], 7, 6, 2), ([12, 13], [1920, 260], [77], 6, 9, 3), ([64], [260], [0, 9], 1, 8, 8), ([40], [256], [500, 2], 3, 16, 8),
    ([3, 3, 3, 3], [128, 0, 50, 1280], [12, 600], 1, 16, 8)]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("sizes,shared,tails,gamma,hq,hkv", CASES)
def test_against_64_bits(mv, sizes, shared, tails, gamma, hq, hkv, d):
    w = _make(sizes, shared, tails, gamma, hq, hkv, d, sum(sizes) + d)
    out, out32, lse, status = _run(mv, w)
    assert status == 0
    _check(w, out, out32, lse)
    again = _run(mv, w)
    assert all(torch.equal(x, y) for x, y in zip((out, out32, lse), again))                    # sums in a fixed order
    assert torch.equal(_run(mv, w, f32=False)[0], out)                                          # and without the optional outputs


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128, 256])
def test_maxima_that_keep_rising(mv, d):
    """The reference of the weights has to move, in both tiles and at other blocks in each row."""
    w = _make([6, 14], [1700, 1100], [40, 3], 5, 14, 2, d, d, slope=0.15)
    out, out32, lse, status = _run(mv, w)
    assert status == 0
    _check(w, out, out32, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128, 256])
def test_sequences_without_room_are_skipped(mv, d):
    """A negative length, one beyond the table: skipped and reported, the output rows left as they were; the others share what they share."""
    w = _make([5, 4], [512, 384], [9, 30, 2], 3, 8, 2, d, d)
    w["seq_lens"][0] = -5                                                 # the first of its group, whose table is then not the one to read
    w["page_table"][0] = -1
    w["seq_lens"][7] = w["page_table"].shape[1] * 16 - 3
    out, out32, lse, status = _run(mv, w)
    assert status == -3
    _check(w, out, out32, lse, skipped=(0, 7))
    for b in (0, 7):
        assert bool((out[b] == 3).all()) and bool(torch.isnan(out32[b]).all()) and bool(torch.isnan(lse[b]).all())


@pytest.mark.gpu
def test_more_shared_than_committed(mv):
    """shared_lens beyond a member's length is that length; negative is none."""
    w = _make([4, 3], [640, 300], [50, 0, 8], 2, 8, 2, 128, 3)
    whole = _run(mv, w)
    w["shared"][0] = 2 ** 31 - 1; w["shared"][1] = -4
    # (what tables have in common ends at the shared pages: the group's shortest member is taken, which is as long as they are here)
    out, out32, lse, status = _run(mv, w)
    assert status == 0 and whole[3] == 0
    _check(w, out, out32, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("start", [[0, 3, 2, 6], [0, 3, 6, 5], [1, 2, 3, 6], [0, 2, 4, 7], [0, -1, 3, 6], [6, 6, 6, 6], [0, 2 ** 31 - 1, 3, 6]])
def test_groups_that_are_none(mv, start):
    """Reported; every sequence is then read by itself, and right."""
    w = _make([2, 2, 2], [256, 256, 256], [10, 20], 1, 4, 2, 64, 1)
    w["start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
    out, out32, lse, status = _run(mv, w)
    assert status == -1
    _check(w, out, out32, lse)


@pytest.mark.gpu
def test_an_unmapped_page_of_the_prefix_is_reported(mv):
    w = _make([3], [512], [10], 1, 4, 2, 128, 1)
    w["page_table"][:, 5] = w["k_pages"].shape[0]
    assert _run(mv, w)[3] == -3


@pytest.mark.gpu
def test_many_groups(mv):
    w = _make([2] * 256, [128 + 16 * (i % 3) for i in range(256)], [1, 30, 5], 0, 2, 1, 64, 9)
    out, out32, lse, status = _run(mv, w)
    assert status == 0
    _check(w, out, out32, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("d,hq,hkv", [(128, 28, 4), (256, 16, 8)])
def test_long_prefix_and_agreement_with_massv_verify_attn(mv, d, hq, hkv):
    w = _make([24, 8], [6000, 3333], [100, 900, 0], 5, hq, hkv, d, 2)
    out, out32, lse, status = _run(mv, w)
    assert status == 0
    desc = mv.attn_desc(32, 5, hq, hkv, d, w["page_table"].shape[1], w["k_pages"].shape[0])
    ws = mv.alloc_workspace(mv.massv_verify_attn_workspace_size(desc), "cuda")
    o2, f2, l2 = torch.empty_like(out), torch.empty_like(out32), torch.empty_like(lse)
    mv.massv_verify_attn(desc, w["q"], w["k_new"], w["v_new"], w["k_pages"], w["v_pages"], w["page_table"], w["seq_lens"], o2, f2, l2, ws, None)
    # two roundings of the weights (2^-8 of the weighted magnitudes at most, far less in the norm)
    assert float(((out32 - f2).norm(dim=-1) / f2.norm(dim=-1)).max()) < 8e-3 and float((lse - l2).abs().max()) < 1e-4
    w["seq_lens"] = w["seq_lens"][:3].contiguous(); w["q"] = w["q"][:3].contiguous()
    for n in ("k_new", "v_new", "page_table"):
        w[n] = w[n][:3].contiguous()
    _check(w, out[:3], out32[:3], lse[:3])


@pytest.mark.gpu
def test_captured_with_lengths_that_change(mv):
    """A captured call takes groups and lengths from the device: replayed after a commit and after the groups changed; a second
    call with a workspace of its own runs beside it on another stream."""
    w = _make([4, 4], [640, 384], [50, 10], 3, 8, 2, 128, 4, extra_pages=4)
    pages = w["k_pages"].shape[0]
    # room for a second block
    table, spare = w["page_table"].clone(), torch.randn((8 * 2, 2, 16, 128), device="cuda").to(torch.bfloat16)
    w["k_pages"], w["v_pages"] = (torch.cat((w[n], spare)).contiguous() for n in ("k_pages", "v_pages"))
    for b in range(8):
        used = (int(w["seq_lens"][b]) + 4 + 15) // 16
        table[b, used:used + 2] = torch.arange(pages + 2 * b, pages + 2 * b + 2, dtype=torch.int32)
    w["page_table"] = table
    desc = mv.attn_desc(8, 3, 8, 2, 128, table.shape[1], w["k_pages"].shape[0])
    new_ws = lambda: mv.alloc_workspace(mv.massv_verify_attn_shared_workspace_size(desc, 2), "cuda")
    ws, status = new_ws(), torch.zeros((1,), dtype=torch.int32, device="cuda")
    out, out32, lse = torch.empty_like(w["q"]), torch.empty(w["q"].shape, device="cuda"), torch.empty(w["q"].shape[:3], device="cuda")
    args = (w["q"], w["k_new"], w["v_new"], w["k_pages"], w["v_pages"], w["page_table"], w["seq_lens"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mv.massv_verify_attn_shared(desc, w["start"], w["shared"], *args, out, out32, lse, ws, status)
    for change in (lambda: None, lambda: w["seq_lens"].add_(2), lambda: w["shared"].copy_(torch.tensor([130, 384])), lambda: (w["start"].copy_(torch.tensor([0, 2, 8])), w["shared"].copy_(torch.tensor([300, 0])))):
        change()
        graph.replay()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = torch.empty_like(out)
            mv.massv_verify_attn_shared(desc, w["start"], w["shared"], *args, other, None, None, new_ws(), status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        _check(w, out, out32, lse)
        assert torch.equal(other, out)
