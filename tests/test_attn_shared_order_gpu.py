"""Shared-prefix attention where one CTA goes through many items of different kinds: what a wait stands for must not depend on how far the
other roles have come.  Against 64 bits, and many calls that have to agree in every bit."""
import pytest
import torch

import test_attn_shared as attn
from test_attn_shared import mv  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def _same_again(mv, w, times):
    """The first call's results; the others' have to equal them."""
    out, out32, lse, status = attn._run(mv, w)
    assert status == 0
    for _ in range(times):
        again = attn._run(mv, w)
        assert all(torch.equal(x, y) for x, y in zip((out, out32, lse), again)) and again[3] == 0
    return out, out32, lse


# 8 query heads to a KV head and 8 block rows: two sequences to a tile.  5, 6 and 9, 10 and 13, 14 sequences: 3, 5 and 7 tiles, so that an item
# on one tile ends a group and an item on two begins the next.
ODD_TILES = [5, 4, 9, 2, 13, 6, 1, 10, 2, 3, 14, 2]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_groups,blocks,hkv", [(256, (1, 2, 3, 4, 5), 1), (256, (1,), 1), (256, (2,), 2), (256, (4, 1), 1), (200, (3, 1, 2), 1), (60, (5, 2, 1, 4, 3), 3), (11, (1, 3, 2), 4)])
def test_items_on_one_tile_ahead_of_items_on_two(mv, d, n_groups, blocks, hkv):
    sizes = [ODD_TILES[(i * 5 + 1) % len(ODD_TILES)] for i in range(n_groups)]
    w = attn._make(sizes, [128 * blocks[i % len(blocks)] for i in range(n_groups)], [0, 3, 20], 7, 8 * hkv, hkv, d, d + n_groups)
    attn._check(w, *_same_again(mv, w, 30))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sizes", [[11, 21, 32], [2, 21, 1, 11, 32], [3, 30, 3, 12]])
def test_long_items_on_one_tile(mv, d, sizes):
    """28 query heads on 4, six rows: three sequences to a tile; long prefixes, so that the ranges of the CTAs cut every kind of item."""
    w = attn._make(sizes, [2048 + 384 * i for i in range(len(sizes))], [100, 7, 260], 5, 28, 4, d, 3)
    attn._check(w, *_same_again(mv, w, 10))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_groups,size", [(256, 4), (251, 3), (243, 4), (230, 6), (214, 4), (199, 5), (187, 8), (150, 7)])
def test_tails_behind_short_items_on_two_tiles(mv, d, n_groups, size):
    """Prefixes of a block or two: one CTA ends several items on two tiles and goes on with tails, which use both tiles' scores and accumulators."""
    w = attn._make([size] * n_groups, [128 * (1 + i % 2) for i in range(n_groups)], [0, 3, 140], 7, 8, 1, d, n_groups)
    attn._check(w, *_same_again(mv, w, 30))


@pytest.mark.parametrize("d", [256, 128, 64])
@pytest.mark.parametrize("sizes,shared,tails,gamma,hq,hkv", [([5, 3], [2048, 0], [0, 1900], 3, 16, 8), ([1, 1, 1], [0, 0, 0], [3000, 2500, 200], 5, 16, 8), ([12], [1536], [700, 30], 7, 8, 2), ([40], [0], [500, 900], 1, 16, 8)])
def test_maxima_that_rise_in_the_second_half_of_every_block(mv, d, sizes, shared, tails, gamma, hq, hkv):
    """The accumulator is rescaled between a block's halves, each time behind a product that may still be waiting for its V."""
    w = attn._make(sizes, shared, tails, gamma, hq, hkv, d, 17)
    g = torch.Generator(device="cuda").manual_seed(d)
    for b in range(sum(sizes)):
        for i, page in enumerate(w["page_table"][b].tolist()):
            if page >= 0 and i % 8 >= 4:                                    # a block is 8 pages; 3 log2 units per block and unit of the row's spread
                w["k_pages"][page] = (torch.randn((hkv, 16, d), dtype=torch.bfloat16, device="cuda", generator=g).float() * (1 + 3 * (i // 8))).to(torch.bfloat16)
    attn._check(w, *_same_again(mv, w, 30))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("sizes,shared,gamma,hq,hkv", [([3], 512, 0, 2, 1), ([3, 4], 2048, 2, 8, 2), ([40, 30], 256, 3, 16, 8)])
def test_keys_that_are_no_numbers(mv, d, sizes, shared, gamma, hq, hkv):
    """A part of a row's context of which no score is a number: the row is none either, and nothing else changes."""
    w = attn._make(sizes, [shared] * len(sizes), [0], gamma, hq, hkv, d, 21)
    want = attn._run(mv, w)
    w["k_new"][1, 0] = float("nan")                                         # all that this sequence's first row has behind the prefix
    got = attn._run(mv, w)
    assert got[3] == 0
    for x, y in zip(got[:3], want[:3]):
        assert bool(torch.isnan(x[1]).all()) and torch.equal(x[0], y[0]) and torch.equal(x[2:], y[2:])
    for block in range(shared // 128):                                      # the first group's prefix, a block at a time
        w = attn._make(sizes, [shared] * len(sizes), [0], gamma, hq, hkv, d, 21)
        w["k_pages"][w["page_table"][0, block * 8:block * 8 + 8].long()] = float("nan")
        got = attn._run(mv, w)
        for x, y in zip(got[:3], want[:3]):
            assert bool(torch.isnan(x[:sizes[0]]).all()) and torch.equal(x[sizes[0]:], y[sizes[0]:])


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("factor", [0.25, 4.0])
def test_an_explicit_scale(mv, d, factor):
    """A power of two times 1 / sqrt(d) is the same as queries times that power."""
    w = attn._make([4, 3], [512, 200], [9, 40], 3, 8, 2, d, 8)
    desc = mv.attn_desc(7, 3, 8, 2, d, w["page_table"].shape[1], w["k_pages"].shape[0], scale=factor * d ** -0.5)
    ws = mv.alloc_workspace(mv.massv_verify_attn_shared_workspace_size(desc, 2), "cuda").fill_(0xff)
    out, out32, lse, status = torch.empty_like(w["q"]), torch.empty(w["q"].shape, device="cuda"), torch.empty(w["q"].shape[:3], device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
    mv.massv_verify_attn_shared(desc, w["start"], w["shared"], w["q"], w["k_new"], w["v_new"], w["k_pages"], w["v_pages"], w["page_table"], w["seq_lens"], out, out32, lse, ws, status)
    assert int(status.item()) == 0
    attn._check(dict(w, q=w["q"] * factor), out, out32, lse)
