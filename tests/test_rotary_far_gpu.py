"""Rotary positions far out: the turned values against angles worked out in many digits from the formula of the frequencies, not from their rounded fractions."""
from decimal import Decimal

import pytest
import torch

from test_rotary import PI, _check, _frequencies, mv  # noqa: F401  (mv: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("rot,base", [(64, 10000.0), (128, 1e6), (36, 500000.0)])
def test_positions_near_the_largest(mv, half, rot, base):
    pos = [0, 1, 4095, 131071, 10 ** 9, 10 ** 9 + 7, 2 ** 30 - 1, 2 ** 31 - 1, -1, -10 ** 9, -2 ** 31]
    turns = [f / (2 * PI) for f in _frequencies(rot, base)]
    # off by 16 * 2^-64 of a turn times 2^31 and by 2^-26 of a turn in the kernel: 2 pi (2^-29 + 2^-26), 1.1e-7 of a
    # radian, beside _check's other terms of 2^-22 within its 2^-20 of the products
    angle = torch.tensor([[float(((p * t) % 1) * 2 * PI) for t in turns] for p in map(Decimal, pos)], dtype=torch.float64, device="cuda")
    d = (rot + 15) // 8 * 8                                               # heads are multiples of 8, with something behind rot_dim to copy
    x = torch.randn((len(pos), 3, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(rot)).to(torch.bfloat16)
    out = torch.empty_like(x)
    desc = mv.rope_desc(1, len(pos), 3, 0, d, rot, layout=mv.ROPE_HALF if half else mv.ROPE_INTERLEAVED)
    mv.massv_rotary(desc, mv.massv_rope_frequencies(rot, base), x, None, out, None, positions=torch.tensor(pos, dtype=torch.int64).to(torch.int32).cuda())
    _check(out, x, angle, rot, half, 1.0)
