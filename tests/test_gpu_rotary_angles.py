"""One angle for a position and a frequency, whichever operator and however many rows at a time; far positions."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_cache import BF, FP, gen, i32, make_table, normal   # noqa: E402

import paper_2410_03355_b200 as lt   # noqa: E402

pytestmark = pytest.mark.gpu


def steep(sections, far, B, R, seed):
    """Frequencies of all sizes and positions of all sizes, negative ones among them."""
    pairs = sum(sections)
    freq = torch.exp(torch.rand(pairs, generator=gen(seed)) * 18.0 - 16.0)   # 1e-7 to 7
    freq[-1] = -freq[-1]
    pos = (torch.exp(torch.rand((len(sections), B, R), generator=gen(seed + 1), dtype=torch.float64) * math.log(far)) - 1).long()
    pos = torch.where(torch.rand(pos.shape, generator=gen(seed + 2)) < 0.3, -pos, pos)
    pos.view(-1)[:3] = torch.tensor([far, -far, 0])
    return freq, pos.clamp(-2 ** 31, 2 ** 31 - 1).int()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("S,D,H,sections,interleaved", [(16, 64, 2, (16, 16), True), (64, 128, 3, (16, 24, 24), False), (32, 80, 1, (5, 9), False)])
def test_the_same_codes_however_rows_are_appended(S, D, H, sections, interleaved, dtype):
    B, R = 3, 8
    table = make_table(B, 2, 2 * B, 300)
    freq, pos = steep(sections, 2 ** 31 - 1, B, R, 301)
    rot = lt.Rotation(freq.cuda(), sections, interleaved=interleaved)
    k, v = normal((B, R, H, D), 304, dtype), normal((B, R, H, D), 305, dtype)
    k[:, 0] *= 4.0   # (the first row sets the scale: no code is made anew)
    v[:, 0] *= 4.0
    caches = []
    for step in (8, 1, 2, 5):
        c = lt.KVCache.empty(2 * B, H, S, D)
        for r in range(0, R, step):
            part = slice(r, min(R, r + step))
            lt.cache_append(k[:, part], v[:, part], c, table, i32([r] * B), positions=pos[:, :, part].contiguous().cuda(), rotation=rot)
        caches.append(c)
    for c in caches[1:]:
        assert torch.equal(c.k.view(torch.uint8), caches[0].k.view(torch.uint8))
        assert torch.equal(c.k_scale, caches[0].k_scale)
    # and they are the codes of the rows that rotary turns
    turned = lt.rotary(k.float(), pos.cuda(), rot)
    c = lt.KVCache.empty(2 * B, H, S, D)
    lt.cache_append(turned, v.float(), c, table, i32([0] * B))
    assert torch.equal(c.k.view(torch.uint8), caches[0].k.view(torch.uint8))


# cos and sin of exact angles: what is left of the angle after 64-bit fractions of a turn is off by 2^-33 turns at most; near and rest are rounded once each
# (2^-25 of half a turn and 2^-24 of that), sincospif is good to two units (2^-23 of at most 1), the turn by the rest is a product and a sum (2^-24 each)
ANGLE = 2 * math.pi * 2.0 ** -33 + math.pi * 2.0 ** -48 + 2.0 ** -23 + 2 * 2.0 ** -24


@pytest.mark.parametrize("inverse", [False, True])
def test_far_positions_turn_as_exactly_as_near_ones(inverse):
    """(1, 0) turned is (cos, sin): against angles reduced with 200 bits."""
    from fractions import Fraction
    pi = Fraction(3141592653589793238462643383279502884197169399375105820974944592307816406286, 10 ** 75)
    R, pairs = 200, 32
    freq, pos = steep((pairs,), 2 ** 31 - 1, 1, R, 310)
    x = torch.zeros(1, R, 1, 2 * pairs)
    x[..., 0::2] = 1.0
    got = lt.rotary(x.cuda(), pos.cuda(), lt.Rotation(freq.cuda(), (pairs,), interleaved=True), inverse=inverse)[0, :, 0].cpu().double()
    for r in range(R):
        for j in range(pairs):
            turns = Fraction(int(pos[0, 0, r])) * Fraction(float(freq[j])) / (2 * pi)
            phi = float((turns - round(turns)) * 2 * pi) * (-1.0 if inverse else 1.0)
            assert abs(got[r, 2 * j] - math.cos(phi)) <= ANGLE and abs(got[r, 2 * j + 1] - math.sin(phi)) <= ANGLE, (r, j)
