"""Attention to the paged cache on the GPU, every kernel and division, against 64 bits and the bound of attention_cases.py."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import attention_cases as cases   # noqa: E402
from test_gpu_cache import close, filled_cache, gen, i32, make_table, normal, random_tree   # noqa: E402

import paper_2410_03355_b200 as lt   # noqa: E402

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32
TYPES = {"bf16": BF, "f32": FP}


def check(q, cache, table, lengths, *, counts=None, starts=None, parents=None, scale=None):
    """One call against the 64-bit reference; rows that `counts` leaves out stay as they are."""
    status = torch.zeros(len(lengths), dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 5.0)
    lt.cache_attention(q, cache, table, i32(lengths), counts=None if counts is None else i32(counts), starts=None if starts is None else i32(starts),
                       tree_parents=None if parents is None else parents.cuda(), scale=scale, out=out, status=status)
    assert not status.any()
    want, bound = cases.attention(q.cpu(), cache, table.tolist(), lengths, counts, starts, None if parents is None else parents.tolist(), scale)
    left_out = want.isnan()
    assert (out.cpu()[left_out] == 5.0).all()
    close(torch.where(left_out.cuda(), torch.zeros_like(out), out), want.nan_to_num(0.0), bound, q.dtype)
    return out, want


# (rows, heads a group, components, room): few, mid (bf16; fp32: wide), wide with at most 64 rows, wide
FORMS = [(1, 4, 128, 8192), (9, 1, 64, 8192), (40, 1, 64, 1984), (40, 1, 128, 960), (33, 1, 64, 8192), (33, 1, 128, 8192), (35, 2, 64, 8192), (50, 3, 96, 8192)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,G,D,room", FORMS)
def test_few_values_on_a_long_axis(R, G, D, room, dtype):
    """Scores are random, but of a component's values all but three are zero: nothing is added up but the weights themselves, whose every bit shows."""
    S, H, B = 64, 2, 2
    lengths, width = [room - R - 3, room // 2], room // S
    table = make_table(B, width, B * width, 220)
    cache = filled_cache(table, [n + R for n in lengths], H, S, D, B * width, 221)
    cache.k_scale.fill_(2.0 ** -8)
    some = torch.rand(cache.v.shape, generator=gen(222)) < 3.0 / lengths[1]
    cache.v.copy_(torch.where(some, torch.randint(1, 8, cache.v.shape, generator=gen(223)).float(), torch.zeros(())).to(torch.float8_e4m3fn))
    q = normal((B, R, H * G, D), 224, TYPES[dtype])
    parents = random_tree(B, R - 1, 6, 225) if R > 1 else None
    check(q, cache, table, lengths, parents=parents)
    check(q, cache, table, lengths, parents=parents, starts=[room // 3, 0], scale=3.0 / D ** 0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,G,D,room", FORMS)
@pytest.mark.parametrize("sink", [0.0, 0.125])
def test_one_token_takes_the_row(R, G, D, room, dtype, sink):
    """A first token far ahead of all others and with little or no value of its own: the output is what the others leave, each 2^-8 to 2^-34 of the first."""
    S, H, B = 64, 1, 2
    lengths, width = [room - R - 3, room // 2], room // S
    table = make_table(B, width, B * width, 230)
    cache = lt.KVCache.empty(B * width, H, S, D)
    cache.v.copy_((1.0 + torch.rand(cache.v.shape, generator=gen(231))).to(torch.float8_e4m3fn))
    k, v = torch.zeros(cache.k.shape), cache.v.float()
    for b in range(B):
        k[table[b, 0], :, 0, 0] = 16.0
        v[table[b, 0], :, 0] = sink
    cache.k.copy_(k.to(torch.float8_e4m3fn))
    cache.v.copy_(v.to(torch.float8_e4m3fn))
    q = torch.zeros((B, R, H * G, D))
    behind = torch.linspace(8.3, 34.3, R * G).view(R, G)   # in powers of two, row by row
    q[..., 0] = (behind / 16.0 * 0.6931471805599453).flatten()[None].expand(B, -1).view(B, R, H * G)
    check(q.to(TYPES[dtype]).cuda(), cache, table, lengths, scale=1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,G,D,room", FORMS)
def test_blocks_of_very_different_scales(R, G, D, room, dtype):
    """Blocks whose values are 2^-28 of others': seen in the components where the others are zero."""
    S, H, B = 16, 1, 2
    lengths, width = [200, 90], room // S
    table = make_table(B, width, B * width, 250)
    cache = filled_cache(table, [n + R for n in lengths], H, S, D, B * width, 251)
    cache.k_scale.fill_(2.0 ** -4)
    small = torch.randint(0, 2, cache.v_scale.shape, generator=gen(252)).bool()
    cache.v_scale.copy_(torch.where(small, 2.0 ** -28, 1.0))
    v = cache.v.float().cpu().nan_to_num(0.0)
    v[..., D // 2:] *= small[:, :, None, None]
    cache.v.copy_(v.to(torch.float8_e4m3fn))
    check(normal((B, R, H * G, D), 253, TYPES[dtype]), cache, table, lengths, scale=0.25)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,G,D,room", FORMS)
def test_scales_that_are_no_powers_of_two(R, G, D, room, dtype):
    """A cache of the caller's own making: any positive scale."""
    S, H, B = 32, 2, 2
    lengths, width = [300, 97], room // S
    table = make_table(B, width, B * width, 240)
    cache = filled_cache(table, [n + R for n in lengths], H, S, D, B * width, 241)
    for i, t in enumerate((cache.k_scale, cache.v_scale)):
        t.mul_(1.0 + torch.rand(t.shape, generator=gen(242 + i)).cuda())
    some = torch.rand(cache.v.shape, generator=gen(244)) < 3.0 / lengths[1]   # (as above: the weights and scales themselves)
    cache.v.copy_(torch.where(some, cache.v.float().cpu().nan_to_num(0.0), torch.zeros(())).to(torch.float8_e4m3fn))
    check(normal((B, R, H * G, D), 245, TYPES[dtype]), cache, table, lengths)
