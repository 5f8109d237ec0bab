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


@pytest.mark.parametrize("case", cases.CASES, ids=cases.name_of)
def test_against_64_bits(case):
    c = case
    B, R, H, D, S = len(c["lengths"]), c["R"], c["H"], c["D"], c["S"]
    width = c["room"] // S
    held = [n + m for n, m in zip(c["lengths"], c.get("counts") or [R] * B)]
    need = [-(-n // S) for n in held]
    pages = sum(need) + 1
    pool = torch.randperm(pages, generator=gen(200)).tolist()
    table = torch.full((B, width), 1 << 20, dtype=torch.int32)   # entries behind a sequence's tokens are not read
    for b in range(B):
        table[b, :need[b]] = torch.tensor([pool.pop() for _ in range(need[b])], dtype=torch.int32)
    cache = filled_cache(table, held, H, S, D, pages, 201)
    q = normal((B, R, H * c["G"], D), 202, TYPES[c["dtype"]])
    check(q, cache, table.cuda(), c["lengths"], counts=c.get("counts"), starts=c.get("starts"),
          parents=random_tree(B, R - 1, c["tree"], 203) if c.get("tree") else None)


# (rows, heads a group, components, room): few, mid (bf16; fp32: wide), wide with at most 64 rows, wide
FORMS = [(1, 4, 128, 8192), (9, 1, 64, 8192), (40, 1, 64, 1984), (40, 1, 128, 960), (33, 1, 64, 8192), (33, 1, 128, 8192), (35, 2, 64, 8192), (50, 3, 96, 8192)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,G,D,room", FORMS)
@pytest.mark.parametrize("whole", [False, True])
def test_every_token_counts(R, G, D, room, dtype, whole):
    """All scores equal; token c has a value in component c % D only, and says in it which of the component's tokens it is: an output is a sum of a few
    integers over the number of tokens seen, of which none can be missing, doubled or another's without its component showing it."""
    S = 32
    B, H = (232, 2) if whole else (2, 1)   # (so many units that none is divided)
    full = min(room - R, (12 if dtype == "bf16" else 60) * D)
    lengths = [full, full // 3 + 5] * (B // 2)
    starts = [7, 0] * (B // 2)
    width = room // S
    one = torch.randperm(2 * width, generator=gen(210)).view(2, width).int()
    table = one.repeat(B // 2, 1).cuda()   # (sequences share their pages)
    cache = lt.KVCache.empty(2 * width, H, S, D)
    # the blocks' scales differ; values are whole numbers up to 8, which all their codes hold
    scale = torch.exp2(torch.randint(-3, 1, (2 * width, H), generator=gen(211)).float())
    cache.v_scale.copy_(scale)
    value = torch.zeros(2 * width, H, S, D)
    at = torch.arange(width * S)
    mark = (1 + (at // D) % 8).float()   # 1 to 8
    for b in range(2):
        value[one[b].long()[at // S], :, at % S, at % D] = mark[:, None].expand(-1, H)
    cache.v.copy_((value / scale[:, :, None, None]).to(torch.float8_e4m3fn))
    cache.k.copy_(torch.ones(2 * width, H, S, D).to(torch.float8_e4m3fn))
    q = torch.ones((B, R, H * G, D), dtype=TYPES[dtype], device="cuda")
    got = lt.cache_attention(q, cache, table, i32(lengths), starts=i32(starts)).cpu().double()
    for b in range(2):
        n = torch.arange(R)[:, None]
        see = (at[None] >= starts[b]) & (at[None] <= lengths[b] + n)
        total = torch.zeros(R, D, dtype=torch.float64).index_add_(1, at % D, (see * mark).double())
        want = (total / see.sum(1, keepdim=True))[:, None]
        # numerators are all the same: what exp2 is off by divides out, and so do the parts' weights; what is left of one is that the sum has it as it is and the
        # products as halves (it is 1 but for the rounding of a score of 16: 2^-20).  A sum is n / 32 + 64 additions of 2^-24, the output whole numbers times
        # one factor; then the rounding to the type
        allow = want * ((see.sum(1).max() / 32 + 128) * 2.0 ** -24 + 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24))
        step = 1.0 / see.sum(1).max()   # what the least token adds
        assert step > 2 * allow.max()
        assert ((got[b::2] - want).abs() <= allow).all()


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
