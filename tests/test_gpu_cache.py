"""The cache operators on the GPU against 64-bit references: rotary positions, append, attention, keep, read."""
import math
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import cache_reference as ref   # noqa: E402

import paper_2410_03355_b200 as lt   # noqa: E402

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(shape, seed, dtype=FP, spread=1.0):
    return (torch.randn(shape, generator=gen(seed)) * spread).to(dtype).cuda()


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def make_table(B, width, pages, seed):
    return i32(torch.randperm(pages, generator=gen(seed))[:B * width].view(B, width))


def blank_cache(pages, H, S, D):
    """A cache of blocks that were never written: NaN codes throughout."""
    c = lt.KVCache.empty(pages, H, S, D)
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(ref.NAN_CODE)
    return c


def filled_cache(table, lengths, H, S, D, pages, seed):
    """Random tokens below `lengths`, scales that differ between blocks, NaN codes everywhere else."""
    c = blank_cache(pages, H, S, D)
    g = gen(seed)
    for code, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        scale.copy_(torch.exp2(torch.randint(-10, -4, scale.shape, generator=g).float()))
        value = (torch.randn(code.shape, generator=g) * 80).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).cuda()
        for b, n in enumerate(lengths):
            for block in range(-(-n // S)):
                page, m = int(table[b, block]), min(S, n - block * S)
                code.view(torch.uint8)[page, :, :m] = value[page, :, :m]
    return c


def snapshot(c):
    return ref.Cache(c.k, c.v, c.k_scale, c.v_scale)


def close(got, want, bound, dtype):
    got = got.detach().cpu().to(ref.F64)
    err = (got - want).abs()
    allow = bound + ref.HALF_STEP[dtype] * (want.abs() + bound)
    bad = ~(err <= allow)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float((err - allow)[bad].max() if bad.any() else 0)} at {torch.nonzero(bad)[0].tolist()}"


# ---- rotary -------------------------------------------------------------------------------------------------------------

# cos and sin: the angle in half turns is rounded to 2^-25, sincospif is good to two units (2^-23 of at most 1); products and sum three roundings
TURN = math.pi * 2.0 ** -25 + 2.0 ** -23 + 3 * 2.0 ** -24


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("B,R,H,D,sections", [(1, 1, 1, 2, (1,)), (2, 61, 5, 64, (16, 16)), (3, 7, 2, 128, (16, 24, 24)), (1, 130, 3, 80, (5, 0, 7, 9)),
                                              (2, 9, 1, 6, (1, 2)), (1, 3, 33, 512, (256,)), (1, 2, 2, 48, (8, 8)), (5, 1, 4, 96, (3,))])
def test_rotary(B, R, H, D, sections, interleaved, dtype):
    x = normal((B, R, H, D), 1, dtype)
    pos = torch.randint(-3, 200_000, (len(sections), B, R), generator=gen(2), dtype=torch.int32)
    pos.view(-1)[0] = 2 ** 31 - 1
    freq = 10000.0 ** (-torch.arange(sum(sections)) / sum(sections))
    rot = lt.Rotation(freq.cuda(), sections, interleaved=interleaved)
    for inverse in (False, True):
        want, mag = ref.rotate(x.cpu(), pos, freq, sections, interleaved, inverse)
        got = lt.rotary(x, pos.cuda(), rot, inverse=inverse)
        close(got, want, TURN * mag, dtype)
    # in place, and components in the middle of a wider row (other strides, odd alignment)
    y = x.clone()
    assert lt.rotary(y, pos.cuda(), rot, out=y, inverse=True) is y and torch.equal(y, got)
    wide = torch.zeros((B, R, H + 2, D + 3), dtype=dtype, device="cuda")
    view = wide[:, :, 1:1 + H, 1:1 + D]
    view.copy_(x)
    lt.rotary(view, pos.cuda(), rot, out=view, inverse=True)
    assert torch.equal(view, got)
    view.zero_()
    assert not wide.any()


def test_rotary_gradient_is_the_formula_and_the_difference():
    """f(x) = sum(g * rotary(x)): its gradient is rotary(g, inverse), and, f being linear, equals differences up to rounding."""
    g, x = normal((1, 4, 2, 32), 3), normal((1, 4, 2, 32), 4)
    pos = i32(torch.randint(0, 5000, (2, 1, 4), generator=gen(5)))
    rot = lt.Rotation((10000.0 ** (-torch.arange(12) / 12)).cuda(), (6, 6), interleaved=False)
    grad = lt.rotary(g, pos, rot, inverse=True).double()
    for i in (0, 11, 12, 23, 24, 31, 77, 255):
        d = torch.zeros_like(x).view(-1)
        d[i] = 1.0
        d = d.view_as(x)
        diff = ((lt.rotary(x + d, pos, rot).double() - lt.rotary(x - d, pos, rot).double()) * g.double()).sum() / 2
        # eight roundings of values up to |x| + 1 < 8, each 2^-24 relative, in two components, weighted by g (< 5)
        assert abs(diff - grad.view(-1)[i]) < 2 * 5 * 8 * (8 * 2.0 ** -24 + 2 * TURN)


# ---- append -------------------------------------------------------------------------------------------------------------

def check_append(cache, before, k, v, table, lengths, counts, pos, freq, sections, interleaved):
    """The cache after an append against the reference."""
    S, R = cache.page_tokens, k.shape[1]
    after = snapshot(cache)
    want_k, mag = (k.cpu().to(ref.F64), k.cpu().to(ref.F64).abs()) if freq is None else ref.rotate(k.cpu(), pos, freq, sections, interleaved)
    err = torch.zeros_like(mag) if freq is None else TURN * mag
    touched = set()
    for b, n in enumerate(counts):
        for block in range(lengths[b] // S, -(-(lengths[b] + n) // S) if n else 0):
            touched.add(int(table[b, block]))
        t = table[b].tolist()
        expect = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
        expect.code = [c.clone() for c in before.code]
        expect.scale = [s.clone() for s in before.scale]
        expect.append(0, want_k[b, :n], t, lengths[b])
        expect.append(1, v[b, :n].cpu().to(ref.F64), t, lengths[b])
        first = lengths[b] // S * S
        got, want = after.tokens(1, t, first, lengths[b] + n), expect.tokens(1, t, first, lengths[b] + n)
        assert torch.equal(got.nan_to_num(1e9), want.nan_to_num(1e9))   # values: no rounding but the codes'
        got, want = after.tokens(0, t, first, lengths[b] + n), expect.tokens(0, t, first, lengths[b] + n)
        held = lengths[b] - first
        if n:
            assert torch.equal(got[:held].nan_to_num(1e9), want[:held].nan_to_num(1e9))
        scale = torch.stack([after.scale[0][t[i // S]] for i in range(lengths[b], lengths[b] + n)]) if n else torch.zeros(0, cache.heads, dtype=ref.F64)
        x, e = want_k[b, :n], err[b, :n]
        finite = torch.isfinite(x)
        half = torch.maximum(2.0 ** -4 * (x.abs() + e), 2.0 ** -10 * scale[..., None]) + e
        assert (((got[held:] - x).abs() <= half) | ~finite).all()
        assert (got[held:].isnan() == ~finite).all()
        if n and finite.all():
            for block in range(lengths[b] // S, -(-(lengths[b] + n) // S)):
                for head in range(cache.heads):
                    assert after.scale[0][t[block], head] in (expect.scale[0][t[block], head], 2 * expect.scale[0][t[block], head], expect.scale[0][t[block], head] / 2)
                    assert after.scale[1][t[block], head] == expect.scale[1][t[block], head]
    rest = [p for p in range(cache.pages) if p not in touched]
    for which in range(2):
        assert torch.equal(after.code[which][rest].nan_to_num(1e9), before.code[which][rest].nan_to_num(1e9))
        assert torch.equal(after.scale[which][rest], before.scale[which][rest])


APPENDS = [   # lengths, counts (None: all R)
    (1, [0, 1, 15, 16, 500], None), (4, [0, 14, 63, 64], [4, 3, 0, 1]), (5, [0, 3, 62], None), (61, [0, 5, 127, 64], [61, 7, 0, 60]), (300, [0, 33], [300, 299]),
]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("S,D,H,sections,interleaved", [(16, 16, 1, (8,), True), (64, 64, 3, (16, 16), True), (128, 128, 2, (16, 24, 24), False),
                                                        (32, 80, 5, (5, 0, 7, 9), False), (64, 112, 1, (11,), True), (16, 128, 2, None, False)])
@pytest.mark.parametrize("R,lengths,counts", APPENDS)
def test_append(R, lengths, counts, S, D, H, sections, interleaved, dtype):
    B = len(lengths)
    width = -(-(max(lengths) + R) // S)
    table = make_table(B, width, B * width + 2, 7)
    cache = filled_cache(table, lengths, H, S, D, B * width + 2, 8)
    before = snapshot(cache)
    k, v = normal((B, R, H, D), 9, dtype, 3.0), normal((B, R, H, D), 10, dtype)
    kw, pos, freq = {}, None, None
    if sections:
        pos = torch.randint(0, 40_000, (len(sections), B, R), generator=gen(11), dtype=torch.int32)
        freq = 10000.0 ** (-torch.arange(sum(sections)) / sum(sections))
        kw = dict(positions=pos.cuda(), rotation=lt.Rotation(freq.cuda(), sections, interleaved=interleaved))
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    n = None if counts is None else i32(counts)
    lt.cache_append(k, v, cache, table, i32(lengths), counts=n, status=status, **kw)
    assert not status.any()
    check_append(cache, before, k, v, table, lengths, counts or [R] * B, pos, freq, sections, interleaved)
    # again: nothing changes; and from the middle of a wider tensor with an odd offset
    first = [t.view(torch.uint8).clone() for t in (cache.k, cache.v)]
    wide = torch.zeros((B, R, 2 * H + 1, D + 1), dtype=dtype, device="cuda")
    wide[:, :, :H, 1:] = k
    wide[:, :, H:2 * H, 1:] = v
    lt.cache_append(wide[:, :, :H, 1:], wide[:, :, H:2 * H, 1:], cache, table, i32(lengths), counts=n, **kw)
    assert torch.equal(cache.k.view(torch.uint8), first[0]) and torch.equal(cache.v.view(torch.uint8), first[1])


@pytest.mark.parametrize("R", [2, 20])
def test_append_extremes(R):
    """Zeros, subnormal and huge values, values at the border between two scales, and values that are not finite."""
    S, D, H = 16, 32, 8
    table = i32([[0, 1], [2, 3]])
    cache = filled_cache(table, [3, 0], H, S, D, 4, 12)
    before = snapshot(cache)
    x = torch.randn(2, R, H, D, generator=gen(13))
    x[:, :, 0] = 0.0
    x[:, :, 1] *= 1e-42
    x[:, :, 2] *= 1e37
    x[:, :, 3].clamp_(-1, 1)[:, 0, 0] = 448.0 / 256          # exactly at the border: fits
    x[:, :, 4].clamp_(-1, 1)[:, 0, 0] = 448.0001 / 256       # just behind it
    x[0, 1, 5, 3], x[1, 0, 5, 4], x[1, R - 1, 6, 0] = math.inf, math.nan, -math.inf
    x[:, :, 7] = math.nan
    x = x.cuda()
    status = i32([64, 0])
    lt.cache_append(x, x, cache, table, i32([3, 0]), status=status)
    assert status.tolist() == [64 | lt.ST_NONFINITE, lt.ST_NONFINITE]
    check_append(cache, before, x, x, table, [3, 0], [R, R], None, None, None, False)


def test_append_faults_leave_the_rest():
    S, D, H, R = 16, 16, 1, 20
    table = i32([[0, 1, 2], [3, -1, 5], [6, 7, 8], [9, 10, 11], [12, 99, 14]])
    lengths, counts = [4, 4, -1, 40, 0], [20, 20, 20, 20, 21]
    cache = filled_cache(table.clamp(0, 14), [4, 4, 0, 40, 0], H, S, D, 15, 14)
    before = snapshot(cache)
    x = normal((5, R, H, D), 15)
    status = torch.zeros(5, dtype=torch.int32, device="cuda")
    lt.cache_append(x, x, cache, table, i32(lengths), counts=i32(counts), status=status)
    assert status.tolist() == [0, lt.ST_BAD_BLOCK, lt.ST_BAD_LENGTH, lt.ST_BAD_LENGTH, lt.ST_BAD_LENGTH]
    after = snapshot(cache)
    for page in [*range(4, 15)]:
        assert torch.equal(after.code[0][page].nan_to_num(1e9), before.code[0][page].nan_to_num(1e9))
    before.append(1, x[0].cpu().to(ref.F64), [0, 1, 2], 4)
    assert torch.equal(after.tokens(1, [0, 1, 2], 0, 24), before.tokens(1, [0, 1, 2], 0, 24))
    before.append(1, x[1, :12].cpu().to(ref.F64), [3], 4)
    assert torch.equal(after.tokens(1, [3], 0, 16), before.tokens(1, [3], 0, 16))


# ---- read ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("S,D,H", [(16, 16, 1), (64, 80, 3), (128, 128, 2)])
def test_read(S, D, H, dtype):
    lengths, first, counts, R = [0, 1, 130, 77], [0, 0, 3, 64], [0, 1, 100, 13], 100
    table = make_table(4, -(-130 // S), 4 * -(-130 // S) + 1, 16)
    cache = filled_cache(table, lengths, H, S, D, 4 * -(-130 // S) + 1, 17)
    out = tuple(torch.full((4, R, H, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert lt.cache_read(cache, table, i32(first), R, counts=i32(counts), out=out, status=status) == out
    was = snapshot(cache)
    for b in range(4):
        for which in range(2):
            want = was.tokens(which, table[b].tolist(), first[b], first[b] + counts[b])
            assert torch.equal(out[which][b, :counts[b]].cpu().to(ref.F64), want)   # (codes and powers of two: exact in both types)
            assert (out[which][b, counts[b]:] == 7.0).all()
    assert not status.any()
    bad = table.clone()
    bad[2, 0] = 10_000
    k, v = lt.cache_read(cache, bad, i32([0, 5, 0, -1]), 40, counts=i32([0, -1, 40, 1]), dtype=dtype, status=status)
    assert status.tolist() == [0, lt.ST_BAD_LENGTH, lt.ST_BAD_BLOCK, lt.ST_BAD_LENGTH]
    assert k[2, :min(S, 40)].isnan().all() and v[1].isnan().all() and k[3].isnan().all() and not k[0].any()
    if S < 40:
        assert not v[2, S:].isnan().any()


# ---- keep ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("S,D,H", [(16, 16, 1), (16, 80, 2), (32, 48, 3), (64, 64, 5), (128, 128, 2)])
def test_keep(S, D, H):
    lengths = [0, 3, 14, 15, 16, 120, 7, 7]
    paths = [[0, 1, 2], [], [1, 4, 9, 20, 59], [2, 3, 17, 18, 40, 41, 42, 43, 44, 45, 46, 50, 51, 52, 58, 59], [0, 7, 8], [5], [*range(60)], [*range(1, 60)]]
    B, N = len(lengths), 60
    width = -(-(120 + 61) // S)
    table = make_table(B, width, B * width, 18)
    cache = filled_cache(table, [n + 61 for n in lengths], H, S, D, B * width, 19)
    was = snapshot(cache)
    path = torch.full((B, N), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    new = lt.cache_keep(cache, table, i32(lengths), i32([len(p) for p in paths]), path.cuda(), status=status)
    assert new.tolist() == [n + 1 + len(p) for n, p in zip(lengths, paths)] and not status.any()
    got = snapshot(cache)
    for b, p in enumerate(paths):
        was.keep(table[b].tolist(), lengths[b], p)
        for which in range(2):
            end = lengths[b] + 1 + len(p)
            assert torch.equal(got.tokens(which, table[b].tolist(), 0, end), was.tokens(which, table[b].tolist(), 0, end)), b


def test_keep_long_chain_and_faults():
    N, S, H, D = 1024, 64, 1, 16
    lengths = [5, 5, 5, 5, 5, -1, 2000, 5]
    B = len(lengths)
    table = make_table(B, 20, B * 20, 20)
    cache = filled_cache(table, [n + N + 1 if 0 <= n < 100 else 0 for n in lengths], H, S, D, B * 20, 21)
    table[7, 3] = -5
    path = torch.arange(N, dtype=torch.int32).repeat(B, 1)
    path[1, 500] = 499                # not increasing
    path[2, 1023] = 1024              # behind the last node
    path[3, 0] = -1
    path[4] = torch.cat([torch.arange(1, N, dtype=torch.int32), torch.tensor([-1], dtype=torch.int32)])
    path[7] = path[4]
    accept = [N, N, N, N, N - 1, 3, 3, N - 1]
    was = snapshot(cache)
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    out = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    new = lt.cache_keep(cache, table, i32(lengths), i32(accept), path.cuda(), out_lengths=out, status=status)
    assert new is out
    assert status.tolist() == [0, lt.ST_BAD_PATH, lt.ST_BAD_PATH, lt.ST_BAD_PATH, 0, lt.ST_BAD_LENGTH, lt.ST_BAD_LENGTH, lt.ST_BAD_BLOCK]
    assert new.tolist() == [5 + 1 + N, 5, 5, 5, 5 + N, -1, 2000, 5]
    got = snapshot(cache)
    was.keep(table[4].tolist(), 5, list(range(1, N)))
    for which in range(2):
        assert torch.equal(got.tokens(which, table[4].tolist(), 0, 5 + N), was.tokens(which, table[4].tolist(), 0, 5 + N))
        others = sorted(set(range(B * 20)) - set(table[4].tolist()))
        assert torch.equal(got.code[which][others].nan_to_num(1e9), was.code[which][others].nan_to_num(1e9))


# ---- attention ----------------------------------------------------------------------------------------------------------

def random_tree(B, N, depth, seed):
    import lantern_inputs as li
    return torch.from_numpy(li.tree_parents(B, N, depth=depth, seed=seed)).int()


def run_attention(lengths, R, H, G, D, S, dtype, *, tree=0, counts=None, starts=None, scale=None, seed=30, spread=1.0):
    B = len(lengths)
    width = max(1, -(-(max(lengths) + R) // S))
    pages = B * width + 1
    table = make_table(B, width, pages, seed)
    n = counts or [R] * B
    cache = filled_cache(table, [a + c for a, c in zip(lengths, n)], H, S, D, pages, seed + 1)
    q = normal((B, R, H * G, D), seed + 2, dtype, spread)
    parents = random_tree(B, R - 1, tree, seed + 3) if tree else None
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 5.0)
    got = lt.cache_attention(q, cache, table, i32(lengths), counts=None if counts is None else i32(counts), starts=None if starts is None else i32(starts),
                             tree_parents=None if parents is None else parents.cuda(), scale=scale, out=out, status=status)
    assert got is out and not status.any()
    want, bound = ref.attention(q.cpu(), snapshot(cache), table.tolist(), lengths, counts, starts, None if parents is None else parents.tolist(), scale)
    left_out = want.isnan()
    assert (got.cpu()[left_out] == 5.0).all()
    close(torch.where(left_out.cuda(), torch.zeros_like(got), got), want.nan_to_num(0.0), bound, dtype)
    return q, cache, table, got


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("H,G,D,S", [(1, 1, 16, 16), (3, 1, 64, 64), (2, 4, 128, 128), (1, 8, 80, 32), (2, 3, 112, 16), (1, 16, 48, 64)])
def test_attention_single_tokens(H, G, D, S, dtype):
    run_attention([0, 1, 14, 15, 16, 63, 64, 200, 777], 1, H, G, D, S, dtype)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("H,G,D,S", [(2, 1, 64, 64), (1, 4, 128, 16), (1, 3, 96, 32), (2, 8, 128, 128)])
def test_attention_trees(H, G, D, S, dtype):
    run_attention([0, 1, 40, 63, 131, 300], 61, H, G, D, S, dtype, tree=6)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("H,G,D,S", [(1, 1, 64, 64), (2, 2, 128, 32), (1, 5, 32, 16)])
def test_attention_chains_with_counts_and_starts(H, G, D, S, dtype):
    run_attention([0, 0, 9, 100, 100, 257], 8, H, G, D, S, dtype, counts=[8, 3, 8, 0, 1, 5], starts=[0, 2, 9, 50, 64, 1000])
    run_attention([0, 30, 129], 150, H, G, D, S, dtype, counts=[150, 77, 129], starts=[0, 31, 64])


@pytest.mark.parametrize("dtype", [BF, FP])
def test_attention_trees_with_counts_and_starts(dtype):
    run_attention([0, 5, 200, 64], 33, 2, 2, 64, 16, dtype, tree=4, counts=[33, 1, 20, 0], starts=[3, 9, 190, 0])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("R,tree", [(1, 0), (7, 0), (40, 5)])
def test_attention_split_over_a_long_axis(R, tree, dtype):
    run_attention([6000], R, 1, 2, 64, 64, dtype, tree=tree)
    run_attention([3000, 100, 0], R, 2, 1, 128, 16, dtype, tree=tree, starts=[2, 99, 0])


@pytest.mark.parametrize("dtype", [BF, FP])
def test_attention_sharp_softmax(dtype):
    """Large scores, of which one or a few tokens take all, early or late; negative and zero scales."""
    run_attention([300, 70], 3, 1, 2, 64, 16, dtype, spread=30.0)
    run_attention([300, 70], 30, 1, 1, 64, 32, dtype, tree=3, spread=30.0)
    run_attention([50, 3], 2, 1, 1, 32, 16, dtype, scale=-0.5)
    run_attention([50, 3], 2, 1, 1, 32, 16, dtype, scale=0.0)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("R", [4, 70])
def test_attention_nan_reaches_only_rows_that_see_it(R, dtype):
    H, G, D, S, lengths = 2, 1, 64, 64, [100, 10]
    B, width = 2, -(-(100 + R) // S)
    table = make_table(B, width, B * width, 40)
    cache = filled_cache(table, [n + R for n in lengths], H, S, D, B * width, 41)
    parents = torch.full((B, R - 1), -1, dtype=torch.int32)   # all drafts below the root
    q = normal((B, R, H * G, D), 42, dtype)
    clean = lt.cache_attention(q, cache, table, i32(lengths), tree_parents=parents.cuda())

    def slot(b, token):
        return int(table[b, token // S]), token % S

    page, at = slot(0, 100 + 2)
    cache.v.view(torch.uint8)[page, 1, at, 5] = ref.NAN_CODE
    page, at = slot(1, 10 + 3)
    cache.k.view(torch.uint8)[page, 0, at, 7] = 0xFF
    got = lt.cache_attention(q, cache, table, i32(lengths), tree_parents=parents.cuda())
    hit = torch.zeros(B, R, H * G, D, dtype=torch.bool)
    hit[0, 2, 1] = hit[1, 3, 0] = True
    assert torch.equal(got.cpu()[~hit], clean.cpu()[~hit])
    assert got[0, 2, 1, 5].isnan() and got[1, 3, 0].isnan().all()
    page, at = slot(0, 3)   # a cached token: everyone sees it, unless it lies ahead of the start
    cache.v.view(torch.uint8)[page, 0, at, 9] = ref.NAN_CODE
    got = lt.cache_attention(q, cache, table, i32(lengths), tree_parents=parents.cuda())
    assert got[0, :, 0, 9].isnan().all() and not got[1, :, 1].isnan().any()
    got = lt.cache_attention(q, cache, table, i32(lengths), tree_parents=parents.cuda(), starts=i32([4, 0]))
    assert not got[0, :, 0].isnan().any()
    q[0, 1, 0, 3], q[1, 0, 1, 0] = math.nan, math.inf
    got = lt.cache_attention(q, cache, table, i32(lengths), tree_parents=parents.cuda(), starts=i32([4, 0]))
    assert got[0, 1, 0].isnan().all() and got[1, 0, 1].isnan().all() and not got[0, 1, 1].isnan().any() and not got[0, 3, 0].isnan().any()


@pytest.mark.parametrize("R", [3, 40])
def test_attention_faults(R):
    H, D, S = 2, 64, 16
    lengths = [20, 20, -1, 60, 20, 20]
    B, width = 6, 5
    table = make_table(B, width, B * width, 50)
    cache = filled_cache(table, [80] * B, H, S, D, B * width, 51)
    table[1, 0] = B * width
    counts = [R, R, R, R, R + 1, R]
    parents = torch.full((B, R - 1), -1, dtype=torch.int32)
    parents[5, 1] = 1
    lengths[3] = 80 - R + 1
    q = normal((B, R, H, D), 52, BF)
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    got = lt.cache_attention(q, cache, table, i32(lengths), counts=i32(counts), tree_parents=parents.cuda(), status=status)
    assert status.tolist() == [0, lt.ST_BAD_BLOCK, lt.ST_BAD_LENGTH, lt.ST_BAD_LENGTH, lt.ST_BAD_LENGTH, lt.ST_BAD_PARENT]
    assert not got[0].isnan().any() and got[1:].isnan().all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("R,G", [(1, 4), (30, 3)])
def test_attention_strided_queries(R, G, dtype):
    """Queries inside a fused projection, at aligned and odd offsets, give the same bits."""
    H, D, S, lengths = 2, 64, 32, [100, 33]
    q, cache, table, got = run_attention(lengths, R, H, G, D, S, dtype)
    for ahead in (16, 3):
        wide = torch.full((2, R, H * G + 2 * H, D + ahead), 9.0, dtype=dtype, device="cuda")
        wide[:, :, :H * G, ahead:] = q
        again = lt.cache_attention(wide[:, :, :H * G, ahead:], cache, table, i32(lengths))
        assert torch.equal(again, got)
    turned = q.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3)   # rows ahead of sequences
    assert torch.equal(lt.cache_attention(turned, cache, table, i32(lengths)), got)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D,R,tree", [(32, 70, 4), (96, 70, 0), (80, 35, 3)])
def test_attention_more_units_than_places(D, R, tree, dtype):
    """More rows and heads than the GPU takes at once, sequences of all lengths, some without rows, some that see nothing."""
    g = gen(62)
    B = 50
    lengths = torch.randint(0, 150, (B,), generator=g).tolist()
    counts = torch.randint(0, R + 1, (B,), generator=g).tolist()
    starts = torch.randint(0, 200, (B,), generator=g).tolist()
    lengths[3], counts[5], counts[6], starts[7] = 0, 0, R, 0
    run_attention(lengths, R, 7, 1, D, 16, dtype, tree=tree, counts=counts, starts=starts)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_blank_units_between_others(D, dtype):
    """Sequences whose rows see nothing, or that are refused, take turns with others on the same CTAs: they change nothing of these."""
    S, R, width, each = 16, 17, 144, 296     # (a multiple of the places for CTAs)
    B = 6 * each
    pages = 40
    table = make_table(pages // 4, 4, pages, 63)
    cache = filled_cache(table, [60] * (pages // 4), 1, S, D, pages, 64)
    g = gen(65)
    wide = torch.zeros(B, width, dtype=torch.int32, device="cuda")
    wide[:, :4] = table[torch.arange(B) % (pages // 4)].to("cuda")
    lengths = torch.randint(1, 40, (B,), generator=g)
    turn = (torch.arange(B) // each) % 6
    starts = torch.where(turn % 3 == 1, 100, 0)
    blank, refused = turn % 3 == 1, turn == 5
    lengths[refused] = -1
    q = normal((B, R, 1, D), 66, dtype)
    some = ~(blank | refused)
    want = lt.cache_attention(q[some.cuda()].contiguous(), cache, wide[some.cuda()].contiguous(), i32(lengths[some].tolist()))
    for _ in range(5):
        status = torch.zeros(B, dtype=torch.int32, device="cuda")
        got = lt.cache_attention(q, cache, wide, i32(lengths.tolist()), starts=i32(starts.tolist()), status=status)
        assert torch.equal(got[some.cuda()], want)
        assert not got[blank.cuda()].any() and got[refused.cuda()].isnan().all()
        assert status.tolist() == [lt.ST_BAD_LENGTH if r else 0 for r in refused.tolist()]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("R,H,D", [(1, 2, 64), (30, 2, 128), (40, 1, 64), (90, 1, 96)])
def test_attention_value_scales_far_apart(R, H, D, dtype):
    S, lengths = 16, [150, 97]
    width = -(-(max(lengths) + R) // S)
    table = make_table(2, width, 2 * width, 67)
    cache = filled_cache(table, [n + R for n in lengths], H, S, D, 2 * width, 68)
    cache.v_scale.copy_(torch.exp2(torch.randint(-60, 30, cache.v_scale.shape, generator=gen(69)).float()))
    q = normal((2, R, H, D), 70, dtype)
    got = lt.cache_attention(q, cache, table, i32(lengths))
    want, bound = ref.attention(q.cpu(), snapshot(cache), table.tolist(), lengths)
    close(got, want, bound, dtype)


def test_caches_and_rotations_are_fixed():
    cache = lt.KVCache.empty(2, 1, 16, 16)
    rotation = lt.Rotation(torch.ones(4, device="cuda"), (4,), interleaved=True)
    for made, name in ((cache, "k"), (cache, "v_scale"), (cache, "heads"), (rotation, "inv_freq"), (rotation, "interleaved")):
        with pytest.raises(AttributeError, match="fixed"):
            setattr(made, name, getattr(made, name))


def test_attention_largest_tree():
    run_attention([70], 1025, 1, 1, 16, 64, BF, tree=100)


def test_shared_prefix_pages():
    """Two sequences that share the pages of their prefix."""
    H, D, S = 2, 64, 16
    table = i32([[0, 1, 2, 4], [0, 1, 3, 5]])
    lengths = [36, 40]
    cache = filled_cache(table, [44, 44], H, S, D, 6, 60)
    q = normal((2, 4, H, D), 61, BF)
    want, bound = ref.attention(q.cpu(), snapshot(cache), table.tolist(), lengths)
    close(lt.cache_attention(q, cache, table, i32(lengths)), want, bound, BF)


# ---- together, and how they are called -----------------------------------------------------------------------------------

def test_decoding_steps_with_verification():
    """Prompts, then steps as a generation loop makes them: rotate, append, attend, verify, keep -- against the same loop in 64 bits."""
    import lantern_inputs as li
    B, H, G, D, S, N, V, depth = 3, 2, 2, 64, 16, 20, 512, 4
    width = 16
    table = make_table(B, width, B * width, 70)
    cache = blank_cache(B * width, H, S, D)
    freq = 10000.0 ** (-torch.arange(16) / 16)
    rot = lt.Rotation(torch.cat([freq, freq]).cuda(), (16, 16), interleaved=True)
    prompt = [37, 5, 64]
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    lengths = i32([0] * B)
    k, v = normal((B, 64, H, D), 71, BF), normal((B, 64, H, D), 72, BF)
    pos = torch.arange(64).repeat(2, B, 1).int()
    lt.cache_append(k, v, cache, table, lengths, counts=i32(prompt), positions=pos.cuda(), rotation=rot, status=status)
    check_append(cache, snapshot(blank_cache(B * width, H, S, D)), k, v, table, [0] * B, prompt, pos, torch.cat([freq, freq]), (16, 16), True)
    lengths, at = i32(prompt), list(prompt)
    idx, _ = lt.build_neighbors(torch.from_numpy(li.codebook_gaussian(V, 8)).cuda(), 20)
    for step in range(4):
        inp = li.verify_inputs(B, N, V, dtype=li.BF16, cfg_scale=3.0, rho=0.95, parents=li.tree_parents(B, N, depth=depth, seed=step), seed=step)
        parents = torch.from_numpy(inp.tree_parents).int()
        R = N + 1
        k, v, q = (normal((B, R, n, D), 80 + 3 * step + i, BF) for i, n in enumerate((H, H, H * G)))
        deep = torch.zeros(B, R, dtype=torch.int32)
        for b in range(B):
            for i in range(N):
                deep[b, i + 1] = deep[b, parents[b, i] + 1] + 1
        pos = torch.stack([(torch.tensor(at)[:, None] + deep) // 16, (torch.tensor(at)[:, None] + deep) % 16]).int()
        before = snapshot(cache)
        turned = lt.rotary(q, pos.cuda(), rot)
        lt.cache_append(k, v, cache, table, lengths, positions=pos.cuda(), rotation=rot, status=status)
        check_append(cache, before, k, v, table, at, [R] * B, pos, torch.cat([freq, freq]), (16, 16), True)
        got = lt.cache_attention(turned, cache, table, lengths, tree_parents=parents.cuda(), status=status)
        want, bound = ref.attention(turned.cpu(), snapshot(cache), table.tolist(), at, parents=parents.tolist())
        close(got, want, bound, BF)
        tl = torch.from_numpy(inp.target_logits).view(torch.int16).view(BF).cuda()
        dl = torch.from_numpy(inp.draft_logits).view(torch.int16).view(BF).cuda()
        out = lt.verify(tl, dl, inp.cfg_scale, inp.T, torch.from_numpy(inp.draft_tokens).cuda(), parents.cuda(), idx, 0.3, torch.from_numpy(inp.uniforms).cuda())
        now = snapshot(cache)
        lengths = lt.cache_keep(cache, table, lengths, out.accept_len, out.accept_path, status=status)
        accepted, path, kept = out.accept_len.tolist(), out.accept_path.tolist(), snapshot(cache)
        for b in range(B):
            now.keep(table[b].tolist(), at[b], path[b][:accepted[b]])
            at[b] += 1 + accepted[b]
            for which in range(2):
                assert torch.equal(kept.tokens(which, table[b].tolist(), 0, at[b]), now.tokens(which, table[b].tolist(), 0, at[b]))
        assert lengths.tolist() == at
    assert not status.any()
    kr, vr = lt.cache_read(cache, table, i32([0] * B), min(at), dtype=FP)
    for b in range(B):
        assert torch.equal(kr[b].cpu().to(ref.F64), snapshot(cache).tokens(0, table[b].tolist(), 0, min(at)))


def small_step(seed, R=9, lengths=(50, 300, 0), H=2, G=2, D=64, S=16):
    B, width = len(lengths), 24
    table = make_table(B, width, B * width, seed)
    cache = filled_cache(table, list(lengths), H, S, D, B * width, seed + 1)
    rows = [normal((B, R, n, D), seed + 2 + i, BF) for i, n in enumerate((H * G, H, H))]
    pos = i32(torch.randint(0, 100, (1, B, R), generator=gen(seed)))
    rot = lt.Rotation((10000.0 ** (-torch.arange(32) / 32)).cuda(), (32,), interleaved=False)
    return cache, table, i32(list(lengths)), rows, pos, rot


def one_step(cache, table, lengths, rows, pos, rot, parents, accept, path, outs):
    q, k, v = rows
    turned = lt.rotary(q, pos, rot, out=outs["q"])
    lt.cache_append(k, v, cache, table, lengths, positions=pos, rotation=rot)
    lt.cache_attention(turned, cache, table, lengths, tree_parents=parents, out=outs["o"], workspace=outs["w"])
    lt.cache_keep(cache, table, lengths, accept, path, out_lengths=outs["n"])
    lt.cache_read(cache, table, lengths, 4, out=(outs["k"], outs["v"]))


def step_outputs(cache, table, rows):
    B, R, HQ, D = rows[0].shape
    need = lt.cache_attention_workspace_bytes(B, R, HQ, cache, table.shape[1])
    new = lambda *s: torch.zeros(s, dtype=BF, device="cuda")   # noqa: E731
    return dict(q=new(B, R, HQ, D), o=new(B, R, HQ, D), w=torch.empty(max(need, 256), dtype=torch.uint8, device="cuda"),
                n=torch.zeros(B, dtype=torch.int32, device="cuda"), k=new(B, 4, cache.heads, D), v=new(B, 4, cache.heads, D))


def test_a_step_recorded_and_replayed():
    cache, table, lengths, rows, pos, rot = small_step(90)
    B, R = rows[0].shape[:2]
    parents = random_tree(B, R - 1, 3, 91).cuda()
    accept, path = i32([2, 1, 0]), i32([[0, 5] + [-1] * 6, [3] + [-1] * 7, [-1] * 8])
    outs = step_outputs(cache, table, rows)
    saved = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    restore = lambda: [a.copy_(b) for a, b in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), saved)]   # noqa: E731
    args = (cache, table, lengths, rows, pos, rot, parents, accept, path, outs)
    one_step(*args)
    torch.cuda.synchronize()
    restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one_step(*args)
    for i in range(3):   # inputs rewritten in place
        for t in rows:
            t.copy_(normal(t.shape, 100 + i, BF))
        lengths.copy_(i32([10 * i, 200 + i, 1]))
        restore()
        one_step(*args)
        want = {n: t.clone() for n, t in outs.items() if n != "w"}
        codes = [t.view(torch.uint8).clone() for t in (cache.k, cache.v)]
        restore()
        for n, t in outs.items():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n in want:   # (bits: the third sequence reads blocks that were never written)
            assert torch.equal(outs[n].view(torch.uint8), want[n].view(torch.uint8)), n
        assert torch.equal(cache.k.view(torch.uint8), codes[0]) and torch.equal(cache.v.view(torch.uint8), codes[1])


def test_two_streams_at_once():
    """Two steps in flight on streams of their own, each with its workspace, give what they give alone."""
    sets, want = [], []
    for seed in (110, 120):
        cache, table, lengths, rows, pos, rot = small_step(seed, lengths=(380, 3, 370), R=4)
        args = (cache, table, lengths, rows, pos, rot, None, i32([1, 0, 2]), i32([[0, -1, -1], [-1] * 3, [0, 2, -1]]), step_outputs(cache, table, rows))
        one_step(*args)   # (settles the scales: the next passes change nothing)
        one_step(*args)
        want.append({n: t.clone() for n, t in args[-1].items() if n != "w"})
        sets.append(args)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for args, s in zip(sets, streams):
            with torch.cuda.stream(s):
                one_step(*args)
    torch.cuda.synchronize()
    for args, w in zip(sets, want):
        for n in w:
            assert torch.equal(args[-1][n], w[n]), n
    # and through the stream argument (the rows are appended again: keep has moved some of them)
    cache, table, lengths, rows, pos, rot = sets[0][:6]
    lt.cache_append(rows[1], rows[2], cache, table, lengths, positions=pos, rotation=rot, stream=streams[0])
    got = lt.cache_attention(sets[0][-1]["q"], cache, table, lengths, stream=streams[0])
    streams[0].synchronize()
    assert torch.equal(got, want[0]["o"])


def test_results_belong_to_the_stream_of_the_call():
    """What a call allocates comes from the pool of the stream it runs on: memory that the current stream has just given back, and still writes
    to, is not the result's."""
    cache, table, lengths, rows, pos, rot = small_step(150, R=20)
    want = lt.rotary(rows[0], pos, rot), lt.cache_attention(rows[0], cache, table, lengths), lt.cache_read(cache, table, lengths, 7, counts=i32([7, 3, 0]))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        for t in (want[0], want[2][0]):
            x = torch.empty_like(t)
            torch.cuda._sleep(20_000_000)   # some ten milliseconds
            x.fill_(3.0)
            del x
        got = (lt.rotary(rows[0], pos, rot, stream=side), lt.cache_attention(rows[0], cache, table, lengths, stream=side),
               lt.cache_read(cache, table, lengths, 7, counts=i32([7, 3, 0]), stream=side))
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1].view(torch.uint8), want[1].view(torch.uint8))
        for a, b in zip(got[2], want[2]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_a_cache_of_more_than_2_to_32_codes():
    H, S, D, pages = 8, 64, 128, 70_000   # 4.6e9 codes of each kind
    k = torch.empty((pages, H, S, D), dtype=torch.float8_e4m3fn, device="cuda")
    v = torch.empty_like(k)
    for t in (k, v):
        t.view(torch.uint8)[-4:].fill_(ref.NAN_CODE)
    scale = torch.ones((pages, H), device="cuda")
    cache = lt.KVCache(k, v, scale, scale.clone())
    table = i32([[pages - 1, pages - 3], [pages - 2, pages - 4]])
    lengths, R = [0, 0], 100
    x = [normal((2, R, H, D), 130 + i, BF) for i in range(3)]
    lt.cache_append(x[0], x[1], cache, table, i32(lengths))
    small = ref.Cache(cache.k[-4:], cache.v[-4:], cache.k_scale[-4:], cache.v_scale[-4:])
    local = [[3, 1], [2, 0]]
    want = ref.Cache(cache.k[-4:], cache.v[-4:], cache.k_scale[-4:], cache.v_scale[-4:])
    for b in range(2):
        for which in range(2):
            want.append(which, x[which][b].cpu().to(ref.F64), local[b], 0)
            assert torch.equal(small.tokens(which, local[b], 0, R), want.tokens(which, local[b], 0, R))
    q = x[2][:, :3]
    got = lt.cache_attention(q, cache, table, i32([97, 97]))
    out, bound = ref.attention(q.cpu(), small, local, [97, 97])
    close(got, out, bound, BF)
    path = torch.full((2, 40), -1, dtype=torch.int32)
    path[0, :2], path[1, 0] = torch.tensor([3, 30], dtype=torch.int32), 39
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    lt.cache_keep(cache, table, i32([60, 20]), i32([2, 1]), path.cuda(), status=status)
    assert not status.any()
    kr, vr = lt.cache_read(cache, table, i32([0, 0]), 63, dtype=FP)
    for b, (n, path) in enumerate(((60, [3, 30]), (20, [39]))):
        small.keep(local[b], n, path)
        assert torch.equal(vr[b, :n + 1 + len(path)].cpu().to(ref.F64), small.tokens(1, local[b], 0, n + 1 + len(path)))


def test_empty_calls():
    cache, table, lengths, rows, pos, rot = small_step(140)
    none = torch.zeros((3, 0, 4, 64), dtype=BF, device="cuda")
    assert lt.cache_attention(none, cache, table, lengths).shape == none.shape
    assert lt.rotary(none, pos[:, :, :0].contiguous(), rot).shape == none.shape
    lt.cache_append(none[:, :, :2], none[:, :, :2], cache, table, lengths)
    assert lt.cache_read(cache, table, lengths, 0)[0].numel() == 0
    assert lt.cache_keep(cache, table, lengths, i32([0, 0, 0]), torch.zeros((3, 0), dtype=torch.int32, device="cuda")).tolist() == [51, 301, 1]
    torch.cuda.synchronize()
    nobody = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")   # noqa: E731
    lt.cache_append(nobody(0, 3, 2, 64, dtype=BF), nobody(0, 3, 2, 64, dtype=BF), cache, nobody(0, 5), nobody(0), positions=nobody(1, 0, 3), rotation=rot)
    assert lt.cache_attention(nobody(0, 3, 4, 64, dtype=BF), cache, nobody(0, 5), nobody(0)).numel() == 0
    assert lt.cache_keep(cache, nobody(0, 5), nobody(0), nobody(0), nobody(0, 7)).numel() == 0
    assert lt.cache_read(cache, nobody(0, 5), nobody(0), 3)[1].numel() == 0
    torch.cuda.synchronize()
