"""Attention whose copies do not come, made without any fault: they are withheld on purpose, the bounded waits run out, nothing is in flight."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_cache import BF, FP, filled_cache, i32, make_table, normal, random_tree   # noqa: E402

import paper_2410_03355_b200 as lt   # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("R,G,D,room", [(1, 4, 128, 2048), (9, 1, 64, 2048), (40, 1, 64, 1984), (40, 1, 128, 960), (33, 1, 64, 8192), (33, 1, 128, 8192),
                                        (35, 2, 64, 8192), (50, 3, 96, 8192), (61, 2, 64, 512)])
def test_a_copy_that_does_not_come(R, G, D, room, dtype):
    S, H, B = 32, 2, 3
    lengths, width = [min(900, room - R), 20, min(700, room - R)], room // S
    table = make_table(B, width, B * width, 500)
    cache = filled_cache(table, [n + R for n in lengths], H, S, D, B * width, 501)
    q = normal((B, R, H * G, D), 502, dtype)
    parents = None if R == 1 else random_tree(B, R - 1, 5, 503).cuda()
    call = lambda status: lt.cache_attention(q, cache, table, i32(lengths), tree_parents=parents, status=status)   # noqa: E731
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    want = call(status)
    assert not status.any()
    for missing in (0, 300, lengths[0]):
        status.fill_(1 << 20)
        try:
            lt.debug_wait_test(max_tries=20_000, withhold_context=missing)
            got = call(status)
            torch.cuda.synchronize()
        finally:
            lt.debug_wait_test(0, -1)
        for b in range(B):
            if missing < lengths[b] // 128 * 128:   # (a tile that it has whole)
                assert got[b].isnan().all() and status[b].item() == 1 << 20 | lt.ST_INTERNAL
            elif status[b].item() == 1 << 20:
                assert torch.equal(got[b], want[b])
            else:
                assert status[b].item() == 1 << 20 | lt.ST_INTERNAL
    status.zero_()
    assert torch.equal(call(status), want) and not status.any()   # the device is as usable as before
