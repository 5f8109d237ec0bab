"""What the cache operators refuse on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2410_03355_b200 as lt
from paper_2410_03355_b200 import cache as binding

NULL, SHAPE, PARAM, WORKSPACE, ALIGN = -1, -2, -3, -4, -8
AT = 1 << 20   # stands for device memory: nothing reads it


def cache(k=AT, v=AT, ks=AT, vs=AT, pages=10, heads=4, S=64, D=64):
    return binding._CacheStruct(k, v, ks, vs, pages, heads, S, D)


def strides(*s):
    return (ctypes.c_int64 * 3)(*(s or (1024, 256, 64)))


def rotation(freq=AT, pos=AT, axes=2, inter=0, section=(16, 16, 0, 0)):
    return binding._RotationStruct(freq, pos, axes, inter, (ctypes.c_int32 * 4)(*section))


def ref(s):
    return None if s is None else ctypes.addressof(s)


def append(c=None, k=AT, v=AT, dtype=lt.BF16, B=2, R=3, ks=None, vs=None, table=AT, width=4, lengths=AT, rot=None):
    c, ks, vs = c or cache(), ks or strides(), vs or strides()
    return lt.load_library().lantern_cache_append(k, v, dtype, B, R, ks, vs, ref(c), table, width, lengths, None, ref(rot), None, None)


def attention(c=None, q=AT, out=AT + 4096, dtype=lt.BF16, B=2, R=3, HQ=8, table=AT, width=4, lengths=AT, parents=None, scale=0.1, ws=None, ws_bytes=0):
    c = c or cache()
    return lt.load_library().lantern_cache_attention(q, out, dtype, B, R, HQ, strides(), ref(c), table, width, lengths, None, None, parents, scale, None,
                                                  ws, ws_bytes, None)


def keep(c=None, table=AT, width=4, lengths=AT, accept=AT, path=AT, B=2, N=3, out=AT + 4096):
    c = c or cache()
    return lt.load_library().lantern_cache_keep(ref(c), table, width, lengths, accept, path, B, N, out, None, None)


def read(c=None, table=AT, width=4, first=AT, B=2, R=3, dtype=lt.BF16, k=AT, v=AT):
    c = c or cache()
    return lt.load_library().lantern_cache_read(ref(c), table, width, first, None, B, R, dtype, k, v, None, None)


def rotary(x=AT, out=AT, dtype=lt.BF16, B=2, R=3, H=4, D=64, rot=None):
    rot = rot or rotation()
    return lt.load_library().lantern_rotary(x, out, dtype, B, R, H, D, strides(), strides(), ref(rot), 0, None)


@pytest.mark.parametrize("call", [append, attention, keep, read])
def test_caches_that_are_refused(call):
    for c, want in [(cache(k=0), NULL), (cache(vs=0), NULL), (cache(S=48), SHAPE), (cache(S=8), SHAPE), (cache(S=256), SHAPE), (cache(D=8), SHAPE),
                    (cache(D=72), SHAPE), (cache(D=144), SHAPE), (cache(pages=0), SHAPE), (cache(heads=0), SHAPE), (cache(pages=1 << 24), SHAPE),
                    (cache(v=AT + 8), ALIGN)]:
        assert call(c) == want
    assert call(table=None) == NULL
    assert call(width=0) == SHAPE and call(width=(1 << 24) + 1) == SHAPE
    assert call(B=-1) == SHAPE


@pytest.mark.parametrize("call", [append, attention, read])
def test_types_and_row_counts(call):
    assert call(dtype=2) == PARAM and call(dtype=-1) == PARAM
    assert call(R=-1) == SHAPE
    assert call(B=0) == 0 and call(R=0) == 0   # nothing to do


def test_append():
    assert append(k=None) == NULL and append(v=None) == NULL and append(lengths=None) == NULL
    assert append(B=65536) == SHAPE
    assert append(k=AT + 1) == ALIGN and append(v=AT + 2, dtype=lt.F32) == ALIGN
    for rot, want in [(rotation(freq=0), NULL), (rotation(pos=0), NULL), (rotation(axes=0), SHAPE), (rotation(axes=5), SHAPE),
                      (rotation(section=(16, 17, 0, 0)), SHAPE), (rotation(section=(0, 0, 0, 0)), SHAPE), (rotation(section=(-1, 8, 0, 0)), SHAPE)]:
        assert append(rot=rot) == want


def test_attention():
    assert attention(q=None) == NULL and attention(out=None) == NULL and attention(lengths=None) == NULL
    assert attention(HQ=0) == SHAPE and attention(HQ=6) == SHAPE
    assert attention(R=1026, parents=AT) == SHAPE
    assert attention(scale=float("nan")) == PARAM and attention(scale=float("inf")) == PARAM
    assert attention(out=AT) == PARAM                  # in place
    assert attention(out=AT + 8) == ALIGN and attention(q=AT + 1) == ALIGN
    assert attention(B=1 << 16, R=1 << 16) == SHAPE
    long = dict(B=1, R=1, width=1000)
    need = lt.cache_attention_workspace_bytes(1, 1, 8, _view(), 1000)
    assert need > 0
    assert attention(**long) == WORKSPACE and attention(**long, ws=AT, ws_bytes=need - 1) == WORKSPACE
    assert attention(**long, ws=AT + 16, ws_bytes=need) == WORKSPACE
    assert lt.cache_attention_workspace_bytes(1, 1, 6, _view(), 1000) == 0


def _view():
    """A cache of which only the sizes are looked at."""
    class View:
        struct = cache()
        _at = ctypes.addressof(struct)
    return View


def test_keep():
    assert keep(lengths=None) == NULL and keep(accept=None) == NULL and keep(path=None) == NULL and keep(out=None) == NULL
    assert keep(N=-1) == SHAPE and keep(N=1025) == SHAPE and keep(B=65536) == SHAPE
    assert keep(out=AT) == PARAM                       # in place
    assert keep(B=0) == 0


def test_keep_results_in_place_of_inputs():
    B, N = 4, 3
    far = dict(B=B, N=N, lengths=AT, accept=AT + 4096, path=AT + 8192)
    for at, size in ((AT, 4 * B), (AT + 4096, 4 * B), (AT + 8192, 4 * B * N)):
        for out in (at, at + size - 4, at - 4 * B + 4):
            assert keep(**far, out=out) == PARAM
    assert keep(**{**far, "N": 0, "path": None}, out=AT) == PARAM


def test_read():
    assert read(first=None) == NULL and read(k=None) == NULL and read(v=None) == NULL
    assert read(k=AT + 8) == ALIGN and read(B=1 << 16, R=1 << 16) == SHAPE


def test_rotary():
    assert rotary(x=None) == NULL and rotary(out=None) == NULL
    assert rotary(dtype=3) == PARAM
    assert rotary(D=63) == SHAPE and rotary(D=514) == SHAPE and rotary(D=0) == SHAPE and rotary(H=-1) == SHAPE
    assert rotary(D=30) == SHAPE                       # 32 pairs of axes in 30 components
    assert rotary(rot=rotation(axes=0)) == SHAPE and rotary(rot=rotation(freq=0)) == NULL
    assert rotary(B=0) == 0 and rotary(R=0) == 0 and rotary(H=0) == 0
    assert rotary(out=AT + 1) == ALIGN


def test_rotary_rows_that_are_one():
    for axis in range(3):
        stride = [4 * 64 * 3, 4 * 64, 64]
        stride[axis] = 0
        call = lambda shape: lt.load_library().lantern_rotary(AT, 2 * AT, lt.BF16, *shape, strides(), (ctypes.c_int64 * 3)(*stride), ref(rotation()), 0, None)
        assert call((2, 3, 4, 64)) == PARAM


def test_binding_refuses_what_it_cannot_marshal():
    f8 = torch.zeros(4, 2, 16, 16, dtype=torch.uint8).view(torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="CUDA"):
        lt.KVCache(f8, f8, torch.ones(4, 2), torch.ones(4, 2))
    with pytest.raises(ValueError, match="pages"):
        lt.KVCache(f8, f8[:2], torch.ones(4, 2), torch.ones(4, 2))
    with pytest.raises(ValueError):
        lt.Rotation(torch.ones(4), (2, 2), interleaved=True)      # on the host
    with pytest.raises(ValueError, match="frequency"):
        lt.Rotation(torch.ones(4), (2, 3), interleaved=True)
    with pytest.raises(ValueError, match="sections"):
        lt.Rotation(torch.ones(5), (1, 1, 1, 1, 1), interleaved=True)
    with pytest.raises(ValueError, match="CUDA"):
        lt.rotary(torch.zeros(1, 1, 1, 4), None, None)
