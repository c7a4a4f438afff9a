"""Rotary positions, the paged cache and windowed attention: calls that are refused, before anything touches a device."""
import ctypes
import math

import pytest
import torch

from paper_2608_26965_b200 import binding, build

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
PTR = 1 << 20          # an aligned address that nothing reads: the calls below are refused


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def rows(data=PTR, b=1 << 16, h=1 << 12, n=128):
    return binding.CaRows(data, b, h, n)


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(binding.CaRows) == 32 and ctypes.sizeof(binding.CaRotary) == 32
    assert ctypes.sizeof(binding.CaCache) == 44 and ctypes.sizeof(binding.CaWindow) == 48


def call_rotary(lib, rot=None, q=None, k=None, oq=None, ok=None, pos=PTR, batch=2, hq=4, hk=2, n=8, d=128, dtype=1, pos_b=24):
    rot = binding.Rotary(128, [16, 24, 24])._struct if rot is None else rot
    r = lambda x: rows() if x is None else x
    return lib.rotary_axes(rot, batch, hq, hk, n, d, dtype, 0, r(q), r(k), pos, pos_b, r(oq), r(ok), None)


def test_rotary_refusals(lib):
    assert call_rotary(lib, pos=None) == INVALID
    for kw in (dict(batch=0), dict(hq=0), dict(hk=-1), dict(n=0), dict(pos_b=-1)):
        assert call_rotary(lib, **kw) == INVALID, kw
    for kw in (dict(d=96), dict(dtype=2), dict(hq=70000)):
        assert call_rotary(lib, **kw) == UNSUPPORTED, kw
    for bad in (rows(0), rows(PTR + 8), rows(b=4), rows(h=1001), rows(n=130)):
        for which in ("q", "k", "oq", "ok"):
            assert call_rotary(lib, **{which: bad}) == INVALID, which
    for bad in (rows(n=0), rows(h=64), rows(b=-128)):       # rows of an output overlap
        assert call_rotary(lib, oq=bad) == INVALID and call_rotary(lib, ok=bad) == INVALID
    # an output that is another tensor of the call, or its input with other strides
    other = [rows(PTR + (i << 24)) for i in range(4)]
    apart = dict(q=other[0], k=other[1], oq=other[2], ok=other[3])
    for kw in (dict(oq=other[1]), dict(ok=other[0]), dict(ok=other[2]), dict(oq=rows(PTR, n=256)), dict(ok=rows(PTR + (1 << 24), b=1 << 17))):
        assert call_rotary(lib, **{**apart, **kw}) == INVALID, kw
    good = (ctypes.c_double * 65)(*([1.0] * 65))
    ptr = ctypes.cast(good, ctypes.POINTER(ctypes.c_double))
    four = ctypes.c_int32 * 4
    for axes, pairs in ((0, (1, 0, 0, 0)), (5, (1, 0, 0, 0)), (1, (0, 0, 0, 0)), (1, (65, 0, 0, 0)), (2, (40, 30, 0, 0)), (2, (-1, 4, 0, 0)),
                        (2, (2 ** 31 - 1, 2, 0, 0))):
        assert call_rotary(lib, rot=binding.CaRotary(axes, four(*pairs), 1, ptr)) == INVALID, pairs
    good[3] = math.inf
    assert call_rotary(lib, rot=binding.CaRotary(1, four(8, 0, 0, 0), 1, ptr)) == INVALID
    assert call_rotary(lib, rot=binding.CaRotary(1, four(8, 0, 0, 0), 1, None)) == INVALID


def test_cache_refusals(lib):
    size = ctypes.c_size_t()
    base = dict(batch=4, heads_q=8, heads_kv=2, head_dim=128, dtype="bf16", page_rows=16, pages=100, pages_per_sequence=20)
    make = lambda **kw: binding.make_cache_problem(**{**base, **kw})
    ask = lambda **kw: lib.ca_cache_workspace_bytes(make(**kw), size)
    assert ask() == OK and size.value > 256
    for kw in (dict(batch=0), dict(heads_q=9), dict(heads_kv=0), dict(pages=0), dict(pages_per_sequence=0), dict(left=-2), dict(sinks=-1),
               dict(softmax_scale=-1.0), dict(softmax_scale=math.nan), dict(softmax_scale=math.inf)):
        assert ask(**kw) == INVALID, kw
    for kw in (dict(head_dim=96), dict(page_rows=8), dict(page_rows=2048), dict(batch=70000),
               dict(page_rows=1024, pages_per_sequence=1 << 21)):
        assert ask(**kw) == UNSUPPORTED, kw
    assert lib.ca_cache_workspace_bytes(None, size) == INVALID
    c = make()

    def append(n=1, k=None, v=None, lengths=PTR, table=PTR, rot=None, pos=None, kp=PTR, vp=PTR, ws=PTR, ws_bytes=1 << 30):
        return lib.cache_append(c, n, k or rows(), v or rows(), lengths, None, table, rot, pos, 0, kp, vp, ws, ws_bytes, None)

    for kw in (dict(n=0), dict(lengths=None), dict(table=None), dict(kp=None), dict(vp=PTR + 2), dict(k=rows(0)), dict(v=rows(h=3)),
               dict(rot=binding.Rotary(128, [4])._struct)):
        assert append(**kw) == INVALID, kw
    for kw in (dict(ws=None), dict(ws=PTR + 4), dict(ws_bytes=size.value - 1)):
        assert append(**kw) == WORKSPACE, kw
    assert append(rot=binding.CaRotary(1, (ctypes.c_int32 * 4)(70, 0, 0, 0), 1, binding.Rotary(128, [4])._struct.freq), pos=PTR) == INVALID

    def paged(q=None, o=None, lengths=PTR, table=PTR, appended=0, kp=PTR, vp=PTR, ws=PTR, ws_bytes=1 << 30):
        return lib.paged_attention_fwd(c, q or rows(), kp, vp, lengths, appended, table, o or rows(), None, ws, ws_bytes, None)

    for kw in (dict(q=rows(PTR + 4)), dict(o=rows(h=0)), dict(lengths=None), dict(table=None), dict(appended=-1), dict(kp=None), dict(vp=PTR + 8)):
        assert paged(**kw) == INVALID, kw
    for kw in (dict(ws=None), dict(ws=PTR + 4), dict(ws_bytes=100)):
        assert paged(**kw) == WORKSPACE, kw


def test_window_refusals(lib):
    size = ctypes.c_size_t()
    base = dict(batch=2, heads_q=8, heads_kv=2, n_q=100, n_k=100, head_dim=64, dtype="bf16", left=10, right=0)
    make = lambda **kw: binding.make_window_problem(**{**base, **kw})
    ask = lambda **kw: lib.ca_window_workspace_bytes(make(**kw), size)
    assert ask() == OK and size.value >= 256
    for kw in (dict(batch=0), dict(heads_q=7), dict(n_q=0), dict(n_k=0), dict(left=-2), dict(right=-2), dict(sinks=-1), dict(flags=1),
               dict(softmax_scale=-0.5), dict(softmax_scale=math.nan)):
        assert ask(**kw) == INVALID, kw
    for kw in (dict(head_dim=32), dict(batch=70000)):
        assert ask(**kw) == UNSUPPORTED, kw
    assert lib.ca_window_workspace_bytes(None, size) == INVALID
    p = make()

    def window(q=None, k=None, v=None, o=None, ws=PTR, ws_bytes=1 << 30):
        r = lambda x: x or rows()
        return lib.window_attention_fwd(p, r(q), r(k), r(v), None, None, r(o), None, ws, ws_bytes, None)

    for name in ("q", "k", "v", "o"):
        for bad in (rows(0), rows(PTR + 8), rows(n=12)):
            assert window(**{name: bad}) == INVALID, name
    assert window(o=rows(n=32)) == INVALID
    for kw in (dict(ws=None), dict(ws=PTR + 4), dict(ws_bytes=255)):
        assert window(**kw) == WORKSPACE, kw
    other = [rows(PTR + (i << 24)) for i in range(4)]
    for i in range(3):                                      # the output is an input
        assert window(*other[:3], o=other[i]) == INVALID


def test_binding_refusals(lib):
    with pytest.raises(binding.ClusterAttnError):
        binding.Rotary(64, [40])
    with pytest.raises(binding.ClusterAttnError):
        binding.Rotary(64, [])
    with pytest.raises(binding.ClusterAttnError):
        binding.Rotary(64, [4], frequencies=[1.0, 2.0, 3.0])
    with pytest.raises(binding.ClusterAttnError):
        binding.Rotary(64, [2], frequencies=[1.0, math.nan])
    with pytest.raises(binding.ClusterAttnError):
        binding.make_window_problem(1, 1, 1, 4, 4, 64, "fp16", 1, 0)
    x = torch.zeros((1, 1, 4, 64))
    with pytest.raises(binding.ClusterAttnError):
        binding.rotary_axes(binding.Rotary(64, [4]), x, None, torch.zeros((1, 4, 1), dtype=torch.int32))
    if not torch.cuda.is_available():
        with pytest.raises(binding.ClusterAttnError):
            binding.WindowPlan(binding.make_window_problem(1, 1, 1, 4, 4, 64, "bf16", 1, 0))
        with pytest.raises(binding.ClusterAttnError):
            binding.PagedCache(binding.make_cache_problem(1, 1, 1, 64, "bf16", 16, 4, 4))
