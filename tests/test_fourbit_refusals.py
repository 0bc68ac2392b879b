"""Arguments that the entry points of the 4-bit cache refuse, on the host and before anything looks into the context or touches
a GPU: a block of zeros stands in for the context, numbers for the device pointers."""
import ctypes as C

import pytest
import torch

from paper_2602_01345_amd import FourBitCache, load_library
from paper_2602_01345_amd import binding as Bn

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
BASE = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return load_library()


_CTX = C.create_string_buffer(4096)


def _cache(at=1, B=2, kv_heads=2, capacity=100, dh=64):
    p = BASE * 64 * at
    return Bn._FourBitCache(p, p + BASE, p + 2 * BASE, p + 3 * BASE, B, kv_heads, capacity, dh)


def _rows(n=3, heads=2, dh=64, at=40, **kw):
    r = Bn._Rows(BASE * 64 * at, n * heads * dh, heads * dh, dh, 1)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _ref(x):
    return None if x is None else C.byref(x)


def _append(lib, cache=None, k=None, v=None, dtype=1, n=3, n_rows=None, kv_len=5, kv_rows=None, kv_next=None, ctx=_CTX):
    cache = _cache() if cache is None else cache
    return lib.nova_fourbit_append(ctx, None, dtype, _ref(cache), n, _ref(k or _rows()), _ref(v or _rows(at=41)), n_rows, kv_len,
                                   kv_rows, kv_next)


@pytest.mark.parametrize("kw,rc", [
    (dict(ctx=None), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(n=-1), INVALID), (dict(kv_len=-1), INVALID),
    (dict(kv_len=98), INVALID), (dict(n=101), INVALID), (dict(cache=_cache(dh=96)), UNSUPPORTED),
    (dict(cache=_cache(kv_heads=0)), INVALID), (dict(cache=_cache(B=-1)), INVALID), (dict(cache=_cache(capacity=-1)), INVALID),
    (dict(cache=_cache(B=70000)), UNSUPPORTED), (dict(cache=_cache(capacity=1 << 27)), UNSUPPORTED),
    (dict(n_rows=BASE + 2), INVALID), (dict(kv_rows=BASE + 1), INVALID), (dict(kv_next=BASE + 3), INVALID),
    (dict(kv_rows=BASE, kv_next=BASE), INVALID), (dict(kv_rows=BASE, kv_next=BASE + 4), INVALID),
    (dict(n_rows=BASE + 4, kv_next=BASE), INVALID),
    (dict(k=_rows(data=0)), INVALID), (dict(v=_rows(data=BASE + 1)), INVALID), (dict(k=_rows(stride_row=-64)), INVALID),
    (dict(v=_rows(stride_channel=-1)), INVALID),
])
def test_append(lib, kw, rc):
    assert _append(lib, **kw) == rc


@pytest.mark.parametrize("field", ["k_codes", "k_scales", "v_codes", "v_scales"])
@pytest.mark.parametrize("value", [0, BASE + 8])
def test_cache_arrays(lib, field, value):
    c = _cache()
    setattr(c, field, value)
    assert _append(lib, cache=c) == INVALID
    assert lib.nova_fourbit_evict(_CTX, None, _ref(c), _ref(_cache(2)), 1, BASE, None, 5, None, None, None, None) == INVALID


def test_nothing_to_do_is_no_error(lib):
    assert _append(lib, cache=_cache(B=0)) == 0
    assert lib.nova_fourbit_unpack(_CTX, None, 1, _ref(_cache()), 0, 0, None, None, None, None) == 0
    assert lib.nova_fourbit_unpack(_CTX, None, 1, _ref(_cache()), 0, 4, None, None, None, None) == 0
    assert _attend(lib, n=0) == 0 and _attend(lib, cache=_cache(B=0)) == 0
    assert _mass(lib, cache=_cache(B=0)) == 0


def _unpack(lib, cache=None, dtype=1, first=0, n=3, first_rows=None, n_rows=None, k=None, v=None):
    return lib.nova_fourbit_unpack(_CTX, None, dtype, _ref(cache or _cache()), first, n, first_rows, n_rows, _ref(k or _rows()),
                                   _ref(v))


@pytest.mark.parametrize("kw,rc", [
    (dict(dtype=-1), UNSUPPORTED), (dict(first=-1), INVALID), (dict(n=-1), INVALID), (dict(first=98), INVALID),
    (dict(first_rows=BASE + 2), INVALID), (dict(n_rows=BASE + 2), INVALID), (dict(k=_rows(stride_channel=0)), INVALID),
    (dict(k=_rows(stride_row=0)), INVALID), (dict(v=_rows(stride_b=0)), INVALID), (dict(v=_rows(stride_head=0)), INVALID),
    (dict(v=_rows(data=0)), INVALID),
])
def test_unpack(lib, kw, rc):
    assert _unpack(lib, **kw) == rc


def _attend(lib, cache=None, dtype=1, heads=4, n=3, q=None, n_rows=None, kv_len=50, kv_rows=None, out=BASE * 8, lse=None,
            ws=BASE * 16, ws_bytes=1 << 40, ctx=_CTX):
    q = _rows(heads=4) if q is None else q
    return lib.nova_fourbit_attention(ctx, None, dtype, _ref(cache or _cache()), heads, n, _ref(q), n_rows, kv_len, kv_rows, 0.125,
                                      out, lse, ws, ws_bytes)


def _mass(lib, cache=None, dtype=1, heads=4, n=3, q=None, n_rows=None, kv_len=50, kv_rows=None, lse=BASE, mass_in=None,
          mass=BASE * 8, ws=BASE * 16, ws_bytes=1 << 40, ctx=_CTX):
    q = _rows(heads=4) if q is None else q
    return lib.nova_fourbit_mass(ctx, None, dtype, _ref(cache or _cache()), heads, n, _ref(q), n_rows, kv_len, kv_rows, 0.125, lse,
                                 mass_in, mass, ws, ws_bytes)


@pytest.mark.parametrize("call", [_attend, _mass])
@pytest.mark.parametrize("kw,rc", [
    (dict(ctx=None), INVALID), (dict(dtype=7), UNSUPPORTED), (dict(heads=0), INVALID), (dict(heads=3), INVALID),
    (dict(n=-1), INVALID), (dict(kv_len=-1), INVALID), (dict(kv_len=101), INVALID), (dict(n=1 << 28), UNSUPPORTED),
    (dict(cache=_cache(dh=32)), UNSUPPORTED), (dict(n_rows=BASE + 1), INVALID), (dict(kv_rows=BASE + 2), INVALID),
    (dict(lse=BASE + 2), INVALID), (dict(q=_rows(heads=4, data=0)), INVALID), (dict(q=_rows(heads=4, data=BASE + 8)), INVALID),
    (dict(q=_rows(heads=4, stride_channel=2)), INVALID), (dict(q=_rows(heads=4, stride_row=260)), INVALID),
    (dict(q=_rows(heads=4, stride_head=65)), INVALID), (dict(q=_rows(heads=4, stride_b=-768)), INVALID),
])
def test_queries(lib, call, kw, rc):
    assert call(lib, **kw) == rc


def test_attention_outputs(lib):
    assert _attend(lib, out=0) == INVALID and _attend(lib, out=BASE + 8) == INVALID
    assert _attend(lib, out=_rows(heads=4).data) == INVALID


def test_mass_outputs(lib):
    assert _mass(lib, mass=None) == INVALID and _mass(lib, lse=None) == INVALID and _mass(lib, mass=BASE * 8 + 2) == INVALID
    assert _mass(lib, mass_in=BASE * 8 + 4) == INVALID        # overlapping, but not the same array


@pytest.mark.parametrize("shape", [dict(n=1, kv_len=4000), dict(n=40, kv_len=4000), dict(n=700, kv_len=20)])
def test_workspaces_too_small(lib, shape):
    c = _cache(capacity=4000)
    for call, size in ((_attend, lib.nova_fourbit_attention_workspace_bytes), (_mass, lib.nova_fourbit_mass_workspace_bytes)):
        need = size(C.byref(c), 4, shape["n"], shape["kv_len"])
        if need:
            for ws, nbytes in ((None, 0), (BASE * 16, need - 1), (BASE * 16 + 8, need)):
                assert call(lib, cache=c, ws=ws, ws_bytes=nbytes, **shape) == WORKSPACE


def test_workspace_of_shapes_that_are_none(lib):
    for size in (lib.nova_fourbit_attention_workspace_bytes, lib.nova_fourbit_mass_workspace_bytes):
        assert size(None, 4, 1, 10) == 0 and size(C.byref(_cache()), 3, 1, 10) == 0
        assert size(C.byref(_cache()), 4, 0, 10) == 0 and size(C.byref(_cache(dh=80)), 4, 1, 10) == 0


# (B, heads, n): products past 2^30, past 2^31, and 2^64 exactly, which is 0 in 64 bits
_TOO_MANY = [(2, 4, 1 << 28), (1, 2, 1 << 30), (2, 1 << 30, 1), (3, 2147483646, 1), (16, 1 << 30, 1 << 30), (4, 1 << 30, 1 << 30),
             (16, 1 << 29, 1 << 30), (65535, 2147483646, 2147483647)]


@pytest.mark.parametrize("call", [_attend, _mass])
@pytest.mark.parametrize("B,heads,n", _TOO_MANY)
def test_sizes_whose_product_wraps(lib, call, B, heads, n):
    for kv_heads in (1, 2):
        assert call(lib, cache=_cache(B=B, kv_heads=kv_heads), heads=heads, n=n, q=_rows(heads=4)) == UNSUPPORTED


@pytest.mark.parametrize("size", ["nova_fourbit_attention_workspace_bytes", "nova_fourbit_mass_workspace_bytes"])
def test_no_workspace_for_sizes_that_the_calls_refuse(lib, size):
    f = getattr(lib, size)
    for B, heads, n in _TOO_MANY:
        for kv_heads in (1, 2):
            assert f(C.byref(_cache(B=B, kv_heads=kv_heads)), heads, n, 10) == 0
    for cache, kv_len in ((_cache(), 101), (_cache(), 2147483647), (_cache(), -1), (_cache(B=65536), 10), (_cache(B=-1), 10),
                          (_cache(kv_heads=32768), 10), (_cache(kv_heads=0), 10), (_cache(capacity=(1 << 24) + 1), 10)):
        for n in (1, 700):
            assert f(C.byref(cache), 2 * max(cache.kv_heads, 1), n, kv_len) == 0


def _evict(lib, src=None, dst=None, k=4, idx=BASE, k_rows=None, kv_len=50, kv_rows=None, kv_next=None, ms=None, md=None):
    return lib.nova_fourbit_evict(_CTX, None, _ref(src or _cache()), _ref(dst or _cache(2, capacity=20)), k, idx, k_rows, kv_len,
                                  kv_rows, kv_next, ms, md)


@pytest.mark.parametrize("kw", [
    dict(k=-1), dict(k=21), dict(kv_len=-1), dict(kv_len=101), dict(idx=None), dict(idx=BASE + 2), dict(k_rows=BASE * 2 + 1),
    dict(dst=_cache(2, B=3)), dict(dst=_cache(2, kv_heads=1)), dict(dst=_cache(2, dh=128)), dict(dst=_cache(1)),
    dict(ms=BASE * 4), dict(md=BASE * 4), dict(ms=BASE * 4, md=BASE * 4), dict(ms=BASE * 4 + 4, md=BASE * 4),
    dict(kv_rows=BASE * 2, kv_next=BASE * 2), dict(k_rows=BASE * 2, kv_next=BASE * 2 + 4), dict(kv_next=BASE + 8),
])
def test_evict(lib, kw):
    assert _evict(lib, **kw) == INVALID


def test_evict_into_a_part_of_its_source(lib):
    src, dst = _cache(), _cache(2, capacity=20)
    dst.v_scales = src.k_scales + 16
    assert _evict(lib, src=src, dst=dst) == INVALID


def test_binding_looks_at_shapes_and_types():
    c = FourBitCache.empty(2, 3, 10, 64, device="cpu")
    assert c.capacity == 10 and c.dh == 64
    assert c.k_codes.shape == (2, 3, 10, 32) and c.v_scales.shape == (2, 3, 10, 2)
    with pytest.raises(ValueError):
        FourBitCache(c.k_codes, c.k_scales, c.v_codes[:, :, :9], c.v_scales).c_struct()
    with pytest.raises(ValueError):
        FourBitCache(c.k_codes, c.k_scales[..., :1], c.v_codes, c.v_scales[..., :1]).c_struct()
    with pytest.raises(AssertionError):
        FourBitCache(c.k_codes.int(), c.k_scales, c.v_codes, c.v_scales).c_struct()
    with pytest.raises(ValueError):
        Bn._rows(torch.zeros(2, 1, 4, 64), 3, 64, "q")
    with pytest.raises(ValueError):
        Bn._shaped("lse", torch.zeros(2, 3), (2, 3, 4), torch.float32)
    with pytest.raises(ValueError):
        Bn._shaped("n_per_row", torch.zeros(2, dtype=torch.int64), (2,), torch.int32)


# ---- the block -------------------------------------------------------------------------------------------------------
def _shape(**kw):
    v = dict(dtype=1, B=2, N=20, C=128, heads=2, ffn_mult=4, kv_len=50, kv_capacity=100, k=10)
    v.update(kw)
    return Bn._Shape(*[v[n] for n, _ in Bn._Shape._fields_])


def _block(lib, shape=None, cache=None, weights=True, variant=None, k_rows=None, kv_rows=None, kv_next=None, x=BASE, idx=BASE,
           mass_in=None, mass=None, y=BASE, ws=BASE, ws_bytes=1 << 40, ctx=_CTX):
    w = Bn._Weights(*[BASE * 4] * 8)
    return lib.nova_pruned_block_fourbit(ctx, None, _ref(shape or _shape()), _ref(w) if weights else None, _ref(variant), k_rows,
                                         kv_rows, kv_next, x, idx, _ref(cache or _cache()), mass_in, mass, y, ws, ws_bytes)


@pytest.mark.parametrize("kw,rc", [
    (dict(ctx=None), INVALID), (dict(weights=False), INVALID), (dict(shape=_shape(dtype=5)), UNSUPPORTED),
    (dict(shape=_shape(k=21)), INVALID), (dict(shape=_shape(kv_len=91)), INVALID), (dict(shape=_shape(kv_len=-1)), INVALID),
    (dict(shape=_shape(C=64)), UNSUPPORTED), (dict(shape=_shape(C=192, dtype=0)), UNSUPPORTED),
    (dict(cache=_cache(B=3)), INVALID), (dict(cache=_cache(kv_heads=1)), INVALID), (dict(cache=_cache(dh=128)), INVALID),
    (dict(cache=_cache(capacity=101)), INVALID), (dict(k_rows=BASE + 1), INVALID), (dict(kv_rows=BASE + 2), INVALID),
    (dict(kv_next=BASE + 3), INVALID), (dict(x=None), INVALID), (dict(idx=None), INVALID), (dict(y=None), INVALID),
    (dict(y=BASE + 8), INVALID), (dict(mass_in=BASE), INVALID), (dict(mass=BASE + 2), INVALID),
    (dict(mass=BASE, mass_in=BASE + 16), INVALID), (dict(variant=Bn._Variant(2, 0)), INVALID),
    (dict(variant=Bn._Variant(0, 1)), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=BASE + 128), WORKSPACE),
])
def test_block(lib, kw, rc):
    assert _block(lib, **kw) == rc


def test_block_workspace(lib):
    size = lib.nova_fourbit_block_workspace_bytes
    need = size(C.byref(_shape()))
    assert need > lib.nova_workspace_bytes(C.byref(_shape(kv_len=0, kv_capacity=64)))
    assert _block(lib, ws_bytes=need - 1) == WORKSPACE
    assert size(None) == 0 and size(C.byref(_shape(k=0))) == 0 and size(C.byref(_shape(kv_len=91))) == 0
    assert _block(lib, shape=_shape(k=0)) == 0 and _block(lib, shape=_shape(B=0), cache=_cache(B=0)) == 0


def test_runner_refuses_what_it_cannot_keep():
    from paper_2602_01345_amd.image import ImageRunner
    for kw in (dict(cache_bits=8), dict(evict_to=10), dict(cache_bits=4, evict_to=0),
               dict(cache_bits=4, evict_to=10 ** 6)):
        with pytest.raises(ValueError):
            ImageRunner(None, B=1, C=128, heads=2, grids=[1, 400], dtype=torch.bfloat16, weights=[{}], device="cpu", **kw)
