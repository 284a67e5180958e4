"""What the paged-cache calls refuse before anything is launched (no GPU needed).

The argument checks come before the device is touched, so they are driven through the C-ABI with a zeroed
stand-in for the context and numbers in the place of device pointers: a refused call reads neither."""
import ctypes as C

import pytest

from paper_2608_25431_b200 import binding, build as B

PTR = 0x10000                      # stands for a device address; never read


@pytest.fixture(scope="module")
def lib():
    B.build_lib()
    return binding.lib()


@pytest.fixture(scope="module")
def ctx():
    return C.create_string_buffer(1 << 16)


def batch(**kw):
    b = binding._Batch(4, 8, 16, 100, PTR, PTR, PTR, PTR)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def pool(**kw):
    p = binding._KvPool(PTR, 100, 16, 8, 128, 0, PTR)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def attn(**kw):
    a = binding._Attn(PTR, 1024, 128, PTR, 1024, 128, 4, 8, 0.1, PTR, 1, PTR, PTR)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BATCHES = [(dict(n_req=8193), binding.E_RANGE), (dict(page_tokens=0), binding.E_INVAL), (dict(page_tokens=65537), binding.E_RANGE),
           (dict(max_blocks=0), binding.E_INVAL), (dict(max_blocks=2 ** 31), binding.E_RANGE), (dict(owner=None), binding.E_INVAL),
           (dict(have=None), binding.E_INVAL), (dict(want=None), binding.E_INVAL), (dict(table=None), binding.E_INVAL),
           (dict(n_pages=2 ** 31 // 16), binding.E_RANGE)]


def tables(lib, ctx, b, free=PTR, cap=10, n_free=PTR, owner_map=PTR, layers=1, status=PTR):
    return lib.gift_block_tables(ctx, C.byref(b) if b else None, free, cap, n_free, owner_map, layers, status, None)


def slots(lib, ctx, b, n=4, out=PTR):
    return lib.gift_slot_map(ctx, C.byref(b) if b else None, None, n, out, None, None, None, None, None, None)


def segments(lib, ctx, b, serial=PTR, layers=2, token=64, flags=0, segs=PTR, pt=PTR, cap=10):
    return lib.gift_kv_segments(ctx, C.byref(b) if b else None, serial, layers, token, flags, segs, pt, cap, None, None)


def append(lib, ctx, p, k=PTR, ks=(1024, 128), v=PTR, vs=(1024, 128), n=4, sl=PTR, who=PTR, status=PTR):
    return lib.gift_kv_append(ctx, C.byref(p) if p else None, k, *ks, v, *vs, n, sl, who, status, None)


def attention(lib, ctx, b, p, a, status=PTR):
    return lib.gift_kv_attention(ctx, C.byref(b) if b else None, C.byref(p) if p else None, C.byref(a) if a else None, status, None)


@pytest.mark.parametrize("change,code", BATCHES)
def test_batches(lib, ctx, change, code):
    b = batch(**change)
    assert tables(lib, ctx, b) == code and slots(lib, ctx, b) == code and segments(lib, ctx, b) == code
    assert attention(lib, ctx, b, pool(), attn()) == code


def test_null_context_and_structures(lib, ctx):
    b = batch()
    for f in (tables, slots, segments):
        assert f(lib, None, b) == binding.E_INVAL and f(lib, ctx, None) == binding.E_INVAL
    assert append(lib, None, pool()) == binding.E_INVAL and append(lib, ctx, None) == binding.E_INVAL
    for args in ((None, b, pool(), attn()), (ctx, None, pool(), attn()), (ctx, b, None, attn()), (ctx, b, pool(), None)):
        assert attention(lib, *args) == binding.E_INVAL


def test_tables_slots_segments(lib, ctx):
    b = batch()
    for kw in (dict(free=None), dict(n_free=None), dict(owner_map=None), dict(layers=0), dict(status=None)):
        assert tables(lib, ctx, b, **kw) == binding.E_INVAL
    assert tables(lib, ctx, b, layers=1025) == binding.E_RANGE and tables(lib, ctx, b, cap=2 ** 31) == binding.E_RANGE
    assert slots(lib, ctx, b, out=None) == binding.E_INVAL and slots(lib, ctx, b, n=2 ** 31) == binding.E_RANGE
    for kw in (dict(serial=None), dict(layers=0), dict(token=0), dict(flags=4), dict(segs=None), dict(pt=None)):
        assert segments(lib, ctx, b, **kw) == binding.E_INVAL
    for kw in (dict(layers=1025), dict(cap=2 ** 31), dict(token=2 ** 31)):
        assert segments(lib, ctx, b, **kw) == binding.E_RANGE
    assert segments(lib, ctx, batch(n_pages=2 ** 27 - 1), layers=17) == binding.E_RANGE
    assert segments(lib, ctx, b, segs=PTR + 4) == binding.E_ALIGN


POOLS = [(dict(pages=None), binding.E_INVAL), (dict(dtype=2), binding.E_INVAL), (dict(n_heads=0), binding.E_INVAL),
         (dict(head_dim=0), binding.E_INVAL), (dict(page_tokens=0), binding.E_INVAL), (dict(n_heads=1025), binding.E_RANGE),
         (dict(head_dim=2048), binding.E_RANGE), (dict(head_dim=12), binding.E_ALIGN), (dict(pages=PTR + 8), binding.E_ALIGN),
         (dict(n_pages=2 ** 31 // 16), binding.E_RANGE)]


@pytest.mark.parametrize("change,code", POOLS)
def test_pools(lib, ctx, change, code):
    assert append(lib, ctx, pool(**change)) == code
    assert attention(lib, ctx, batch(), pool(**change), attn()) == code


def test_append(lib, ctx):
    p = pool()
    for kw in (dict(k=None), dict(v=None), dict(sl=None), dict(who=None), dict(status=None)):
        assert append(lib, ctx, p, **kw) == binding.E_INVAL
    for kw in (dict(k=PTR + 2), dict(v=PTR + 8), dict(ks=(1028, 128)), dict(vs=(1024, 100))):
        assert append(lib, ctx, p, **kw) == binding.E_ALIGN
    assert append(lib, ctx, p, ks=(2 ** 41, 128)) == append(lib, ctx, p, vs=(1024, 2 ** 38)) == binding.E_RANGE
    assert append(lib, ctx, p, n=2 ** 31) == binding.E_RANGE
    assert append(lib, ctx, p, n=0) == binding.OK


def test_attention(lib, ctx):
    b, p = batch(), pool()
    for kw in (dict(q=None), dict(out=None), dict(n_heads=0), dict(n_heads=12), dict(mask_words=0), dict(out_row_stride=0),
               dict(out_head_stride=0)):
        assert attention(lib, ctx, b, p, attn(**kw)) == binding.E_INVAL, kw
    for kw in (dict(n_heads=2048), dict(n_rows=2 ** 29), dict(mask_words=2 ** 24), dict(q_row_stride=2 ** 41)):
        assert attention(lib, ctx, b, p, attn(**kw)) == binding.E_RANGE, kw
    for kw in (dict(q=PTR + 2), dict(out=PTR + 8), dict(q_head_stride=12), dict(out_row_stride=1025)):
        assert attention(lib, ctx, b, p, attn(**kw)) == binding.E_ALIGN, kw
    assert attention(lib, ctx, b, p, attn(), status=None) == binding.E_INVAL
    assert attention(lib, ctx, b, pool(head_dim=96), attn()) == binding.E_RANGE
    assert attention(lib, ctx, b, pool(n_pages=99), attn()) == binding.E_INVAL
    assert attention(lib, ctx, b, pool(page_tokens=8), attn()) == binding.E_INVAL
    assert attention(lib, ctx, batch(n_req=0), p, attn()) == binding.OK


def test_what_is_accepted_reaches_the_device(lib, ctx):
    import torch
    if torch.cuda.is_available():
        pytest.skip("these calls would run")
    b, p = batch(), pool()
    assert tables(lib, ctx, b) == slots(lib, ctx, b) == segments(lib, ctx, b) == append(lib, ctx, p) == binding.E_CUDA
    assert attention(lib, ctx, b, p, attn()) == binding.E_CUDA
    one = dict(n_rows=1, out_row_stride=0)
    assert attention(lib, ctx, b, p, attn(**one)) == binding.E_CUDA


def test_tensor_checks_of_the_binding():
    import torch
    x = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.Batch(x, x, x, torch.zeros(4, 2, dtype=torch.int32), 16, 8)      # not on a GPU
    with pytest.raises(ValueError):
        binding.Batch(x, x, x, torch.zeros(3, 2, dtype=torch.int32), 16, 8)      # table of another batch
    with pytest.raises(ValueError):
        binding.Batch(x, x, x, x, 16, 8)
    with pytest.raises(ValueError):
        binding._rows3(torch.zeros(4, 2, 8), 0, "k", 2, 8, torch.float32)
