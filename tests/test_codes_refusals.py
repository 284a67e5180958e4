"""What the calls on rows and 8-bit pages refuse before anything is launched (no GPU needed): as test_paged_refusals.py does,
through the C-ABI with a zeroed stand-in for the context and numbers in the place of device pointers."""
import ctypes as C
import math

import pytest
import torch

from paper_2608_25431_b200 import binding, build as B

PTR = 0x10000                      # stands for a device address; never read


@pytest.fixture(scope="module")
def lib():
    B.build_lib()
    return binding.lib()


@pytest.fixture(scope="module")
def ctx():
    return C.create_string_buffer(1 << 16)


def pool(**kw):
    p = binding._KvPool(PTR, 100, 16, 8, 128, binding.E4M3, PTR)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def rows(**kw):
    a = binding._KvRows(PTR, 4096, 128, PTR, 4096, 128, PTR, 1024, 128, PTR, 1024, 128, 4, 32, 0, 0, PTR, PTR, 1e-6, 64, 1,
                        (C.c_uint32 * 4)(64, 0, 0, 0), PTR, PTR, 4)
    for k, v in kw.items():
        setattr(a, k, (C.c_uint32 * 4)(*v) if k == "sections" else v)
    return a


def attn(**kw):
    a = binding._AttnCodes(binding._Attn(PTR, 1024, 128, PTR, 1024, 128, 4, 8, 0.1, None, 0, PTR, PTR), 0, 0.0, 0, None)
    for k, v in kw.items():
        setattr(a if hasattr(a, k) and k != "attn" else a.attn, k, v)
    return a


def batch(**kw):
    b = binding._Batch(4, 8, 16, 100, PTR, PTR, PTR, PTR)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def write(lib, ctx, p, r, slots=PTR, who=PTR, status=PTR):
    return lib.gift_kv_write(ctx, C.byref(p) if p else None, C.byref(r) if r else None, slots, who, status, None)


def read(lib, ctx, p, dtype=0, n=4, slots=PTR, who=PTR, k=PTR, ks=(1024, 128), v=PTR, vs=(1024, 128), status=PTR):
    return lib.gift_kv_read(ctx, C.byref(p) if p else None, dtype, n, slots, who, k, *ks, v, *vs, status, None)


def attention(lib, ctx, b, p, a, status=PTR):
    return lib.gift_kv_attention_codes(ctx, C.byref(b) if b else None, C.byref(p) if p else None, C.byref(a) if a else None, status, None)


POOLS = [(dict(pages=None), binding.E_INVAL), (dict(n_heads=0), binding.E_INVAL), (dict(head_dim=0), binding.E_INVAL),
         (dict(page_tokens=0), binding.E_INVAL), (dict(n_heads=1025), binding.E_RANGE), (dict(head_dim=2048), binding.E_RANGE),
         (dict(head_dim=24), binding.E_ALIGN), (dict(pages=PTR + 8), binding.E_ALIGN), (dict(n_pages=2 ** 31 // 16), binding.E_RANGE)]


@pytest.mark.parametrize("change, code", POOLS)
def test_pools(lib, ctx, change, code):
    p = pool(**change)
    assert write(lib, ctx, p, rows()) == read(lib, ctx, p) == attention(lib, ctx, batch(), p, attn()) == code


def test_types_of_pools(lib, ctx):
    assert write(lib, ctx, pool(dtype=3), rows()) == read(lib, ctx, pool(dtype=3)) == binding.E_INVAL
    # rows of a 16-bit pool are of its type
    assert write(lib, ctx, pool(dtype=1), rows(dtype=0)) == read(lib, ctx, pool(dtype=1), dtype=0) == binding.E_INVAL
    assert write(lib, ctx, pool(), rows(dtype=2)) == read(lib, ctx, pool(), dtype=2) == binding.E_INVAL
    for d in (0, 1):
        assert attention(lib, ctx, batch(), pool(dtype=d), attn()) == binding.E_INVAL


def test_null_context_and_structures(lib, ctx):
    assert write(lib, None, pool(), rows()) == write(lib, ctx, None, rows()) == write(lib, ctx, pool(), None) == binding.E_INVAL
    assert read(lib, None, pool()) == read(lib, ctx, None) == binding.E_INVAL
    for args in ((None, batch(), pool(), attn()), (ctx, None, pool(), attn()), (ctx, batch(), None, attn()), (ctx, batch(), pool(), None)):
        assert attention(lib, *args) == binding.E_INVAL


def test_write(lib, ctx):
    for kw in (dict(k=None), dict(v=None), dict(q_out=None), dict(q=None), dict(n_heads=0), dict(flags=2), dict(eps=-1.0), dict(eps=math.nan),
               dict(eps=math.inf), dict(freq=None), dict(pos=None), dict(n_axes=0), dict(sections=(63, 0, 0, 0)), dict(n_axes=2, sections=(60, 8, 0, 0)),
               dict(n_axes=2, sections=(2 ** 32 - 1, 65, 0, 0)), dict(q_out_row_stride=0), dict(q_out_head_stride=0)):
        assert write(lib, ctx, pool(), rows(**kw)) == binding.E_INVAL, kw
    for kw in (dict(n_heads=1025), dict(n_freq=68, sections=(68, 0, 0, 0)), dict(n_axes=5), dict(n_rows=2 ** 31), dict(q_row_stride=2 ** 41)):
        assert write(lib, ctx, pool(), rows(**kw)) == binding.E_RANGE, kw
    for kw in (dict(n_freq=30, sections=(30, 0, 0, 0)), dict(q=PTR + 2), dict(k=PTR + 8), dict(q_out=PTR + 4), dict(k_row_stride=1028),
               dict(v_head_stride=100), dict(q_norm=PTR + 8), dict(k_norm=PTR + 2)):
        assert write(lib, ctx, pool(), rows(**kw)) == binding.E_ALIGN, kw
    assert write(lib, ctx, pool(head_dim=272), rows()) == binding.E_RANGE
    for kw in (dict(slots=None), dict(who=None), dict(status=None)):
        assert write(lib, ctx, pool(), rows(), **kw) == binding.E_INVAL
    assert write(lib, ctx, pool(), rows(n_rows=0)) == binding.OK


def test_read(lib, ctx):
    for kw in (dict(k=None), dict(v=None), dict(slots=None), dict(who=None), dict(status=None), dict(ks=(0, 128)), dict(vs=(1024, 0))):
        assert read(lib, ctx, pool(), **kw) == binding.E_INVAL, kw
    for kw in (dict(k=PTR + 2), dict(v=PTR + 8), dict(ks=(1028, 128)), dict(vs=(1024, 100))):
        assert read(lib, ctx, pool(), **kw) == binding.E_ALIGN, kw
    assert read(lib, ctx, pool(), n=2 ** 31) == read(lib, ctx, pool(), ks=(2 ** 41, 128)) == binding.E_RANGE
    assert read(lib, ctx, pool(), n=0) == binding.OK


def test_attention(lib, ctx):
    b, p = batch(), pool()
    for kw in (dict(q=None), dict(out=None), dict(n_heads=0), dict(n_heads=12), dict(tree_mask=PTR), dict(out_row_stride=0), dict(out_head_stride=0),
               dict(dtype=2), dict(softcap=-1.0), dict(softcap=math.nan), dict(softcap=math.inf), dict(scale=math.nan), dict(scale=math.inf),
               dict(tree_mask=PTR, mask_words=1, window=4), dict(tree_mask=PTR, mask_words=1, slopes=PTR)):
        assert attention(lib, ctx, b, p, attn(**kw)) == binding.E_INVAL, kw
    for kw in (dict(n_heads=2048), dict(n_rows=2 ** 29), dict(mask_words=2 ** 24), dict(q_row_stride=2 ** 41), dict(window=2 ** 31),
               dict(scale=3e38), dict(softcap=3e38), dict(scale=1e30, softcap=1e-20)):
        assert attention(lib, ctx, b, p, attn(**kw)) == binding.E_RANGE, kw
    for kw in (dict(q=PTR + 2), dict(out=PTR + 8), dict(q_head_stride=12), dict(out_row_stride=1025)):
        assert attention(lib, ctx, b, p, attn(**kw)) == binding.E_ALIGN, kw
    assert attention(lib, ctx, b, p, attn(), status=None) == binding.E_INVAL
    assert attention(lib, ctx, b, pool(head_dim=96), attn()) == binding.E_RANGE
    assert attention(lib, ctx, b, pool(n_pages=99), attn()) == attention(lib, ctx, b, pool(page_tokens=8), attn()) == binding.E_INVAL
    assert attention(lib, ctx, batch(n_req=8193), p, attn()) == binding.E_RANGE
    assert attention(lib, ctx, batch(n_req=0), p, attn()) == binding.OK


def test_what_is_accepted_reaches_the_device(lib, ctx):
    if torch.cuda.is_available():
        pytest.skip("these calls would run")
    for p, r in ((pool(), rows()), (pool(dtype=0), rows()), (pool(), rows(q=None, q_out=None, q_norm=None)), (pool(), rows(n_freq=0, freq=None, pos=None)),
                 (pool(head_dim=256), rows()), (pool(owner_map=None), rows())):
        assert write(lib, ctx, p, r, who=PTR if p.owner_map else None) == binding.E_CUDA
    assert read(lib, ctx, pool()) == read(lib, ctx, pool(head_dim=1024)) == read(lib, ctx, pool(dtype=1), dtype=1) == binding.E_CUDA
    assert attention(lib, ctx, batch(), pool(), attn(softcap=30.0, window=5, slopes=PTR)) == binding.E_CUDA
    assert attention(lib, ctx, batch(), pool(), attn(tree_mask=PTR, mask_words=1, softcap=30.0)) == binding.E_CUDA


def test_checks_of_the_binding():
    """On CPU tensors: everything is refused, at the latest for where it lies."""
    ctx = binding.Ctx.__new__(binding.Ctx)
    ctx.device, ctx._h = 0, None
    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    slots, who = torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int32)
    pages = torch.zeros((3, 16, binding.kv8_token_bytes(2, 64)), dtype=torch.uint8)
    bad = [dict(pages=pages[:, :, :-16]), dict(pages=pages.float()), dict(pages=pages), dict(k=k.float()), dict(k=k[0])]
    for kw in bad:
        a = dict(pages=pages, k=k) | kw
        with pytest.raises(ValueError):
            ctx.kv_write(a["pages"], a["k"], k, slots, who, who)
        with pytest.raises(ValueError):
            ctx.kv_read(a["pages"], a["k"], k, slots, who, who)
    with pytest.raises(ValueError):
        ctx.kv_attention_codes(None, pages, 2, k.float(), k, who)
    with pytest.raises(ValueError):
        ctx.kv_attention_codes(None, pages, 3, k, k, who)
    assert binding.kv8_token_bytes(3, 80) == 512
