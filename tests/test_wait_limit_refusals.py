"""The limit of the attention's waits: what is refused, without a GPU (a zeroed stand-in is the context)."""
import ctypes as C

from paper_2608_25431_b200 import binding, build as B


def test_wait_limits():
    B.build_lib()
    lib, ctx = binding.lib(), C.create_string_buffer(1 << 16)
    assert lib.gift_ctx_wait_limit(None, 5) == binding.E_INVAL
    assert lib.gift_ctx_wait_limit(ctx, 10 ** 9 + 1) == binding.E_RANGE
    for ns in (0, 1, 10 ** 9):
        assert lib.gift_ctx_wait_limit(ctx, ns) == binding.OK
