"""What the entry points around the projection refuse on the host beyond `test_around_refusals.py`; an opaque block of zeros stands in for a context."""
import ctypes

import pytest

from paper_2603_05035_b200 import binding

P = 1 << 20                     # an address that is aligned and never followed
INVALID, WORKSPACE, OK = binding.ERR_INVALID, binding.ERR_WORKSPACE, binding.OK


@pytest.fixture(scope="module")
def lib():
    from paper_2603_05035_b200 import build
    build.build()
    return binding.load_library()


@pytest.fixture()
def ctx():
    return ctypes.create_string_buffer(1 << 16)


def test_attention_workspace(lib, ctx):
    need = lib.gelo_attention_workspace_bytes()
    assert lib.gelo_set_attention_workspace(None, P, need) == INVALID
    assert lib.gelo_set_attention_workspace(ctx, P + 16, need) == INVALID
    assert lib.gelo_set_attention_workspace(ctx, P, need - 1) == WORKSPACE
    assert lib.gelo_set_attention_workspace(ctx, P, need) == OK
    assert lib.gelo_set_attention_workspace(ctx, None, 0) == OK


def test_norm_in_place_keeps_the_stride(lib, ctx):
    """One row's results must not land on rows that others have yet to read."""
    A, B, C = P, 2 * P, 3 * P

    def norm(x=A, ldx=64, r=None, ldr=0, w=None, rows=3, d=64, ro=None, ldro=0, y=B, ldy=64, c=None, ldc=0, s=None):
        return lib.gelo_rms_norm(ctx, x, ldx, r, ldr, w, rows, d, 1e-5, binding.BF16, ro, ldro, y, ldy, c, ldc, s, None)

    for bad in (dict(y=A, ldy=128), dict(y=A, ldx=128), dict(r=B, ldr=128), dict(r=C, ldr=64, ro=C, ldro=72), dict(r=C, ldr=64, ro=A, ldro=128), dict(r=C, ldr=64, ro=B, ldro=64),
                dict(r=C, ldr=64, y=A, ro=A, ldro=64), dict(w=B), dict(r=C, ldr=64, w=C, ro=C, ldro=64), dict(c=A, ldc=64, s=P), dict(c=B, ldc=64, s=P),
                dict(c=C, ldc=64, s=P, r=C, ldr=64), dict(c=C, ldc=64, s=P, w=C), dict(rows=1, r=C, ldr=64, ro=B, ldro=64)):
        assert norm(**bad) == INVALID, bad


def test_attention_scales_whose_product_overflows(lib, ctx):
    def call(scale, k_scale, dtype=binding.E4M3):
        c = binding._CacheStruct(k_dev=P, v_dev=P, table_dev=P, page_stride=16 * 4 * 128, token_stride=4 * 128, head_stride=128, dtype=dtype, pages=10, page_size=16,
                                 kv_heads=4, head_dim=128, seqs=0, max_pages=5, table_ld=5, k_scale=k_scale, v_scale=1.0)
        return lib.gelo_paged_attention(ctx, ctypes.addressof(c), P, 1024, 8, P, scale, 0, binding.BF16, P, 1024, None, None)

    for scale, k_scale in ((1e30, 1e10), (-1e30, 1e10), (3e38, 1.0), (1.0, 3e38)):
        assert call(scale, k_scale) == INVALID, (scale, k_scale)
    assert call(3e38, 1.0, binding.BF16) == INVALID
    assert call(2e38, 1.0, binding.BF16) == call(-1e20, 1e18) == call(1e30, 1e-10) == OK       # (no sequences: nothing is launched)
