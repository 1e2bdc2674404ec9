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
