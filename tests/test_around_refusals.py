"""What the entry points around the projection refuse, on the host: every check stands before the first use of the context or the GPU, so an opaque
block of zeros can stand in for a context."""
import ctypes

import pytest
import torch

from paper_2603_05035_b200 import binding

P = 1 << 20                     # an address that is aligned and never followed
INVALID, UNSUPPORTED, OK = binding.ERR_INVALID, binding.ERR_UNSUPPORTED, binding.OK


@pytest.fixture(scope="module")
def lib():
    from paper_2603_05035_b200 import build
    build.build()
    return binding.load_library()


@pytest.fixture(scope="module")
def ctx():
    return ctypes.create_string_buffer(1 << 16)


def cache(**kw):
    c = dict(k_dev=P, v_dev=P, table_dev=P, page_stride=16 * 4 * 128, token_stride=4 * 128, head_stride=128, dtype=binding.BF16, pages=10, page_size=16,
             kv_heads=4, head_dim=128, seqs=3, max_pages=5, table_ld=5, k_scale=1.0, v_scale=1.0)
    c.update(kw)
    return binding._CacheStruct(**c)


def rope(**kw):
    r = dict(turns_dev=P, rot=128, interleaved=0, magnitude=1.0)
    r.update(kw)
    return binding._RopeStruct(**r)


BAD_CACHES = [dict(k_dev=None), dict(v_dev=P + 8), dict(table_dev=None), dict(table_dev=P + 2), dict(page_stride=100), dict(token_stride=64), dict(head_stride=0),
              dict(token_stride=4 * 128 + 4), dict(dtype=4), dict(dtype=-1), dict(pages=0), dict(page_size=0), dict(kv_heads=0), dict(head_dim=4), dict(head_dim=260),
              dict(head_dim=264), dict(head_dim=100), dict(seqs=-1), dict(max_pages=0), dict(table_ld=4), dict(k_scale=0.0), dict(v_scale=-1.0),
              dict(k_scale=float("nan")), dict(v_scale=2.0), dict(dtype=binding.E4M3, k_scale=float("inf")), dict(dtype=binding.E4M3, head_dim=120),
              dict(dtype=binding.E4M3, token_stride=4 * 128 + 8), dict(kv_heads=1 << 30, head_dim=128)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches(lib, ctx, bad):
    c = cache(**bad)
    assert lib.gelo_paged_attention(ctx, ctypes.addressof(c), P, 1024, 8, P, 0.1, 0, binding.BF16, P, 1024, None, None) == INVALID
    assert lib.gelo_append_kv(ctx, ctypes.addressof(c), P, 512, P, 512, None, 0, 0, 3, None, P, None, binding.BF16, None, 0, None) == INVALID


def test_cache_types(lib, ctx):
    for store, act in ((binding.F32, binding.BF16), (binding.BF16, binding.F16), (binding.F16, binding.F32), (binding.E4M3, binding.F32)):
        c = cache(dtype=store)
        assert lib.gelo_paged_attention(ctx, ctypes.addressof(c), P, 1024, 8, P, 0.1, 0, act, P, 1024, None, None) == UNSUPPORTED
    assert lib.gelo_paged_attention(ctx, None, P, 1024, 8, P, 0.1, 0, binding.BF16, P, 1024, None, None) == INVALID


def test_attention(lib, ctx):
    def call(h=ctx, c=cache(), q=P, ldq=1024, heads=8, ln=P, scale=0.1, window=0, dt=binding.BF16, o=P, ldo=1024, lse=None):
        return lib.gelo_paged_attention(h, ctypes.addressof(c), q, ldq, heads, ln, scale, window, dt, o, ldo, lse, None)

    for bad in (dict(h=None), dict(q=None), dict(q=P + 2), dict(ldq=1016), dict(ldq=1028), dict(heads=6), dict(heads=0), dict(ln=None), dict(scale=float("nan")),
                dict(window=-1), dict(dt=3), dict(o=None), dict(o=P + 4), dict(ldo=512), dict(lse=P + 2), dict(heads=1 << 28), dict(ldo=2048)):
        assert call(**bad) == INVALID, bad
    assert call(c=cache(seqs=0)) == OK
    assert lib.gelo_attention_workspace_bytes() > 0


def test_append_and_rotary(lib, ctx):
    def append(h=ctx, c=cache(), k=P, ldk=512, v=P, ldv=512, q=None, ldq=0, heads=0, n=3, seq=None, pos=P, r=None, dt=binding.BF16, qo=None, ldqo=0):
        return lib.gelo_append_kv(h, ctypes.addressof(c), k, ldk, v, ldv, q, ldq, heads, n, seq, pos, ctypes.addressof(r) if r else None, dt, qo, ldqo, None)

    for bad in (dict(h=None), dict(k=None), dict(k=P + 2), dict(v=None), dict(ldk=500), dict(ldk=516), dict(ldv=256), dict(n=-1), dict(n=4), dict(pos=None), dict(dt=9),
                dict(q=P), dict(qo=P), dict(q=P, qo=P, heads=8, ldq=512, ldqo=1024), dict(q=P, qo=P, heads=8, ldq=1024, ldqo=2048), dict(q=P, qo=P, heads=0, ldq=8, ldqo=8),
                dict(r=rope(rot=127)), dict(r=rope(rot=130)), dict(r=rope(rot=-2)), dict(r=rope(turns_dev=None)), dict(r=rope(turns_dev=P + 4)),
                dict(r=rope(magnitude=float("nan")))):
        assert append(**bad) == INVALID, bad
    assert append(n=0) == OK and append(n=0, k=None, v=None, pos=None) == OK

    def rotary(x=P, ldx=512, n=3, heads=4, dh=128, pos=P, r=rope(), dt=binding.BF16, y=P, ldy=512):
        return lib.gelo_rotary(ctx, x, ldx, n, heads, dh, pos, ctypes.addressof(r) if r else None, dt, y, ldy, None)

    for bad in (dict(x=None), dict(y=None), dict(ldx=504), dict(ldy=520), dict(heads=0), dict(dh=12), dict(dh=0), dict(dh=264), dict(pos=None), dict(r=None),
                dict(r=rope(rot=256)), dict(dt=3), dict(n=-1), dict(heads=1 << 30)):
        assert rotary(**bad) == INVALID, bad
    assert rotary(n=0) == OK

    def turns(rot=64, base=1e4, factor=1.0, original=0.0, low=1.0, high=32.0, out=P):
        return lib.gelo_rope_turns(ctx, rot, base, factor, original, low, high, out, None)

    for bad in (dict(rot=3), dict(rot=-2), dict(rot=258), dict(base=0.0), dict(base=float("inf")), dict(factor=0.0), dict(factor=float("nan")), dict(original=-1.0),
                dict(original=10.0, low=2.0, high=2.0), dict(original=10.0, low=float("nan")), dict(out=None), dict(out=P + 4)):
        assert turns(**bad) == INVALID, bad
    assert turns(rot=0, out=None) == OK


def test_norm_and_row_product(lib, ctx):
    def norm(x=P, ldx=64, r=None, ldr=0, w=None, rows=3, d=64, eps=1e-5, dt=binding.BF16, ro=None, ldro=0, y=P, ldy=64, c=None, ldc=0, s=None):
        return lib.gelo_rms_norm(ctx, x, ldx, r, ldr, w, rows, d, eps, dt, ro, ldro, y, ldy, c, ldc, s, None)

    for bad in (dict(x=None), dict(x=P + 8), dict(ldx=56), dict(ldx=68), dict(r=P, ldr=32), dict(ro=P, ldro=64), dict(r=P, ldr=64, ro=P, ldro=60), dict(w=P + 2), dict(rows=-1),
                dict(d=60), dict(d=0), dict(eps=-1.0), dict(dt=3), dict(y=None), dict(ldy=0), dict(c=P, ldc=64), dict(s=P), dict(c=P, ldc=72, s=P), dict(c=P + 8, ldc=64, s=P),
                dict(c=P, ldc=64, s=P + 2), dict(d=72, ldx=72, ldy=72, c=P, ldc=80, s=P)):
        assert norm(**bad) == INVALID, bad
    assert norm(d=65544, ldx=65544, ldy=65544) == UNSUPPORTED
    assert norm(rows=0) == OK

    def rows(u=P, su=P, w=P, sw=P, m=3, d=64, p=64, y=P):
        return lib.gelo_project_e4m3_rows(ctx, u, su, w, sw, m, d, p, y, None)

    for bad in (dict(u=None), dict(su=None), dict(w=P + 8), dict(sw=None), dict(m=0), dict(d=72), dict(p=8), dict(y=P + 2)):
        assert rows(**bad) == INVALID, bad


def test_descriptions_of_tensors_that_do_not_fit():
    k = torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16)
    table = torch.zeros((2, 2), dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.PagedCache(k, k, table)                       # not on a GPU
    with pytest.raises(ValueError):
        binding.PagedCache(k.double(), k, table)
    with pytest.raises(ValueError):
        binding.Rope(torch.zeros(32, dtype=torch.float64))


def test_marshalling_looks_before_it_calls(lib, ctx):
    """Tensors of the wrong kind are refused in words before the library sees an address."""
    m = binding._marshal
    handle = ctypes.addressof(ctx)
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="X must be 4 x 64 of BFloat16 on cuda:0"):
        m.rms_norm(handle, 0, x, x, None, 1e-5, None, None, None, None, 0)
    with pytest.raises(ValueError, match="unsupported dtype of X"):
        m.rms_norm(handle, 0, x.double(), x, None, 1e-5, None, None, None, None, 0)
    with pytest.raises(ValueError, match="X"):
        m.rms_norm(handle, 0, x[0], x, None, 1e-5, None, None, None, None, 0)
    with pytest.raises(ValueError, match="X must be"):
        m.rms_norm(handle, 0, "x", x, None, 1e-5, None, None, None, None, 0)
    with pytest.raises(TypeError):
        m.rms_norm(handle, 0, x)
    with pytest.raises(ValueError, match="multiple of heads"):
        m.rotary(handle, 0, x, 3, x, 0, None, 0)
    c = cache()
    with pytest.raises(ValueError, match="multiple of head_dim"):
        m.paged_attention(handle, 0, ctypes.addressof(c), x, x, x, 0.1, 0, None, 0)
    with pytest.raises(ValueError, match="K must be"):
        m.append_kv(handle, 0, ctypes.addressof(c), x, x, x, None, None, None, None, 0)
    with pytest.raises(ValueError, match="U8 must hold"):
        m.project_e4m3_rows(handle, 0, x, x, x, x, 4, 64, 64, x, 0)
    with pytest.raises((TypeError, ValueError)):
        m.paged_attention(handle, 0, "cache", x, x, x, 0.1, 0, None, 0)
    with pytest.raises(ValueError, match="out of range"):
        m.rotary(handle, 0, x, 1 << 40, x, 0, None, 0)
