"""Norm, rotation, paged cache and attention of one new token, through the binding, against plain 64-bit forms.

Guard rows and columns around every output are filled beforehand and must stay as they were."""
import math

import pytest
import torch

import around_ref as ref
from paper_2603_05035_b200 import binding

pytestmark = pytest.mark.gpu
DT = ref.DT


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    c.ensure_attention_workspace()
    yield c
    c.close()


def rnd(seed, *shape, scale=1.0, dtype="f32"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(DT[dtype])


def inside(rows, cols, dtype, fill=7.0, left=16, right=16, below=2):
    """A rows x cols view inside a larger matrix that is filled with `fill`, and that matrix."""
    whole = torch.full((rows + below, left + cols + right), fill, device="cuda").to(dtype)
    return whole[:rows, left:left + cols], whole


def untouched(whole, rows, cols, fill=7.0, left=16):
    kept = whole.clone().float()
    kept[:rows, left:left + cols] = fill
    assert (kept == fill).all(), "written outside the result"


# ---- norm ------------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d", [(1, 8), (5, 64), (3, 256), (129, 1000), (7, 2048), (2, 4096), (300, 4096), (3, 8200), (2, 16384), (2, 16392), (1, 65536)])
def test_norm(ctx, dt, rows, d):
    eps = 1e-5
    x, r, w = rnd(1, rows, d, dtype=dt), rnd(2, rows, d, scale=3.0, dtype=dt), (1 + 0.2 * rnd(3, d)).to(DT[dt])
    x[0] *= 1000
    r[-1] = -x[-1]                                              # a sum of zeros
    # a thread adds up to 129 terms in a row, and their sum goes through ten more additions; the root halves that, eight more roundings
    off = (139 / 2 + 8) * 2.0 ** -24
    for res, gain in ((None, w), (r, w), (r, None)):
        h64, y64 = ref.norm(x, res, gain, eps)
        y, whole = inside(rows, d, DT[dt])
        ro, ro_whole = inside(rows, d, DT[dt])
        ctx.rms_norm(x, y, weight=gain, eps=eps, residual=res, residual_out=ro if res is not None else None)
        assert ((y.double() - y64).abs() <= y64.abs() * (ref.HALF_STEP[dt] + off) + 2.0 ** -25).all()
        untouched(whole, rows, d)
        if res is not None:
            assert torch.equal(ro, (x.float() + res.float()).to(DT[dt]))
            untouched(ro_whole, rows, d)
        else:
            assert (ro_whole.float() == 7).all()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d", [(1, 16), (66, 256), (5, 4096), (130, 1040), (2, 20000), (1100, 1104), (1000, 4096), (1300, 4096), (400, 8192)])
def test_norm_codes(ctx, dt, rows, d):
    x, r, w = rnd(4, rows, d, dtype=dt), rnd(5, rows, d, dtype=dt), (1 + 0.2 * rnd(6, d)).to(DT[dt])
    if rows > 1:
        x[1] = 0
        r[1] = 0
    _, y64 = ref.norm(x, r, w, 1e-5)
    codes, whole = inside(rows, d, torch.uint8)
    scale = torch.full((rows + 2,), 7.0, device="cuda")
    y = torch.empty_like(x)
    ctx.rms_norm(x, y, weight=w, residual=r, codes=codes, row_scale=scale[:rows])
    alone = torch.empty_like(codes.contiguous())
    ctx.rms_norm(x, None, weight=w, residual=r, codes=alone, row_scale=torch.empty(rows, device="cuda"))
    assert torch.equal(alone, codes)
    s64 = y64.abs().max(1).values / 448
    s64 = torch.where(s64 > 0, s64, 1.0)
    off = (139 / 2 + 12) * 2.0 ** -24
    s = scale[:rows].double()
    assert ((s - s64).abs() <= s64 * off).all() and (scale[rows:] == 7).all()
    untouched(whole, rows, d)
    z, got = y64 / s[:, None], ref.values(codes.contiguous())
    # the code next to z, or the other neighbour where z lies within `off` of the middle
    assert ((got - z).abs() <= (ref.to_e4m3(z) - z).abs() + 2 * off * z.abs()).all()
    assert (got.abs().max(1).values[s64 != 1] == 448).all()
    if rows > 1:
        assert (codes[1] == 0).all() and scale[1] == 1


def test_norm_in_place_and_strided(ctx):
    x, r, w = rnd(7, 20, 4096, dtype="bf16"), rnd(8, 20, 4096, dtype="bf16"), rnd(9, 4096, dtype="bf16")
    want_y, want_r = torch.empty_like(x), torch.empty_like(x)
    ctx.rms_norm(x, want_y, weight=w, residual=r, residual_out=want_r)
    big = torch.zeros((40, 4096 + 64), dtype=torch.bfloat16, device="cuda")
    xs, rs = big[::2, 32:32 + 4096], r.clone()
    xs.copy_(x)
    ctx.rms_norm(xs, xs, weight=w, residual=rs, residual_out=rs)
    assert torch.equal(xs, want_y) and torch.equal(rs, want_r) and (big[1::2] == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_norm_of_a_row_that_is_not_finite(ctx, bad):
    x = rnd(10, 3, 512, dtype="bf16")
    want, codes0, s0 = torch.empty_like(x), torch.empty((3, 512), dtype=torch.uint8, device="cuda"), torch.empty(3, device="cuda")
    ctx.rms_norm(x, want, codes=codes0, row_scale=s0)
    x[1, 77] = bad
    y, codes, s = torch.empty_like(x), torch.empty_like(codes0), torch.empty_like(s0)
    ctx.rms_norm(x, y, codes=codes, row_scale=s)
    assert s[1].isnan() and ref.values(codes[1]).isnan().all() and y[1, 77].isnan()
    for i in (0, 2):
        assert torch.equal(y[i], want[i]) and torch.equal(codes[i], codes0[i]) and s[i] == s0[i]


def test_rows_of_the_e4m3_product(ctx):
    """Codes and scales of the norm through the product: the tensor core's sum of d products, one rounding to bf16."""
    for m, d, p in ((1, 256, 768), (67, 512, 400), (300, 4096, 1024), (513, 2048, 272)):
        x = rnd(11, m, d, dtype="bf16") * torch.logspace(-2, 2, m, device="cuda")[:, None].bfloat16()
        w8, ws = torch.empty((d, p), dtype=torch.uint8, device="cuda"), torch.empty(2, device="cuda")
        ctx.quantize_e4m3(rnd(12, d, p, scale=0.02, dtype="bf16"), d, p, "bf16", w8, ws)
        codes, s = torch.empty((m, d), dtype=torch.uint8, device="cuda"), torch.empty(m, device="cuda")
        ctx.rms_norm(x, None, codes=codes, row_scale=s)
        s *= torch.logspace(-3, 3, m, device="cuda")
        y = torch.full((m + 1, p), 7.0, dtype=torch.bfloat16, device="cuda")
        ctx.project_e4m3_rows(codes, s, w8, ws, m, d, p, y[:m])
        a, b = ref.values(codes) * s.double()[:, None], ref.values(w8) * ws[0].double()
        want, size = a @ b, a.abs() @ b.abs()
        # products of codes are exact in fp32; the tensor core may keep as few as 22 bits of a partial sum over 32 of them
        assert ((y[:m].double() - want).abs() <= 2.0 ** -8 * want.abs() + (d / 32 + 4) * 2.0 ** -22 * size).all()
        assert (y[m] == 7).all()
        one = torch.full_like(s, 0.5)
        same, scalar = torch.empty_like(y[:m]), torch.empty_like(y[:m])
        ctx.project_e4m3_rows(codes, one, w8, ws, m, d, p, same)
        ctx.project_e4m3(codes, one, w8, ws, m, d, p, scalar)
        assert torch.equal(same, scalar)
    assert ctx.last_status() == binding.OK


# ---- rotation and append -----------------------------------------------------------------------

@pytest.mark.parametrize("rot,kw", [(128, {}), (64, dict(factor=4.0)), (64, dict(base=500000.0, factor=8.0, original=8192.0, low=1.0, high=4.0)),
                                    (2, {}), (256, dict(factor=32.0, original=4096.0)), (10, {})])
def test_turns(ctx, rot, kw):
    t = torch.full((rot // 2 + 1,), 7.0, dtype=torch.float64, device="cuda")
    ctx.rope_turns(t[:rot // 2], **kw)
    want = ref.turns(rot, **kw)
    assert ((t[:rot // 2].cpu() - want).abs() <= 1e-14 * want).all() and t[rot // 2] == 7


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,dh,rot,inter", [(1, 8, 8, False), (4, 64, 64, False), (4, 64, 64, True), (3, 80, 40, False), (3, 80, 20, False), (3, 80, 22, True),
                                                (32, 128, 128, False), (5, 96, 48, True), (2, 256, 256, False), (2, 256, 256, True), (2, 128, 2, False),
                                                (7, 16, 0, False)])
def test_rotary(ctx, dt, heads, dh, rot, inter):
    n = 9
    pos = torch.tensor([0, 1, 2, -1, 4095, 131071, 1000003, 2 ** 31 - 1, 17], dtype=torch.int32, device="cuda")
    x = rnd(20, n, heads * dh, dtype=dt)
    t = torch.empty(rot // 2, dtype=torch.float64, device="cuda")
    ctx.rope_turns(t)
    rope = binding.Rope(t, interleaved=inter, magnitude=1.25)
    want, size = ref.rotate(x, heads, dh, pos, ref.turns(rot), inter, 1.25)
    y, whole = inside(n, heads * dh, DT[dt])
    ctx.rotary(x, heads, pos, rope, y)
    live = pos >= 0
    w, z = want.reshape(n, -1)[live], size.reshape(n, -1)[live]
    # 64-bit turns at the far end: position * 2^-53 * 4 units, far below the fp32 angle
    assert ((y[live].double() - w).abs() <= ref.HALF_STEP[dt] * w.abs() + ref.ROTATED * z).all()
    assert (y[3] == 7).all()
    untouched(whole, n, heads * dh)
    own = x.clone()
    ctx.rotary(own, heads, pos, rope)
    assert torch.equal(own[live], y[live]) and torch.equal(own[3], x[3])


def pool(pages, ps, hk, dh, order, dtype, fill=float("nan")):
    """A cache half as (page, token, head, component); codes are bytes."""
    shape = {"token": (pages, ps, hk, dh), "head": (pages, hk, ps, dh), "wide": (pages, ps, hk, dh + 16)}[order]
    x = torch.full(shape, 0x7F, dtype=torch.uint8, device="cuda") if dtype == "e4m3" else torch.full(shape, fill, dtype=DT[dtype], device="cuda")
    return x.transpose(1, 2) if order == "head" else x[..., :dh]


@pytest.mark.parametrize("dt,cache", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("hq,hk,dh,rot,inter,ps,order", [(4, 4, 64, 64, False, 16, "token"), (8, 2, 128, 64, True, 7, "head"), (6, 3, 80, 80, False, 1, "wide"),
                                                         (2, 1, 96, 24, False, 33, "token"), (2, 2, 16, 10, False, 16, "head")])
def test_append(ctx, dt, cache, hq, hk, dh, rot, inter, ps, order):
    g = torch.Generator().manual_seed(5)
    lens, start = [5, 1, 40, 0, 3], [0, 30, 9, 0, 100]
    seq, pos = [], []
    for s, n in enumerate(lens):
        for j in range(n):
            seq.append(s)
            pos.append(start[s] + j if (s, j) != (2, 11) else -5)          # one padded token in the middle
    n, columns = len(seq), -(-110 // ps)
    order_of = torch.randperm(5 * columns + 3, generator=g)[:5 * columns].to(torch.int32)
    table = order_of.reshape(5, columns).cuda()
    k, v = pool(5 * columns + 3, ps, hk, dh, order, cache), pool(5 * columns + 3, ps, hk, dh, order, cache)
    k0, v0 = ref.bits(k).clone(), ref.bits(v).clone()
    ks, vs = (0.02, 0.3) if cache == "e4m3" else (1.0, 1.0)
    qkv = rnd(30, n, (hq + 2 * hk) * dh, dtype=dt)
    Q, K, V = qkv[:, :hq * dh], qkv[:, hq * dh:(hq + hk) * dh], qkv[:, (hq + hk) * dh:]
    t = torch.empty(rot // 2, dtype=torch.float64, device="cuda")
    ctx.rope_turns(t, factor=4.0, original=64.0, low=1.0, high=8.0)
    rope = binding.Rope(t, interleaved=inter)
    paged = binding.PagedCache(k, v, table, k_scale=ks, v_scale=vs)
    perm = torch.randperm(n, generator=g).cuda()                          # tokens in no order
    seq_t, pos_t = torch.tensor(seq, dtype=torch.int32, device="cuda")[perm], torch.tensor(pos, dtype=torch.int32, device="cuda")[perm]
    qo, whole = inside(n, hq * dh, DT[dt])
    ctx.append_kv(paged, K, V, pos_t, seq=seq_t, rope=rope, Q=Q, Q_out=qo)
    assert ctx.last_status() == binding.OK

    t64 = ref.turns(rot, factor=4.0, original=64.0, low=1.0, high=8.0)
    kr, ksize = ref.rotate(K, hk, dh, pos_t, t64, inter)
    qr, qsize = ref.rotate(Q, hq, dh, pos_t, t64, inter)
    live = pos_t >= 0
    w, z = qr.reshape(n, -1)[live], qsize.reshape(n, -1)[live]
    assert ((qo[live].double() - w).abs() <= ref.HALF_STEP[dt] * w.abs() + ref.ROTATED * z).all()
    assert (qo[~live] == 7).all()
    untouched(whole, n, hq * dh)
    p, s = pos_t[live].long(), seq_t[live].long()
    page, at = table.long()[s, p // ps], p % ps
    for half, before, want, size, scale in ((k, k0, kr, ksize, ks), (v, v0, V.double().reshape(n, hk, dh), None, vs)):
        got, want = ref.values(half)[page, at], want[live] / scale
        slack = ref.ROTATED * size[live] / scale if size is not None else torch.zeros_like(want)
        if cache == "e4m3":
            # the division is rounded too
            assert ((got - want).abs() <= (ref.to_e4m3(want) - want).abs() + 2 * (slack + 2.0 ** -24 * want.abs())).all()
        else:
            assert ((got - want).abs() <= ref.HALF_STEP[dt] * want.abs() + slack).all()
            if size is None:
                assert torch.equal(got, want)
        after = ref.bits(half).clone()
        after[page, at] = before[page, at]
        assert torch.equal(after, before), "an entry that belongs to no token was written"
    # the same without Q, and one token per sequence without a list of sequences
    k2, v2 = pool(5 * columns + 3, ps, hk, dh, order, cache), pool(5 * columns + 3, ps, hk, dh, order, cache)
    again = binding.PagedCache(k2, v2, table, k_scale=ks, v_scale=vs)
    ctx.append_kv(again, K, V, pos_t, seq=seq_t, rope=rope)
    assert torch.equal(ref.bits(k2), ref.bits(k)) and torch.equal(ref.bits(v2), ref.bits(v))
    first = torch.tensor([3, 2, 1, -1, 0], dtype=torch.int32, device="cuda")
    ctx.append_kv(again, K[:5], V[:5], first, rope=None)
    for i in (0, 1, 2, 4):
        got = ref.values(v2)[table[i, int(first[i]) // ps].long(), int(first[i]) % ps]
        want = V[i].double().reshape(hk, dh) / vs
        assert torch.equal(got, ref.to_e4m3((V[i].float().reshape(hk, dh) / vs).double()) if cache == "e4m3" else want)


def test_append_outside_the_cache(ctx):
    """Sequences, positions and pages that do not exist: nothing is written, the status word says so, the other tokens are right."""
    hk, dh, ps = 2, 64, 4
    k, v = pool(6, ps, hk, dh, "token", "bf16"), pool(6, ps, hk, dh, "token", "bf16")
    table = torch.tensor([[0, 1], [2, 6], [-1, 5]], dtype=torch.int32, device="cuda")
    paged = binding.PagedCache(k, v, table)
    K = rnd(31, 8, hk * dh, dtype="bf16")
    seq = torch.tensor([0, 1, 1, 2, 2, 3, -1, 0], dtype=torch.int32, device="cuda")
    pos = torch.tensor([7, 3, 4, 0, 7, 0, 0, 8], dtype=torch.int32, device="cuda")       # right, right, page 6, page -1, right, 3 bad places
    ctx.append_kv(paged, K, K, pos, seq=seq, Q=K.clone())
    assert ctx.last_status() == binding.ERR_INVALID and ctx.last_status() == binding.OK
    wrote = torch.zeros((6, ps), dtype=torch.bool, device="cuda")
    for i, page, at in ((0, 1, 3), (1, 2, 3), (4, 5, 3)):
        assert torch.equal(v[page, at], K[i].reshape(hk, dh)) and torch.equal(k[page, at], K[i].reshape(hk, dh))
        wrote[page, at] = True
    assert v[~wrote].isnan().all() and k[~wrote].isnan().all()


# ---- attention ------------------------------------------------------------------------------------

def filled(seed, lens, ps, hk, dh, order, cache, scale=1.0):
    """A cache with random entries where sequences have positions and NaN everywhere else, its table (-1 where nothing is), its scales."""
    g = torch.Generator().manual_seed(seed)
    per = [-(-max(n, 0) // ps) for n in lens]
    pages = sum(per) + 3
    ids = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), max(per) + 1), -1, dtype=torch.int32)
    at = 0
    for s, c in enumerate(per):
        table[s, :c] = ids[at:at + c]
        at += c
    table = table.cuda()
    halves = []
    for h in range(2):
        x = pool(pages, ps, hk, dh, order, cache)
        for s, n in enumerate(lens):
            if n > 0:
                t = torch.arange(n, device="cuda")
                new = rnd(100 * seed + 10 * s + h, n, hk, dh, scale=scale)
                new = (new * 16).to(torch.float8_e4m3fn).view(torch.uint8) if cache == "e4m3" else new.to(DT[cache])
                x[table[s].long()[t // ps], t % ps] = new
        halves.append(x)
    scales = dict(k_scale=1 / 16, v_scale=1 / 20) if cache == "e4m3" else {}
    return binding.PagedCache(halves[0], halves[1], table, **scales), scales


def check_attention(ctx, paged, Q, lens, dt, cache, scale=None, window=0, status=binding.OK):
    seqs, hq, dh = paged.seqs, Q.shape[1] // paged.head_dim, paged.head_dim
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, whole = inside(seqs, hq * dh, DT[dt])
    lse = torch.full((seqs + 1, hq), 7.0, device="cuda")
    ctx.paged_attention(paged, Q, ln, o, scale=scale, window=window, lse=lse[:seqs])
    assert ctx.last_status() == status
    ks, vs = paged.struct.k_scale, paged.struct.v_scale
    o64, l64, weight, slack = ref.attend(Q.reshape(seqs, hq, dh), paged.k, paged.v, paged.table, lens, scale or dh ** -0.5, window, ks, vs)
    vmax = ref.values(paged.v).nan_to_num().abs().max() * vs
    tol_o, tol_l = ref.attend_tolerance(o64, l64, weight, slack, [max(n, 1) for n in lens], vmax, dt, cache)
    got = o.reshape(seqs, hq, dh).double()
    assert torch.isfinite(got).all()
    worst = ((got - o64).abs() / tol_o).max()
    assert worst <= 1, f"output off by {worst:.3g} tolerances"
    empty = torch.isinf(l64)
    assert torch.equal(torch.isneginf(lse[:seqs]), empty) and (got[empty] == 0).all()
    assert ((lse[:seqs].double() - l64).abs()[~empty] <= tol_l[~empty]).all()
    if dt == "f32" and not empty.all():                         # well inside the worst case: random roundings
        assert (got - o64).norm() <= 4e-6 * o64.norm()
    assert (lse[seqs:] == 7).all()
    untouched(whole, seqs, hq * dh)
    bare = torch.empty((seqs, hq * dh), dtype=DT[dt], device="cuda")
    ctx.paged_attention(paged, Q, ln, bare, scale=scale, window=window)
    assert torch.equal(bare, o) and ctx.last_status() == status  # the same twice, and without lse
    return o, lse[:seqs]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dh", [8, 24, 72])
def test_attention_of_narrow_heads(ctx, dt, dh):
    """Widths that are no multiple of 16."""
    lens = [70, 0, 1, 33]
    paged, _ = filled(dh, lens, 3, 2, dh, "wide", dt)
    check_attention(ctx, paged, rnd(48, 4, 6 * dh, scale=2.0, dtype=dt), lens, dt, dt)


TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")]


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("hq,hk,dh,ps,order", [(4, 4, 64, 16, "token"), (32, 32, 128, 16, "token"), (32, 8, 128, 64, "head"), (6, 1, 128, 5, "wide"),
                                               (16, 2, 80, 24, "head"), (16, 1, 96, 1, "token"), (40, 1, 64, 128, "head"), (3, 3, 256, 16, "token"),
                                               (10, 2, 16, 33, "head"), (24, 2, 256, 7, "token"), (34, 2, 112, 48, "head")])
def test_attention(ctx, dt, cache, hq, hk, dh, ps, order):
    lens = [1, 0, 17, 16, 15, 333, 64, 130, -4, 2]
    paged, _ = filled(hq + dh, lens, ps, hk, dh, order, cache)
    Q = rnd(40, len(lens), hq * dh, scale=2.0, dtype=dt)
    check_attention(ctx, paged, Q, lens, dt, cache)
    check_attention(ctx, paged, Q, lens, dt, cache, scale=0.3, window=20)


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("lens,hq,hk", [([5000], 4, 4), ([5000], 16, 2), ([3, 2000, 1, 999], 8, 1), ([1], 1, 1), ([700] * 3, 32, 32)])
def test_attention_is_cut_along_the_length(ctx, dt, cache, lens, hq, hk):
    paged, _ = filled(hq, lens, 16, hk, 128, "token", cache)
    Q = rnd(41, len(lens), hq * 128, scale=2.0, dtype=dt)
    check_attention(ctx, paged, Q, lens, dt, cache)
    for window in (1, 16, 100, 1 << 30):
        check_attention(ctx, paged, Q, lens, dt, cache, window=window)


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("lens,hq,hk,dh", [([21000], 1, 1, 128), ([21000], 32, 1, 64), ([30001], 16, 1, 256), ([9001, 20000], 3, 1, 96),
                                           ([24000] + [5, 900, 0] * 13, 8, 2, 128), ([700] * 20 + [16000] + [300] * 20 + [16001], 2, 1, 64)])
def test_attention_of_heads_in_many_parts(ctx, dt, cache, lens, hq, hk, dh):
    """Heads cut over so many blocks that the sums are added up in rounds; with few sequences, and in the midst of many."""
    paged, _ = filled(dh, lens, 32, hk, dh, "token", cache)
    Q = rnd(49, len(lens), hq * dh, scale=2.0, dtype=dt)
    check_attention(ctx, paged, Q, lens, dt, cache)
    check_attention(ctx, paged, Q, lens, dt, cache, window=14000)


@pytest.mark.parametrize("dt,cache", TYPES[1:])
@pytest.mark.parametrize("scale", [3e3, 1e6, 1e7, 3e8])
def test_attention_of_huge_logits(ctx, dt, cache, scale):
    """Logits whose neighbours in fp32 are further apart than the exponents of a half are wide: nothing overflows, one key takes all."""
    lens = [300, 1, 4000, 33]
    paged, _ = filled(19, lens, 16, 2, 64, "token", cache)
    Q = rnd(52, 4, 6 * 64, scale=2.0, dtype=dt)
    check_attention(ctx, paged, Q, lens, dt, cache, scale=scale)


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("n", [400, 20000])
def test_attention_of_many_small_weights(ctx, dt, cache, n):
    """A key far above the others has a value of zero: what is left is the sum of weights of 2^-26 of the largest."""
    paged, _ = filled(17, [n], 16, 1, 64, "token", cache)
    at = torch.arange(n, device="cuda")
    page = paged.table[0].long()[at // 16]
    keys, vals = torch.zeros((n, 1, 64), device="cuda"), 0.5 + rnd(18, n, 1, 64).abs().clamp(max=2.0)
    keys[n // 2, 0, 0] = 2.25
    vals[n // 2] = 0
    for x, new, f in ((paged.k, keys, 16), (paged.v, vals, 20)):
        x[page, at % 16] = (new * f).to(torch.float8_e4m3fn).view(torch.uint8) if cache == "e4m3" else new.to(DT[cache])
    Q = torch.zeros((1, 64), dtype=DT[dt], device="cuda")
    Q[0, 0] = 8.0
    ln, o, lse = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.empty_like(Q), torch.empty((1, 1), device="cuda")
    ctx.paged_attention(paged, Q, ln, o, scale=1.0, lse=lse)
    ks, vs = paged.struct.k_scale, paged.struct.v_scale
    o64, l64, weight, slack = ref.attend(Q.reshape(1, 1, 64), paged.k, paged.v, paged.table, [n], 1.0, 0, ks, vs)
    tol_o, tol_l = ref.attend_tolerance(o64, l64, weight, slack, [n], 0.0, dt, cache)          # (nothing but errors relative to each weight)
    assert ((o.reshape(1, 1, 64).double() - o64).abs() <= tol_o).all() and ((lse.double() - l64).abs() <= tol_l).all()


@pytest.mark.parametrize("dt,cache", TYPES)
def test_attention_with_one_key_that_counts(ctx, dt, cache):
    """Logits hundreds apart: the sums are rescaled on the way, and the weight of all others vanishes."""
    lens = [200, 37, 90]
    paged, scales = filled(3, lens, 16, 2, 64, "token", cache)
    Q = rnd(42, 3, 4 * 64, scale=30.0, dtype=dt)
    check_attention(ctx, paged, Q, lens, dt, cache, scale=1.0)


@pytest.mark.parametrize("dt,cache", TYPES)
def test_attention_shares_of_many_sequences(ctx, dt, cache):
    """More sequences than threads in a block, most of them short, one long; strided and in-place rows."""
    lens = [(37 * i) % 23 for i in range(700)]
    lens[611] = 1500
    paged, _ = filled(9, lens, 8, 1, 32, "token", cache)
    Q = rnd(43, 700, 2 * 32, scale=2.0, dtype=dt)
    o, lse = check_attention(ctx, paged, Q, lens, dt, cache)
    big = torch.zeros((700, 3, 64), dtype=DT[dt], device="cuda")
    rows = big[:, 1]
    rows.copy_(Q)
    ctx.paged_attention(paged, rows, torch.tensor(lens, dtype=torch.int32, device="cuda"), rows)
    assert torch.equal(rows, o) and (big[:, 0] == 0).all() and (big[:, 2] == 0).all()


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("seqs,hq,hk,dh,ps,longest", [(650, 1, 1, 64, 16, 190), (300, 6, 2, 128, 16, 380), (200, 48, 3, 80, 8, 60), (130, 5, 5, 256, 32, 100),
                                                      (2500, 1, 1, 16, 4, 9)])
def test_attention_of_many_short_sequences(ctx, dt, cache, seqs, hq, hk, dh, ps, longest):
    """So many short heads that every warp takes some of its own, lengths of zero among them; fewer, and a CTA takes each."""
    lens = [(37 * i * i + 11 * i) % (longest + 1) for i in range(seqs)]
    paged, _ = filled(seqs, lens, ps, hk, dh, "token", cache)
    Q = rnd(47, seqs, hq * dh, scale=2.0, dtype=dt)
    check_attention(ctx, paged, Q, lens, dt, cache)
    few = binding.PagedCache(paged.k, paged.v, paged.table[:70], paged.struct.k_scale, paged.struct.v_scale)
    check_attention(ctx, few, Q[:70], lens[:70], dt, cache, window=33)


@pytest.mark.parametrize("dt,cache", TYPES)
def test_attention_pages_and_lengths_that_do_not_exist(ctx, dt, cache):
    lens = [100, 50, 64, 33]
    paged, _ = filled(11, lens, 16, 2, 64, "head", cache)
    paged.table[0, 2] = paged.pages
    paged.table[1, 0] = -7
    paged.table[3, :3] = 1 << 30
    Q = rnd(44, 4, 4 * 64, dtype=dt)
    check_attention(ctx, paged, Q, lens, dt, cache, status=binding.ERR_INVALID)
    paged, _ = filled(12, [32, 16], 16, 2, 64, "head", cache)
    table = paged.table[:, :1].contiguous()                     # one page of sequence 0 is beyond the table
    cut = binding.PagedCache(paged.k, paged.v, table, paged.struct.k_scale, paged.struct.v_scale)
    check_attention(ctx, cut, rnd(45, 2, 4 * 64, dtype=dt), [32, 16], dt, cache, status=binding.ERR_INVALID)
    check_attention(ctx, cut, rnd(45, 2, 4 * 64, dtype=dt), [2 ** 31 - 1, 0], dt, cache, status=binding.ERR_INVALID)


@pytest.mark.parametrize("dt,cache", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16")])
def test_attention_of_infinities(ctx, dt, cache):
    """A key that takes its logit to minus infinity does not count; a NaN in a value that counts is seen, one in a key too."""
    lens = [40, 40, 40, 40]
    paged, _ = filled(13, lens, 16, 1, 64, "token", cache)
    Q = rnd(46, 4, 64, dtype=dt)
    Q[0, 0] = 1.0
    t = paged.table.long()
    paged.k[t[0, 0], :16, 0, 0] = -math.inf                     # sequence 0: its first 16 positions
    paged.k[t[1, 1], 3, 0, 5] = math.nan
    paged.v[t[2, 2], 2, 0, 9] = math.nan
    o = torch.empty((4, 64), dtype=DT[dt], device="cuda")
    lse = torch.empty((4, 1), device="cuda")
    ctx.paged_attention(paged, Q, torch.tensor(lens, dtype=torch.int32, device="cuda"), o, lse=lse)
    assert o[1].isnan().all() and lse[1].isnan()
    assert o[2, 9].isnan() and o[2].isnan().sum() == 1
    assert torch.isfinite(o[0]).all() and torch.isfinite(o[3]).all()
    k, v = ref.values(paged.k), ref.values(paged.v)
    at = torch.arange(16, 40, device="cuda")
    z = k[t[0][at // 16], at % 16, 0] @ Q[0].double() / 8
    want = torch.softmax(z, 0) @ v[t[0][at // 16], at % 16, 0]
    assert ((o[0].double() - want).abs() <= 2 * ref.HALF_STEP[dt] * want.abs() + 2.0 ** -10).all()
    paged.k[t[0, :3]] = -math.inf * torch.sign(Q[0]).to(paged.k.dtype)[None, None, None, :]       # every logit is minus infinity
    ctx.paged_attention(paged, Q, torch.tensor(lens, dtype=torch.int32, device="cuda"), o, lse=lse)
    assert (o[0] == 0).all() and lse[0] == -math.inf and ctx.last_status() == binding.OK


def test_attention_far_into_a_large_cache(ctx):
    """Offsets beyond 2^31 elements: the last pages of a 6 GB half."""
    ps, hk, dh, pages = 16, 8, 128, 200_000
    k = torch.empty((pages, ps, hk, dh), dtype=torch.bfloat16, device="cuda")
    k[-4:] = rnd(50, 4, ps, hk, dh, dtype="bf16")
    table = torch.tensor([[pages - 1, pages - 3, pages - 2]], dtype=torch.int32, device="cuda")
    small = binding.PagedCache(k[-4:].clone(), k[-4:].clone(), torch.tensor([[3, 1, 2]], dtype=torch.int32, device="cuda"))
    Q, ln = rnd(51, 1, 16 * dh, dtype="bf16"), torch.tensor([45], dtype=torch.int32, device="cuda")
    outs = []
    for cache in (small, binding.PagedCache(k, k, table)):
        K = rnd(52, 1, hk * dh, dtype="bf16")
        ctx.append_kv(cache, K, K, torch.tensor([44], dtype=torch.int32, device="cuda"))
        outs.append(torch.empty_like(Q))
        ctx.paged_attention(cache, Q, ln, outs[-1])
    assert ctx.last_status() == binding.OK and torch.equal(outs[0], outs[1])
    assert torch.equal(k[-4:], small.k)


# ---- together -----------------------------------------------------------------------------------------

def layer_inputs(dt, steps, seqs, d, heads):
    dh = d // heads
    W = rnd(60, d, 3 * d, scale=0.02, dtype=dt)
    xs = [rnd(61 + i, seqs, d, dtype=dt) for i in range(steps)]
    return dh, W, xs


@pytest.mark.parametrize("dt,cache,d,heads", [("f32", "f32", 256, 4), ("bf16", "bf16", 1024, 8), ("bf16", "e4m3", 1024, 8)])
def test_decode_steps(dt, cache, d, heads):
    """Norm, projection (obfuscated), append and attention, a few tokens in a row, against the same in 64 bits from the stored inputs."""
    c = binding.Context(0)
    seqs, steps, eps = 5, 4, 1e-5
    dh, W, xs = layer_inputs(dt, steps, seqs, d, heads)
    c.ensure_workspace(seqs, 2, d, 3 * d, dt)
    c.ensure_attention_workspace()
    t = torch.empty(dh // 2, dtype=torch.float64, device="cuda")
    c.rope_turns(t)
    rope = binding.Rope(t)
    k, v = pool(8, 4, heads, dh, "token", cache), pool(8, 4, heads, dh, "token", cache)
    table = torch.tensor([[0, 1], [2, 3], [4, -1], [5, -1], [6, 7]], dtype=torch.int32, device="cuda")
    scales = dict(k_scale=0.01, v_scale=0.01) if cache == "e4m3" else {}
    paged = binding.PagedCache(k, v, table, **scales)
    start = torch.tensor([0, 2, -100, 0, 1], dtype=torch.int32, device="cuda")         # sequence 2 is not running
    h, r = torch.empty_like(xs[0]), torch.zeros_like(xs[0])
    q, kn, vn, o = (torch.empty_like(xs[0]) for _ in range(4))
    keys = [[] for _ in range(seqs)]
    r64 = torch.zeros((seqs, d), dtype=torch.float64, device="cuda")
    for s in (1, 4):                                            # two of them begin with positions that hold zeros
        page, before = int(table[s, 0]), int(start[s])
        k[page, :before] = 0
        v[page, :before] = 0
        keys[s] = [(torch.zeros((heads, dh), dtype=torch.float64, device="cuda"),) * 2] * before
    live = [s for s in range(seqs) if s != 2]
    for step in range(steps):
        pos = torch.where(start >= 0, start + step, -1).to(torch.int32)
        c.rms_norm(xs[step], h, residual=r, residual_out=r)
        c.qkv_offload(h, W, seqs, 2, d, 3 * d, binding.ORTHOGONAL, 7 + step, 10.0, dt, q, kn, vn)
        c.append_kv(paged, kn, vn, pos, rope=rope, Q=q)
        lens = torch.where(pos >= 0, pos + 1, 0).to(torch.int32)
        c.paged_attention(paged, q, lens, o)
        assert c.last_status() == binding.OK
        h64, y64 = ref.norm(xs[step], r64, None, eps)
        r64 = h64
        y = y64 @ W.double()
        q64, k64 = (ref.rotate(y[:, i * d:(i + 1) * d], heads, dh, pos.clamp_min(0), ref.turns(dh), False)[0] for i in (0, 1))
        v64 = y[:, 2 * d:].reshape(seqs, heads, dh)
        want = torch.zeros((seqs, heads, dh), dtype=torch.float64, device="cuda")
        for s in live:
            keys[s].append((k64[s], v64[s]))
            ks, vs = torch.stack([a for a, _ in keys[s]]), torch.stack([b for _, b in keys[s]])
            z = torch.einsum("hd,nhd->hn", q64[s], ks) * dh ** -0.5
            want[s] = torch.einsum("hn,nhd->hd", torch.softmax(z, 1), vs)
        got = o.double().reshape(seqs, heads, dh)
        assert (got[2] == 0).all()
        # the projection's own budget (1e-4 and 2e-2), an E4M3 rounding of every key and value (2^-4 at most each way)
        rel = (got - want).norm() / want.norm()
        assert rel <= {"f32": 2e-4, "bf16": 4e-2}[dt] + (2.0 ** -4 if cache == "e4m3" else 0.0), (step, float(rel))
    c.close()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_captured_step_replays_on_new_inputs(ctx, cache):
    """Norm, append and attention in a CUDA graph; positions, lengths and inputs change between replays."""
    seqs, hq, hk, dh, ps = 6, 8, 2, 64, 16
    d = (hq + 2 * hk) * dh
    paged, _ = filled(21, [300] * seqs, ps, hk, dh, "token", cache)
    x, h = torch.empty((seqs, d), dtype=torch.bfloat16, device="cuda"), torch.empty((seqs, d), dtype=torch.bfloat16, device="cuda")
    pos, lens = (torch.zeros(seqs, dtype=torch.int32, device="cuda") for _ in range(2))
    o, lse = torch.empty((seqs, hq * dh), dtype=torch.bfloat16, device="cuda"), torch.empty((seqs, hq), device="cuda")
    t = torch.empty(dh // 2, dtype=torch.float64, device="cuda")
    ctx.rope_turns(t)
    rope = binding.Rope(t)

    def step(out, l):
        ctx.rms_norm(x, h)
        ctx.append_kv(paged, h[:, hq * dh:(hq + hk) * dh], h[:, (hq + hk) * dh:], pos, rope=rope, Q=h[:, :hq * dh])
        ctx.paged_attention(paged, h[:, :hq * dh], lens, out, lse=l)

    x.copy_(rnd(70, seqs, d))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(o, lse)
        with torch.cuda.graph(graph, stream=side):
            step(o, lse)
    torch.cuda.current_stream().wait_stream(side)
    for i, at in enumerate(([0, 1, 15, 16, 200, 299], [1, 2, 16, 17, 201, -1], [299, 0, 3, 100, 17, 18])):
        x.copy_(rnd(71 + i, seqs, d))
        pos.copy_(torch.tensor(at, dtype=torch.int32))
        lens.copy_((pos + 1).clamp_min(0))
        graph.replay()
        got, got_lse = o.clone(), lse.clone()
        step(o, lse)
        assert torch.equal(got, o) and torch.equal(got_lse, lse) and torch.isfinite(o).all()
    assert ctx.last_status() == binding.OK


def test_first_calls_of_a_context_can_be_captured():
    """No call before the capture: nothing that a kernel's first use does is forbidden there."""
    c = binding.Context(0)
    c.ensure_attention_workspace()
    lens = [90, 7, 0]
    paged, _ = filled(33, lens, 16, 1, 144, "token", "f16")
    Q, x = rnd(90, 3, 5 * 144, dtype="f16"), rnd(91, 3, 720, dtype="f16")
    o, y, ln = torch.zeros_like(Q), torch.empty_like(x), torch.tensor(lens, dtype=torch.int32, device="cuda")
    pos = torch.tensor([3, 4, -1], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.rms_norm(x, y)
        c.append_kv(paged, y[:, :144], y[:, 144:288], pos)
        c.paged_attention(paged, Q, ln, o)
    graph.replay()
    again = torch.empty_like(o)
    c.paged_attention(paged, Q, ln, again)
    assert torch.equal(o, again) and (o[2] == 0).all() and c.last_status() == binding.OK
    c.close()


def test_attention_on_two_streams_with_contexts_of_their_own():
    """Calls that may overlap on the GPU: each context has its own workspace."""
    ctxs = [binding.Context(0) for _ in range(2)]
    for c in ctxs:
        c.ensure_attention_workspace()
    sets = []
    for i in range(2):
        lens = [3000 + 500 * i, 7, 900]
        paged, _ = filled(30 + i, lens, 16, 4, 128, "token", "bf16")
        sets.append((paged, rnd(80 + i, 3, 16 * 128, dtype="bf16"), torch.tensor(lens, dtype=torch.int32, device="cuda")))
    want = []
    for c, (paged, Q, ln) in zip(ctxs, sets):
        want.append(torch.empty_like(Q))
        c.paged_attention(paged, Q, ln, want[-1])
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(s[1]) for _ in range(20)] for s in sets]
    torch.cuda.synchronize()
    for j in range(20):
        for i in range(2):
            ctxs[i].paged_attention(sets[i][0], sets[i][1], sets[i][2], outs[i][j], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in outs[i])
        assert ctxs[i].last_status() == binding.OK
        ctxs[i].close()


# ---- refusals -------------------------------------------------------------------------------------------

def test_two_graphs_share_a_workspace(ctx):
    """Replayed in turn on one stream, with heads in many parts and in few."""
    runs = []
    for lens, hq, hk in (([20000], 4, 1), ([900, 0, 3000, 17], 8, 2)):
        paged, _ = filled(hq, lens, 16, hk, 64, "token", "bf16")
        Q, ln = rnd(50, len(lens), hq * 64, dtype="bf16"), torch.tensor(lens, dtype=torch.int32, device="cuda")
        want, o = torch.empty_like(Q), torch.zeros_like(Q)
        ctx.paged_attention(paged, Q, ln, want)
        runs.append([paged, Q, ln, o, want, torch.cuda.CUDAGraph()])
    torch.cuda.synchronize()
    for paged, Q, ln, o, _, graph in runs:
        with torch.cuda.graph(graph):
            ctx.paged_attention(paged, Q, ln, o)
    for turn in range(6):
        for run in runs:
            run[3].zero_()
        for i in (0, 1, 1, 0)[turn % 3:]:
            runs[i][5].replay()
        torch.cuda.synchronize()
        for i in set((0, 1, 1, 0)[turn % 3:]):
            assert torch.equal(runs[i][3], runs[i][4])


def test_rotation_of_another_device(ctx):
    turns = torch.empty(32, dtype=torch.float64, device="cuda")
    ctx.rope_turns(turns)
    rope = binding.Rope(turns)
    rope.index = 1                                             # as if the tensor were there
    paged, _ = filled(1, [5], 4, 2, 64, "token", "bf16")
    x, pos = rnd(51, 1, 128, dtype="bf16"), torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        ctx.rotary(x, 2, pos, rope)
    with pytest.raises(ValueError):
        ctx.append_kv(paged, x, x, pos, rope=rope)


def test_refusals(ctx):
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    for kw in (dict(Y=None), dict(Y=x, row_scale=torch.zeros(4, device="cuda")), dict(Y=x, residual_out=x), dict(Y=x, eps=-1.0), dict(Y=x, eps=float("nan"))):
        with pytest.raises(binding.GeloError) as e:
            ctx.rms_norm(x, **kw)
        assert e.value.status == binding.ERR_INVALID
    for kw in (dict(Y=x.float()), dict(Y=x[:3]), dict(Y=x.cpu()), dict(Y=torch.empty((64, 4), dtype=torch.bfloat16, device="cuda").T), dict(Y=x, weight=x[0].float())):
        with pytest.raises(ValueError):
            ctx.rms_norm(x, **kw)
    ctx.rms_norm(x[:0], x[:0])
    paged, _ = filled(1, [5, 5], 4, 2, 64, "token", "bf16")
    Q = rnd(1, 2, 4 * 64, dtype="bf16")
    ln = torch.tensor([5, 5], dtype=torch.int32, device="cuda")
    bare = binding.Context(0)
    with pytest.raises(binding.GeloError) as e:
        bare.paged_attention(paged, Q, ln, torch.empty_like(Q))
    assert e.value.status == binding.ERR_WORKSPACE
    bare.close()
    wide, _ = filled(1, [5, 5], 4, 2, 64, "token", "f32")
    codes, _ = filled(1, [5, 5], 4, 2, 64, "token", "e4m3")
    for cache, q in ((wide, Q), (codes, Q.float())):
        with pytest.raises(binding.GeloError) as e:
            ctx.paged_attention(cache, q, ln, torch.empty_like(q))
        assert e.value.status == binding.ERR_UNSUPPORTED
        with pytest.raises(binding.GeloError) as e:
            ctx.append_kv(cache, q[:, :128], q[:, :128], ln)
        assert e.value.status == binding.ERR_UNSUPPORTED
    for bad in (dict(window=-1), dict(scale=float("inf"))):
        with pytest.raises(binding.GeloError) as e:
            ctx.paged_attention(paged, Q, ln, torch.empty_like(Q), **bad)
        assert e.value.status == binding.ERR_INVALID
    with pytest.raises(binding.GeloError):                     # three query heads on two key-value heads
        ctx.paged_attention(paged, Q[:, :192], ln, torch.empty_like(Q)[:, :192])
    with pytest.raises(ValueError):
        ctx.paged_attention(paged, Q, ln.long(), torch.empty_like(Q))
    u8, w8, y = torch.zeros((4, 64), dtype=torch.uint8, device="cuda"), torch.zeros((64, 32), dtype=torch.uint8, device="cuda"), torch.zeros((4, 32), dtype=torch.bfloat16, device="cuda")
    su, sw = torch.ones(4, device="cuda"), torch.ones(2, device="cuda")
    ctx.project_e4m3_rows(u8, su, w8, sw, 4, 64, 32, y)
    ctx.project_e4m3_rows(u8.view(torch.float8_e4m3fn), su, w8, sw[:1], 4, 64, 32, y)
    for bad in ((u8[:3], su, w8, sw, y), (u8, su[:3], w8, sw, y), (u8, su, w8.float(), sw, y), (u8, su, w8, torch.ones(3, device="cuda"), y), (u8, su, w8, sw, y.float())):
        with pytest.raises(ValueError):
            ctx.project_e4m3_rows(*bad[:4], 4, 64, 32, bad[4])
    with pytest.raises(ValueError):
        ctx.paged_attention(paged, Q, ln, torch.empty_like(Q), window=1 << 40)
    with pytest.raises(ValueError):
        binding.PagedCache(paged.k, paged.v, paged.table.expand(2, -1)[:1].expand(2, -1))
    with pytest.raises(binding.GeloError):                     # more tokens than sequences and no list of them
        K = rnd(1, 3, 128, dtype="bf16")
        ctx.append_kv(paged, K, K, torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert ctx.last_status() == binding.OK
