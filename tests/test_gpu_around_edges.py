"""Orders, captures and values at the edges of what the calls around the projection allow."""
import math
import threading
from decimal import Decimal, localcontext
from fractions import Fraction

import pytest
import torch

import around_ref as ref
from paper_2603_05035_b200 import binding
from test_gpu_around_projection import filled, rnd

pytestmark = pytest.mark.gpu
DT = ref.DT


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    c.ensure_attention_workspace()
    yield c
    c.close()


# ---- scratch of the attention ---------------------------------------------------------------------

def long_attention(seed=60):
    """One sequence whose heads are cut into parts, so that scratch is used: the call, its result and what it has to be."""
    paged, _ = filled(seed, [9000], 16, 2, 64, "token", "bf16")
    Q, ln = rnd(seed + 1, 1, 8 * 64, dtype="bf16"), torch.tensor([9000], dtype=torch.int32, device="cuda")
    other = binding.Context(0)
    other.ensure_attention_workspace()
    want, o = torch.empty_like(Q), torch.zeros_like(Q)
    other.paged_attention(paged, Q, ln, want)
    torch.cuda.synchronize()
    other.close()
    return (lambda c: c.paged_attention(paged, Q, ln, o)), o, want


def captured(call, c):
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c)
    return graph


def test_attention_leaves_the_batches_workspace_alone():
    """A replay cannot hold back a batch, so it must not write where batches sample, whichever workspace was set first and however large."""
    call, o, want = long_attention()
    for first in (True, False):
        c = binding.Context(0)
        ws = torch.full((16 << 20,), 0x5A, dtype=torch.uint8, device="cuda")
        if first:
            c.set_workspace(ws)
        c.ensure_attention_workspace()
        if not first:
            c.set_workspace(ws)
        graph = captured(call, c)
        graph.replay()
        call(c)
        torch.cuda.synchronize()
        assert (ws == 0x5A).all() and torch.equal(o, want)
        c.close()


def test_replayed_attention_between_two_batches():
    """Batch, replay and batch of the same shape on one stream, against the same with waits in between."""
    n, k, d, p, calls = 512, 26, 512, 1536, 4
    c = binding.Context(0)
    c.set_lanes(calls)
    c.ensure_batch_workspace(n, k, d, p, "bf16", calls)
    c.ensure_attention_workspace()
    call, o, want = long_attention(62)
    H = [rnd(64 + i, n, d, dtype="bf16") for i in range(calls)]
    W = [rnd(70, d, p, scale=0.02, dtype="bf16")] * calls

    def run(between):
        outs = []
        graph = captured(call, c)
        o.zero_()
        for step in range(6):
            q = [torch.empty((n, p), dtype=torch.bfloat16, device="cuda") for _ in range(calls)]
            between()
            c.qkv_offload_batch(H, W, n, k, d, p, [binding.ORTHOGONAL] * calls, [100 * step + i for i in range(calls)], 10.0, "bf16", q)
            between()
            graph.replay()
            between()
            outs += q + [o.clone()]
        torch.cuda.synchronize()
        return outs

    apart = run(torch.cuda.synchronize)
    close = run(lambda: None)
    assert all(torch.equal(a, b) for a, b in zip(apart, close)) and torch.equal(o, want)
    assert c.last_status() == binding.OK
    c.close()


def test_captured_attention_outlives_a_larger_workspace():
    """A later call that needs a larger workspace lets go of the old one; what was captured before does not use it."""
    c = binding.Context(0)
    c.ensure_attention_workspace()
    call, o, want = long_attention(66)
    graph = captured(call, c)
    c.set_workspace(torch.empty(12 << 20, dtype=torch.uint8, device="cuda"))
    c.ensure_workspace(512, 26, 512, 1536, "bf16")
    c.set_workspace(None)
    taken = [torch.full((12 << 20,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want) and all((t == 0x5A).all() for t in taken)
    c.close()


def test_attention_in_the_shared_workspace():
    """Without scratch of its own a call works in the general workspace, unless it is being captured."""
    call, o, want = long_attention(68)
    c = binding.Context(0)
    c.set_workspace(torch.empty(c._lib.gelo_attention_workspace_bytes(), dtype=torch.uint8, device="cuda"))
    call(c)
    torch.cuda.synchronize()
    assert torch.equal(o, want)
    x, graph = torch.zeros(4, device="cuda"), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x += 1
        with pytest.raises(binding.GeloError) as e:
            call(c)
    assert e.value.status == binding.ERR_WORKSPACE
    c.ensure_attention_workspace()
    o.zero_()
    captured(call, c).replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want)
    c.close()


# ---- keys whose logit is minus infinity ---------------------------------------------------------------

def entries(lens, ps, paged):
    """Page and place of every position of each sequence."""
    out = []
    for s, n in enumerate(lens):
        t = torch.arange(n, device="cuda")
        out.append((paged.table[s].long()[t // ps], t % ps))
    return out


def compacted(paged, where, keep):
    """The positions of each sequence that `keep` leaves, as a cache of pages of one token: keys, values, table, lengths."""
    most = max(int(k.sum()) for k in keep)
    table = torch.full((len(keep), most + 1), -1, dtype=torch.int32, device="cuda")
    ks, vs, at = [], [], 0
    for s, ((page, place), on) in enumerate(zip(where, keep)):
        n = int(on.sum())
        table[s, :n] = torch.arange(at, at + n, dtype=torch.int32, device="cuda")
        ks.append(paged.k[page[on], place[on]])
        vs.append(paged.v[page[on], place[on]])
        at += n
    return torch.cat(ks)[:, None], torch.cat(vs)[:, None], table, [int(on.sum()) for on in keep]


def attend_to(ctx, paged, Q, lens, dt):
    o, lse = torch.full_like(Q, 7.0), torch.full((len(lens), Q.shape[1] // paged.head_dim), 7.0, device="cuda")
    ctx.paged_attention(paged, Q, torch.tensor(lens, dtype=torch.int32, device="cuda"), o, lse=lse)
    assert ctx.last_status() == binding.OK
    return o.reshape(len(lens), -1, paged.head_dim).double(), lse.double()


def assert_near(got, got_lse, want, lens, vmax, dt, cache, heads=slice(None)):
    o64, l64, weight, slack = want
    tol_o, tol_l = ref.attend_tolerance(o64, l64, weight, slack, [max(n, 1) for n in lens], vmax, dt, cache)
    empty = torch.isinf(l64)
    assert ((got - o64).abs() <= tol_o)[:, heads].all()
    assert torch.equal(torch.isneginf(got_lse)[:, heads], empty[:, heads])
    assert (((got_lse - l64).abs() <= tol_l) | empty)[:, heads].all()


LENS = [[40, 5000, 17, 1], [(37 * i) % 23 + 1 for i in range(700)], [33] * 40]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lens", LENS, ids=["cut", "alone", "whole"])
@pytest.mark.parametrize("hq,hk,dh", [(1, 1, 64), (8, 2, 128), (14, 1, 64), (11, 1, 256), (3, 1, 80)])
def test_values_behind_keys_of_minus_infinity(ctx, dt, lens, hq, hk, dh):
    """Keys of minus infinity, whole tiles of them too: their values do not count, be they infinite or NaN."""
    ps = 8
    paged, _ = filled(dh + hq, lens, ps, hk, dh, "token", dt)
    where, keep = entries(lens, ps, paged), []
    for s, (page, place) in enumerate(where):
        t = torch.arange(lens[s], device="cuda")
        gone = (t * t * 7 + s) % 5 == 0
        gone |= (t >= 96) & (t < 160)
        if s % 4 == 3:
            gone |= True
        keep.append(~gone)
        paged.k[page[gone], place[gone], :, 0] = -math.inf
        bad = torch.tensor([math.nan, math.inf, -math.inf], device="cuda").to(DT[dt])[t[gone] % 3]
        paged.v[page[gone], place[gone]] = bad[:, None, None]
    Q = rnd(80, len(lens), hq * dh, scale=2.0, dtype=dt)
    Q.reshape(len(lens), hq, dh)[..., 0] = 0.75
    got, lse = attend_to(ctx, paged, Q, lens, dt)
    k, v, table, left = compacted(paged, where, keep)
    want = ref.attend(Q.reshape(len(lens), hq, dh), k, v, table, left, dh ** -0.5)
    assert torch.isfinite(got).all()
    assert_near(got, lse, want, left, ref.values(v).abs().max(), dt, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lens", LENS, ids=["cut", "alone", "whole"])
@pytest.mark.parametrize("hq,dh", [(4, 64), (8, 128), (14, 64), (11, 256)])
def test_keys_of_minus_infinity_for_some_heads(ctx, dt, lens, hq, dh):
    """Keys so large that the logits of every other head overflow: those heads pass over the value, the others do not, and see an infinity in it."""
    ps = 16
    paged, _ = filled(dh + hq, lens, ps, 1, dh, "head", dt)
    where, keep = entries(lens, ps, paged), []
    for s, (page, place) in enumerate(where):
        t = torch.arange(lens[s], device="cuda")
        gone = (t * 11 + s) % 13 == 3
        keep.append(~gone)
        paged.k[page, place, :, 0] = 0.0
        paged.v[page[gone], place[gone], :, 5] = math.inf
    Q = rnd(81, len(lens), hq * dh, scale=2.0, dtype=dt)
    q = Q.reshape(len(lens), hq, dh)
    q[:, 0::2, 0] = 4.0
    q[:, 1::2, 0] = 0.0
    vmax = 8.0
    k, v, table, left = compacted(paged, where, keep)
    passed = ref.attend(q, k, v, table, left, dh ** -0.5)
    counted = ref.attend(q, paged.k, paged.v, paged.table, lens, dh ** -0.5)
    for (page, place), on in zip(where, keep):
        paged.k[page[~on], place[~on], :, 0] = -3e38
    got, lse = attend_to(ctx, paged, Q, lens, dt)
    assert torch.isfinite(got[:, 0::2]).all()
    assert_near(got, lse, passed, left, vmax, dt, dt, slice(0, None, 2))
    some = torch.tensor([not bool(on.all()) for on in keep], device="cuda")
    assert not torch.isfinite(got[some][:, 1::2, 5]).any()     # infinite, or NaN where a weight is too small for fp32
    got[some, :, 5] = 0.0
    for x in counted[0], counted[2]:
        x[some, :, 5] = 0.0
    assert_near(got, lse, counted, lens, vmax, dt, dt, slice(1, None, 2))


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("lens", LENS, ids=["cut", "alone", "whole"])
@pytest.mark.parametrize("hq,dh", [(2, 64), (8, 128), (14, 64), (11, 256)])
def test_logits_of_minus_infinity_on_codes(ctx, dt, lens, hq, dh):
    """A query of minus infinity makes every logit of its head one: that head is zero whatever the values hold, and sees none of its neighbours'."""
    ps = 16
    paged, scales = filled(dh + hq, lens, ps, 1, dh, "token", "e4m3")
    for page, place in entries(lens, ps, paged):
        paged.k[page, place, :, 0] = 0x38                      # one, before its scale
    Q = rnd(82, len(lens), hq * dh, scale=2.0, dtype=dt)
    q = Q.reshape(len(lens), hq, dh)
    clean = ref.attend(q, paged.k, paged.v, paged.table, lens, dh ** -0.5, 0, *scales.values())
    q[:, 0::2, 0] = -math.inf
    got, lse = attend_to(ctx, paged, Q, lens, dt)
    assert (got[:, 0::2] == 0).all() and torch.isneginf(lse[:, 0::2]).all()
    assert_near(got, lse, clean, lens, 448 / 20, dt, "e4m3", slice(1, None, 2))
    for page, place in entries(lens, ps, paged):
        paged.v[page, place] = 0x7F
    got, lse = attend_to(ctx, paged, Q, lens, dt)
    assert (got[:, 0::2] == 0).all() and got[:, 1::2].isnan().all()


# ---- precision of the weights ---------------------------------------------------------------------------

@pytest.mark.parametrize("dt,cache", [("bf16", "e4m3"), ("f16", "e4m3"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("n,hq", [(2, 1), (40, 1), (400, 12)])
def test_weights_of_more_than_half_precision(ctx, dt, cache, n, hq):
    """Two kinds of keys whose values all but cancel: the weight of one kind lies next to 7/8, so close that eleven bits of it would leave a zero."""
    dh = 64
    to_store = (lambda x: x.to(torch.float8_e4m3fn).view(torch.uint8)) if cache == "e4m3" else (lambda x: x.to(DT[cache]))
    k, v = torch.zeros((n, 1, 1, dh), device="cuda"), torch.full((n, 1, 1, dh), 0.875, device="cuda")
    k[1::2, 0, 0, 0], v[1::2] = -1.0, -1.0
    table = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    paged = binding.PagedCache(to_store(k), to_store(v), table)
    Q = torch.zeros((1, hq * dh), dtype=DT[dt], device="cuda")
    Q[:, ::dh] = 1.0
    off = 0.9 * 2.0 ** -12 if cache != "bf16" else 0.9 * 2.0 ** -10
    scale = -math.log(0.875 * (1 + off))
    scale = torch.tensor(scale, dtype=torch.float32).item()
    ln, o, lse = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.empty_like(Q), torch.empty((1, hq), device="cuda")
    ctx.paged_attention(paged, Q, ln, o, scale=scale, lse=lse)
    o64, l64, weight, slack = ref.attend(Q.reshape(1, hq, dh), paged.k, paged.v, table, [n], scale)
    # the stored result's rounding; the logit and exp as in attend_tolerance, a pair of 16-bit values for each weight, sums of n terms
    rel = 2 * slack[..., None] + 2.0 ** -21 * (1 + l64.abs())[..., None] + (n + 16) * 2.0 ** -24 + (2.0 ** -16 if cache == "bf16" else 2.0 ** -21)
    tol = ref.HALF_STEP[dt] * o64.abs() + rel * weight + 2.0 ** -25
    assert (o64.abs() > 2 * tol).all()                          # a zero would be seen
    assert ((o.reshape(1, hq, dh).double() - o64).abs() <= tol).all()


# ---- norm ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d", [512, 4096, 20000])
def test_norm_in_the_place_of_either_input(ctx, d):
    x, r, w = rnd(90, 9, d, dtype="bf16"), rnd(91, 9, d, dtype="bf16"), rnd(92, d, dtype="bf16")
    y, h = torch.empty_like(x), torch.empty_like(x)
    ctx.rms_norm(x, y, weight=w, residual=r, residual_out=h)
    for out, out_h in ((0, 1), (1, 0), (1, None), (0, None), (None, 0), (None, 1)):
        xs, rs = x.clone(), r.clone()
        spare = torch.empty_like(x)
        ys = spare if out is None else (xs, rs)[out]
        hs = None if out_h is None else (xs, rs)[out_h]
        ctx.rms_norm(xs, ys, weight=w, residual=rs, residual_out=hs)
        assert torch.equal(ys, y) and (hs is None or torch.equal(hs, h))
    wide = torch.empty((18, d), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(binding.GeloError) as e:
        ctx.rms_norm(wide[::2], wide[:9], weight=w)
    assert e.value.status == binding.ERR_INVALID
    one = wide[:1]
    one.copy_(x[:1])
    ctx.rms_norm(one, one, weight=w, residual=r[:1])
    assert torch.equal(one, y[:1])


# ---- rotation ------------------------------------------------------------------------------------------

FAR = [0, 1, 8191, 131071, 1 << 24, (1 << 26) - 1, (1 << 30) + 12345, 2 ** 31 - 1]


def unit_pairs(heads, dh, rot, inter):
    """Heads whose pairs are (1, 0), so that a rotation writes cosines and sines; where they stand."""
    x = torch.zeros((len(FAR), heads, dh), device="cuda")
    i = torch.arange(rot // 2, device="cuda")
    a, b = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
    x[:, :, a] = 1.0
    return x.reshape(len(FAR), -1), a, b


def circle(parts):
    """Cosines and sines of exact fractions of a circle."""
    angle = torch.tensor([[2 * math.pi * float(t - round(t)) for t in row] for row in parts], dtype=torch.float64, device="cuda")
    return angle.cos(), angle.sin()


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dh,rot", [(128, 128), (64, 20)])
def test_rotation_is_exact_about_the_turns_it_is_given(ctx, dh, rot, inter):
    """Each cosine and sine is that of the exact product of position and turns, rounded once (and the angle to binary64, 2^-50 radians)."""
    turns = torch.empty(rot // 2, dtype=torch.float64, device="cuda")
    ctx.rope_turns(turns)
    x, a, b = unit_pairs(2, dh, rot, inter)
    y = torch.empty_like(x)
    ctx.rotary(x, 2, torch.tensor(FAR, dtype=torch.int32, device="cuda"), binding.Rope(turns, interleaved=inter), y)
    c, s = circle([[pos * Fraction(t) for t in turns.tolist()] for pos in FAR])
    y = y.reshape(len(FAR), 2, dh).double()
    for want, at in ((c, a), (s, b)):
        assert ((y[:, :, at] - want[:, None]).abs() <= 2.0 ** -24 * want.abs()[:, None] + 2.0 ** -50).all()


@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_rotation_of_far_positions(ctx, base):
    """The whole angle against one worked out with 60 digits: the stored rounding, and what the turns' own costs."""
    rot = 128
    turns = torch.empty(rot // 2, dtype=torch.float64, device="cuda")
    ctx.rope_turns(turns, base=base)
    with localcontext() as digits:
        digits.prec = 60
        pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494")
        exact = [Fraction((Decimal(base).ln() * (-2 * i) / rot).exp() / (2 * pi)) for i in range(rot // 2)]
    x, a, b = unit_pairs(1, rot, rot, False)
    y = torch.empty_like(x)
    pos = torch.tensor(FAR, dtype=torch.int32, device="cuda")
    ctx.rotary(x, 1, pos, binding.Rope(turns), y)
    c, s = circle([[p * t for t in exact] for p in FAR])
    for want, at in ((c, a), (s, b)):
        assert ((y[:, at].double() - want).abs() <= 2.0 ** -24 * want.abs() + 2.0 ** -50 * (1 + pos.double())[:, None]).all()


# ---- what the roundings leave, no more ----------------------------------------------------------------------

def tight(o64, l64, weight, slack, lens, vmax, dt, cache):
    """As attend_tolerance, with weights held as pairs on every cache: 16 bits (bf16) or 22, and on halves, kept relative to 2^-14 of the
    largest, 2^-39 of it absolute."""
    n = torch.as_tensor(lens, device=o64.device).clamp_min(1).double()[:, None, None]
    exp = 2.0 ** -21 * (1 + l64.abs().nan_to_num(posinf=0, neginf=0))
    rel = 2 * slack[..., None] + exp[..., None] + (n + 16) * 2.0 ** -24 + (2.0 ** -16 if cache == "bf16" else 2.0 ** -22)
    return ref.HALF_STEP[dt] * o64.abs() + rel * weight + n * 2.0 ** -39 * vmax + 2.0 ** -25, slack + (n[..., 0] + 16) * 2.0 ** -24 + exp


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("lens,hq,hk,dh,window", [([21000], 1, 1, 128, 0), ([21000], 32, 1, 64, 14000), ([30001], 16, 1, 256, 0), ([9001, 20000], 3, 1, 96, 0),
                                                  ([24000] + [5, 900, 0] * 13, 8, 2, 128, 0), ([5000], 16, 2, 128, 100), ([700] * 3, 32, 32, 128, 0),
                                                  ([(37 * i) % 23 for i in range(700)], 2, 1, 32, 0), ([1, 0, 17, 16, 15, 333, 64, 130, -4, 2], 40, 1, 64, 20)])
def test_attention_on_codes_to_the_last_part(ctx, dt, lens, hq, hk, dh, window):
    """E4M3 caches within what is rounded: a missing part of a head, however small, would stand out."""
    paged, scales = filled(dh + 1, lens, 32, hk, dh, "token", "e4m3")
    Q = rnd(83, len(lens), hq * dh, scale=2.0, dtype=dt)
    o, lse = torch.empty_like(Q), torch.empty((len(lens), hq), device="cuda")
    ctx.paged_attention(paged, Q, torch.tensor(lens, dtype=torch.int32, device="cuda"), o, window=window, lse=lse)
    want = ref.attend(Q.reshape(len(lens), hq, dh), paged.k, paged.v, paged.table, lens, dh ** -0.5, window, *scales.values())
    tol_o, tol_l = tight(*want, lens, ref.values(paged.v).nan_to_num().abs().max() / 20, dt, "e4m3")
    assert ((o.reshape(want[0].shape).double() - want[0]).abs() <= tol_o).all()
    empty = torch.isinf(want[1])
    assert (((lse.double() - want[1]).abs() <= tol_l) | empty).all() and torch.isneginf(lse[empty]).all()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rows,d", [(40, 64), (40, 512), (300, 1024), (40, 2048), (1000, 2048), (40, 4096), (1000, 4096), (400, 8192), (20, 20000)])
def test_norm_codes_on_middles(ctx, dt, rows, d):
    """Rows whose quotients by the largest are the middles of two codes: the rounding of the stored scale decides, the same way for all of a row.
    The row's factor in fp32 would take the wrong side by the hundred."""
    g = torch.Generator(device="cuda").manual_seed(d)
    odd = 17.0 + 2 * torch.randint(0, 8, (rows, d), generator=g, device="cuda")
    x = odd * torch.exp2(torch.randint(-6, 4, (rows, d), generator=g, device="cuda").float())
    x = torch.where(torch.rand((rows, d), generator=g, device="cuda") < 0.5, x, -x)
    x[:, 0] = 448.0
    x = (x * 2.0 ** -4).to(DT[dt])
    codes, scale = torch.empty((rows, d), dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda")
    ctx.rms_norm(x, None, eps=1e-5, codes=codes, row_scale=scale)
    _, y64 = ref.norm(x, None, None, 1e-5)
    want = ref.to_e4m3(y64 / scale.double()[:, None])
    inv = torch.rsqrt(x.float().square().mean(1, keepdim=True) + 1e-5)
    fp32 = ref.to_e4m3((x.float() * (inv / scale[:, None])).double())
    assert (fp32 != want).sum() > rows * d / 100
    # binary64 sums of exact squares and a factor of 48 bits: the side is right unless the scale's rounding is below 2^-46
    assert ((y64 / scale.double()[:, None])[:, 0] / 448 - 1).abs().min() > 2.0 ** -46
    assert torch.equal(ref.values(codes), want)


# ---- threads --------------------------------------------------------------------------------------------

def test_threads_with_contexts_of_their_own():
    """Three threads, each with a context and a stream, make the calls of a step at once; the results are those of the calls one by one."""
    def step(c, set_, out, stream):
        x, w, paged, pos, ln, rope = set_
        n, hk, dh = x.shape[0], paged.kv_heads, paged.head_dim
        h, q, o = out
        c.rms_norm(x, h, weight=w, stream=stream)
        c.append_kv(paged, h[:, -2 * hk * dh:-hk * dh], h[:, -hk * dh:], pos, rope=rope, Q=h[:, :4 * hk * dh], Q_out=q, stream=stream)
        c.paged_attention(paged, q, ln, o, stream=stream)

    ctxs, sets, want = [], [], []
    for i, hk in enumerate((1, 2, 4)):
        c = binding.Context(0)
        c.ensure_attention_workspace()
        lens = [2000 + 300 * i, 9, 700]
        paged, _ = filled(94 + i, lens, 16, hk, 64, "token", "bf16")
        turns = torch.empty(32, dtype=torch.float64, device="cuda")
        c.rope_turns(turns)
        d = 6 * hk * 64
        sets.append((rnd(95 + i, 3, d, dtype="bf16"), rnd(98 + i, d, dtype="bf16"), paged, torch.tensor(lens, dtype=torch.int32, device="cuda") - 1,
                     torch.tensor(lens, dtype=torch.int32, device="cuda"), binding.Rope(turns)))
        ctxs.append(c)
    outs = [[tuple(torch.empty((3, w), dtype=torch.bfloat16, device="cuda") for w in (s[0].shape[1], 4 * s[2].kv_heads * 64, 4 * s[2].kv_heads * 64))
             for _ in range(60)] for s in sets]
    for c, s, o in zip(ctxs, sets, outs):
        step(c, s, o[0], None)
        torch.cuda.synchronize()
        want.append([t.clone() for t in o[0]])
    streams, failed = [torch.cuda.Stream() for _ in ctxs], []

    def run(i):
        try:
            for o in outs[i]:
                step(ctxs[i], sets[i], o, streams[i])
        except Exception as e:                                   # (reported by the test's own thread)
            failed.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(ctxs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for c, out, w in zip(ctxs, outs, want):
        assert all(torch.equal(a, b) for o in out for a, b in zip(o, w))
        assert c.last_status() == binding.OK
        c.close()
