"""Norms of heads with rotary positions, their gradients, and rows of the cache in 4 bits, on a GPU: against 64-bit formulas,
differences and, bit for bit, the definition of the pages.

Tolerances.  e = 2^-24, u = finfo(dtype).eps / 2: the largest relative errors of one rounding in 32 bits and in the type.
Forward: a sum of squares of positive terms, at most 16 of a lane in turn and 5 additions over lanes, is off by 22 e, its mean
and eps by 2 e more; the inverse root halves that and is itself good to 2 ulp, 4 e: 16 e in all.  Two products, 2 e.  The turn
of 32-bit factors, 4 e (|y_a| + |y_b|).  So |z - exact| <= 24 e A + u |exact|, A = (|y_a| + |y_b|) factor (|y| where nothing
turns), and half the type's smallest step.
Backward: B = the same of the outputs' gradients.  dy off by 4 e B, w = dy g by 5 e B |g|, its sum with x by 28 e S,
S = sum B |g| |x|; times r^2 / D (2 x 16 e and two products): 66 e S r^2 / D; r in front: 16 e more.  So
|dx - exact| <= 84 e r (B |g| + |x| r^2 S / D) + u |exact| and the smallest step.
Gains: a term dy x r is off by 24 e B |x| r; a lane adds up its terms in turn, n of them, then lanes, warps and blocks: at most
n + 5 + 4 + 128 + 8 additions, each e of the sum of magnitudes."""
import numpy as np
import pytest
import torch

from paper_2609_03311_gb300 import dopr

pytestmark = pytest.mark.gpu
DEV = "cuda"
E = 2.0 ** -24
EPS = 1e-6
BLOCKS = 608  # of the backward kernel, at least on 152 SMs; fewer make a lane's turn longer
SMALLEST = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}


def word():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def unit(dt):
    return torch.finfo(dt).eps / 2


# ------------------------------------------------------------------ the formulas, in 64 bits
def turn(x, pos, rope, back=False, magnitudes=False):
    """The rotation of x [T, h, D] float64; magnitudes: the sum of the pair's instead (the bounds' A and B)."""
    if rope is None:
        return x.abs() if magnitudes else x.clone()
    d = rope.cfg.rotary_dim
    f = rope.cfg.theta ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    gain = 1.0
    if rope.cfg.scaling == dopr.ROPE_RAMP:
        gain = rope.cfg.attention_factor  # (the tests' factor is 1: the frequencies stay)
    y = x.clone()
    a, b = (y[..., 0:d:2], y[..., 1:d:2]) if rope.cfg.layout == dopr.ROPE_INTERLEAVED else (y[..., :d // 2], y[..., d // 2:d])
    if magnitudes:
        y = x.abs()
        a, b = (y[..., 0:d:2], y[..., 1:d:2]) if rope.cfg.layout == dopr.ROPE_INTERLEAVED else (y[..., :d // 2], y[..., d // 2:d])
        s = (a + b) * gain
        a.copy_(s), b.copy_(s)
        return y
    w = torch.outer(pos.double(), f)[:, None]
    c, s = torch.cos(w) * gain, torch.sin(w) * gain * (-1 if back else 1)
    u, v = a.clone(), b.clone()
    a.copy_(u * c - v * s), b.copy_(v * c + u * s)
    return y


def gain64(g, D):
    return torch.ones(D, dtype=torch.float64, device=DEV) if g is None else g.double()


def forward64(x, g, pos, rope, eps=EPS):
    x = x.double()
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain64(g, x.shape[-1])
    return turn(y, pos, rope), turn(y, pos, rope, magnitudes=True)


def backward64(dz, x, g, pos, rope, eps=EPS):
    dz, x, g = dz.double(), x.double(), gain64(g, x.shape[-1])
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    dy, B = turn(dz, pos, rope, back=True), turn(dz, pos, rope, magnitudes=True)
    w = dy * g
    dx = r * (w - x * r * r * (w * x).mean(-1, keepdim=True))
    bound = r * (B * g.abs() + x.abs() * r * r * (B * g.abs() * x.abs()).mean(-1, keepdim=True))
    return dx, bound, (dy * x * r).sum((0, 1)), (B * x.abs() * r).sum((0, 1))


def near(got, want, bound32, n32, what):
    dt = got.dtype
    off = (got.double() - want).abs()
    lim = n32 * E * bound32 * (1 + unit(dt)) + unit(dt) * want.abs() + SMALLEST[dt]
    assert torch.isfinite(got).all(), what
    worst = (off / lim).max().item() if off.numel() else 0.0
    assert worst <= 1.0, (what, worst)


def rows(T, hq, hkv, D, dt, seed=0, layout="qkv"):
    """q and k views: of a product's packed rows, heads before tokens, or plain (off: not aligned to 16 bytes)."""
    g = torch.Generator(DEV).manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    if layout == "qkv":
        x = rand(T, (hq + 2 * hkv) * D).to(dt).view(T, -1, D)
        return x[:, :hq], x[:, hq:hq + hkv]
    if layout == "heads":
        return rand(hq, T, D).to(dt).transpose(0, 1), rand(hkv, T, D).to(dt).transpose(0, 1)
    flat = rand(T * (hq + hkv) * D + 1).to(dt)[1:]
    return flat[:T * hq * D].view(T, hq, D), flat[T * hq * D:].view(T, hkv, D)


def make(T, D, rotary, layout=dopr.ROPE_HALF, far=5000, seed=0, factor=1.0):
    pos = torch.randint(0, far, (T,), generator=torch.Generator(DEV).manual_seed(seed + 1), device=DEV, dtype=torch.int32)
    if not rotary:
        return None, None
    more = dict(scaling=dopr.ROPE_RAMP, original_max_position=4096, attention_factor=factor) if factor != 1.0 else {}
    return dopr.Rope(far, rotary, theta=1e6, layout=layout, **more), pos


def gain(D, dt, seed):
    return (1 + 0.3 * torch.randn(D, generator=torch.Generator(DEV).manual_seed(seed), device=DEV)).to(dt)


SHAPES = [  # tokens, q heads, kv heads, D, rotary, view
    (1, 32, 8, 128, 128, "qkv"), (7, 5, 1, 128, 64, "qkv"), (301, 16, 8, 64, 64, "heads"), (33, 4, 4, 96, 48, "qkv"),
    (130, 3, 1, 80, 80, "qkv"), (65, 8, 2, 80, 40, "qkv"), (9, 2, 2, 256, 256, "off"), (17, 6, 2, 128, 128, "off"),
    (12, 3, 1, 2, 2, "qkv"), (40, 2, 1, 34, 10, "heads"), (1300, 8, 2, 128, 0, "qkv"), (3, 40, 8, 256, 128, "qkv")]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T,hq,hkv,D,rotary,view", SHAPES)
def test_norm_and_turn_match_the_formula(T, hq, hkv, D, rotary, view, inter, dt):
    q, k = rows(T, hq, hkv, D, dt, seed=T, layout=view)
    rope, pos = make(T, D, rotary, dopr.ROPE_INTERLEAVED if inter else dopr.ROPE_HALF, seed=T, factor=1.5 if T == 33 else 1.0)
    qg, kg = gain(D, torch.bfloat16, 1), gain(D, torch.bfloat16, 2)
    st = word()
    qo, ko = dopr.head_norm_rope(q, k, qg, kg, eps=EPS, rope=rope, positions=pos, status=st)
    assert st.item() == 0
    for got, x, g in ((qo, q, qg), (ko, k, kg)):
        want, A = forward64(x, g, pos, rope)
        near(got, want, A, 24, "row")


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T,hq,hkv,D,rotary,view", SHAPES)
def test_gradients_match_the_formula(T, hq, hkv, D, rotary, view, inter, dt):
    q, k = rows(T, hq, hkv, D, dt, seed=T + 1, layout=view)
    dqo, dko = rows(T, hq, hkv, D, dt, seed=T + 2, layout="qkv" if view == "heads" else view)
    rope, pos = make(T, D, rotary, dopr.ROPE_INTERLEAVED if inter else dopr.ROPE_HALF, seed=T, factor=1.5 if T == 33 else 1.0)
    qg, kg = gain(D, torch.float32, 3), gain(D, torch.float32, 4)
    st = word()
    dq, dk, dqg, dkg = dopr.head_norm_rope_backward(dqo, q, dko, k, qg, kg, eps=EPS, rope=rope, positions=pos, status=st)
    again = dopr.head_norm_rope_backward(dqo, q, dko, k, qg, kg, eps=EPS, rope=rope, positions=pos)
    assert st.item() == 0
    for a, b in zip((dq, dk, dqg, dkg), again):
        assert torch.equal(a, b)
    for got, gg, x, dz, g in ((dq, dqg, q, dqo, qg), (dk, dkg, k, dko, kg)):
        dx, bound, dg, dg_bound = backward64(dz, x, g, pos, rope)
        near(got, dx, bound, 84, "dx")
        n = -(-T // BLOCKS) * -(-(hq + hkv) // 4)
        near(gg, dg, dg_bound, 24 + n + 145, "gain")


def test_gradients_match_differences():
    # the 64-bit formula's loss, moved along a direction; the kernel's gradient in 32 bits.  Differences are off by h^2 of the third
    # derivative and 2^-53 / h of the loss: with h = 1e-4 and numbers near one, both below 1e-7 of the sums of magnitudes
    T, hq, D = 6, 3, 64
    q, _ = rows(T, hq, 1, D, torch.float32, seed=5)
    dz, _ = rows(T, hq, 1, D, torch.float32, seed=6)
    rope, pos = make(T, D, 32, dopr.ROPE_INTERLEAVED)
    g = gain(D, torch.float32, 7)
    dq, _, dg, _ = dopr.head_norm_rope_backward(dz, q, q_gain=g, eps=1e-2, rope=rope, positions=pos)
    loss = lambda x, gg: (forward64(x, gg, pos, rope, 1e-2)[0] * dz.double()).sum()  # noqa: E731
    h = 1e-4
    for seed in range(4):
        v = torch.randn(T, hq, D, generator=torch.Generator(DEV).manual_seed(seed), device=DEV, dtype=torch.float64)
        w = torch.randn(D, generator=torch.Generator(DEV).manual_seed(seed + 9), device=DEV, dtype=torch.float64)
        by_x = (loss(q.double() + h * v, g) - loss(q.double() - h * v, g)) / (2 * h)
        by_g = (loss(q, g.double() + h * w) - loss(q, g.double() - h * w)) / (2 * h)
        assert abs((dq.double() * v).sum() - by_x) <= 2e-6 * (dq.double() * v).abs().sum()
        assert abs((dg.double() * w).sum() - by_g) <= 2e-6 * (dg.double() * w).abs().sum()


@pytest.mark.parametrize("gd", [torch.float16, torch.bfloat16, torch.float32, None])
def test_gains_of_every_type_and_none(gd):
    T, D = 50, 128
    q, k = rows(T, 8, 2, D, torch.bfloat16, seed=8)
    qg = None if gd is None else gain(D, gd, 1)
    rope, pos = make(T, D, D)
    qo, ko = dopr.head_norm_rope(q, k, qg, qg, rope=rope, positions=pos)
    for got, x in ((qo, q), (ko, k)):
        want, A = forward64(x, qg, pos, rope)
        near(got, want, A, 24, gd)
    dq, dk, a, b = dopr.head_norm_rope_backward(qo, q, ko, k, qg, None, rope=rope, positions=pos)
    assert (a is None) == (gd is None) and b is None
    near(dq, *backward64(qo, q, qg, pos, rope)[:2], 84, "dq")
    near(dk, *backward64(ko, k, None, pos, rope)[:2], 84, "dk")


def test_rows_without_a_position_are_left_and_bad_positions_are_errors():
    T, D = 9, 128
    q, k = rows(T, 4, 2, D, torch.float16, seed=3)
    rope, pos = make(T, D, D, far=100)
    pos[2], pos[5] = -1, 100
    qo, ko = torch.full((T, 4, D), 3.0, device=DEV).half(), torch.full((T, 2, D), 3.0, device=DEV).half()
    st = word()
    g = gain(D, torch.float32, 1)
    dopr.head_norm_rope(q, k, g, g, rope=rope, positions=pos, q_out=qo, k_out=ko, status=st)
    assert st.item() == dopr.ERR_INVALID_ARG
    live = [i for i in range(T) if i not in (2, 5)]
    for got, x in ((qo, q), (ko, k)):
        assert (got[[2, 5]] == 3.0).all()
        want, A = forward64(x[live], g, pos[live], rope)
        near(got[live], want, A, 24, "live")
    st.zero_()
    dz, dzk = rows(T, 4, 2, D, torch.float16, seed=4)
    dq, dk, dqg, dkg = dopr.head_norm_rope_backward(dz, q, dzk, k, g, g, rope=rope, positions=pos, dq=qo, dk=ko, status=st)
    assert st.item() == dopr.ERR_INVALID_ARG
    kept = torch.tensor(live, device=DEV)
    for gg, x, d in ((dqg, q, dz), (dkg, k, dzk)):
        _, _, want, bound = backward64(d[kept], x[kept], g, pos[kept], rope)
        near(gg, want, bound, 24 + 10 + 145, "gain")
    assert torch.equal(dq[[2, 5]], qo[[2, 5]]) and st.item()


def test_in_place_repeated_rows_and_no_rows():
    T, D = 70, 64
    q, k = rows(T, 8, 2, D, torch.bfloat16, seed=2)
    rope, pos = make(T, D, D)
    g = gain(D, torch.bfloat16, 1)
    qo, ko = dopr.head_norm_rope(q, k, g, g, rope=rope, positions=pos)
    a, b = q.clone(), k.clone()
    dopr.head_norm_rope(a, b, g, g, rope=rope, positions=pos, q_out=a, k_out=b)
    assert torch.equal(a, qo) and torch.equal(b, ko)
    # gradients over the outputs' gradients, and over the inputs
    want = dopr.head_norm_rope_backward(qo, q, ko, k, g, g, rope=rope, positions=pos)
    a, b = qo.clone(), ko.clone()
    got = dopr.head_norm_rope_backward(a, q, b, k, g, g, rope=rope, positions=pos, dq=a, dk=b)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and got[0] is a
    a, b = q.clone(), k.clone()
    got = dopr.head_norm_rope_backward(qo, a, ko, b, g, g, rope=rope, positions=pos, dq=a, dk=b)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    # one row for all tokens
    one, _ = dopr.head_norm_rope(q[:1].expand(T, -1, -1), None, g, rope=rope, positions=pos)
    many, _ = dopr.head_norm_rope(q[:1].repeat(T, 1, 1), None, g, rope=rope, positions=pos)
    assert torch.equal(one, many)
    # none
    z = q[:0]
    qo, _ = dopr.head_norm_rope(z, None, g)
    assert qo.shape == (0, 8, D)
    _, _, dg, _ = dopr.head_norm_rope_backward(z, z, q_gain=g)
    assert (dg == 0).all()


def test_bad_numbers_stay_in_their_head():
    T, D = 40, 128
    q, _ = rows(T, 4, 1, D, torch.bfloat16, seed=1)
    q = q.clone()
    rope, pos = make(T, D, D)
    clean, _ = dopr.head_norm_rope(q, rope=rope, positions=pos)
    q[3, 1, 5], q[7, 2, 9], q[9, 0] = float("nan"), float("inf"), 0.0
    got, _ = dopr.head_norm_rope(q, rope=rope, positions=pos)
    bad = torch.zeros(T, 4, dtype=torch.bool, device=DEV)
    bad[3, 1], bad[7, 2], bad[9, 0] = True, True, True
    assert torch.equal(got[~bad], clean[~bad])
    assert got[3, 1].isnan().all() and got[7, 2].isnan().any() and (got[9, 0] == 0).all()


# ------------------------------------------------------------------ the pages
def scales64():
    return torch.tensor([(8 + i % 8) * 2.0 ** (i // 8 - 18) if i >= 8 else i * 2.0 ** -17 for i in range(0xe2)],
                        dtype=torch.float64, device=DEV)


def codes_of(x):
    """(c, scale byte) of rows [..., D] by the definition: the smallest scale, the nearest code, ties away from zero."""
    g = x.double().unflatten(-1, (-1, 32))
    most = g.abs().amax(-1)
    ok = (g.abs() <= 65504).all(-1)  # (false for a NaN)
    byte = torch.searchsorted(7 * scales64(), torch.where(ok, most, 0.0)).clamp(max=0xe1)
    s = scales64()[byte][..., None]
    c = torch.where(s > 0, torch.sign(g) * torch.floor(g.abs() / torch.where(s > 0, s, 1.0) + 0.5), 0.0)
    c = torch.where(ok[..., None], c, 0.0)
    return c.long().flatten(-2), torch.where(ok, byte, 0xff)


def packed(x):
    """The bytes of a row's codes and scales, [..., D / 2] and [..., D / 32]."""
    c, byte = codes_of(x)
    n = (c + 8).unflatten(-1, (-1, 8))
    word = sum(n[..., i] << (4 * (i // 2) + 16 * (i % 2)) for i in range(8))
    return torch.stack([word >> (8 * j) & 255 for j in range(4)], -1).flatten(-2).to(torch.uint8), byte.to(torch.uint8)


def put(pool, page, D, slots, x):
    """Rows x [T, kv heads, D] into a copy of the pool's bytes."""
    pool = pool.clone()
    codes, scales = packed(x)
    block, at = slots // page, slots % page
    a = pool[..., :page * D // 2].view(pool.shape[0], pool.shape[1], page, D // 2)
    b = pool[..., page * D // 2:].view(pool.shape[0], pool.shape[1], page, D // 32)
    live = slots >= 0
    a[block[live], :, at[live]] = codes[live]
    b[block[live], :, at[live]] = scales[live]
    return pool


def pools(layout, seed=0):
    g = torch.Generator(DEV).manual_seed(seed)
    return tuple(torch.randint(0, 256, p.shape, generator=g, device=DEV, dtype=torch.uint8) for p in dopr.cache_pools_4bit(layout))


def slots_of(T, n, seed=0):
    return torch.randperm(n, generator=torch.Generator(DEV).manual_seed(seed), device=DEV)[:T]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("T,hkv,D", [(1, 8, 128), (1, 1, 64), (37, 3, 128), (300, 2, 64), (700, 8, 128)])
def test_append_writes_the_definitions_bytes(T, hkv, D, page, dt):
    blocks = -(-T // page) + 2
    layout = dopr.make_cache_layout(blocks, page, hkv, D, dt, 1, blocks)
    kp, vp = pools(layout, T)
    slots = slots_of(T, blocks * page, T)
    slots[T // 2] = -1 if T > 1 else slots[0]
    g = torch.Generator(DEV).manual_seed(T)
    qkv = torch.randn(T, 4 * hkv * D, generator=g, device=DEV)
    qkv *= torch.exp(3 * torch.randn(T, 1, generator=g, device=DEV))  # rows of all sizes
    qkv = qkv.clamp(-60000, 60000).to(dt).view(T, 4 * hkv, D)
    k, v = qkv[:, hkv:2 * hkv], qkv[:, 3 * hkv:]
    want = put(kp, page, D, slots, k), put(vp, page, D, slots, v)
    st = word()
    dopr.cache_append_4bit(layout, slots, k, v, kp, vp, status=st)
    assert st.item() == 0
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])
    # and what they stand for comes back exactly, within half a step of the row
    ko, vo = torch.full((T + 1, hkv, D), 3.0, device=DEV).to(dt), torch.full((T + 1, hkv, D), 3.0, device=DEV).to(dt)
    dopr.cache_read_4bit(layout, torch.cat([slots, slots[:1]]), kp, vp, k_out=ko, v_out=vo, status=st)
    assert st.item() == 0
    for got, x in ((ko, k), (vo, v)):
        c, byte = codes_of(x)
        s = scales64()[byte].repeat_interleave(32, -1)
        live = slots >= 0
        assert torch.equal(got[:T][live].double(), (c * s)[live]) and (got[:T][~live] == 3.0).all()
        assert ((got[:T].double() - x.double()).abs() <= s / 2)[live].all()
        assert torch.equal(got[T], got[0])


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
def test_groups_of_every_size_ties_and_the_scales_ends(dt):
    # every exponent of the rows' type that counts, group maxima at and beside each scale, elements half way between codes
    vals = []
    for s in scales64().tolist():
        for top in (6.9 * s, 7 * s, 7.1 * s):
            row = torch.tensor([min(top, 65504.0)] + [(i - 15) * s / 2 for i in range(31)], dtype=torch.float64)
            vals.append(row.clamp(-65504, 65504))
    x = torch.stack(vals).to(DEV).to(dt)
    x = x.clamp(-65504, 65504)
    x = torch.cat([x, torch.zeros(-len(x) % 2, 32, device=DEV, dtype=dt)]).view(-1, 1, 64)
    T = len(x)
    layout = dopr.make_cache_layout(T // 16 + 1, 16, 1, 64, dt, 1, T // 16 + 1)
    kp, vp = pools(layout)
    slots = slots_of(T, T)
    st = word()
    want = put(kp, 16, 64, slots, x)
    dopr.cache_append_4bit(layout, slots, x, -x, kp, vp, status=st)
    assert torch.equal(kp, want)
    # bf16 rounds 65504 up to 65536, which is too large
    assert st.item() == (0 if dt == torch.float16 else dopr.ERR_RANGE)
    k, v = dopr.cache_read_4bit(layout, slots, kp, vp)
    assert torch.equal(torch.nan_to_num(k), torch.nan_to_num(-v))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), 70000.0])
def test_groups_that_cannot_be_held_are_nan_and_an_error(bad):
    T, D = 20, 128
    layout = dopr.make_cache_layout(2, 16, 2, D, torch.bfloat16, 1, 2)
    k, v = (torch.randn(T, 2, D, device=DEV).bfloat16() for _ in range(2))
    slots = slots_of(T, 32)
    kp, vp = pools(layout)
    clean = put(kp, 16, D, slots, k), put(vp, 16, D, slots, v)
    v[4, 1, 70] = bad
    want = put(vp, 16, D, slots, v)
    st = word()
    dopr.cache_append_4bit(layout, slots, k, v, kp, vp, status=st)
    assert st.item() == dopr.ERR_RANGE and torch.equal(kp, clean[0]) and torch.equal(vp, want)
    _, vo = dopr.cache_read_4bit(layout, slots, kp, vp)
    nan = torch.zeros(T, 2, D, dtype=torch.bool, device=DEV)
    nan[4, 1, 64:96] = True
    assert torch.equal(vo.isnan(), nan)


def test_slots_outside_the_pool_are_errors_and_write_nothing():
    layout = dopr.make_cache_layout(3, 16, 2, 64, torch.float16, 1, 3)
    k = torch.randn(4, 2, 64, device=DEV).half()
    slots = torch.tensor([5, 48, 2 ** 40, 47], device=DEV)
    kp, vp = pools(layout)
    want = put(kp, 16, 64, torch.tensor([5, -1, -1, 47], device=DEV), k)
    st = word()
    dopr.cache_append_4bit(layout, slots, k, k, kp, vp, status=st)
    assert st.item() == dopr.ERR_INVALID_ARG and torch.equal(kp, want)
    st.zero_()
    out = torch.full((4, 2, 64), 3.0, device=DEV).half()
    dopr.cache_read_4bit(layout, slots, kp, vp, k_out=out, status=st)
    assert st.item() == dopr.ERR_INVALID_ARG and (out[1:3] == 3.0).all() and not (out[[0, 3]] == 3.0).all()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T,hq,hkv,D,rotary", [(1, 32, 8, 128, 128), (50, 8, 2, 128, 64), (333, 5, 5, 64, 64), (20, 4, 1, 64, 16),
                                               (9, 2, 1, 128, 0)])
def test_norm_turn_and_append_at_once_give_the_bits_of_one_after_another(T, hq, hkv, D, rotary, inter, dt):
    layout = dopr.make_cache_layout(T // 16 + 2, 16, hkv, D, dt, 1, T // 16 + 2)
    q, k = rows(T, hq, hkv, D, dt, seed=T)
    v = k.flip(0).contiguous()
    rope, pos = make(T, D, rotary, dopr.ROPE_INTERLEAVED if inter else dopr.ROPE_HALF, far=1000)
    qg, kg = gain(D, torch.bfloat16, 1), gain(D, torch.bfloat16, 2)
    slots = slots_of(T, T)
    if T > 3 and rotary:
        slots[1], pos[2] = -1, -1
    qo, ko = torch.zeros(T, hq, D, device=DEV, dtype=dt), torch.zeros(T, hkv, D, device=DEV, dtype=dt)
    dopr.head_norm_rope(q, k, qg, kg, rope=rope, positions=pos, q_out=qo, k_out=ko)
    kp, vp = pools(layout)
    ka, va = kp.clone(), vp.clone()
    where = slots if pos is None else torch.where(pos < 0, -1, slots)
    dopr.cache_append_4bit(layout, where, ko, v, ka, va)
    q2 = torch.zeros_like(qo)
    st = word()
    dopr.cache_append_4bit(layout, slots, k, v, kp, vp, k_gain=kg, eps=EPS, rope=rope, positions=pos, q=q, q_gain=qg, q_out=q2,
                           status=st)
    assert st.item() == 0 and torch.equal(kp, ka) and torch.equal(vp, va) and torch.equal(q2, qo)
    # a turn without a norm: what the 16-bit cache stores
    if rotary:
        k16, v16 = (torch.zeros(layout.n_blocks, hkv, 16, D, device=DEV, dtype=dt) for _ in range(2))
        dopr.cache_append(layout, where, k, v, k16, v16, rope=rope, positions=pos, q=q, q_out=qo)
        kp, vp = pools(layout, 5)
        live = where[where >= 0]
        dopr.cache_append_4bit(layout, where, k, v, kp, vp, rope=rope, positions=pos, q=q, q_out=q2)
        got, _ = dopr.cache_read_4bit(layout, live, kp, vp)
        c, byte = codes_of(k16[live // 16, :, live % 16])
        assert torch.equal(got.double(), c * scales64()[byte].repeat_interleave(32, -1)) and torch.equal(q2, qo)


def test_pools_beyond_32_bits_of_bytes():
    page, hkv, D = 128, 8, 128
    blocks = 2 ** 32 // (hkv * page * 68) + 3
    layout = dopr.make_cache_layout(blocks, page, hkv, D, torch.bfloat16, 1, 8)
    kp, vp = dopr.cache_pools_4bit(layout)
    assert kp.numel() > 2 ** 32
    slots = torch.tensor([0, blocks * page - 1, (blocks - 1) * page, blocks // 2 * page + 77], device=DEV)
    k, v = (torch.randn(4, hkv, D, device=DEV).bfloat16() for _ in range(2))
    dopr.cache_append_4bit(layout, slots, k, v, kp, vp)
    got = dopr.cache_read_4bit(layout, slots, kp, vp)
    for x, y in zip(got, (k, v)):
        c, byte = codes_of(y)
        assert torch.equal(x.double(), c * scales64()[byte].repeat_interleave(32, -1))
    assert int((kp != 0).sum()) <= 4 * hkv * 68


def test_on_another_stream_and_in_a_graph():
    T, D = 64, 128
    layout = dopr.make_cache_layout(8, 16, 2, D, torch.bfloat16, 1, 8)
    rope, pos = make(T, D, D)
    g = gain(D, torch.float32, 1)
    q, k = rows(T, 8, 2, D, torch.bfloat16, seed=1)
    q, k = q.clone(), k.clone()
    slots = slots_of(T, 128)
    kp, vp = dopr.cache_pools_4bit(layout)
    ws = dopr.head_norm_rope_workspace(D)
    out = [torch.empty(T, 8, D, device=DEV, dtype=torch.bfloat16) for _ in range(2)] + \
          [torch.empty(T, 2, D, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    dg = [torch.empty(D, device=DEV) for _ in range(2)]

    def step(stream=None):
        dopr.cache_append_4bit(layout, slots, k, k, kp, vp, k_gain=g, eps=EPS, rope=rope, positions=pos, q=q, q_gain=g, q_out=out[0],
                               stream=stream)
        dopr.cache_read_4bit(layout, slots, kp, vp, k_out=out[2], v_out=out[3], stream=stream)
        dopr.head_norm_rope_backward(out[0], q, out[2], k, g, g, rope=rope, positions=pos, dq=out[1], dk=out[3], dq_gain=dg[0],
                                     dk_gain=dg[1], workspace=ws, stream=stream)
        return [x.clone() for x in out + dg + [kp, vp]]

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    q.mul_(-0.5), k.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    new = step()
    assert all(torch.equal(a, b) for a, b in zip(captured, new)) and not torch.equal(new[0], want[0])


def test_tensors_that_require_gradients_are_refused():
    q = torch.randn(4, 2, 64, device=DEV, requires_grad=True)
    with pytest.raises(ValueError, match="gradient"):
        dopr.head_norm_rope(q)
    with pytest.raises(ValueError, match="gradient"):
        dopr.head_norm_rope(q.detach(), q_gain=torch.ones(64, device=DEV, requires_grad=True))
    with torch.no_grad():
        dopr.head_norm_rope(q)


def test_wrong_tensors_are_refused():
    q = torch.randn(4, 2, 64, device=DEV)
    for bad in (dict(k=torch.randn(4, 2, 64, device=DEV).half()), dict(k=torch.randn(3, 2, 64, device=DEV)),
                dict(q_gain=torch.ones(63, device=DEV)), dict(q_gain=torch.ones(64, device=DEV), k_gain=torch.ones(64, device=DEV).half()),
                dict(q_gain=torch.ones(64)), dict(positions=torch.zeros(4, device=DEV, dtype=torch.int64))):
        with pytest.raises(ValueError):
            dopr.head_norm_rope(q, **bad)
    layout = dopr.make_cache_layout(2, 16, 2, 64, torch.float16, 1, 2)
    kp, vp = dopr.cache_pools_4bit(layout)
    h, s = q.half(), torch.arange(4, device=DEV)
    for args in ((s.int(), h, h, kp, vp), (s, q, q, kp, vp), (s, h, h, kp.view(-1)[1:], vp), (s, h, h, kp, vp.float())):
        with pytest.raises((ValueError, dopr.DoprError)):
            dopr.cache_append_4bit(layout, *args)
    with pytest.raises(dopr.DoprError):  # 16-byte alignment of the rows
        dopr.cache_append_4bit(layout, s, torch.randn(4 * 2 * 64 + 1, device=DEV).half()[1:].view(4, 2, 64), h, kp, vp)
