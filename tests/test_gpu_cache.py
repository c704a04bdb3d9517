"""The paged prefix cache on a GPU: cache_extend bit for bit against plain loops, rotary positions and stored rows
against 64-bit formulas, shared attention against 64-bit softmax, and a program's steps of them together.

Tolerances.  u = finfo(dtype).eps / 2 is the largest relative error of one rounding.
Rotation: x cos - y sin of 32-bit factors, each product and the sum rounded (2^-24 relative each, a fused product less)
and cos, sin rounded once: below 4 * 2^-24 (|x| + |y|) gain, then one rounding u of the result.
Attention: probabilities rounded to the type (u relative), scores summed in 32 bits: with |q k| summing to at most S
over the head the score is off by at most 128 * 2^-24 S scale, for the inputs here (S scale < 30) below 2^-12, which
moves a probability and their sum by 2^-12 each; exponentials, sums and rescaling by a few 2^-22, which 2^-11 in all
covers.  So |out - exact| <= (u + 2^-11) A + u |exact|, A the softmax average of |v|, and |lse - exact| <= 2^-12 +
2^-22 |exact|."""
import math

import numpy as np
import pytest
import torch

from paper_2609_03311_gb300 import dopr

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def word():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------ extend
class Tables:
    """A cache's rows on the host, by plain loops."""

    def __init__(self, lens, page, max_blocks, n_blocks, seed):
        r = np.random.default_rng(seed)
        self.page, self.n_blocks = page, n_blocks
        self.lens = [int(x) for x in lens]
        order = r.permutation(n_blocks)
        self.tables = r.integers(0, n_blocks, (len(lens), max_blocks)).astype(np.int32)
        at = 0
        for i, n in enumerate(self.lens):
            k = -(-n // page)
            self.tables[i, :k] = order[at:at + k]
            at += k
        self.free = r.integers(0, n_blocks, n_blocks).astype(np.int32)
        self.free[:n_blocks - at] = order[at:]
        self.top = n_blocks - at

    def device(self):
        return i32(self.lens), i32(self.tables), i32(self.free), i32([self.top])

    def extend(self, new, prefix):
        for i, n in enumerate(new):
            if n < 0:
                for p in range(-(-self.lens[i] // self.page)):
                    self.free[self.top] = self.tables[i, p]
                    self.top += 1
                self.lens[i] = 0
        off, slots, where = [0], [], []
        for i, n in enumerate(new):
            for _ in range(max(int(n), 0)):
                if self.lens[i] % self.page == 0:
                    self.top -= 1
                    self.tables[i, self.lens[i] // self.page] = self.free[self.top]
                slots.append(int(self.tables[i, self.lens[i] // self.page]) * self.page + self.lens[i] % self.page)
                where.append((i, self.lens[i]))
                self.lens[i] += 1
            off.append(len(slots))
        pos = [p + (self.lens[prefix[i]] if prefix is not None and prefix[i] >= 0 else 0) for i, p in where]
        return off, slots, pos


def check_extend(t, new, prefix, max_tokens, in_place=False):
    lens, tables, free, n_free = t.device()
    layout = dopr.make_cache_layout(t.n_blocks, t.page, 2, 64, torch.float16, len(t.lens), t.tables.shape[1])
    st, out = word(), dopr.cache_batch(layout, max_tokens)
    if in_place:
        out.seq_lens, out.n_free = lens, n_free
    b = dopr.cache_extend(layout, lens, tables, free, n_free, i32(new), max_tokens, out=out, status=st,
                          prefix=None if prefix is None else i32(prefix))
    off, slots, pos = t.extend(new, prefix)
    rest = [-1] * (max_tokens - len(slots))
    assert st.item() == 0
    assert b.seq_lens.tolist() == t.lens and b.n_free.item() == t.top
    assert b.tok_off.tolist() == off
    assert b.slots.tolist() == slots + rest and b.positions.tolist() == pos + rest
    assert np.array_equal(tables.cpu().numpy(), t.tables) and np.array_equal(free.cpu().numpy(), t.free)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("rows,hi,spare", [(1, 1, 0), (1, 300, 5), (7, 40, 0), (33, 129, 3), (1024, 3, 0), (1025, 9, 7),
                                           (2500, 20, 0)])
def test_extend_equals_plain_loops(page, rows, hi, spare):
    r = np.random.default_rng(rows * page + hi)
    held, new = r.integers(0, 3 * page + 2, rows), r.integers(0, hi + 1, rows)
    mb = -(-(3 * page + 2 + hi) // page)
    t = Tables(held, page, mb, rows * mb + 1, seed=rows)
    check_extend(t, new, None, int(new.sum()) + spare, in_place=rows % 2 == 1)


@pytest.mark.parametrize("rows,hi", [(3, 5), (70, 90), (1500, 10)])
def test_extend_with_prefixes_and_released_rows(rows, hi):
    r = np.random.default_rng(rows)
    docs, page = max(1, rows // 10), 16
    held, new = r.integers(0, 100, rows), r.integers(0, hi + 1, rows)
    new[r.random(rows) < 0.3] = -1
    prefix = np.full(rows, -1)
    prefix[docs:] = r.integers(-1, docs, rows - docs)
    mb = -(-(100 + hi) // page)
    t = Tables(held, page, mb, rows * mb, seed=rows)
    check_extend(t, new, prefix, rows * hi, in_place=True)


def test_extend_takes_the_last_page_and_then_refuses():
    t = Tables([16, 5], 16, 4, 3, seed=1)  # two pages held, one free
    check_extend(t, [1, 11], None, 12)
    lens, tables, free, n_free = t.device()
    layout = dopr.make_cache_layout(3, 16, 2, 64, torch.float16, 2, 4)
    before = [x.clone() for x in (lens, tables, free, n_free)]
    st = word()
    b = dopr.cache_extend(layout, lens, tables, free, n_free, i32([1, 1]), 5, status=st)
    assert st.item() == dopr.ERR_OUT_OF_MEMORY
    assert all(torch.equal(x, y) for x, y in zip((b.seq_lens, tables, free, b.n_free), before))
    assert b.tok_off.tolist() == [0, 0, 0] and b.slots.tolist() == [-1] * 5 and b.positions.tolist() == [-1] * 5


@pytest.mark.parametrize("change", [dict(lens=[-1, 5]), dict(lens=[65, 5]), dict(new=[-2, 1]), dict(new=[60, 1]),
                                    dict(new=[2 ** 31 - 1, 1]), dict(prefix=[0, -1]), dict(prefix=[2, -1]),
                                    dict(prefix=[1, 0]), dict(prefix=[-2, -1]), dict(n_free=[-1]), dict(n_free=[7]),
                                    dict(n_free=[6], new=[-1, 0]), dict(new=[9, 8])])
def test_extend_refuses_bad_device_values_and_leaves_everything(change):
    a = dict(lens=[16, 5], new=[1, 1], prefix=[-1, -1], n_free=[3])
    a.update(change)
    layout = dopr.make_cache_layout(6, 16, 2, 64, torch.float16, 2, 4)
    tables, free = i32([[0, 0, 0, 0], [1, 0, 0, 0]]), i32([2, 3, 4, 5, 0, 0])
    lens, n_free = i32(a["lens"]), i32(a["n_free"])
    before = [x.clone() for x in (lens, tables, free, n_free)]
    st = word()
    b = dopr.cache_extend(layout, lens, tables, free, n_free, i32(a["new"]), 16, prefix=i32(a["prefix"]), status=st)
    assert st.item() == dopr.ERR_INVALID_ARG
    assert all(torch.equal(x, y) for x, y in zip((b.seq_lens, tables, free, b.n_free), before))
    assert b.tok_off.tolist() == [0, 0, 0] and b.slots.tolist() == [-1] * 16
    # an error that stands keeps its place
    st.fill_(dopr.ERR_TIMEOUT)
    dopr.cache_extend(layout, lens, tables, free, n_free, i32(a["new"]), 16, prefix=i32(a["prefix"]), status=st)
    assert st.item() == dopr.ERR_TIMEOUT


@pytest.mark.parametrize("bad", [-1, 6, 2 ** 31 - 1])
def test_extend_gives_no_slot_in_a_page_outside_the_pool(bad):
    layout = dopr.make_cache_layout(6, 16, 2, 64, torch.float16, 2, 4)
    st = word()
    b = dopr.cache_extend(layout, i32([0, 15]), i32([[0] * 4, [bad, 0, 0, 0]]), i32([1, bad, 2, 0, 0, 0]), i32([3]),
                          i32([17, 1]), 20, status=st)
    assert st.item() == dopr.ERR_INVALID_ARG
    assert b.slots.tolist() == [2 * 16 + i for i in range(16)] + [-1] * 4


# ------------------------------------------------------------------ rotary positions
def frequencies(d, theta, scaling, s, original, low, high, att):
    """From include/dopr.h, in 64 bits."""
    i = np.arange(d // 2, dtype=np.float64)
    base = theta * s ** (d / (d - 2)) if scaling == dopr.ROPE_NTK else theta
    f, gain = base ** (-2 * i / d), 1.0
    if scaling == dopr.ROPE_LINEAR:
        f = f / s
    if scaling == dopr.ROPE_BANDS:
        n = original * f / (2 * math.pi)
        f = np.where(n >= high, f, np.where(n <= low, f / s, f / s + (f - f / s) * (n - low) / (high - low)))
    if scaling == dopr.ROPE_RAMP:
        c = lambda n: d * math.log(original / (2 * math.pi * n)) / (2 * math.log(theta))  # noqa: E731
        lo, hi = max(0, math.floor(c(high))), min(d - 1, math.ceil(c(low)))
        r = np.clip((i - lo) / max(hi - lo, 0.001), 0, 1)
        f, gain = f * (1 - r) + f / s * r, att if att > 0 else 0.1 * math.log(s) + 1
    return f, gain


def turned(x, pos, f, gain, rd, interleaved, inverse):
    """64-bit rotation and, for the tolerance, |x| + |y| of each element's pair."""
    y, mag = x.double().clone(), torch.zeros_like(x, dtype=torch.float64)
    a = pos.double()[:, None, None] * torch.from_numpy(f).to(DEV)
    c, s = torch.cos(a) * gain, torch.sin(a) * gain * (-1 if inverse else 1)
    ia = torch.arange(rd // 2, device=DEV) * 2 if interleaved else torch.arange(rd // 2, device=DEV)
    ib = ia + 1 if interleaved else ia + rd // 2
    u, w = x.double()[..., ia], x.double()[..., ib]
    y[..., ia], y[..., ib] = u * c - w * s, w * c + u * s
    mag[..., ia] = mag[..., ib] = (u.abs() + w.abs()) * gain
    return y, mag


def assert_turned(got, x, pos, f, gain, rd, interleaved, inverse):
    want, mag = turned(x, pos, f, gain, rd, interleaved, inverse)
    u = torch.finfo(x.dtype).eps / 2
    tol = 4 * 2.0 ** -24 * mag + (u * want.abs() + u * 4 * 2.0 ** -24 * mag + 2.0 ** -25 if x.dtype != torch.float32 else 0)
    err = (got.double() - want).abs()
    live = pos >= 0
    assert bool((err <= tol)[live].all()), float((err - tol)[live].max())
    assert torch.equal(got[..., rd:][live], x[..., rd:][live])


SCALED = [dict(), dict(scaling=dopr.ROPE_LINEAR, factor=4.0), dict(scaling=dopr.ROPE_NTK, factor=8.0),
          dict(scaling=dopr.ROPE_BANDS, factor=8.0, original_max_position=4096, low=1.0, high=4.0),
          dict(scaling=dopr.ROPE_RAMP, factor=16.0, original_max_position=4096, low=1.0, high=32.0),
          dict(scaling=dopr.ROPE_RAMP, factor=2.0, original_max_position=64, low=1.0, high=2.0, attention_factor=0.8)]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,K,D,rd,inter,inv,far,more", [
    (1, 1, 1, 2, 2, False, False, 10, 0), (1, 32, 8, 128, 128, False, False, 8192, 0),
    (77, 5, 1, 64, 64, True, False, 300000, 1), (300, 16, 8, 128, 64, True, True, 300000, 2),
    (5, 3, 2, 80, 20, False, True, 5000, 3), (64, 4, 4, 128, 32, False, False, 100000, 4),
    (9, 7, 3, 256, 256, True, True, 4000000, 5), (13, 2, 1, 66, 34, False, False, 100, 0),
    (3, 2, 2, 250, 250, True, False, 777, 0)])
def test_rotary_positions(dt, T, H, K, D, rd, inter, inv, far, more):
    g = torch.Generator(DEV).manual_seed(T * D)
    kw = dict(dict(scaling=dopr.ROPE_PLAIN, factor=1.0, original_max_position=0, low=1.0, high=32.0, attention_factor=0.0),
              **SCALED[more])
    f, gain = frequencies(rd, 1e6, kw["scaling"], kw["factor"], kw["original_max_position"], kw["low"], kw["high"],
                          kw["attention_factor"])
    rope = dopr.Rope(far, rd, theta=1e6, layout=int(inter), **kw)
    pos = torch.randint(0, far, (T,), generator=g, device=DEV, dtype=torch.int32)
    pos[0] = far - 1
    packed = torch.randn(T, H + 2 * K, D, generator=g, device=DEV).to(dt)
    q, k = packed[:, :H], packed[:, H:H + K]
    st = word()
    qo, ko = dopr.rope_apply(rope, pos, q, k, inverse=inv, status=st)
    assert_turned(qo, q, pos, f, gain, rd, inter, inv)
    assert_turned(ko, k, pos, f, gain, rd, inter, inv)
    # in place, on a view that is not 16-byte aligned, and q alone: the same bits
    room = torch.zeros(T * (H * D + 1) + 1, dtype=dt, device=DEV)
    odd = room[1:1 + T * (H * D + 1)].view(T, H * D + 1)[:, :H * D].unflatten(1, (H, D))
    odd.copy_(q)
    dopr.rope_apply(rope, pos, odd, q_out=odd, inverse=inv, status=st)
    assert torch.equal(odd, qo) and st.item() == 0


def test_rotary_rows_without_a_position_and_beyond_the_table():
    rope = dopr.Rope(100, 64)
    x = torch.randn(4, 2, 64, device=DEV)
    out = torch.full_like(x, 7.0)
    st = word()
    dopr.rope_apply(rope, i32([3, -1, 100, 99]), x, q_out=out, status=st)
    assert st.item() == dopr.ERR_INVALID_ARG
    assert bool((out[1:3] == 7).all()) and not bool((out[0] == 7).any()) and not bool((out[3] == 7).any())
    dopr.rope_apply(rope, i32([]), x[:0])  # no rows


def test_the_gradient_is_the_inverse_turn():
    # <g, R x> = <R^T g, x>, and differences of a loss along one element
    rope = dopr.Rope(5000, 32, scaling=dopr.ROPE_RAMP, factor=4.0, original_max_position=512, low=1.0, high=16.0)
    g = torch.Generator(DEV).manual_seed(5)
    pos = torch.randint(0, 5000, (31,), generator=g, device=DEV, dtype=torch.int32)
    x, w = (torch.randn(31, 3, 64, generator=g, device=DEV) for _ in range(2))
    y, back = dopr.rope_apply(rope, pos, x)[0], dopr.rope_apply(rope, pos, w, inverse=True)[0]
    lhs, rhs = (w.double() * y.double()).sum(), (back.double() * x.double()).sum()
    size = (w.double() * y.double()).abs().sum()
    assert abs(float(lhs - rhs)) <= 16 * 2.0 ** -24 * float(size)
    for t, h, d in ((0, 0, 0), (30, 2, 17), (7, 1, 63)):
        step = torch.zeros_like(x)
        step[t, h, d] = 1.0  # the turn is linear: a difference of any size
        dy = dopr.rope_apply(rope, pos, x + step)[0].double() - y.double()
        assert abs(float((w.double() * dy).sum()) - float(back[t, h, d])) <= 64 * 2.0 ** -24 * float(w[t, h].abs().sum() + 1) * 8


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,H,K,D,page,rd", [(1, 4, 2, 64, 16, 64), (50, 32, 8, 128, 64, 128), (333, 6, 3, 128, 128, 64),
                                             (70, 5, 1, 64, 32, 20)])
def test_append_stores_turned_keys_and_values(dt, T, H, K, D, page, rd):
    g = torch.Generator(DEV).manual_seed(T)
    blocks = -(-T // page) + 2
    layout = dopr.make_cache_layout(blocks, page, K, D, dt, 1, blocks)
    rope, f = dopr.Rope(4096, rd), frequencies(rd, 1e6, 0, 1, 0, 0, 0, 0)[0]
    pos = torch.randint(0, 4096, (T,), generator=g, device=DEV, dtype=torch.int32)
    slots = torch.randperm(blocks * page, generator=g, device=DEV)[:T]
    if T > 3:
        slots[1], pos[2] = -1, -1  # not stored; not touched at all
    packed = torch.randn(T, H + 2 * K, D, generator=g, device=DEV).to(dt)
    q, k, v = packed[:, :H], packed[:, H:H + K], packed[:, H + K:]
    pools = [torch.randn(blocks, K, page, D, generator=g, device=DEV).to(dt) for _ in range(2)]
    want = [p.clone() for p in pools]
    st, qo = word(), torch.full((T, H, D), 7.0, dtype=dt, device=DEV)
    dopr.cache_append(layout, slots, k, v, *pools, rope=rope, positions=pos, q=q, q_out=qo, status=st)
    assert st.item() == 0
    assert_turned(qo, q, pos, f, 1.0, rd, False, False)
    kt = dopr.rope_apply(rope, pos, k)[0]
    assert_turned(kt, k, pos, f, 1.0, rd, False, False)
    live = (slots >= 0) & (pos >= 0)
    b, at = slots[live] // page, slots[live] % page
    want[0][b, :, at], want[1][b, :, at] = kt[live], v[live]
    assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])
    if T > 3:
        assert bool((qo[2] == 7).all()) and not bool((qo[1] == 7).all())
    # without rotary positions: rows as they are; a slot outside the pool is refused and left out
    plain = [p.clone() for p in want]
    slots[0] = blocks * page
    dopr.cache_append(layout, slots, k, v, *pools, status=st)
    live = (slots >= 0) & (slots < blocks * page)
    b, at = slots[live] // page, slots[live] % page
    plain[0][b, :, at], plain[1][b, :, at] = k[live], v[live]
    assert st.item() == dopr.ERR_INVALID_ARG
    assert torch.equal(pools[0], plain[0]) and torch.equal(pools[1], plain[1])


# ------------------------------------------------------------------ attention
class Batch:
    """Documents (rows without a prefix) and requests in a paged cache, and the 64-bit answer."""

    def __init__(self, hq, hkv, d, dt, page, docs, reqs, seed, dirt=math.nan, own_rows=(), spare=3):
        """docs: their lengths; reqs: (document or -1, own length, new tokens) in row order; own_rows: documents'
        own new tokens {row: n}; dirt fills every page's places past its row's end and all spare pages."""
        g = torch.Generator(DEV).manual_seed(seed)
        self.hq, self.hkv, self.d, self.dt, self.page = hq, hkv, d, dt, page
        self.lens = list(docs) + [r[1] for r in reqs]
        self.prefix = [-1] * len(docs) + [r[0] for r in reqs]
        own_rows = dict(own_rows)
        self.new = [own_rows.get(i, 0) for i in range(len(docs))] + [r[2] for r in reqs]
        n = len(self.lens)
        pages = [-(-x // page) for x in self.lens]
        self.mb, blocks = max(1, max(pages)), sum(pages) + spare
        order = np.random.default_rng(seed).permutation(blocks)
        self.tables = np.full((n, self.mb), -5, dtype=np.int32)  # entries past a row's pages are never read
        shape = (blocks, hkv, page, d)
        self.k = torch.full(shape, dirt, dtype=dt, device=DEV)
        self.v = torch.full(shape, dirt, dtype=dt, device=DEV)
        self.rows, at = [], 0
        for i, x in enumerate(self.lens):
            self.tables[i, :pages[i]] = order[at:at + pages[i]]
            at += pages[i]
            kv = [torch.randn(x, hkv, d, generator=g, device=DEV).to(dt) for _ in range(2)]
            self.rows.append(kv)
            t = torch.arange(x, device=DEV)
            b = torch.from_numpy(self.tables[i]).to(DEV).long()[t // page]
            self.k[b, :, t % page], self.v[b, :, t % page] = kv[0], kv[1]
        self.T = sum(self.new)
        self.q = torch.randn(self.T, hq, d, generator=g, device=DEV).to(dt)
        self.off = np.concatenate([[0], np.cumsum(self.new)])
        self.layout = dopr.make_cache_layout(blocks, page, hkv, d, dt, n, self.mb)

    def args(self, max_tokens=None):
        return (i32(self.off), i32(self.lens), i32(self.prefix), max_tokens or self.T)

    def run(self, pad=0, **kw):
        st = word()
        q = torch.cat([self.q, torch.full((pad, self.hq, self.d), math.nan, dtype=self.dt, device=DEV)]) if pad else self.q
        T = self.T + pad
        plan = dopr.shared_attention_plan(self.layout, self.hq, i32(self.off), i32(self.lens), i32(self.prefix), T, status=st)
        out = torch.full((T, self.hq, self.d), 7.0, dtype=self.dt, device=DEV)
        lse = torch.full((T, self.hq), 7.0, device=DEV)
        dopr.shared_attention(self.layout, plan, q, self.k, self.v, i32(self.tables), out=out, lse=lse, status=st, **kw)
        assert st.item() == 0
        assert bool((out[self.T:] == 7).all()) and bool((lse[self.T:] == 7).all())
        return out[:self.T], lse[:self.T]

    def exact(self, scale=None):
        """(out, lse, softmax average of |v|) in 64 bits."""
        scale = self.d ** -0.5 if scale is None else scale
        out, avg = (torch.zeros(self.T, self.hq, self.d, dtype=torch.float64, device=DEV) for _ in range(2))
        lse = torch.full((self.T, self.hq), -math.inf, dtype=torch.float64, device=DEV)
        G = self.hq // self.hkv
        for i, n in enumerate(self.new):
            if n == 0:
                continue
            p = self.prefix[i]
            k, v = (torch.cat([self.rows[p][j], self.rows[i][j]] if p >= 0 else [self.rows[i][j]]).double() for j in (0, 1))
            m = self.lens[p] if p >= 0 else 0
            seen = m + torch.clamp(self.lens[i] - n + torch.arange(n, device=DEV) + 1, min=0)
            q = self.q[self.off[i]:self.off[i + 1]].double()
            a = torch.einsum("thd,khd->thk", q, k.repeat_interleave(G, 1)) * scale
            a = a.masked_fill((torch.arange(k.shape[0], device=DEV) >= seen[:, None])[:, None], -math.inf)
            s = slice(self.off[i], self.off[i + 1])
            if k.shape[0] == 0:
                continue
            lse[s] = torch.logsumexp(a, -1)
            w = torch.nan_to_num(torch.softmax(a, -1), nan=0.0)
            out[s] = torch.einsum("thk,khd->thd", w, v.repeat_interleave(G, 1))
            avg[s] = torch.einsum("thk,khd->thd", w, v.abs().repeat_interleave(G, 1))
        return out, lse, avg

    def check(self, got, scale=None):
        out, lse, avg = self.exact(scale)
        u = torch.finfo(self.dt).eps / 2
        err, tol = (got[0].double() - out).abs(), (u + 2.0 ** -11) * avg + u * out.abs() + 2.0 ** -24
        assert bool((err <= tol).all()), (float((err / tol).max()), int((~(err <= tol)).sum()))
        empty = lse == -math.inf
        assert torch.equal(got[1] == -math.inf, empty) and bool((got[0][empty] == 0).all())
        e2 = (got[1].double() - lse).abs()[~empty]
        assert bool((e2 <= 2.0 ** -12 + 2.0 ** -22 * lse.abs()[~empty]).all()), float(e2.max()) if e2.numel() else 0


BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attention_of_queries_on_one_document(page, d, dt):
    Batch(8, 2, d, dt, page, [300], [(0, 24, 1), (0, 1, 1), (0, 64, 1)], seed=page + d).check(
        Batch(8, 2, d, dt, page, [300], [(0, 24, 1), (0, 1, 1), (0, 64, 1)], seed=page + d).run())


@pytest.mark.parametrize("m", [0, 1, 15, 16, 17, 127, 128, 129, 255, 256, 257, 1000, 5000])
@pytest.mark.parametrize("own,new", [(0, 1), (1, 1), (5, 5), (130, 3), (129, 129)])
def test_attention_lengths(m, own, new):
    b = Batch(4, 1, 128, BF, 32, [m], [(0, own, new)], seed=m + own)
    b.check(b.run())


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (5, 1), (6, 2), (7, 1), (8, 8), (16, 1), (33, 1), (40, 8), (64, 1),
                                    (128, 2)])
def test_attention_head_counts(hq, hkv):
    b = Batch(hq, hkv, 64, HF, 16, [200, 77], [(0, 30, 2), (1, 50, 9), (0, 3, 3), (1, 1, 1)], seed=hq)
    b.check(b.run())


@pytest.mark.parametrize("dt,d", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("seed", range(6))
def test_attention_of_ragged_batches_in_any_order(seed, dt, d):
    r = np.random.default_rng(seed)
    docs = [int(x) for x in r.integers(0, [40, 700, 3000][seed % 3], 5)]
    reqs = []
    for _ in range(int(r.integers(1, 60))):
        own = int(r.integers(0, 150))
        reqs.append((int(r.integers(-1, 5)), own, int(r.integers(0, own + 2)) if seed % 2 else 1))
    if sum(x[2] for x in reqs) == 0:
        reqs.append((0, 1, 1))
    b = Batch(8, 2, d, dt, [16, 64, 128][seed % 3], docs, reqs, seed, dirt=[math.nan, math.inf, 6e4][seed % 3],
              own_rows={1: min(docs[1], 70)})
    b.check(b.run(pad=seed * 3))


def test_attention_rows_that_see_nothing():
    # more new tokens than own keys, an empty prefix, no prefix: the first rows see no key
    b = Batch(4, 2, 128, BF, 16, [0, 33], [(0, 2, 5), (-1, 0, 3), (1, 0, 2), (-1, 1, 4)], seed=3)
    got = b.run()
    b.check(got)
    assert int((got[1] == -math.inf).sum()) == (3 + 3 + 3) * 4


@pytest.mark.parametrize("n,new,m", [(40, 32, 900), (3, 600, 513), (1, 2000, 100), (70, 64, 40)])
def test_attention_of_many_rows(n, new, m):
    b = Batch(8, 2, 128, BF, 64, [m, 1], [(0, new + (i % 3), new) for i in range(n)], seed=n)
    b.check(b.run())


@pytest.mark.parametrize("m", [40000, 131072])
def test_attention_of_a_long_document(m):
    b = Batch(4, 1, 128, BF, 128, [m], [(0, 9, 1), (0, 100, 1)], seed=1)
    b.check(b.run())


def test_attention_with_large_scores_and_one_heavy_key():
    # scores in the hundreds: the running maximum grows by more than any fixed step, and late
    b = Batch(4, 1, 128, BF, 64, [1500], [(0, 70, 3)], seed=8)
    for at, by in ((3, 4.0), (700, 9.0), (1499, 30.0)):
        b.rows[0][0][at] = (b.q[0, 0] * by).to(BF)
        blk = int(b.tables[0, at // 64])
        b.k[blk, :, at % 64] = b.rows[0][0][at]
    out, lse, avg = b.exact()
    got = b.run()
    # scores reach 30 |q|^2 / sqrt(128) ~ 340: off by up to 128 * 2^-24 * 340 = 2.6e-3, in place of 2^-12
    u = torch.finfo(BF).eps / 2
    assert bool(((got[0].double() - out).abs() <= (u + 8e-3) * avg + u * out.abs() + 2.0 ** -24).all())
    assert bool(((got[1].double() - lse).abs() <= 3e-3).all())


def test_attention_of_infinite_and_nan_inputs_stays_in_its_rows():
    b = Batch(4, 2, 128, BF, 16, [100], [(0, 20, 1), (0, 30, 1), (-1, 40, 1)], seed=2)
    clean = b.run()
    b.q[1] = math.nan
    got = b.run()
    assert bool(torch.isnan(got[0][1]).all())
    for t in (0, 2):
        assert torch.equal(got[0][t], clean[0][t]) and torch.equal(got[1][t], clean[1][t])
    # a visible key of minus infinity on one side gives scores of minus infinity or NaN; a NaN value reaches its rows
    b.q[1] = 1.0
    at = 99
    b.v[int(b.tables[0, at // 16]), 0, at % 16] = math.nan
    got = b.run()
    assert bool(torch.isnan(got[0][:2, :2]).all()) and not bool(torch.isnan(got[0][:, 2:]).any())
    assert not bool(torch.isnan(got[0][2]).any())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_rows_are_not_touched_by_values_that_only_others_see(bad, d):
    # the last own value of one row is bad: its last token alone sees it, not its others, nor rows beside it
    b = Batch(4, 2, d, BF, 16, [50], [(0, 20, 5), (0, 30, 2), (0, 9, 9)], seed=6)
    want = b.run()
    b.check(want)
    at = 19
    b.v[int(b.tables[1, at // 16]), 1, at % 16] = bad
    got = b.run()
    other = torch.ones(b.T, dtype=torch.bool, device=DEV)
    other[4] = False
    u = torch.finfo(BF).eps / 2
    # the rows beside are computed alone, in another order and without rounded probabilities
    assert bool(((got[0] - want[0]).double().abs()[other] <= (3 * u + 2.0 ** -10) * b.exact()[2][other] + 2.0 ** -24).all())
    assert torch.equal(got[0][4, :2], want[0][4, :2]) and not bool(torch.isfinite(got[0][4, 2:]).any())
    assert bool(((got[1] - want[1]).abs() <= 2.0 ** -11).all())


def test_attention_refuses_a_plan_of_other_sizes():
    b = Batch(4, 2, 64, HF, 16, [20], [(0, 5, 2), (0, 6, 1)], seed=1)
    plan = dopr.shared_attention_plan(b.layout, b.hq, *b.args())
    room = torch.zeros(plan.numel() * 4, dtype=torch.uint8, device=DEV)
    room[:plan.numel()] = plan
    st, q = word(), torch.cat([b.q, b.q])
    out = torch.full_like(q, 7.0)
    dopr.shared_attention(b.layout, room, q, b.k, b.v, i32(b.tables), out=out, status=st)
    assert st.item() == dopr.ERR_INVALID_ARG and bool((out == 7).all())


def test_attention_scale_and_strided_views():
    b = Batch(8, 2, 64, HF, 32, [400], [(0, 20, 7), (0, 9, 9)], seed=4)
    want = b.run(scale=0.31)
    b.check(want, scale=0.31)
    plan = dopr.shared_attention_plan(b.layout, b.hq, *b.args())
    wide = torch.randn(b.T, 12, 80, dtype=torch.float32, device=DEV).to(HF)
    q = wide[:, 2:10, 8:72]
    q.copy_(b.q)
    out = torch.zeros(b.hq, b.T, 72, dtype=HF, device=DEV).transpose(0, 1)[:, :, :64]
    dopr.shared_attention(b.layout, plan, q, b.k, b.v, i32(b.tables), scale=0.31, out=out)
    assert torch.equal(out, want[0])


def test_attention_of_one_query_for_all_tokens():
    # a broadcast view: the same row for every token
    b = Batch(8, 2, 64, HF, 32, [400], [(0, 20, 7), (0, 9, 9)], seed=4)
    b.q = b.q[:1].expand(b.T, -1, -1)
    b.check(b.run())


def test_attention_plan_refuses_bad_device_values_and_attention_then_writes_nothing():
    b = Batch(4, 2, 64, HF, 16, [20], [(0, 5, 2), (0, 6, 1)], seed=1)
    for off, lens, prefix in (([0, 0, 2, 1], b.lens, b.prefix), ([1, 1, 2, 3], b.lens, b.prefix),
                              ([0, 0, 2, 4], b.lens, b.prefix), (b.off, [20, -1, 6], b.prefix),
                              (b.off, [20, 16 * b.mb + 1, 6], b.prefix), (b.off, b.lens, [-1, 3, 0]),
                              (b.off, b.lens, [-1, 1, 0]), (b.off, b.lens, [-1, 0, 1]), (b.off, b.lens, [-1, -2, 0])):
        st = word()
        plan = dopr.shared_attention_plan(b.layout, b.hq, i32(off), i32(lens), i32(prefix), b.T, status=st)
        assert st.item() == dopr.ERR_INVALID_ARG
        out = torch.full_like(b.q, 7.0)
        dopr.shared_attention(b.layout, plan, b.q, b.k, b.v, i32(b.tables), out=out)
        assert bool((out == 7).all())


def test_attention_reads_page_zero_for_a_page_outside_the_pool_and_says_so():
    b = Batch(4, 2, 64, HF, 16, [40], [(0, 5, 2), (-1, 6, 1)], seed=1, dirt=0.0)
    st = word()
    plan = dopr.shared_attention_plan(b.layout, b.hq, *b.args())
    for bad in (-1, b.layout.n_blocks, 2 ** 31 - 1):
        tables = b.tables.copy()
        tables[0, 1] = bad
        st.zero_()
        out = dopr.shared_attention(b.layout, plan, b.q, b.k, b.v, i32(tables), status=st)
        assert st.item() == dopr.ERR_INVALID_ARG
        tables[0, 1] = 0
        st.zero_()
        assert torch.equal(out, dopr.shared_attention(b.layout, plan, b.q, b.k, b.v, i32(tables), status=st))
        assert st.item() == 0


def test_attention_on_other_streams_and_twice_at_once():
    bs = [Batch(8, 2, 128, BF, 64, [3000], [(0, 50, 1)] * 20, seed=s) for s in (1, 2)]
    want = [b.run() for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for b, s in zip(bs, streams):
            plan = dopr.shared_attention_plan(b.layout, b.hq, *b.args(), stream=s)
            got.append((b, dopr.shared_attention(b.layout, plan, b.q, b.k, b.v, i32(b.tables), stream=s)))
            s.synchronize()
    torch.cuda.synchronize()
    for b, out in got:
        assert torch.equal(out, want[bs.index(b)][0])


# ------------------------------------------------------------------ together
class Program:
    """A two-layer cache as a user's program keeps it: documents stored once, then requests token by token."""

    def __init__(self, dt=BF, hq=8, hkv=2, d=128, page=16, docs=(200, 35), reqs=5, cap=40):
        self.n, self.docs, self.hq, self.hkv, self.d, self.dt = len(docs) + reqs, len(docs), hq, hkv, d, dt
        mb = -(-max(max(docs), cap) // page)
        blocks = sum(-(-x // page) for x in docs) + reqs * -(-cap // page)
        self.layout = dopr.make_cache_layout(blocks, page, hkv, d, dt, self.n, mb)
        self.pools = [[torch.full((blocks, hkv, page, d), math.nan, dtype=dt, device=DEV) for _ in range(2)] for _ in range(2)]
        self.seq_lens, self.n_free = i32([0] * self.n), i32([blocks])
        self.tables, self.free = i32(np.full((self.n, mb), -1)), i32(np.arange(blocks))
        self.prefix = i32([-1] * self.docs + [i % self.docs for i in range(reqs)])
        self.rope, self.status = dopr.Rope(1024, d), word()
        self.keys = [[[] for _ in range(self.n)] for _ in range(2)]  # host record, by layer and row, in 64 bits

    def batch(self, max_tokens):
        out = dopr.cache_batch(self.layout, max_tokens)
        out.seq_lens, out.n_free = self.seq_lens, self.n_free
        return out

    def step(self, out, new, qkv, outs):
        """All calls of one step; qkv[layer] [max_tokens, hq + 2 hkv, d]."""
        T = out.max_tokens
        dopr.cache_extend(self.layout, self.seq_lens, self.tables, self.free, self.n_free, new, T, prefix=self.prefix, out=out,
                          status=self.status)
        plan = dopr.shared_attention_plan(self.layout, self.hq, out.tok_off, self.seq_lens, self.prefix, T, status=self.status)
        for l in range(2):
            q, k, v = qkv[l][:, :self.hq], qkv[l][:, self.hq:self.hq + self.hkv], qkv[l][:, self.hq + self.hkv:]
            qr = dopr.cache_append(self.layout, out.slots, k, v, *self.pools[l], rope=self.rope, positions=out.positions, q=q,
                                   status=self.status)
            dopr.shared_attention(self.layout, plan, qr, *self.pools[l], self.tables, out=outs[l], status=self.status)

    def expect(self, new, lens, qkv, l):
        """The step's outputs of layer l in 64 bits from the record, with roundings of turned rows to the type."""
        f = frequencies(self.d, 1e6, 0, 1, 0, 0, 0, 0)[0]
        pre = self.prefix.tolist()
        out, avg, at = [], [], 0
        after = [a + b for a, b in zip(lens, new)]
        rows = []
        for i, n in enumerate(new):
            x = qkv[l][at:at + n]
            base = after[pre[i]] if pre[i] >= 0 else 0
            pos = torch.arange(base + lens[i], base + after[i], device=DEV)
            turn = lambda z: turned(z, pos, f, 1.0, self.d, False, False)[0].to(self.dt).double()  # noqa: E731
            k, v = turn(x[:, self.hq:self.hq + self.hkv]), x[:, self.hq + self.hkv:].double()
            self.keys[l][i].append((k, v))
            rows.append(turn(x[:, :self.hq]))
            at += n
        cat = lambda i, j: torch.cat([p[j] for p in self.keys[l][i]] + [torch.zeros(0, self.hkv, self.d, dtype=torch.float64, device=DEV)])  # noqa: E731,E501
        G = self.hq // self.hkv
        for i, n in enumerate(new):
            if n == 0:
                continue
            ks, vs = ([cat(pre[i], j)] if pre[i] >= 0 else [] for j in (0, 1))
            k, v = torch.cat(ks + [cat(i, 0)]), torch.cat(vs + [cat(i, 1)])
            seen = k.shape[0] - n + 1 + torch.arange(n, device=DEV)
            a = torch.einsum("thd,khd->thk", rows[i], k.repeat_interleave(G, 1)) * self.d ** -0.5
            a = a.masked_fill((torch.arange(k.shape[0], device=DEV) >= seen[:, None])[:, None], -math.inf).softmax(-1)
            out.append(torch.einsum("thk,khd->thd", a, v.repeat_interleave(G, 1)))
            avg.append(torch.einsum("thk,khd->thd", a, v.abs().repeat_interleave(G, 1)))
        return torch.cat(out), torch.cat(avg)

    def rows_of(self, seed, T):
        g = torch.Generator(DEV).manual_seed(seed)
        return [torch.randn(T, self.hq + 2 * self.hkv, self.d, generator=g, device=DEV).to(self.dt) for _ in range(2)]

    def check(self, outs, new, lens, qkv):
        # a turned q or k that rounds the other way than the 64-bit one's moves scores like another rounding u of one
        # operand element: covered by a second u in the average's factor
        u = torch.finfo(self.dt).eps / 2
        T = sum(new)
        for l in range(2):
            want, avg = self.expect(new, lens, qkv, l)
            err = (outs[l][:T].double() - want).abs()
            assert bool((err <= (2 * u + 2.0 ** -11) * avg + u * want.abs() + 2.0 ** -24).all()), float(err.max())


def test_a_program_stores_documents_and_answers_token_by_token():
    p = Program()
    lens = [0] * p.n
    steps = [[200, 35] + [0] * 5, [0, 0, 7, 3, 1, 12, 0], [0, 0, 1, 1, 1, 1, 5], [0, 0, 1, 0, 1, 1, 1], [0, 0] + [1] * 5,
             [0, 0] + [20] * 5]
    for n, new in enumerate(steps):
        T = sum(new) + n  # a few rows behind the last token
        qkv = p.rows_of(n, T)
        outs = [torch.full((T, p.hq, p.d), 7.0, dtype=p.dt, device=DEV) for _ in range(2)]
        p.step(p.batch(T), i32(new), qkv, outs)
        assert p.status.item() == 0
        p.check(outs, new, lens, qkv)
        assert all(bool((o[sum(new):] == 7).all()) for o in outs)
        lens = [a + b for a, b in zip(lens, new)]
        assert p.seq_lens.tolist() == lens


def test_a_captured_step_is_replayed_as_the_sequences_grow():
    p = Program()
    lens = [0] * p.n
    new = [200, 35] + [4] * 5
    qkv = p.rows_of(99, sum(new))
    outs = [torch.zeros(sum(new), p.hq, p.d, dtype=p.dt, device=DEV) for _ in range(2)]
    p.step(p.batch(sum(new)), i32(new), qkv, outs)
    p.check(outs, new, lens, qkv)
    lens = list(new)
    # one graph for a token of each request and a row that is free: what changes lies on the device
    T = 6
    b, add = p.batch(T), i32([0, 0, 1, 1, 1, 1, 1])
    outs, qkv = [torch.zeros(T, p.hq, p.d, dtype=p.dt, device=DEV) for _ in range(2)], p.rows_of(0, T)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        p.step(b, add, qkv, outs)
    for n in range(20):
        new = [0, 0] + [int(x) for x in np.random.default_rng(n).integers(0, 2, 5)]
        if sum(new) == 0:
            new[2] = 1
        add.copy_(i32(new))
        for x, y in zip(qkv, p.rows_of(n, T)):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert p.status.item() == 0
        p.check(outs, new, lens, qkv)
        lens = [a + c for a, c in zip(lens, new)]
        assert p.seq_lens.tolist() == lens


# ------------------------------------------------------------------ more rows and tokens than a plan holds close by
@pytest.mark.parametrize("n,docs,busy,in_order", [(1500, 40, 1500, False), (1500, 1400, 1500, True), (5000, 9, 5000, False),
                                                  (16000, 384, 700, False)])
def test_attention_of_thousands_of_rows(n, docs, busy, in_order):
    # rows in any order of their prefixes (or in it), most of them with one token; beyond 1,024 rows the lists are made in
    # parts, beyond some 3,000 they no longer lie in shared memory
    r = np.random.default_rng(n + docs)
    of = r.integers(-1, docs, n)
    of = np.sort(of) if in_order else of
    live = np.zeros(n, dtype=bool)
    live[r.permutation(n)[:busy]] = True
    reqs = [(int(p), int(x), int(t)) for p, x, t in zip(of, np.where(live, r.integers(0, 4, n), 0),
                                                        np.where(live, r.choice([0, 1, 1, 1, 2], n), 0))]
    b = Batch(2, 1, 64, BF, 16, [int(x) for x in r.integers(0, 20, docs)], reqs, seed=n)
    b.check(b.run())


def test_attention_of_more_tokens_than_items_in_shared_memory():
    r = np.random.default_rng(3)
    reqs = [(int(r.integers(-1, 2)), 70, int(t)) for t in r.integers(60, 71, 300)]
    b = Batch(4, 1, 64, HF, 32, [40, 0], reqs, seed=4)
    b.check(b.run())


@pytest.mark.parametrize("rows,hi", [(16384, 1), (16384, 2), (129, 4), (128, 4), (100, 3)])
def test_extend_of_many_and_few_rows(rows, hi):
    # both counts of threads, and offsets found in two steps over all rows
    r = np.random.default_rng(rows + hi)
    held, new = r.integers(0, 20, rows), r.integers(0, hi + 1, rows)
    new[r.random(rows) < 0.4] = -1
    mb = -(-(20 + hi) // 16)
    t = Tables(held, 16, mb, rows * mb, seed=rows)
    check_extend(t, new, None, int(np.maximum(new, 0).sum()) + hi)


def test_extend_refuses_a_batch_of_another_layout():
    # a step's buffers made for 3 rows, every tensor but the workspace replaced by one that 40 rows fit
    t = Tables([5] * 40, 16, 2, 90, seed=1)
    small = dopr.make_cache_layout(90, 16, 2, 64, torch.float16, 3, 2)
    layout = dopr.make_cache_layout(90, 16, 2, 64, torch.float16, 40, 2)
    out, whole = dopr.cache_batch(small, 40), dopr.cache_batch(layout, 40)
    lens, tables, free, n_free = t.device()
    for name in ("tok_off", "seq_lens", "slots", "positions", "n_free"):
        setattr(out, name, getattr(whole, name))
    with pytest.raises(ValueError, match="workspace"):
        dopr.cache_extend(layout, lens, tables, free, n_free, i32([1] * 40), 40, out=out)
    dopr.cache_extend(layout, lens, tables, free, n_free, i32([1] * 40), 40, out=whole)
    assert whole.seq_lens.tolist() == [6] * 40


@pytest.mark.parametrize("m", [0, 100, 128, 129, 256, 300, 1000, 4100])
@pytest.mark.parametrize("d,page,own,new", [(128, 64, 90, 20), (64, 16, 300, 9), (128, 32, 5, 5)])
def test_attention_of_one_tile_with_blocks_in_turn(d, page, own, new, m):
    # 17 to 128 rows a kv head: two groups take the blocks in turn, and one adds up both; of one block, of rows that see the
    # keys of one group alone, behind another document's tile and before a tile of its own
    b = Batch(8, 2, d, BF, page, [m, 150], [(0, own, new), (1, 40, 25), (0, 3, 6), (-1, 70, 30)], seed=m + d, dirt=math.inf)
    b.check(b.run())


# ------------------------------------------------------------------ calls that the documentation speaks of
@pytest.mark.parametrize("change", [dict(n_blocks=11), dict(n_blocks=20), dict(page=32), dict(n_kv_heads=1), dict(n_kv_heads=4),
                                    dict(head_dim=128), dict(dtype=BF), dict(n_seqs=2), dict(n_seqs=4), dict(max_blocks=1),
                                    dict(max_blocks=6), dict(max_blocks=8), dict(hq=8), dict()])
def test_attention_refuses_a_plan_of_another_layout(change):
    # every field by itself; tables, pools and the plan's room are large enough for any of them
    b = Batch(4, 2, 64, HF, 16, [100], [(0, 5, 2), (0, 6, 1)], seed=1)
    a = dict(n_blocks=b.layout.n_blocks, page=16, n_kv_heads=2, head_dim=64, dtype=HF, n_seqs=3, max_blocks=b.mb, hq=4)
    assert (a["n_blocks"], a["max_blocks"]) == (12, 7)
    plan = dopr.shared_attention_plan(b.layout, b.hq, *b.args())
    a.update(change)
    hq = a.pop("hq")
    layout = dopr.make_cache_layout(**a)
    room = torch.zeros(plan.numel() * 8, dtype=torch.uint8, device=DEV)
    room[:plan.numel()] = plan
    pool = torch.zeros(2 * b.k.numel() * 8, dtype=a["dtype"], device=DEV)
    q = torch.ones(b.T, hq, a["head_dim"], dtype=a["dtype"], device=DEV)
    st, out, lse = word(), torch.full_like(q, 7.0), torch.full((b.T, hq), 7.0, device=DEV)
    dopr.shared_attention(layout, room, q, pool, pool, i32(np.zeros(64)), out=out, lse=lse, status=st)
    if change:
        assert st.item() == dopr.ERR_INVALID_ARG and bool((out == 7).all()) and bool((lse == 7).all())
    else:
        assert st.item() == 0 and bool((out == 0).all())


def test_rotary_positions_of_the_largest_number_of_tokens():
    # 2^31 - 1 rows of one pair: the kernel's step behind the last of them passes 31 bits
    T = 2 ** 31 - 1
    rope = dopr.Rope(4, 2)
    x = torch.empty(T, 1, 2, dtype=HF, device=DEV).normal_()
    pos = torch.zeros(T, dtype=torch.int32, device=DEV)
    ends = torch.cat([torch.arange(100, device=DEV), torch.arange(T - 70000, T, device=DEV)])
    pos[ends] = 3
    out, st = torch.full_like(x, 7.0), word()
    dopr.rope_apply(rope, pos, x, q_out=out, status=st)
    assert st.item() == 0
    assert_turned(out[ends], x[ends], pos[ends], *frequencies(2, 1e6, 0, 1, 0, 0, 0, 0), 2, False, False)
    out[ends] = x[ends]  # the rows between are at position 0, which turns nothing
    assert all(torch.equal(out[i:i + 2 ** 28], x[i:i + 2 ** 28]) for i in range(0, T, 2 ** 28))
    del x, out
    with pytest.raises(ValueError, match="at most"):
        wide = torch.zeros(1, dtype=HF, device=DEV).expand(2 ** 31, 1, 2)
        dopr.rope_apply(rope, torch.zeros(2 ** 31, dtype=torch.int32, device=DEV), wide, q_out=wide)


def test_extend_by_the_largest_number_of_tokens():
    # one row takes every page of the largest pool; the step's extent is the largest, 127 places longer
    n = 2 ** 24 - 1
    layout = dopr.make_cache_layout(n, 128, 1, 64, HF, 2, n)
    free = torch.arange(n, dtype=torch.int32, device=DEV)
    tables = torch.zeros(2, n, dtype=torch.int32, device=DEV)
    st, T = word(), 2 ** 31 - 1
    b = dopr.cache_extend(layout, i32([0, 0]), tables, free, i32([n]), i32([0, n * 128]), T, status=st)
    assert st.item() == 0 and b.tok_off.tolist() == [0, 0, n * 128] and b.seq_lens.tolist() == [0, n * 128]
    assert b.n_free.item() == 0 and torch.equal(tables[1], free.flip(0))
    for i in range(0, n * 128, 2 ** 28):
        t = torch.arange(i, min(i + 2 ** 28, n * 128), device=DEV)
        assert torch.equal(b.slots[i:i + t.numel()], (n - 1 - t // 128) * 128 + t % 128)
        assert torch.equal(b.positions[i:i + t.numel()], t.int())
    assert b.slots[n * 128:].tolist() == [-1] * 127 and b.positions[n * 128:].tolist() == [-1] * 127
    with pytest.raises(ValueError, match="at most"):
        dopr.cache_extend(layout, i32([0, 0]), tables, free, i32([n]), i32([0, 1]), 2 ** 32 + 4, out=b)


def refused_by_the_plan(layout, hq, off, lens, prefix, tables):
    T = int(off[-1])
    st = word()
    plan = dopr.shared_attention_plan(layout, hq, i32(off), i32(lens), i32(prefix), T, status=st)
    assert st.item() == dopr.ERR_UNSUPPORTED
    pool = torch.zeros(layout.n_blocks, layout.n_kv_heads, layout.page, layout.head_dim, dtype=HF, device=DEV)
    q, st = torch.ones(T, hq, layout.head_dim, dtype=HF, device=DEV), word()
    out, lse = torch.full_like(q, 7.0), torch.full((T, hq), 7.0, device=DEV)
    dopr.shared_attention(layout, plan, q, pool, pool, tables, out=out, lse=lse, status=st)
    assert st.item() == 0 and bool((out == 7).all()) and bool((lse == 7).all())


@pytest.mark.parametrize("tokens", [1, 40])
def test_plan_refuses_more_work_than_it_counts(tokens):
    # 2^30 keys for each of 16 kv heads: 2^30 units for a single row a head, 48 * 2^24 for forty
    layout = dopr.make_cache_layout(1, 128, 16, 64, HF, 2, 2 ** 23)
    refused_by_the_plan(layout, 16, [0, 0, tokens], [2 ** 30, 0], [-1, 0], torch.zeros(2, 2 ** 23, dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("tokens", [1, 40])
def test_plan_refuses_keys_that_31_bits_do_not_count(tokens):
    # tables may name a page more than once: a prefix of 2^30 keys and as many own ones, by pieces of 16 and by tiles
    layout = dopr.make_cache_layout(1, 128, 1, 64, HF, 3, 2 ** 23)
    refused_by_the_plan(layout, 1, [0, 0, tokens, tokens], [2 ** 30, 2 ** 30, 0], [-1, 0, -1],
                        torch.zeros(3, 2 ** 23, dtype=torch.int32, device=DEV))
    # rows of a tile whose own keys alone are too many
    if tokens > 1:
        refused_by_the_plan(layout, 1, [0, tokens, 2 * tokens, 3 * tokens], [2 ** 30, 2 ** 30, 2 ** 30], [-1] * 3,
                            torch.zeros(3, 2 ** 23, dtype=torch.int32, device=DEV))
    # a page less is planned
    st = word()
    dopr.shared_attention_plan(layout, 1, i32([0, 0, tokens, tokens]), i32([2 ** 30, 2 ** 30 - 256, 0]), i32([-1, 0, -1]), tokens,
                               status=st)
    assert st.item() == 0


MIXED = {  # documents and requests whose rows share items in every way: (hq, docs, reqs)
    "one tile": (4, [20 + 3 * i for i in range(40)], [(i % 40, 20 - i % 7, 9) for i in range(80)]),
    "two tiles": (8, [20 + 5 * i for i in range(30)], [(i % 30, 30 - i % 4, 20) for i in range(60)]),
    "few rows": (4, [5 + 11 * i for i in range(30)], [(i % 30, 3 + i % 40, 1 + i % 2) for i in range(60)]),
    "own keys beside tiles": (4, [3000], [(0, 5 + i, 1) for i in range(50)]),
    "few rows, cut": (4, [9000, 700], [(0, 30, 1), (0, 17, 2), (1, 40, 1), (1, 33, 1)]),
    "cut": (8, [20000], [(0, 9 + i, 9) for i in range(3)]),
    "no prefix": (8, [10], [(-1, 50 + i, 1 + 13 * (i % 3)) for i in range(20)]),
}


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", list(MIXED))
def test_attention_of_values_that_other_rows_of_an_item_see(kind, d, bad):
    # one element of the last own value of every third request is bad: its last token sees it, nobody else
    hq, docs, reqs = MIXED[kind]
    b = Batch(hq, 2, d, BF, 16, docs, reqs, seed=len(reqs) + d)
    want = b.run()
    b.check(want)
    sees = torch.zeros(b.T, dtype=torch.bool, device=DEV)
    for i in range(len(docs), len(b.lens), 3):
        at = b.lens[i] - 1
        b.v[int(b.tables[i, at // 16]), 1, at % 16, 5] = bad
        sees[b.off[i + 1] - 1] = True
    got = b.run()
    G = hq // 2
    same = torch.ones_like(want[0], dtype=torch.bool)
    same[:, G:, 5] = False
    assert torch.equal(got[0][same], want[0][same]) and torch.equal(got[1], want[1])
    mine = got[0][:, G:, 5]
    assert not bool(torch.isfinite(mine[sees]).any())
    if not math.isnan(bad):
        assert bool((mine[sees] == bad).all())
    out, _, avg = (x[:, G:, 5] if x.dim() == 3 else x for x in b.exact())
    u = torch.finfo(BF).eps / 2
    err, tol = (mine.double() - out).abs(), (u + 2.0 ** -11) * avg + u * out.abs() + 2.0 ** -24
    assert bool((err <= tol)[~sees].all()), float((err / tol)[~sees].max())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_attention_of_a_bad_value_in_a_long_document(bad):
    # every row sees it: the results hold it at once, in its element alone, and nothing runs into a limit
    b = Batch(32, 8, 128, BF, 64, [131072, 200], [(0, 20 + i, 4) for i in range(64)] + [(1, 9, 9), (1, 30, 1)], seed=5)
    want = b.run()
    b.v[int(b.tables[0, 700 // 64]), 1, 700 % 64, 5] = bad
    got = b.run()
    T = 64 * 4
    assert bool(torch.isnan(got[0][:T, 4:8, 5]).all() if math.isnan(bad) else (got[0][:T, 4:8, 5] == bad).all())
    same = torch.ones_like(want[0], dtype=torch.bool)
    same[:T, 4:8, 5] = False
    assert torch.equal(got[0][same], want[0][same]) and torch.equal(got[1], want[1])
    # no longer than a few times what it takes without (a walk over the document by a warp a row takes hundreds of times that)
    plan, tables = dopr.shared_attention_plan(b.layout, b.hq, *b.args()), i32(b.tables)
    ws = dopr.shared_attention_workspace(b.layout, b.hq, b.T)
    a, z = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    dopr.shared_attention(b.layout, plan, b.q, b.k, b.v, tables, workspace=ws)
    z.record()
    z.synchronize()
    assert a.elapsed_time(z) < 20


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tokens", [1, 3, 40, 200])
@pytest.mark.parametrize("m", [1000, 131072])
def test_attention_of_one_heavy_key_among_many_light_ones(m, tokens, d, dt):
    # one key has 2^26 times the weight of each other: together they matter, and each is below the steps of fp16 near one.
    # Its place is late, so that the maximum grows over sums of the others, or first.
    for at in (0, m - 1, m // 2):
        b = Batch(1, 1, d, dt, 64, [m], [(0, tokens + 2, tokens)], seed=3)
        b.q.zero_()
        b.q[:, :, 0] = 16.0
        k, v = b.rows[0]
        k.zero_()
        k[at, :, 0] = 26 * math.log(2) * d ** 0.5 / 16
        v.copy_(1 + torch.rand_like(v.float()) / 2)
        v[at] = 0.0
        t = torch.arange(m, device=DEV)
        blk = torch.from_numpy(b.tables[0]).to(DEV).long()[t // 64]
        b.k[blk, :, t % 64], b.v[blk, :, t % 64] = k, v
        out, lse, avg = b.exact()
        got = b.run()
        # beside the roundings above, probabilities of fp16 lie on steps of 2^-35 of the largest: off by 2^-36 a key at most
        u = torch.finfo(dt).eps / 2
        tol = (u + 2.0 ** -11) * avg + u * out.abs() + 2.0 ** -24 + (m * 2.0 ** -36 * 1.5 if dt == HF else 0)
        err = (got[0].double() - out).abs()
        assert bool((err <= tol).all()), (at, float((err / tol).max()), float(out.abs().max()))
        assert bool(((got[1].double() - lse).abs() <= 2.0 ** -12 + 2.0 ** -22 * lse.abs()).all())


def test_append_refuses_a_closed_rotary_table():
    layout = dopr.make_cache_layout(2, 16, 1, 64, HF, 1, 2)
    rope, x = dopr.Rope(8, 64), torch.ones(3, 1, 64, dtype=HF, device=DEV)
    pools = [torch.zeros(2, 1, 16, 64, dtype=HF, device=DEV) for _ in range(2)]
    rope.close()
    with pytest.raises(ValueError, match="closed"):
        dopr.cache_append(layout, torch.arange(3, device=DEV), x, x, *pools, rope=rope, positions=i32([1, 2, 3]))
    assert not bool(pools[0].any()) and not bool(pools[1].any())


def test_tensors_that_require_a_gradient_are_refused_unless_gradients_are_off():
    b = Batch(4, 2, 64, HF, 16, [20], [(0, 5, 2)], seed=1)
    rope, pos, x = dopr.Rope(64, 64), i32([1, 2]), b.q.clone().requires_grad_()
    y = torch.zeros(2, 2, 64, dtype=HF, device=DEV, requires_grad=True)
    plan, tables, z = dopr.shared_attention_plan(b.layout, 4, *b.args()), i32(b.tables), y.detach()
    pools = [p.clone().requires_grad_() for p in (b.k, b.v)]
    slots = torch.tensor([3, 4], device=DEV)
    calls = [lambda: dopr.rope_apply(rope, pos, x), lambda: dopr.rope_apply(rope, pos, b.q, y),
             lambda: dopr.rope_apply(rope, pos, b.q, q_out=x),
             lambda: dopr.cache_append(b.layout, slots, y, z, b.k, b.v), lambda: dopr.cache_append(b.layout, slots, z, y, b.k, b.v),
             lambda: dopr.cache_append(b.layout, slots, z, z, pools[0], b.v),
             lambda: dopr.cache_append(b.layout, slots, z, z, b.k, b.v, rope=rope, positions=pos, q=x),
             lambda: dopr.shared_attention(b.layout, plan, x, b.k, b.v, tables),
             lambda: dopr.shared_attention(b.layout, plan, b.q, b.k, pools[1], tables)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()


def test_a_rotation_in_a_graph_of_autograd_by_its_inverse():
    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, rope, pos):
            ctx.more = rope, pos
            return dopr.rope_apply(rope, pos, x)[0]

        @staticmethod
        def backward(ctx, g):
            return dopr.rope_apply(*ctx.more, g.contiguous(), inverse=True)[0], None, None

    rope, pos = dopr.Rope(64, 32), i32([1, 2, 3])
    x = torch.randn(3, 2, 64, device=DEV, requires_grad=True)
    w = torch.randn(3, 2, 64, device=DEV)
    (Turn.apply(x, rope, pos) * w).sum().backward()
    assert torch.equal(x.grad, dopr.rope_apply(rope, pos, w, inverse=True)[0])


@pytest.mark.parametrize("rows", [2, 300])
@pytest.mark.parametrize("bad", [-1, 6, 2 ** 31 - 1])
def test_extend_says_so_when_a_released_page_is_outside_the_pool(bad, rows):
    layout = dopr.make_cache_layout(6, 16, 2, 64, torch.float16, rows, 4)
    tables, lens, new = np.zeros((rows, 4)), np.zeros(rows), np.zeros(rows)
    tables[rows - 1, :2] = 3, bad
    lens[rows - 1], new[rows - 1] = 20, -1
    st, free = word(), i32([1, 2, 0, 0, 0, 0])
    b = dopr.cache_extend(layout, i32(lens), i32(tables), free, i32([2]), i32(new), 20, status=st)
    assert st.item() == dopr.ERR_INVALID_ARG and b.n_free.item() == 4 and free.tolist()[:4] == [1, 2, 3, bad]
    assert not any(b.seq_lens.tolist())


def test_outputs_whose_rows_overlap_are_refused():
    b = Batch(4, 2, 64, HF, 16, [20], [(0, 5, 3)], seed=1)
    rope, pos = dopr.Rope(64, 64), i32([1, 2, 3])
    one = torch.zeros(1, 4, 64, dtype=HF, device=DEV).expand(3, 4, 64)
    sliding = torch.zeros(1000, dtype=HF, device=DEV).as_strided((3, 4, 64), (128, 64, 1))
    plan, tables, kv = dopr.shared_attention_plan(b.layout, 4, *b.args()), i32(b.tables), b.q[:, :2].contiguous()
    for out in (one, sliding):
        for call in (lambda: dopr.rope_apply(rope, pos, b.q, q_out=out), lambda: dopr.rope_apply(rope, pos, b.q, b.q, k_out=out),
                     lambda: dopr.rope_apply(rope, pos, out, q_out=out),
                     lambda: dopr.cache_append(b.layout, torch.arange(3, device=DEV), kv, kv, b.k, b.v, rope=rope, positions=pos, q=b.q,
                                               q_out=out),
                     lambda: dopr.shared_attention(b.layout, plan, b.q, b.k, b.v, tables, out=out)):
            with pytest.raises(dopr.DoprError, match="overlap"):
                call()
    assert torch.equal(dopr.rope_apply(rope, pos, one)[0], torch.zeros(3, 4, 64, dtype=HF, device=DEV))


def test_attention_of_two_streams_at_the_same_time():
    # calls of two streams queue up behind a short wait of each, so that they run beside one another: tiles that fill tensor
    # memory, few items and joins of both, with plans, workspaces and outputs of their own
    bs = [Batch(8, 2, 128, BF, 64, [3000, 500], [(i % 2, 50, 1 + i) for i in range(20)], seed=1),
          Batch(4, 2, 64, HF, 16, [700] * 9, [(i % 9, 9 + i, 1 + i % 2) for i in range(40)], seed=2)]
    want = [b.run() for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    rounds, jobs = 12, []
    for b, s in zip(bs, streams):
        args, tables = b.args(), i32(b.tables)
        plan = torch.empty(dopr.shared_attention_plan(b.layout, b.hq, *args).numel(), dtype=torch.uint8, device=DEV)
        outs = [torch.full_like(b.q, 7.0) for _ in range(rounds)]
        lses = [torch.zeros(b.T, b.hq, device=DEV) for _ in range(rounds)]
        jobs.append((b, s, args, tables, plan, dopr.shared_attention_workspace(b.layout, b.hq, b.T), outs, lses, word()))
    torch.cuda.synchronize()

    def queue(i):
        for b, s, args, tables, plan, ws, outs, lses, st in jobs:
            dopr.shared_attention_plan(b.layout, b.hq, *args, plan=plan, status=st, stream=s)
            dopr.shared_attention(b.layout, plan, b.q, b.k, b.v, tables, out=outs[i], lse=lses[i], workspace=ws, status=st, stream=s)

    def check():
        torch.cuda.synchronize()
        for (b, _, _, _, _, _, outs, lses, st), (out, lse) in zip(jobs, want):
            assert st.item() == 0
            assert all(torch.equal(x, out) for x in outs) and all(torch.equal(x, lse) for x in lses)
            for x in outs + lses:
                x.fill_(7.0)
        torch.cuda.synchronize()

    for s in streams:
        with torch.cuda.stream(s):
            torch.cuda._sleep(3000000)  # about 2 ms, in which everything is queued
    for i in range(rounds):
        queue(i)
    check()
    # the same as two branches of one graph
    graph, fork = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=fork):
        for s in streams:
            s.wait_stream(fork)
        for i in range(rounds):
            queue(i)
        for s in streams:
            fork.wait_stream(s)
    for _ in range(3):
        graph.replay()
        check()


@pytest.mark.parametrize("d,dt", [(128, BF), (64, HF)])
def test_pages_beyond_32_bits_of_elements(d, dt):
    # pools of more than 2^32 elements, of which the last pages are used: append, few rows and tiles
    hkv, page, blocks = 8, 128, 2 ** 32 // (8 * 128 * d) + 700
    layout = dopr.make_cache_layout(blocks, page, hkv, d, dt, 4, 40)
    pools = [torch.empty(blocks, hkv, page, d, dtype=dt, device=DEV) for _ in range(2)]
    lens, new, prefix = [3000, 20, 50, 9], [0, 1, 30, 9], [-1, 0, 0, -1]
    tables = np.zeros((4, 40))
    tables[0, :24], tables[1, 0], tables[2, 0], tables[3, 0] = blocks - 1 - 20 * np.arange(24), blocks - 2, blocks - 3, blocks - 4
    tables, g = i32(tables), torch.Generator(DEV).manual_seed(d)
    rows = []
    for i, n in enumerate(lens):
        k, v = (torch.randn(n, hkv, d, generator=g, device=DEV).to(dt) for _ in range(2))
        t = torch.arange(n, device=DEV)
        dopr.cache_append(layout, tables[i].long()[t // page] * page + t % page, k, v, *pools)
        rows.append((k, v))
        b, at = int(tables[i, (n - 1) // page]), (n - 1) % page
        assert torch.equal(pools[0][b, :, at], k[-1]) and torch.equal(pools[1][b, :, at], v[-1])
    b = Batch(16, hkv, d, dt, page, lens[:1], [(0, 20, 1), (0, 50, 30), (-1, 9, 9)], seed=1)
    b.rows, b.layout, b.tables, b.k, b.v = rows, layout, tables.cpu().numpy(), *pools
    assert b.lens == lens and b.new == new and b.prefix == prefix
    b.check(b.run())


def test_a_step_of_no_tokens():
    b = Batch(4, 2, 64, HF, 16, [40], [(0, 5, 1), (-1, 3, 0)], seed=1)
    none, st, off = b.q[:0], word(), i32([0, 0, 0, 0])
    for T in (0, 7):
        plan = dopr.shared_attention_plan(b.layout, b.hq, off, i32(b.lens), i32(b.prefix), T, status=st)
        q, out = (torch.full((T, 4, 64), x, dtype=HF, device=DEV) for x in (1.0, 7.0))
        dopr.shared_attention(b.layout, plan, q, b.k, b.v, i32(b.tables), out=out, status=st)
        assert bool((out == 7).all())
        e = dopr.cache_extend(b.layout, i32(b.lens), i32(b.tables), i32([0] * 8), i32([0]), i32([0, 0, 0]), T, status=st)
        assert e.seq_lens.tolist() == b.lens and e.tok_off.tolist() == [0] * 4 and e.slots.tolist() == [-1] * T
    rope = dopr.Rope(8, 64)
    dopr.cache_append(b.layout, torch.empty(0, dtype=torch.int64, device=DEV), none[:, :2], none[:, :2], b.k, b.v, rope=rope,
                      positions=i32([]), q=none)
    assert st.item() == 0


@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_attention_of_a_step_whose_new_rows_are_all_bad(what):
    # a model that has come apart: queries, new keys or new values are NaN, on a long document and beside a good request
    b = Batch(32, 8, 128, BF, 64, [131072, 200], [(0, 4, 4) for i in range(64)] + [(1, 9, 9)], seed=5)
    want = b.run()
    T = 64 * 4
    if what == "q":
        b.q[:T] = math.nan
    else:
        pool = b.k if what == "k" else b.v
        for i in range(2, 66):
            pool[int(b.tables[i, 0]), :, :4] = math.nan
    plan, tables = dopr.shared_attention_plan(b.layout, b.hq, *b.args()), i32(b.tables)
    ws, st = dopr.shared_attention_workspace(b.layout, b.hq, b.T), word()
    dopr.shared_attention(b.layout, plan, b.q, b.k, b.v, tables, workspace=ws)
    a, z = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    got = dopr.shared_attention(b.layout, plan, b.q, b.k, b.v, tables, workspace=ws, status=st)
    z.record()
    z.synchronize()
    assert st.item() == 0 and bool(torch.isnan(got[:T]).all()) and torch.equal(got[T:], want[0][T:])
    assert a.elapsed_time(z) < 20


def test_a_refused_allocation_does_not_fail_the_calls_behind_it():
    from paper_2609_03311_gb300 import synth

    shape = synth.ModelShape("oom", n_layers=2, hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=128, ffn=384, vocab=512)
    b = Batch(4, 2, 64, HF, 16, [20], [(0, 5, 2)], seed=1)
    want = b.run()
    for call in (lambda: b.run(), lambda: dopr.Rope(64, 64)):
        with pytest.raises(dopr.DoprError):
            dopr.Store(dopr.make_config(shape, max_position=512), max_doc_id=15, pool_bytes=1 << 50)
        got = call()
    got = b.run()
    assert torch.equal(got[0], want[0])
