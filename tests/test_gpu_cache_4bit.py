"""Attention over the paged cache in 4 bits, on a GPU: against 64-bit softmax over the values that the pages hold, and a program's
steps of norm, append and attention together.

Tolerances: those of the 16-bit cache's attention (tests/test_gpu_cache.py).  The values that pages hold are exact in the products'
type, so nothing is added for them: |out - exact| <= (u + 2^-11) A + u |exact| + 2^-24, A the softmax average of |v|, and
|lse - exact| <= 2^-12 + 2^-22 |exact|."""
import math

import numpy as np
import pytest
import torch

from paper_2609_03311_gb300 import dopr
from test_gpu_cache import BF, HF, MIXED, Batch, i32, word
from test_gpu_heads import EPS, codes_of, gain, pools, put, scales64

pytestmark = pytest.mark.gpu
DEV = "cuda"


def held(x):
    c, byte = codes_of(x)
    return (c * scales64()[byte].repeat_interleave(32, -1)).to(x.dtype)


class Batch4(Batch):
    """The same documents and requests in 4-bit pages; bytes that no row's keys are in are random, scales' bytes among them."""

    def __init__(self, *args, seed, size=1.0, **kw):
        super().__init__(*args, seed=seed, **kw)
        self.k4, self.v4 = pools(self.layout, seed)
        for i, x in enumerate(self.lens):
            self.rows[i] = [(r.float() * size).to(self.dt) for r in self.rows[i]]
            self.write(i, torch.arange(x, device=DEV))

    def write(self, i, t):
        """Row i's keys and values at the positions t into the pages; the record then has what is held."""
        slots = torch.from_numpy(self.tables[i]).to(DEV).long()[t // self.page] * self.page + t % self.page
        self.k4 = put(self.k4, self.page, self.d, slots, self.rows[i][0][t])
        self.v4 = put(self.v4, self.page, self.d, slots, self.rows[i][1][t])
        for r in self.rows[i]:
            r[t] = held(r[t])

    def run(self, pad=0, want=0, **kw):
        st = word()
        q = torch.cat([self.q, torch.full((pad, self.hq, self.d), math.nan, dtype=self.dt, device=DEV)]) if pad else self.q
        T = self.T + pad
        plan = dopr.shared_attention_plan(self.layout, self.hq, i32(self.off), i32(self.lens), i32(self.prefix), T, status=st)
        assert st.item() == 0
        out = torch.full((T, self.hq, self.d), 7.0, dtype=self.dt, device=DEV)
        lse = torch.full((T, self.hq), 7.0, device=DEV)
        dopr.shared_attention_4bit(self.layout, plan, q, self.k4, self.v4, i32(self.tables), out=out, lse=lse, status=st, **kw)
        assert st.item() == want
        assert bool((out[self.T:] == 7).all()) and bool((lse[self.T:] == 7).all())
        return out[:self.T], lse[:self.T]


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_few_rows(page, d, dt):
    b = Batch4(8, 2, d, dt, page, [300], [(0, 24, 1), (0, 1, 1), (0, 64, 1)], seed=page + d)
    b.check(b.run())


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_tiles(page, d, dt):
    b = Batch4(8, 2, d, dt, page, [300, 40], [(0, 24, 20), (0, 70, 30), (1, 64, 64), (-1, 140, 90)], seed=page + d)
    b.check(b.run())


@pytest.mark.parametrize("m", [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 5000])
@pytest.mark.parametrize("own,new", [(0, 1), (1, 1), (5, 5), (130, 3), (129, 129)])
def test_lengths(m, own, new):
    b = Batch4(4, 1, 128, BF, 32, [m], [(0, own, new)], seed=m + own)
    b.check(b.run())


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (5, 1), (6, 2), (7, 1), (8, 8), (16, 1), (33, 1), (40, 8), (64, 1), (128, 2)])
def test_head_counts(hq, hkv):
    b = Batch4(hq, hkv, 64, HF, 16, [200, 77], [(0, 30, 2), (1, 50, 9), (0, 3, 3), (1, 1, 1)], seed=hq)
    b.check(b.run())


@pytest.mark.parametrize("dt,d", [(BF, 128), (HF, 64), (HF, 128)])
@pytest.mark.parametrize("seed", range(6))
def test_ragged_batches_in_any_order(seed, dt, d):
    r = np.random.default_rng(seed)
    docs = [int(x) for x in r.integers(0, [40, 700, 3000][seed % 3], 5)]
    reqs = []
    for _ in range(int(r.integers(1, 60))):
        own = int(r.integers(0, 150))
        reqs.append((int(r.integers(-1, 5)), own, int(r.integers(0, own + 2)) if seed % 2 else 1))
    if sum(x[2] for x in reqs) == 0:
        reqs.append((0, 1, 1))
    b = Batch4(8, 2, d, dt, [16, 64, 128][seed % 3], docs, reqs, seed=seed, own_rows={1: min(docs[1], 70)})
    b.check(b.run(pad=seed * 3))


def test_rows_that_see_nothing():
    b = Batch4(4, 2, 128, BF, 16, [0, 33], [(0, 2, 5), (-1, 0, 3), (1, 0, 2), (-1, 1, 4)], seed=3)
    got = b.run()
    b.check(got)
    assert int((got[1] == -math.inf).sum()) == (3 + 3 + 3) * 4


@pytest.mark.parametrize("n,new,m", [(40, 32, 900), (3, 600, 513), (1, 2000, 100), (70, 64, 40)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_many_rows(n, new, m, dt):
    b = Batch4(8, 2, 128, dt, 64, [m, 1], [(0, new + (i % 3), new) for i in range(n)], seed=n)
    b.check(b.run())


@pytest.mark.parametrize("m", [0, 100, 128, 129, 192, 256, 300, 1000, 4100])
@pytest.mark.parametrize("d,page,own,new", [(128, 64, 90, 20), (64, 16, 300, 9), (128, 32, 5, 5), (64, 128, 70, 30)])
def test_one_tile_with_blocks_in_turn(d, page, own, new, m):
    b = Batch4(8, 2, d, BF, page, [m, 150], [(0, own, new), (1, 40, 25), (0, 3, 6), (-1, 70, 30)], seed=m + d)
    b.check(b.run())


@pytest.mark.parametrize("m", [40000, 131072])
@pytest.mark.parametrize("tokens", [1, 20])
def test_a_long_document(m, tokens):
    b = Batch4(4, 1, 128, BF, 128, [m], [(0, 9 + tokens, tokens), (0, 100, tokens)], seed=1)
    b.check(b.run())


@pytest.mark.parametrize("kind", list(MIXED))
@pytest.mark.parametrize("d,dt", [(128, BF), (64, HF)])
def test_rows_that_share_items_in_every_way(kind, d, dt):
    hq, docs, reqs = MIXED[kind]
    b = Batch4(hq, 2, d, dt, 16, docs, reqs, seed=len(reqs) + d)
    b.check(b.run())


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("tokens", [1, 40])
@pytest.mark.parametrize("size", [2.0 ** -14, 2.0 ** -9, 2.0 ** 13])
def test_values_of_every_size(size, tokens, dt):
    # scales of a bit and of the largest: keys' scores stay about one by q, values come out as they are
    b = Batch4(4, 2, 128, dt, 16, [500], [(0, 40 + tokens, tokens)] * 3, seed=7, size=size)
    scale = 128 ** -0.5 * (2.0 ** -13 if size > 1 else min(1 / size, 512.0))
    out, lse, avg = b.exact(scale)
    got = b.run(scale=scale)
    u = torch.finfo(dt).eps / 2
    tiny = 2.0 ** -25 if dt == HF else 0.0  # half of fp16's smallest step
    err, tol = (got[0].double() - out).abs(), (u + 2.0 ** -11) * avg + u * out.abs() + tiny
    assert bool((err <= tol).all()), float((err / tol).max())
    assert bool(((got[1].double() - lse).abs() <= 2.0 ** -12 + 2.0 ** -22 * lse.abs()).all())


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tokens", [1, 3, 40, 200])
def test_one_heavy_key_among_many_light_ones(tokens, d, dt):
    m = 131072
    for at in (0, m - 1):
        b = Batch4(1, 1, d, dt, 64, [m], [(0, tokens + 2, tokens)], seed=3)
        b.q.zero_()
        b.q[:, :, 0] = 16.0
        k, v = b.rows[0]
        k.zero_()
        k[at, :, 0] = 26 * math.log(2) * d ** 0.5 / 16
        v.copy_(1 + torch.rand_like(v.float()) / 2)
        v[at] = 0.0
        b.write(0, torch.arange(m, device=DEV))
        out, lse, avg = b.exact()
        got = b.run()
        # fp16's probabilities lie on steps of 2^-35 of the largest
        u = torch.finfo(dt).eps / 2
        tol = (u + 2.0 ** -11) * avg + u * out.abs() + 2.0 ** -24 + (m * 2.0 ** -36 * 1.6 if dt == HF else 0)
        err = (got[0].double() - out).abs()
        assert bool((err <= tol).all()), (at, float((err / tol).max()))
        assert bool(((got[1].double() - lse).abs() <= 2.0 ** -12 + 2.0 ** -22 * lse.abs()).all())


# Parts of few rows long enough that a warp takes 8 rows of one run at once, with codes as they are: some 16 pieces of 16 keys and more for
# each of 8 warps an SM.  P times the scale of a value is rounded once, to 11 bits, in P's place.
LONG = {
    "a row a token": (8, 8, 0, [(-1, 2100 + 37 * i, 1) for i in range(24)]),
    "four rows a token": (32, 8, 0, [(-1, 1500 + 91 * i, 1) for i in range(24)]),
    "five rows a token": (20, 4, 0, [(-1, 1900 + 53 * i, 1) for i in range(50)]),
    "eight rows a token": (64, 8, 0, [(-1, 2400 + 29 * (i % 7), 1) for i in range(20)]),
    "two tokens of each": (16, 8, 0, [(-1, 1700 + 111 * i, 2) for i in range(20)]),
    "five of each, more than 8 rows": (16, 8, 0, [(-1, 2200 + 13 * i, 5) for i in range(20)]),
    "long and short": (32, 8, 0, [(-1, [40, 5000, 3, 2600, 0, 16, 17][i % 7], 1) for i in range(49)]),
    "one sequence": (8, 2, 0, [(-1, 250001, 1)]),
    "two tokens of one": (8, 2, 0, [(-1, 250017, 2)]),
    "three tokens of one": (8, 2, 0, [(-1, 250002, 3)]),
    "two on a document": (8, 2, 230000, [(0, 25, 1), (0, 400, 1)]),
}


@pytest.mark.parametrize("dt,d,page", [(BF, 128, 64), (HF, 128, 16), (HF, 64, 128), (BF, 64, 32)])
@pytest.mark.parametrize("kind", list(LONG))
def test_long_parts_of_few_rows(kind, dt, d, page):
    hq, hkv, m, reqs = LONG[kind]
    b = Batch4(hq, hkv, d, dt, page, [m] if m else [], reqs, seed=len(kind) + d)
    got = b.run()
    b.check(got)
    again = b.run()
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("bad", [math.nan, math.inf, 1e30])
def test_bad_queries_stay_in_their_rows_of_long_parts(bad):
    hq, hkv, _, reqs = LONG["four rows a token"]
    b = Batch4(hq, hkv, 128, BF, 64, [], reqs, seed=2)
    clean = b.run()
    b.q[3, 5] = bad
    got = b.run()
    rest = torch.ones(b.T, hq, dtype=torch.bool, device=DEV)
    rest[3, 5] = False
    assert not bool(torch.isfinite(got[0][3, 5]).all()) or bad == 1e30
    assert torch.equal(got[0][rest], clean[0][rest]) and torch.equal(got[1][rest], clean[1][rest])


@pytest.mark.parametrize("byte", [0xe2, 0xff])
@pytest.mark.parametrize("pool", ["k", "v"])
@pytest.mark.parametrize("kind", ["a row a token", "four rows a token", "one sequence"])
def test_scales_that_stand_for_nan_in_long_parts(kind, pool, byte):
    hq, hkv, _, reqs = LONG[kind]
    b = Batch4(hq, hkv, 128, HF, 16, [], reqs, seed=5)
    p = b.k4 if pool == "k" else b.v4
    places = [(int(b.tables[i, at // 16]), i % hkv, 16 * 64 + at % 16 * 4 + i % 4)
              for i in range(0, len(reqs), 2) for at in (0, 777, b.lens[i] - 1)]
    for x in places:
        p[x] = byte
    got = b.run(want=dopr.ERR_RANGE)
    for x in places:
        p[x] = 0
    again = b.run()
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("dt", [BF, HF])
def test_values_of_very_different_sizes_in_long_parts(dt):
    # a sequence's values grow 2^16 times over its keys, one group of elements is 2^6 times the others, and every other sequence is larger
    # still.  P's largest is 2^11 or more, the largest scale comes as 1 / 2 or more, and their products are rounded to 11 bits, or to
    # steps of 2^-24: a key adds at most 7 2^-25 / (2^11 / 2) = 7 2^-35 of the run's largest scale.
    hq, hkv, _, reqs = LONG["four rows a token"]
    b = Batch4(hq, hkv, 128, dt, 64, [], reqs, seed=9)
    for i, n in enumerate(b.lens):
        grow = torch.exp2(torch.linspace(-16, 0, n, device=DEV))[:, None, None] * (16.0 if i % 2 else 1.0)
        v = b.rows[i][1].float() * grow
        v[:, :, 32:64] *= 64
        b.rows[i][1] = v.to(dt)
        b.write(i, torch.arange(n, device=DEV))
    out, lse, avg = b.exact()
    got = b.run()
    u = torch.finfo(dt).eps / 2
    largest = max(float(r[1].float().abs().max()) for r in b.rows) / 7 * 1.125
    tol = (u + 2.0 ** -11) * avg + u * out.abs() + 7 * 2.0 ** -35 * largest * max(b.lens) + 2.0 ** -24
    err = (got[0].double() - out).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("bad", [math.nan, math.inf, 1e30])
@pytest.mark.parametrize("tokens", [1, 30])
def test_bad_queries_stay_in_their_rows(bad, tokens):
    b = Batch4(4, 2, 128, BF, 16, [100], [(0, 20 + tokens, tokens), (0, 30 + tokens, tokens), (-1, 40, 1)], seed=2)
    clean = b.run()
    b.q[0] = bad
    got = b.run()
    assert not bool(torch.isfinite(got[0][0]).all()) or bad == 1e30
    assert torch.equal(got[0][1:], clean[0][1:]) and torch.equal(got[1][1:], clean[1][1:])


@pytest.mark.parametrize("kind", list(MIXED))
@pytest.mark.parametrize("byte", [0xe2, 0xf8, 0xff])
@pytest.mark.parametrize("pool", ["k", "v"])
def test_scales_that_stand_for_nan_count_as_zero_and_are_an_error(kind, byte, pool):
    # of the last own key of every third request: the others' results keep their bits
    hq, docs, reqs = MIXED[kind]
    b = Batch4(hq, 2, 128, BF, 16, docs, reqs, seed=len(reqs))
    want = b.run()
    zero = byte
    p = b.k4 if pool == "k" else b.v4
    sees = torch.zeros(b.T, dtype=torch.bool, device=DEV)
    places = []
    for i in range(len(docs), len(b.lens), 3):
        at = b.lens[i] - 1
        places.append((int(b.tables[i, at // 16]), 1, 16 * 64 + at % 16 * 4 + 2))
        sees[b.off[i + 1] - 1] = True
    for x in places:
        p[x] = byte
    got = b.run(want=dopr.ERR_RANGE)
    assert torch.equal(got[0][~sees], want[0][~sees]) and torch.equal(got[1][~sees], want[1][~sees])
    for x in places:
        p[x] = 0
    again = b.run()
    assert zero and torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_pages_outside_the_pool_are_read_as_page_zero():
    for reqs in ([(0, 5, 2), (-1, 6, 1)], [(0, 30, 30), (-1, 60, 50)]):
        b = Batch4(4, 2, 64, HF, 16, [40], reqs, seed=1)
        b.k4[0], b.v4[0] = b.k4[1] & 0x7f, b.v4[1] & 0x7f  # (any page, with scales)
        st = word()
        plan = dopr.shared_attention_plan(b.layout, b.hq, *b.args())
        for bad in (-1, b.layout.n_blocks, 2 ** 31 - 1):
            tables = b.tables.copy()
            tables[0, 1] = bad
            st.zero_()
            out = dopr.shared_attention_4bit(b.layout, plan, b.q, b.k4, b.v4, i32(tables), status=st)
            assert st.item() == dopr.ERR_INVALID_ARG
            tables[0, 1] = 0
            assert torch.equal(out, dopr.shared_attention_4bit(b.layout, plan, b.q, b.k4, b.v4, i32(tables)))


def test_a_plan_of_other_sizes_and_strided_views():
    b = Batch4(8, 2, 64, HF, 32, [400], [(0, 20, 7), (0, 9, 9)], seed=4)
    want = b.run(scale=0.31)
    b.check(want, scale=0.31)
    plan = dopr.shared_attention_plan(b.layout, b.hq, *b.args())
    wide = torch.zeros(b.T, 12, 64, dtype=HF, device=DEV)
    wide[:, 2:10] = b.q
    out = torch.zeros(8, b.T, 64, dtype=HF, device=DEV).transpose(0, 1)
    dopr.shared_attention_4bit(b.layout, plan, wide[:, 2:10], b.k4, b.v4, i32(b.tables), scale=0.31, out=out)
    assert torch.equal(out, want[0])
    room = torch.zeros(plan.numel() * 4, dtype=torch.uint8, device=DEV)
    room[:plan.numel()] = plan
    st, q = word(), torch.cat([b.q, b.q])
    out = torch.full_like(q, 7.0)
    dopr.shared_attention_4bit(b.layout, room, q, b.k4, b.v4, i32(b.tables), out=out, status=st)
    assert st.item() == dopr.ERR_INVALID_ARG and bool((out == 7).all())
    # one row for all tokens
    b.q = b.q[:1].expand(b.T, -1, -1)
    b.check(b.run())


def test_pools_beyond_32_bits_of_bytes():
    hkv, page, d = 8, 128, 128
    blocks = 2 ** 32 // (hkv * page * 68) + 100
    layout = dopr.make_cache_layout(blocks, page, hkv, d, BF, 4, 40)
    k4, v4 = dopr.cache_pools_4bit(layout)
    lens = [3000, 20, 50, 9]
    tables = np.zeros((4, 40))
    tables[0, :24], tables[1, 0], tables[2, 0], tables[3, 0] = blocks - 1 - 4 * np.arange(24), blocks - 2, blocks - 3, blocks - 4
    b = Batch(16, hkv, d, BF, page, lens[:1], [(0, 20, 1), (0, 50, 30), (-1, 9, 9)], seed=1)
    st = word()
    for i, n in enumerate(lens):
        t = torch.arange(n, device=DEV)
        slots = torch.from_numpy(tables[i]).to(DEV).long()[t // page] * page + t % page
        dopr.cache_append_4bit(layout, slots, *b.rows[i], k4, v4, status=st)
        b.rows[i] = list(dopr.cache_read_4bit(layout, slots, k4, v4, status=st))
    plan = dopr.shared_attention_plan(layout, 16, *b.args())
    lse = torch.empty(b.T, 16, device=DEV)
    out = dopr.shared_attention_4bit(layout, plan, b.q, k4, v4, i32(tables), lse=lse, status=st)
    assert st.item() == 0
    b.check((out, lse))


class Program:
    """A two-layer 4-bit cache as a program of a model with head norms keeps it: documents stored once, then requests token by token."""

    def __init__(self, dt=BF, hq=8, hkv=2, d=128, page=16, docs=(200, 35), reqs=5, cap=40):
        self.n, self.docs, self.hq, self.hkv, self.d, self.dt = len(docs) + reqs, len(docs), hq, hkv, d, dt
        mb = -(-max(max(docs), cap) // page)
        blocks = sum(-(-x // page) for x in docs) + reqs * -(-cap // page)
        self.page, self.layout = page, dopr.make_cache_layout(blocks, page, hkv, d, dt, self.n, mb)
        self.pools = [pools(self.layout, i) for i in range(2)]
        self.seq_lens, self.n_free = i32([0] * self.n), i32([blocks])
        self.tables, self.free = i32(np.full((self.n, mb), -1)), i32(np.arange(blocks))
        self.prefix = i32([-1] * self.docs + [i % self.docs for i in range(reqs)])
        self.rope, self.status = dopr.Rope(1024, d), word()
        self.gains = [(gain(d, BF, 2 * i), gain(d, BF, 2 * i + 1)) for i in range(2)]

    def batch(self, max_tokens):
        out = dopr.cache_batch(self.layout, max_tokens)
        out.seq_lens, out.n_free = self.seq_lens, self.n_free
        return out

    def step(self, out, new, qkv, outs, qs):
        T, st = out.max_tokens, self.status
        dopr.cache_extend(self.layout, self.seq_lens, self.tables, self.free, self.n_free, new, T, prefix=self.prefix, out=out, status=st)
        plan = dopr.shared_attention_plan(self.layout, self.hq, out.tok_off, self.seq_lens, self.prefix, T, status=st)
        for l in range(2):
            q, k, v = qkv[l][:, :self.hq], qkv[l][:, self.hq:self.hq + self.hkv], qkv[l][:, self.hq + self.hkv:]
            dopr.cache_append_4bit(self.layout, out.slots, k, v, *self.pools[l], k_gain=self.gains[l][1], eps=EPS, rope=self.rope,
                                   positions=out.positions, q=q, q_gain=self.gains[l][0], q_out=qs[l], status=st)
            dopr.shared_attention_4bit(self.layout, plan, qs[l], *self.pools[l], self.tables, out=outs[l], status=st)

    def rows_of(self, seed, T):
        g = torch.Generator(DEV).manual_seed(seed)
        return [torch.randn(T, self.hq + 2 * self.hkv, self.d, generator=g, device=DEV).to(self.dt) for _ in range(2)]

    def check(self, outs, qs, new, qkv, positions):
        """The step's attention in 64 bits, from its q and what the pages hold; and the new rows there, from the norm's outputs."""
        lens, tables, pre = self.seq_lens.tolist(), self.tables.long(), self.prefix.tolist()
        T, G = sum(new), self.hq // self.hkv
        for l in range(2):
            def row(i):
                t = torch.arange(lens[i], device=DEV)
                return [x.double() for x in dopr.cache_read_4bit(self.layout, tables[i][t // self.page] * self.page + t % self.page, *self.pools[l])]

            q, k = dopr.head_norm_rope(qkv[l][:T, :self.hq], qkv[l][:T, self.hq:self.hq + self.hkv], *self.gains[l], eps=EPS, rope=self.rope,
                                       positions=positions[:T])
            assert torch.equal(q, qs[l][:T])
            at = 0
            for i, n in enumerate(new):
                if n == 0:
                    continue
                mine = row(i)
                assert torch.equal(mine[0][lens[i] - n:], held(k[at:at + n]).double())
                assert torch.equal(mine[1][lens[i] - n:], held(qkv[l][at:at + n, self.hq + self.hkv:]).double())
                ks, vs = (torch.cat([a, b]) for a, b in zip(row(pre[i]), mine)) if pre[i] >= 0 else mine
                seen = ks.shape[0] - n + 1 + torch.arange(n, device=DEV)
                a = torch.einsum("thd,khd->thk", q[at:at + n].double(), ks.repeat_interleave(G, 1)) * self.d ** -0.5
                a = a.masked_fill((torch.arange(ks.shape[0], device=DEV) >= seen[:, None])[:, None], -math.inf).softmax(-1)
                want = torch.einsum("thk,khd->thd", a, vs.repeat_interleave(G, 1))
                avg = torch.einsum("thk,khd->thd", a, vs.abs().repeat_interleave(G, 1))
                u = torch.finfo(self.dt).eps / 2
                err = (outs[l][at:at + n].double() - want).abs()
                assert bool((err <= (u + 2.0 ** -11) * avg + u * want.abs() + 2.0 ** -24).all()), float(err.max())
                at += n


def test_a_program_stores_documents_and_answers_token_by_token():
    p = Program()
    steps = [[200, 35] + [0] * 5, [0, 0, 7, 3, 1, 12, 0], [0, 0, 1, 1, 1, 1, 5], [0, 0, 1, 0, 1, 1, 1], [0, 0] + [1] * 5,
             [0, 0] + [20] * 5]
    for n, new in enumerate(steps):
        T = sum(new) + n  # a few rows behind the last token
        qkv = p.rows_of(n, T)
        outs, qs = ([torch.full((T, p.hq, p.d), 7.0, dtype=p.dt, device=DEV) for _ in range(2)] for _ in range(2))
        b = p.batch(T)
        p.step(b, i32(new), qkv, outs, qs)
        assert p.status.item() == 0
        p.check(outs, qs, new, qkv, b.positions)
        assert all(bool((o[sum(new):] == 7).all()) for o in outs + qs)


def test_a_captured_step_is_replayed_as_the_sequences_grow():
    p = Program(dt=HF, d=64, page=32)
    new = [200, 35] + [4] * 5
    qkv = p.rows_of(99, sum(new))
    outs, qs = ([torch.zeros(sum(new), p.hq, p.d, dtype=p.dt, device=DEV) for _ in range(2)] for _ in range(2))
    b = p.batch(sum(new))
    p.step(b, i32(new), qkv, outs, qs)
    p.check(outs, qs, new, qkv, b.positions)
    T = 6
    b, add = p.batch(T), i32([0, 0, 1, 1, 1, 1, 1])
    outs, qs = ([torch.zeros(T, p.hq, p.d, dtype=p.dt, device=DEV) for _ in range(2)] for _ in range(2))
    qkv = p.rows_of(0, T)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        p.step(b, add, qkv, outs, qs)
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
        p.check(outs, qs, new, qkv, b.positions)


def test_two_streams_at_the_same_time():
    bs = [Batch4(8, 2, 128, BF, 64, [3000, 500], [(i % 2, 50, 1 + i) for i in range(20)], seed=1),
          Batch4(4, 2, 64, HF, 16, [700] * 9, [(i % 9, 9 + i, 1 + i % 2) for i in range(40)], seed=2)]
    want = [b.run() for b in bs]
    jobs = []
    for b in bs:
        plan = dopr.shared_attention_plan(b.layout, b.hq, *b.args())
        outs = [torch.full_like(b.q, 7.0) for _ in range(12)]
        jobs.append((b, torch.cuda.Stream(), plan, i32(b.tables), dopr.shared_attention_workspace(b.layout, b.hq, b.T), outs, word()))
    torch.cuda.synchronize()
    for _, s, *_ in jobs:
        with torch.cuda.stream(s):
            torch.cuda._sleep(3000000)  # about 2 ms, in which everything is queued
    for i in range(12):
        for b, s, plan, tables, ws, outs, st in jobs:
            dopr.shared_attention_4bit(b.layout, plan, b.q, b.k4, b.v4, tables, out=outs[i], workspace=ws, status=st, stream=s)
    torch.cuda.synchronize()
    for (_, _, _, _, _, outs, st), (out, _) in zip(jobs, want):
        assert st.item() == 0 and all(torch.equal(x, out) for x in outs)


@pytest.mark.parametrize("d,dt,page", [(128, HF, 16), (128, BF, 32), (64, BF, 16), (128, BF, 128)])
def test_calls_one_after_another_give_the_same_bits(d, dt, page):
    # tiles whose blocks end in their first half or in their second, so that the raw rings' stages change hands, beside few items
    r = np.random.default_rng(page + d)
    docs = [79, 724, 40, 200, 129, 16, 1000, 50]
    reqs = [(i % 8, int(r.integers(1, 90)), 1) for i in range(100)] + [(2, 90, 30), (-1, 70, 70), (3, 20, 20)]
    bs = [Batch4(16, 8, d, dt, page, docs, reqs, seed=s) for s in (1, 2)]
    want = [b.run() for b in bs]
    for b, w in zip(bs, want):
        b.check(w)
    jobs = [(b, dopr.shared_attention_plan(b.layout, b.hq, *b.args()), i32(b.tables), torch.empty_like(b.q),
             dopr.shared_attention_workspace(b.layout, b.hq, b.T)) for b in bs]
    same, st = torch.ones((), dtype=torch.bool, device=DEV), word()
    for _ in range(1500):
        for (b, plan, tables, out, ws), w in zip(jobs, want):
            dopr.shared_attention_4bit(b.layout, plan, b.q, b.k4, b.v4, tables, out=out, workspace=ws, status=st)
            same &= (out == w[0]).all()
    assert bool(same) and st.item() == 0


def test_thousands_of_rows_and_steps_of_no_tokens():
    r = np.random.default_rng(5)
    reqs = [(int(x), int(r.integers(0, 4)), int(r.choice([0, 1, 1, 2]))) for x in r.integers(-1, 40, 1500)]
    b = Batch4(2, 1, 64, BF, 16, [int(x) for x in r.integers(0, 20, 40)], reqs, seed=1)
    b.check(b.run())
    b = Batch4(4, 2, 64, HF, 16, [40], [(0, 5, 1), (-1, 3, 0)], seed=1)
    for T in (0, 7):
        plan = dopr.shared_attention_plan(b.layout, b.hq, i32([0, 0, 0, 0]), i32(b.lens), i32(b.prefix), T)
        q, out = (torch.full((T, 4, 64), x, dtype=HF, device=DEV) for x in (1.0, 7.0))
        dopr.shared_attention_4bit(b.layout, plan, q, b.k4, b.v4, i32(b.tables), out=out)
        assert bool((out == 7).all())


def test_wrong_pools_are_refused():
    b = Batch4(4, 2, 64, HF, 16, [40], [(0, 5, 1)], seed=1)
    plan = dopr.shared_attention_plan(b.layout, b.hq, *b.args())
    flat = b.k4.flatten()
    for k in (b.k, flat[1:], flat.cpu(), flat[:-1], b.k4.view(torch.int8)):
        with pytest.raises(ValueError):
            dopr.shared_attention_4bit(b.layout, plan, b.q, k, b.v4, i32(b.tables))
    odd = torch.cat([flat[:8], flat])[8:]
    with pytest.raises(dopr.DoprError):
        dopr.shared_attention_4bit(b.layout, plan, b.q, odd, b.v4, i32(b.tables))
    with pytest.raises(ValueError, match="gradient"):
        dopr.shared_attention_4bit(b.layout, plan, b.q.clone().requires_grad_(), b.k4, b.v4, i32(b.tables))
