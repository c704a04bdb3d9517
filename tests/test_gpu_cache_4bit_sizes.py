"""Attention over the paged cache in 4 bits where values of one part differ very much in size, on a GPU: what a row does not see, or
sees at next to no weight, costs it nothing.

Tolerances.  Where up to 8 rows share many keys, a probability times a value's scale is rounded to 11 bits, or, where it is
small, to a step of 2^-24.  A row's largest such product is 2^10 or more: 2^11 times the half of a power of two that its scale lies above
(scales below 2^-15 count as 2^-15 there).  So a key adds at most 7 2^-25 / 2^10 = 7 2^-35 of the largest P max(s, 2^-15) among the
keys that the row sees, and |out - exact| <= (u + 2^-11) A + u |exact| + 2^-24 + n 7 2^-35 X: n those keys, X that largest
product over the sum of P, A the softmax average of |v|."""
import math

import pytest
import torch

from paper_2609_03311_gb300 import dopr
from test_gpu_cache import BF, HF
from test_gpu_cache_4bit import LONG, Batch4
from test_gpu_heads import scales64

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Sized(Batch4):
    """Sequences without a prefix."""

    def scales(self, i):
        """The largest of the scales of each key's values, [keys, kv heads]."""
        t = torch.arange(self.lens[i], device=DEV)
        page = self.v4[torch.from_numpy(self.tables[i]).to(DEV).long()[t // self.page]]
        at = self.page * self.d // 2 + (t % self.page)[:, None] * (self.d // 32) + torch.arange(self.d // 32, device=DEV)
        return scales64()[page.gather(2, at[:, None].expand(-1, self.hkv, -1)).long()].amax(-1)

    def steps(self):
        """n 7 2^-35 X of each row, [tokens, q heads, 1]."""
        out = torch.zeros(self.T, self.hq, 1, dtype=torch.float64, device=DEV)
        for i, n in enumerate(self.new):
            if n == 0:
                continue
            rows, G = slice(self.off[i], self.off[i + 1]), self.hq // self.hkv
            a = torch.einsum("thd,khd->thk", self.q[rows].double(), self.rows[i][0].double().repeat_interleave(G, 1)) * self.d ** -0.5
            seen = self.lens[i] - n + torch.arange(n, device=DEV) + 1
            a = a.masked_fill((torch.arange(self.lens[i], device=DEV) >= seen[:, None])[:, None], -math.inf).softmax(-1)
            s = self.scales(i).clamp(min=2.0 ** -15).repeat_interleave(G, 1).T
            out[rows, :, 0] = (a * s).amax(-1) * 7 * 2.0 ** -35 * seen[:, None]
        return out

    def check(self, got):
        out, lse, avg = self.exact()
        u = torch.finfo(self.dt).eps / 2
        err, tol = (got[0].double() - out).abs(), (u + 2.0 ** -11) * avg + u * out.abs() + 2.0 ** -24 + self.steps()
        assert bool((err <= tol).all()), (float((err / tol).max()), int((~(err <= tol)).sum()))
        assert bool(((got[1].double() - lse).abs() <= 2.0 ** -12 + 2.0 ** -22 * lse.abs()).all())

    def light_beside_heavy(self, i, heavy):
        """Row i: the keys `heavy` have no value, the others 2^-18 or 2^-19 of their weight and values of 2^-4 and half as much again."""
        k, v = self.rows[i]
        k.zero_()
        k[heavy, :, 0] = 18 * math.log(2) * self.d ** 0.5 / 16
        v.copy_((1 + torch.rand(v.shape, generator=torch.Generator(DEV).manual_seed(i), device=DEV) / 2) * 2.0 ** -4)
        v[heavy] = 0.0
        self.q.zero_()
        self.q[:, :, 0] = 16.0


FORMS = [(BF, 128, 64), (HF, 128, 16), (HF, 64, 128), (BF, 64, 32)]
SEVERAL = {  # several new tokens of a sequence, with up to 8 rows and with more: (hq, hkv, requests)
    "two of each": (16, 8, [(-1, 1700 + 111 * i, 2) for i in range(20)]),
    "two, four rows a token": (8, 2, [(-1, 250010, 2)]),
    "three, four rows a token": (8, 2, [(-1, 250009, 3)]),
    "eight of each": (8, 8, [(-1, 2300 + 41 * i, 8) for i in range(20)]),
    "a few of each": (8, 8, [(-1, 2000 + 113 * i, 1 + i % 8) for i in range(24)]),
}


@pytest.mark.parametrize("dt,d,page", FORMS)
@pytest.mark.parametrize("kind", list(SEVERAL))
def test_large_values_that_a_row_does_not_see(kind, dt, d, page):
    # The last key, which the last token alone sees, has a value some 2^20 times those of the keys just before it, which hold all that
    # the others see.
    hq, hkv, reqs = SEVERAL[kind]
    b = Sized(hq, hkv, d, dt, page, [], reqs, seed=len(kind) + d)
    got = []
    for last in (2.0 ** -4, 60000.0):
        for i, n in enumerate(b.lens):
            b.light_beside_heavy(i, n - 9)
            b.rows[i][1][:-16] = 0.0
            b.rows[i][1][-1, :, 32:64] = last
            b.write(i, torch.arange(n, device=DEV))
        got.append(b.run())
        b.check(got[-1])
    others = torch.ones(b.T, dtype=torch.bool, device=DEV)
    others[torch.from_numpy(b.off[1:] - 1).to(DEV)] = False
    assert int(others.sum()) > 0
    assert torch.equal(got[0][0][others], got[1][0][others]) and torch.equal(got[0][1][others], got[1][1][others])


@pytest.mark.parametrize("dt,d,page", FORMS)
@pytest.mark.parametrize("kind", ["a row a token", "four rows a token", "eight rows a token", "one sequence"])
def test_large_values_of_next_to_no_weight(kind, dt, d, page):
    # every 64th key has 2^-60 of the heaviest one's weight, and a value some 2^20 times the others'
    hq, hkv, _, reqs = LONG[kind]
    b = Sized(hq, hkv, d, dt, page, [], reqs, seed=len(kind) + d)
    for i, n in enumerate(b.lens):
        b.light_beside_heavy(i, slice(0, None, 16))
        b.rows[i][0][5::64, :, 0] = -42 * math.log(2) * d ** 0.5 / 16
        b.rows[i][1][5::64, :, 32:64] = 60000.0
        b.write(i, torch.arange(n, device=DEV))
    b.check(b.run())


@pytest.mark.parametrize("dt,d,page", FORMS)
def test_sequences_of_different_sizes_do_not_meet(dt, d, page):
    # a sequence's values grow 2^16 times over its keys, one group of elements is 2^6 times the others, and every other sequence 16 times
    # larger: each row is held to what it sees itself
    hq, hkv, _, reqs = LONG["four rows a token"]
    b = Sized(hq, hkv, d, dt, page, [], reqs, seed=9)
    for i, n in enumerate(b.lens):
        v = b.rows[i][1].float() * torch.exp2(torch.linspace(-16, 0, n, device=DEV))[:, None, None] * (16.0 if i % 2 else 1.0)
        v[:, :, 32:64] *= 64
        b.rows[i][1] = v.to(dt)
        b.write(i, torch.arange(n, device=DEV))
    b.check(b.run())


@pytest.mark.parametrize("dt", [BF, HF])
def test_values_that_are_all_zero_and_ones_behind_them(dt):
    # keys of no value (scales of zero) weigh in the sums alone, wherever they stand
    hq, hkv, _, reqs = LONG["four rows a token"]
    b = Sized(hq, hkv, 128, dt, 64, [], reqs, seed=4)
    for i, n in enumerate(b.lens):
        at = [slice(0, n // 2), slice(n // 2, n), slice(0, n), slice(0, n, 2)][i % 4]
        b.rows[i][1][at] = 0.0
        b.write(i, torch.arange(n, device=DEV))
    got = b.run()
    b.check(got)
    for i in range(2, len(b.lens), 4):
        assert bool((got[0][i] == 0).all())


@pytest.mark.parametrize("S,n,hq,hkv,d,dt", [(128, 32768, 8, 8, 64, HF), (128, 32771, 8, 2, 128, HF), (128, 30001, 8, 8, 128, BF),
                                             (256, 20011, 8, 4, 64, BF)])
@pytest.mark.parametrize("mean", [0.0, 2.0])
def test_many_long_sequences(S, n, hq, hkv, d, dt, mean):
    # A warp's part has hundreds of pieces, of keys of about one weight.  Roundings are independent of one another and of the values: of
    # P times a scale at most 2^-11 of each term, whose squares add up to those of the values' part that has no mean, and of the result u;
    # uniform ones have a third of their bounds' squares on the mean.  32-bit sums add next to nothing.  Twice that is allowed.
    page, pages = 64, -(-n // 64)
    layout = dopr.make_cache_layout(S * pages, page, hkv, d, dt, S, pages)
    k4, v4 = dopr.cache_pools_4bit(layout)
    g = torch.Generator(DEV).manual_seed(n)
    tables = torch.randperm(S * pages, generator=g, device=DEV).view(S, pages)
    t = torch.arange(n, device=DEV)
    slots = lambda i: tables[i][t // page] * page + t % page  # noqa: E731
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    for i in range(S):
        k, v = (torch.randn(n, hkv, d, generator=g, device=DEV) for _ in range(2))
        dopr.cache_append_4bit(layout, slots(i), k.to(dt), (v + mean).to(dt), k4, v4, status=st)
    q = (torch.randn(S, hq, d, generator=g, device=DEV) / 4).to(dt)
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    plan = dopr.shared_attention_plan(layout, hq, i32(range(S + 1)), i32([n] * S), i32([-1] * S), S, status=st)
    out = dopr.shared_attention_4bit(layout, plan, q, k4, v4, i32(tables), status=st)
    assert st.item() == 0
    G, err, room = hq // hkv, 0.0, 0.0
    for i in range(0, S, 16):
        k, v = dopr.cache_read_4bit(layout, slots(i), k4, v4)
        for h in range(hkv):
            a = (q[i, h * G:h * G + G].double() @ k[:, h].double().T * d ** -0.5).softmax(-1)
            want = a @ v[:, h].double()
            u = torch.finfo(dt).eps / 2
            err += float((out[i, h * G:h * G + G].double() - want).square().sum())
            room += float((2.0 ** -22 * (a.square() @ v[:, h].double().square()) + u ** 2 * want.square()).sum()) / 3
    assert err <= 4 * room, math.sqrt(err / room)


@pytest.mark.parametrize("dt,d,page", FORMS)
@pytest.mark.parametrize("kind", ["a row a token", "four rows a token", "eight rows a token"])
def test_light_values_beside_a_heavy_key_whose_codes_are_zero(kind, dt, d, page):
    # Every second element of the heavy key's value is zero, beside others of 4; the keys around it have 2^-18 of its weight and all that there
    # is of those elements.  The heavy key has the largest product, so a key adds at most 7 2^-35 of 4 / 7.
    hq, hkv, _, reqs = LONG[kind]
    b = Sized(hq, hkv, d, dt, page, [], reqs, seed=len(kind) + d)
    for i, n in enumerate(b.lens):
        b.light_beside_heavy(i, n - 9)
        v = b.rows[i][1]
        v *= 16.0
        v[:-16] = 0.0
        v[n - 9, :, 1::2] = 4.0
        b.write(i, torch.arange(n, device=DEV))
    b.check(b.run())


@pytest.mark.parametrize("dt,d,page", FORMS)
@pytest.mark.parametrize("size", [1, 16, 256])
def test_scores_are_as_good_as_a_product_in_32_bits(size, dt, d, page):
    # A score is a sum of a head's products, exact in 32 bits, in 16 steps at most, each of which is off by a last bit of what has been
    # added up, below 2^-23 of the sum M of the magnitudes; independent of one another (half of that on the root of the mean squares): the
    # root of 16 half bits, and 2^-22 |score| of the last two products.  One key outweighs the others there, so its score is what is seen.
    # Twice that is allowed on the root mean square over the rows, beside 2^-12 of the softmax's sum in the worst row.
    hq, hkv, _, reqs = LONG["four rows a token"]
    b = Sized(hq, hkv, d, dt, page, [], reqs, seed=size)
    for i, n in enumerate(b.lens):
        b.rows[i][0] = (b.rows[i][0].float() * size ** 0.5).to(dt)
        b.write(i, torch.arange(n, device=DEV))
    b.q = (b.q.float() * 4 * size ** 0.5).to(dt)
    lse, got = b.exact()[1], b.run()[1].double()
    bound = torch.zeros_like(lse)
    for i in range(len(b.lens)):
        k = b.rows[i][0].double().repeat_interleave(hq // hkv, 1)
        a = torch.einsum("hd,khd->hk", b.q[i].double(), k) * d ** -0.5
        at = a.argmax(-1)
        M = (b.q[i].double().abs() * k[at, torch.arange(hq, device=DEV)].abs()).sum(-1) * d ** -0.5
        bound[i] = M * 4 * 2.0 ** -24 + a.amax(-1).abs() * 2.0 ** -22 + 2.0 ** -20
    err = (got - lse).abs()
    assert float(err.square().mean().sqrt()) <= 2 * float(bound.square().mean().sqrt()), float(err.square().mean().sqrt() / bound.square().mean().sqrt())
    assert bool((err <= 2.0 ** -12 + 8 * bound).all()), float((err / bound).max())
