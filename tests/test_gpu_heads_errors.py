"""What device errors of the head norms and of the append that norms and turns leave behind, on a GPU: bad rows are left as they were
and reported, the others get what they get without them.

Pages are compared byte for byte with the definition (tests/test_gpu_heads.py) of the rows that dopr.head_norm_rope gives, gradients
with the 64-bit formula at that file's tolerances."""
import pytest
import torch

from paper_2609_03311_gb300 import dopr
from test_gpu_heads import BLOCKS, EPS, backward64, gain, make, near, pools, put, rows, slots_of, word

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,hq,hkv,D,rotary,view", [(9, 4, 2, 128, 128, "qkv"), (700, 16, 8, 64, 32, "heads"), (41, 3, 1, 34, 10, "off")])
def test_gradients_of_rows_without_a_position_are_left(T, hq, hkv, D, rotary, view, dt):
    q, k = rows(T, hq, hkv, D, dt, seed=T, layout=view)
    dz, dzk = rows(T, hq, hkv, D, dt, seed=T + 1)
    rope, pos = make(T, D, rotary, far=100)
    skipped = torch.zeros(T, dtype=torch.bool, device=DEV)
    for i, p in ((0, -1), (2, 100), (T // 2, -7), (T - 1, 2 ** 31 - 1)):
        pos[i], skipped[i] = p, True
    g = gain(D, torch.float32, 1)
    dq, dk = torch.full((T, hq, D), 3.0, device=DEV, dtype=dt), torch.full((T, hkv, D), 3.0, device=DEV, dtype=dt)
    st = word()
    _, _, dqg, dkg = dopr.head_norm_rope_backward(dz, q, dzk, k, g, g, rope=rope, positions=pos, dq=dq, dk=dk, status=st)
    assert st.item() == dopr.ERR_INVALID_ARG
    for got, gg, x, d in ((dq, dqg, q, dz), (dk, dkg, k, dzk)):
        assert bool((got[skipped] == 3.0).all())
        dx, bound, dg, dg_bound = backward64(d[~skipped], x[~skipped], g, pos[~skipped], rope)
        near(got[~skipped], dx, bound, 84, "dx")
        near(gg, dg, dg_bound, 24 + -(-T // BLOCKS) * -(-(hq + hkv) // 4) + 145, "gain")
    # in place, and without any bad position: rows without one are no error
    pos[2], pos[T - 1] = -1, -1
    st.zero_()
    a, b = dz.clone(), dzk.clone()
    dopr.head_norm_rope_backward(a, q, b, k, g, g, rope=rope, positions=pos, dq=a, dk=b, status=st)
    assert st.item() == 0 and torch.equal(a[skipped], dz[skipped]) and torch.equal(b[skipped], dzk[skipped])
    assert torch.equal(a[~skipped], dq[~skipped]) and torch.equal(b[~skipped], dk[~skipped])


class Fused:
    """Rows for an append that norms and turns, the pools and outputs before it, and what it has to leave there."""

    def __init__(self, dt, D, inter, T=60, hq=6, hkv=3, page=16, rotary=None):
        self.dt, self.D, self.page, self.T, self.hkv = dt, D, page, T, hkv
        self.layout = dopr.make_cache_layout(T // page + 2, page, hkv, D, dt, 1, T // page + 2)
        self.n_slots = self.layout.n_blocks * page
        q, k = rows(T, hq, hkv, D, dt, seed=D)
        self.q, self.k, self.v = q.clone(), k.clone(), k.flip(0).contiguous()
        self.rope, self.pos = make(T, D, rotary or D, dopr.ROPE_INTERLEAVED if inter else dopr.ROPE_HALF, far=1000)
        self.qg, self.kg = gain(D, torch.bfloat16, 1), gain(D, torch.float32, 2).to(torch.bfloat16)
        self.slots = slots_of(T, self.n_slots)
        self.q_out = torch.full((T, hq, D), 3.0, device=DEV, dtype=dt)

    def check(self, want, left=(), unstored=()):
        """left: rows of which nothing may be written; unstored: rows that only q is written of."""
        kp, vp = pools(self.layout, 3)
        pos = self.pos.clone()
        pos[list(left)] = -1
        q, k = torch.full_like(self.q_out, 3.0), torch.zeros(self.T, self.hkv, self.D, device=DEV, dtype=self.dt)
        dopr.head_norm_rope(self.q, self.k, self.qg, self.kg, eps=EPS, rope=self.rope, positions=pos, q_out=q, k_out=k)
        slots = self.slots.clone()
        slots[list(left) + list(unstored)] = -1
        k_want, v_want = put(kp, self.page, self.D, slots, k), put(vp, self.page, self.D, slots, self.v)
        st = word()
        dopr.cache_append_4bit(self.layout, self.slots, self.k, self.v, kp, vp, k_gain=self.kg, eps=EPS, rope=self.rope,
                               positions=self.pos, q=self.q, q_gain=self.qg, q_out=self.q_out, status=st)
        assert st.item() == want
        assert torch.equal(kp, k_want) and torch.equal(vp, v_want)
        assert torch.equal(torch.nan_to_num(self.q_out, nan=-5.0), torch.nan_to_num(q, nan=-5.0))
        assert bool((self.q_out[list(left)] == 3.0).all())


KINDS = [(torch.float16, 128, False), (torch.bfloat16, 128, True), (torch.bfloat16, 64, False), (torch.float16, 64, True)]


@pytest.mark.parametrize("dt,D,inter", KINDS)
def test_bad_slots_of_an_append_that_norms_leave_their_rows(dt, D, inter):
    f = Fused(dt, D, inter)
    f.slots[0], f.slots[31], f.slots[59] = f.n_slots, 2 ** 40, 2 ** 63 - 1
    f.slots[7], f.pos[9] = -1, -1
    f.check(dopr.ERR_INVALID_ARG, left=(0, 31, 59, 9), unstored=(7,))


@pytest.mark.parametrize("dt,D,inter", KINDS)
def test_bad_positions_of_an_append_that_norms_leave_their_rows(dt, D, inter):
    f = Fused(dt, D, inter, rotary=32)
    f.pos[0], f.pos[30], f.pos[59] = 1000, 2 ** 31 - 1, 5000
    f.check(dopr.ERR_INVALID_ARG, left=(0, 30, 59))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dt,D,inter", KINDS)
def test_bad_numbers_of_an_append_that_norms_are_nan_and_an_error(dt, D, inter, bad):
    f = Fused(dt, D, inter)
    f.k[4, 1, 40], f.v[50, 2, 7] = bad, bad
    f.check(dopr.ERR_RANGE)


@pytest.mark.parametrize("dt,D,inter", KINDS)
def test_bad_queries_of_an_append_that_norms_are_no_error(dt, D, inter):
    f = Fused(dt, D, inter)
    f.q[4, 1, 40] = float("nan")
    f.check(0)


@pytest.mark.parametrize("dt,D,inter", KINDS)
def test_normed_keys_beyond_the_range_are_nan_and_an_error(dt, D, inter):
    # finite keys whose normed values are not fp16's, or more than pages hold: one head of a row has all of its weight in one element
    f = Fused(dt, D, inter)
    f.kg[3] = 65536.0
    f.k[11, 0] = 0.0
    f.k[11, 0, 3] = 1.0
    f.check(dopr.ERR_RANGE)
    # and what is just held: half the range and less
    f = Fused(dt, D, inter)
    f.kg[:] = 65504.0 / 2 / D ** 0.5
    f.check(0)


@pytest.mark.parametrize("dt,D", [(torch.float16, 128), (torch.bfloat16, 64)])
def test_an_append_that_only_turns_leaves_bad_rows(dt, D):
    f = Fused(dt, D, False)
    f.pos[5], f.slots[8], f.k[20, 0, 0], f.pos[30] = 1000, f.n_slots, float("nan"), -1
    kp, vp = pools(f.layout, 3)
    q, k = f.q_out.clone(), f.k.clone()
    slots, pos = f.slots.clone(), f.pos.clone()
    slots[[5, 8, 30]], pos[[5, 8, 30]] = -1, -1
    dopr.rope_apply(f.rope, pos, f.q, f.k, q_out=q, k_out=k)
    want = put(kp, f.page, D, slots, k), put(vp, f.page, D, slots, f.v)
    st = word()
    dopr.cache_append_4bit(f.layout, f.slots, f.k, f.v, kp, vp, rope=f.rope, positions=f.pos, q=f.q, q_out=f.q_out, status=st)
    assert st.item() in (dopr.ERR_INVALID_ARG, dopr.ERR_RANGE)
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1]) and torch.equal(f.q_out, q)
