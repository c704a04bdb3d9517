"""Refusals of the head norms' and the 4-bit cache's C entry points: host arguments are checked before any device work, so none
of these needs a GPU (device pointers are never followed)."""
import ctypes

import pytest
import torch

from paper_2609_03311_gb300 import build as libbuild
from paper_2609_03311_gb300 import dopr

P = ctypes.c_void_p(4096)  # stands for a device buffer
ODD, FOUR, EIGHT = ctypes.c_void_p(4097), ctypes.c_void_p(4100), ctypes.c_void_p(4104)
F16, BF16, F32 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return dopr.load()


def layout(**kw):
    a = dict(n_blocks=8, page=64, n_kv_heads=2, head_dim=128, dtype=torch.bfloat16, n_seqs=3, max_blocks=4)
    a.update(kw)
    return dopr.make_cache_layout(**a)


def heads(data=4096, tok=512, head=128, n=4):
    return ctypes.byref(dopr.Heads(data, tok, head, n))


def norm(**kw):
    a = dict(rope=None, dtype=BF16, D=128, T=4, pos=None, eps=1e-6, gd=F32, q=heads(), qg=P, qo=heads(), k=heads(n=2), kg=P,
             ko=heads(n=2), st=None)
    a.update(kw)
    return [a[x] for x in ("rope", "dtype", "D", "T", "pos", "eps", "gd", "q", "qg", "qo", "k", "kg", "ko", "st")] + [None]


BAD = [(dict(dtype=3), dopr.ERR_INVALID_ARG), (dict(T=-1), dopr.ERR_INVALID_ARG), (dict(D=127), dopr.ERR_UNSUPPORTED),
       (dict(D=258), dopr.ERR_UNSUPPORTED), (dict(D=0), dopr.ERR_UNSUPPORTED), (dict(eps=0.0), dopr.ERR_INVALID_ARG),
       (dict(eps=-1.0), dopr.ERR_INVALID_ARG), (dict(eps=float("nan")), dopr.ERR_INVALID_ARG),
       (dict(eps=float("inf")), dopr.ERR_INVALID_ARG), (dict(gd=3), dopr.ERR_INVALID_ARG), (dict(qg=ODD), dopr.ERR_INVALID_ARG),
       (dict(kg=ctypes.c_void_p(4098)), dopr.ERR_INVALID_ARG), (dict(k=None), dopr.ERR_INVALID_ARG),
       (dict(q=None), dopr.ERR_INVALID_ARG), (dict(qo=None), dopr.ERR_INVALID_ARG), (dict(qo=heads(n=3)), dopr.ERR_INVALID_ARG),
       (dict(q=heads(data=4097)), dopr.ERR_INVALID_ARG), (dict(q=heads(tok=-1)), dopr.ERR_INVALID_ARG),
       (dict(q=heads(head=64)), dopr.ERR_INVALID_ARG), (dict(qo=heads(tok=256)), dopr.ERR_INVALID_ARG),
       (dict(ko=heads(tok=0, n=2)), dopr.ERR_INVALID_ARG), (dict(st=ODD), dopr.ERR_INVALID_ARG)]


@pytest.mark.parametrize("kw,status", BAD)
def test_bad_norms_are_refused(lib, kw, status):
    assert lib.dopr_head_norm_rope(*norm(**kw)) == status
    assert lib.dopr_last_error()


def back(**kw):
    a = dict(rope=None, dtype=BF16, D=128, T=4, pos=None, eps=1e-6, gd=F32, dqo=heads(), q=heads(), qg=P, dq=heads(), dqg=P,
             dko=heads(n=2), k=heads(n=2), kg=P, dk=heads(n=2), dkg=P, ws=P, st=None)
    a.update(kw)
    names = ("rope", "dtype", "D", "T", "pos", "eps", "gd", "dqo", "q", "qg", "dq", "dqg", "dko", "k", "kg", "dk", "dkg", "ws", "st")
    return [a[x] for x in names] + [None]


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=-1), dopr.ERR_INVALID_ARG), (dict(T=-1), dopr.ERR_INVALID_ARG), (dict(D=130 + 128), dopr.ERR_UNSUPPORTED),
    (dict(eps=0.0), dopr.ERR_INVALID_ARG), (dict(dqo=None), dopr.ERR_INVALID_ARG), (dict(dqo=heads(n=2)), dopr.ERR_INVALID_ARG),
    (dict(dq=heads(n=2)), dopr.ERR_INVALID_ARG), (dict(dq=heads(tok=256)), dopr.ERR_INVALID_ARG), (dict(dk=None), dopr.ERR_INVALID_ARG),
    (dict(dko=None), dopr.ERR_INVALID_ARG), (dict(k=None, dko=None, dk=None), dopr.ERR_INVALID_ARG),  # dk_gain is left
    (dict(ws=None), dopr.ERR_INVALID_ARG), (dict(ws=EIGHT), dopr.ERR_INVALID_ARG), (dict(dqg=ctypes.c_void_p(4098)), dopr.ERR_INVALID_ARG),
    (dict(dkg=ctypes.c_void_p(4098)), dopr.ERR_INVALID_ARG), (dict(gd=7), dopr.ERR_INVALID_ARG)])
def test_bad_gradients_are_refused(lib, kw, status):
    assert lib.dopr_head_norm_rope_backward(*back(**kw)) == status
    assert lib.dopr_last_error()


def test_no_rows_are_no_work(lib):
    assert lib.dopr_head_norm_rope(*norm(T=0, q=None, qo=None, k=None, ko=None)) == dopr.OK
    l = ctypes.byref(layout())
    assert lib.dopr_cache_append_4bit(l, None, 0, None, None, 0.0, 0, None, None, None, None, None, None, None, None, None, None) == dopr.OK
    assert lib.dopr_cache_read_4bit(l, 0, None, None, None, None, None, None, None) == dopr.OK


def test_workspaces_and_pools_have_their_sizes(lib):
    assert lib.dopr_head_norm_rope_workspace(128) > 0
    assert lib.dopr_head_norm_rope_workspace(127) == -1 and lib.dopr_head_norm_rope_workspace(0) == -1
    # 4.25 bits an element
    assert lib.dopr_cache_4bit_pool_bytes(ctypes.byref(layout())) == 8 * 2 * 64 * (64 + 4)
    assert lib.dopr_cache_4bit_pool_bytes(ctypes.byref(layout(head_dim=64, page=16))) == 8 * 2 * 16 * (32 + 2)
    k, v = dopr.cache_pools_4bit(layout(), "cpu")
    assert k.shape == (8, 2, 64 * 68) and v.shape == k.shape and not k.any()


BAD_LAYOUTS = [(dict(n_blocks=0), dopr.ERR_INVALID_ARG), (dict(page=48), dopr.ERR_UNSUPPORTED), (dict(head_dim=96), dopr.ERR_UNSUPPORTED),
               (dict(dtype=torch.float32), dopr.ERR_UNSUPPORTED), (dict(n_blocks=2 ** 26, page=32), dopr.ERR_UNSUPPORTED)]


def append(**kw):
    a = dict(l=ctypes.byref(layout()), rope=None, T=4, pos=None, slots=P, eps=1e-6, gd=F32, q=heads(), qg=P, qo=heads(), k=heads(n=2),
             kg=P, v=heads(n=2), kp=P, vp=P, st=None)
    a.update(kw)
    return [a[x] for x in ("l", "rope", "T", "pos", "slots", "eps", "gd", "q", "qg", "qo", "k", "kg", "v", "kp", "vp", "st")] + [None]


def read(**kw):
    a = dict(l=ctypes.byref(layout()), T=4, slots=P, kp=P, vp=P, ko=heads(n=2), vo=heads(n=2), st=None)
    a.update(kw)
    return [a[x] for x in ("l", "T", "slots", "kp", "vp", "ko", "vo", "st")] + [None]


@pytest.mark.parametrize("kw,status", BAD_LAYOUTS)
def test_bad_layouts_are_refused(lib, kw, status):
    l = ctypes.byref(layout(**kw))
    assert lib.dopr_cache_4bit_pool_bytes(l) == -1
    assert lib.dopr_cache_append_4bit(*append(l=l)) == status
    assert lib.dopr_cache_read_4bit(*read(l=l)) == status
    assert lib.dopr_last_error()


@pytest.mark.parametrize("kw", [
    dict(T=-1), dict(slots=None), dict(slots=FOUR), dict(kp=None), dict(vp=None), dict(kp=EIGHT), dict(vp=EIGHT), dict(k=None),
    dict(v=None), dict(k=heads()), dict(v=heads(n=1)), dict(q=None), dict(qo=None), dict(qo=heads(n=2)), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=0.0),  # gains without a norm
    dict(eps=0.0, qg=None, kg=None),  # q without norm and rope
    dict(q=heads(data=4104)), dict(k=heads(data=4104, n=2)), dict(v=heads(tok=516, n=2)), dict(qo=heads(tok=256)), dict(st=ODD),
    dict(qg=ODD), dict(gd=5)])
def test_bad_appends_are_refused(lib, kw):
    assert lib.dopr_cache_append_4bit(*append(**kw)) == dopr.ERR_INVALID_ARG
    assert lib.dopr_last_error()


@pytest.mark.parametrize("kw", [dict(T=-1), dict(slots=None), dict(slots=FOUR), dict(kp=None), dict(vp=EIGHT), dict(ko=None), dict(vo=None),
                                dict(ko=heads(n=4)), dict(vo=heads(tok=128, n=2)), dict(ko=heads(data=4104, n=2)), dict(st=ODD)])
def test_bad_reads_are_refused(lib, kw):
    assert lib.dopr_cache_read_4bit(*read(**kw)) == dopr.ERR_INVALID_ARG
    assert lib.dopr_last_error()


def test_the_binding_takes_device_tensors_and_open_tables_only(lib):
    x, s = torch.zeros(4, 2, 128, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    pool = torch.zeros(8 * 2 * 64 * 68, dtype=torch.uint8)
    for call in (lambda: dopr.head_norm_rope(x), lambda: dopr.head_norm_rope_backward(x, x),
                 lambda: dopr.cache_append_4bit(layout(), s, x, x, pool, pool), lambda: dopr.cache_read_4bit(layout(), s, pool, pool)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    rope = dopr.Rope.__new__(dopr.Rope)
    rope._h = ctypes.c_void_p()
    for call in (lambda: dopr.head_norm_rope(x, rope=rope, positions=s.int()), lambda: dopr.head_norm_rope_backward(x, x, rope=rope),
                 lambda: dopr.cache_append_4bit(layout(), s, x, x, pool, pool, rope=rope)):
        with pytest.raises(ValueError, match="closed"):
            call()
    with pytest.raises(ValueError):
        dopr.head_norm_rope(x.long())


def attention(**kw):
    a = dict(l=ctypes.byref(layout()), plan=P, T=4, q=heads(), kp=P, vp=P, tables=P, scale=0.1, out=heads(), lse=None, ws=P, st=None)
    a.update(kw)
    return [a[x] for x in ("l", "plan", "T", "q", "kp", "vp", "tables", "scale", "out", "lse", "ws", "st")] + [None]


@pytest.mark.parametrize("kw,status", [
    (dict(plan=None), 1), (dict(q=None), 1), (dict(kp=None), 1), (dict(vp=None), 1), (dict(tables=None), 1), (dict(out=None), 1),
    (dict(ws=None), 1), (dict(T=-1), 1), (dict(T=2 ** 30), dopr.ERR_UNSUPPORTED), (dict(q=heads(n=3)), dopr.ERR_UNSUPPORTED),
    (dict(out=heads(n=2)), 1), (dict(q=heads(data=4104)), 1), (dict(out=heads(tok=128)), 1), (dict(scale=0.0), 1),
    (dict(scale=float("inf")), 1), (dict(kp=EIGHT), 1), (dict(ws=ctypes.c_void_p(4112)), 1), (dict(plan=EIGHT), 1), (dict(lse=ODD), 1),
    (dict(l=ctypes.byref(layout(head_dim=96))), dopr.ERR_UNSUPPORTED)])
def test_bad_attention_over_4_bits_is_refused(lib, kw, status):
    assert lib.dopr_shared_attention_4bit(*attention(**kw)) == status
    assert lib.dopr_last_error()
