"""Refusals of the paged prefix cache's C entry points: host arguments are checked before any device work, so none of
these needs a GPU (device pointers are never followed)."""
import ctypes

import pytest
import torch

from paper_2609_03311_gb300 import build as libbuild
from paper_2609_03311_gb300 import dopr

P = ctypes.c_void_p(4096)  # stands for a device buffer


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


BAD_LAYOUTS = [(dict(n_blocks=0), dopr.ERR_INVALID_ARG), (dict(n_kv_heads=-1), dopr.ERR_INVALID_ARG),
               (dict(n_seqs=0), dopr.ERR_INVALID_ARG), (dict(max_blocks=0), dopr.ERR_INVALID_ARG),
               (dict(page=48), dopr.ERR_UNSUPPORTED), (dict(page=256), dopr.ERR_UNSUPPORTED),
               (dict(head_dim=96), dopr.ERR_UNSUPPORTED), (dict(dtype=torch.float32), dopr.ERR_UNSUPPORTED),
               (dict(n_seqs=16385), dopr.ERR_UNSUPPORTED), (dict(max_blocks=2 ** 26, page=64), dopr.ERR_UNSUPPORTED),
               (dict(n_blocks=2 ** 26, page=32), dopr.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", BAD_LAYOUTS)
def test_bad_layouts_are_refused_by_every_call(lib, kw, status):
    l = ctypes.byref(layout(**kw))
    assert lib.dopr_cache_extend_workspace(l) == -1
    assert lib.dopr_shared_attention_plan_bytes(l, 8, 4) == -1
    assert lib.dopr_shared_attention_workspace(l, 8, 4) == -1
    assert lib.dopr_cache_extend(l, P, P, P, P, None, P, 4, P, P, P, P, P, P, None, None) == status
    assert lib.dopr_cache_append(l, None, 1, None, P, None, None, heads(n=2), heads(n=2), P, P, None, None) == status
    assert lib.dopr_shared_attention_plan(l, 8, 4, P, P, None, P, None, None) == status
    assert lib.dopr_shared_attention(l, P, 4, heads(), P, P, P, 0.1, heads(), None, P, None, None) == status
    assert lib.dopr_last_error()


def test_null_layouts_and_pointers_are_refused(lib):
    assert lib.dopr_cache_extend_workspace(None) == -1
    l = ctypes.byref(layout())
    good = [l, P, P, P, P, None, P, 4, P, P, P, P, P, P, None, None]
    for i in (0, 1, 2, 3, 4, 6, 8, 9, 10, 11, 12, 13):
        a = list(good)
        a[i] = None
        assert lib.dopr_cache_extend(*a) == dopr.ERR_INVALID_ARG, i
    a = list(good)
    a[7] = -1
    assert lib.dopr_cache_extend(*a) == dopr.ERR_INVALID_ARG
    a = list(good)
    a[13] = ctypes.c_void_p(4100)  # the workspace, not 16-byte aligned
    assert lib.dopr_cache_extend(*a) == dopr.ERR_INVALID_ARG
    for i in (3, 4, 6):
        a = [l, 8, 4, P, P, None, P, None, None]
        a[i] = None
        assert lib.dopr_shared_attention_plan(*a) == dopr.ERR_INVALID_ARG, i
    for i in (1, 3, 4, 5, 6, 8, 10):
        a = [l, P, 4, heads(), P, P, P, 0.1, heads(), None, P, None, None]
        a[i] = None
        assert lib.dopr_shared_attention(*a) == dopr.ERR_INVALID_ARG, i
    for i in (4, 7, 8, 9, 10):
        a = [l, None, 1, None, P, None, None, heads(n=2), heads(n=2), P, P, None, None]
        a[i] = None
        assert lib.dopr_cache_append(*a) == dopr.ERR_INVALID_ARG, i


@pytest.mark.parametrize("bad,status", [
    (dict(q=heads(n=3)), dopr.ERR_UNSUPPORTED),            # 3 q heads on 2 kv heads
    (dict(q=heads(n=2 * 65)), dopr.ERR_UNSUPPORTED),       # 65 q heads a kv head
    (dict(out=heads(n=2)), dopr.ERR_INVALID_ARG),          # heads differ
    (dict(q=heads(data=4104)), dopr.ERR_INVALID_ARG),      # 8-byte aligned
    (dict(q=heads(tok=516)), dopr.ERR_INVALID_ARG),        # a stride of 1,032 bytes
    (dict(out=heads(head=64)), dopr.ERR_INVALID_ARG),      # heads overlap
    (dict(out=heads(tok=-512)), dopr.ERR_INVALID_ARG),
    (dict(scale=0.0), dopr.ERR_INVALID_ARG),
    (dict(scale=float("nan")), dopr.ERR_INVALID_ARG),
    (dict(scale=float("inf")), dopr.ERR_INVALID_ARG),
    (dict(pool=ctypes.c_void_p(4104)), dopr.ERR_INVALID_ARG),
    (dict(tokens=-1), dopr.ERR_INVALID_ARG),
    (dict(tokens=2 ** 30), dopr.ERR_UNSUPPORTED),
])
def test_bad_attention_arguments_are_refused(lib, bad, status):
    a = dict(q=heads(), out=heads(), scale=0.1, pool=P, tokens=4)
    a.update(bad)
    assert lib.dopr_shared_attention(ctypes.byref(layout()), P, a["tokens"], a["q"], a["pool"], P, P, a["scale"], a["out"],
                                     None, P, None, None) == status
    assert lib.dopr_last_error()


@pytest.mark.parametrize("plan,workspace", [(4104, 4096), (4096, 4112), (4096, 4100)])
def test_misaligned_plans_and_workspaces_are_refused(lib, plan, workspace):
    # a plan by 16 bytes, a workspace by 32
    assert lib.dopr_shared_attention(ctypes.byref(layout()), ctypes.c_void_p(plan), 4, heads(), P, P, P, 0.1, heads(), None,
                                     ctypes.c_void_p(workspace), None, None) == dopr.ERR_INVALID_ARG
    assert lib.dopr_last_error()


@pytest.mark.parametrize("bad,status", [
    (dict(max_position=0), dopr.ERR_INVALID_ARG), (dict(rotary_dim=0), dopr.ERR_INVALID_ARG),
    (dict(rotary_dim=63), dopr.ERR_UNSUPPORTED), (dict(rotary_dim=258), dopr.ERR_UNSUPPORTED),
    (dict(max_position=2 ** 22 + 1), dopr.ERR_UNSUPPORTED), (dict(layout=2), dopr.ERR_INVALID_ARG),
    (dict(scaling=5), dopr.ERR_INVALID_ARG), (dict(theta=1.0), dopr.ERR_INVALID_ARG),
    (dict(theta=float("nan")), dopr.ERR_INVALID_ARG), (dict(scaling=1, factor=0.5), dopr.ERR_INVALID_ARG),
    (dict(scaling=2, factor=float("inf")), dopr.ERR_INVALID_ARG),
    (dict(scaling=2, factor=2.0, rotary_dim=2), dopr.ERR_INVALID_ARG),
    (dict(scaling=3, factor=2.0), dopr.ERR_INVALID_ARG),  # no original_max_position
    (dict(scaling=4, factor=2.0, original_max_position=100, low=4.0, high=1.0), dopr.ERR_INVALID_ARG),
    (dict(scaling=4, factor=2.0, original_max_position=100, attention_factor=-1.0), dopr.ERR_INVALID_ARG),
])
def test_bad_rotary_tables_are_refused(lib, bad, status):
    a = dict(max_position=16, rotary_dim=64)
    a.update(bad)
    with pytest.raises(dopr.DoprError) as e:
        dopr.Rope(**a)
    assert e.value.status == status
    assert lib.dopr_rope_create(None, ctypes.byref(ctypes.c_void_p())) == dopr.ERR_INVALID_ARG
    assert lib.dopr_rope_create(ctypes.byref(dopr.RopeConfig()), None) == dopr.ERR_INVALID_ARG
    assert lib.dopr_rope_destroy(None) == dopr.OK


def test_the_binding_takes_device_tensors_only(lib):
    l = layout()
    z = torch.zeros(64, dtype=torch.int32)
    with pytest.raises(ValueError):
        dopr.cache_extend(l, z, z, z, z, z, 4)
    with pytest.raises(ValueError):
        dopr.shared_attention_plan(l, 8, z, z, z, 4)
    with pytest.raises(ValueError):
        dopr.shared_attention(l, z, torch.zeros(4, 4, 128, dtype=torch.bfloat16), z, z, z)


def test_workspace_and_plan_sizes_grow_with_their_work(lib):
    l = ctypes.byref(layout())
    assert lib.dopr_cache_extend_workspace(l) >= 3 * 3 * 4
    sizes = [lib.dopr_shared_attention_plan_bytes(l, 8, t) for t in (0, 1, 64, 1000)]
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_the_binding_refuses_a_closed_rotary_table(lib):
    # its handle is NULL, with which the library would store keys as they are
    rope = dopr.Rope.__new__(dopr.Rope)
    rope._h = ctypes.c_void_p()
    x, pos = torch.zeros(4, 2, 128, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    pool = torch.zeros(8, 2, 64, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="closed"):
        dopr.cache_append(layout(), pos.long(), x, x, pool, pool, rope=rope, positions=pos)
    with pytest.raises(ValueError, match="closed"):
        dopr.rope_apply(rope, pos, x)
    rope.close()


def test_buffers_that_are_not_aligned_to_their_type_are_refused(lib):
    # a kernel's access to one would fault
    l, odd, four = ctypes.byref(layout()), ctypes.c_void_p(4098), ctypes.c_void_p(4100)
    good = [l, P, P, P, P, None, P, 4, P, P, P, P, P, P, None, None]
    for i in (1, 2, 3, 4, 5, 6, 8, 9, 10, 11, 12, 13, 14):
        a = list(good)
        a[i] = odd
        assert lib.dopr_cache_extend(*a) == dopr.ERR_INVALID_ARG, i
    a = list(good)
    a[11] = four  # slots, 64-bit
    assert lib.dopr_cache_extend(*a) == dopr.ERR_INVALID_ARG
    for i in (3, 4, 5, 6, 7):
        a = [l, 8, 4, P, P, None, P, None, None]
        a[i] = odd
        assert lib.dopr_shared_attention_plan(*a) == dopr.ERR_INVALID_ARG, i
    for i in (6, 9, 11):
        a = [l, P, 4, heads(), P, P, P, 0.1, heads(), None, P, None, None]
        a[i] = odd
        assert lib.dopr_shared_attention(*a) == dopr.ERR_INVALID_ARG, i
    for i, p in ((4, odd), (4, four), (11, odd)):
        a = [l, None, 1, None, P, None, None, heads(n=2), heads(n=2), P, P, None, None]
        a[i] = p
        assert lib.dopr_cache_append(*a) == dopr.ERR_INVALID_ARG, i
    assert b"aligned" in lib.dopr_last_error()


@pytest.mark.parametrize("tok,head,n,tokens,good", [
    (512, 128, 4, 4, True), (128, 512, 4, 4, True), (128, 520, 4, 4, True), (640, 160, 4, 9, True), (512, 0, 1, 4, True), (128, 0, 1, 4, True), (0, 0, 1, 4, False),
    (0, 128, 4, 4, False), (0, 128, 4, 1, True), (128, 128, 4, 4, False), (384, 128, 4, 4, False), (504, 128, 4, 4, False),
    (128, 504, 4, 4, False), (128, 512, 4, 5, False), (64, 512, 4, 2, False), (120, 512, 4, 2, False), (2 ** 40, 2 ** 60, 4, 4, True),
    (2 ** 40, 2 ** 40, 4, 4, False)])
def test_outputs_whose_rows_overlap_are_refused(lib, tok, head, n, tokens, good):
    # rows of 128 elements.  The workspace is misaligned, which is looked at last: nothing gets as far as a launch
    l, q = layout(n_kv_heads=1), heads(n=n)
    assert lib.dopr_shared_attention(ctypes.byref(l), P, tokens, q, P, P, P, 0.1, heads(tok=tok, head=head, n=n), None,
                                     ctypes.c_void_p(4096 + 16), None, None) == dopr.ERR_INVALID_ARG
    assert (b"workspace" if good else b"overlap") in lib.dopr_last_error()
