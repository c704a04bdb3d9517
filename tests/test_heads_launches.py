"""Rules of the launches of norms of heads and of the 4-bit cache, checked on the CUDA sources (no GPU needed)."""
import re

import pytest

from test_dependent_launches import _kernels, _source

HEADS = {"k_head_norm", "k_append_4bit", "k_head_norm_back", "k_head_norm_gains", "k_read_4bit"}


def test_the_kernels_are_those_that_are_known_here():
    assert {k for k, _, _ in _kernels(_source("k_head_norm.cu"))} == HEADS
    assert {k for k, _, _ in _kernels(_source("k_shared_attn_4bit.cu"))} == {"k_shared_attn_4bit"}


@pytest.mark.parametrize("name", sorted(HEADS))
def test_nothing_is_read_before_the_wait(name):
    body = {k: b for k, _, b in _kernels(_source("k_head_norm.cu"))}[name]
    assert body.count("pdl_wait()") == 1 and body.count("pdl_trigger()") == 1
    before = body[:body.index("pdl_wait()")]
    assert "pdl_trigger()" not in before and "return" not in before
    for read in (r"\ba\.\w+\s*\[", r"\bws\s*\[", r"gain_at\(", r"__ldg\(", r"\bStream\b.*\(", r"\bWalk<", r"\*reinterpret_cast"):
        assert not re.search(read, re.sub(r"using S = [^;]*;", "", before)), read


def test_all_of_them_are_launched_dependent():
    text = _source("k_head_norm.cu")
    assert "<<<" not in text and "launch_ordinary" not in text
    for name in HEADS:
        assert re.search(r"launch_dependent\(%s\b" % name, text), name


def test_the_attention_is_an_ordinary_launch_ahead_of_the_join():
    text = _source("k_shared_attn_4bit.cu")
    body = next(b for _, _, b in _kernels(text))
    assert body.count("pdl_trigger()") == 1 and "pdl_wait" not in body
    assert "<<<" not in text and "launch_dependent" not in text
    assert text.index("launch_ordinary(k_shared_attn_4bit<T, D>") < text.index("launch_shared_join(")


def test_both_warps_that_expand_free_each_stage_of_the_raw_rings():
    # a stage is freed by two arrivals, one a warp; a wait by parity holds only for a warp that passes each of a stage's phases
    text = _source("shared_attn_device.cuh")
    body = text[text.index("void expand_4bit("):]
    body = body[:body.index("template <typename T, int D, bool FOUR>")]
    assert body.count("raw.next(raw_stages)") == 1 and body.count("L::RAW_EMPTY") == 1 and "part)" not in body.split("raw.next")[1]
    assert re.search(r"i >= L::RAW_EMPTY\) \? 2", text)
