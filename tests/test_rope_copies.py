"""Copies and settings of a rotation (no GPU needed: the handle is host memory)."""
import copy
import gc
import math
import pickle

import pytest


@pytest.mark.parametrize("make", [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r)), lambda r: copy.deepcopy({"layer": [r]})["layer"][0]])
def test_copies_have_their_own_handle(make):
    """Each destroys its own: the other goes on working."""
    from paper_2607_27692_b200 import build, paged
    build.build()
    rope = paged.Rope(128, 64, base=500000.0, interleaved=True, scaling="yarn", factor=4.0, original_len=8192, beta_fast=16.0, attn_factor=1.5)
    want = rope.frequencies()
    other = make(rope)
    assert type(other) is paged.Rope and other.h != rope.h
    assert other.frequencies() == want and (other.d, other.rot_dim) == (rope.d, rope.rot_dim)
    rope.close()
    del rope
    gc.collect()
    assert other.frequencies() == want
    again = make(other)
    del other
    gc.collect()
    assert again.frequencies() == want
    again.close()
    with pytest.raises(paged._rt.RetopkError):
        make(again)


@pytest.mark.parametrize("factor", [1.1e30, 1e39, 1e300, math.inf, math.nan, -0.1])
def test_factors_on_cosine_and_sine_that_fp32_does_not_hold(factor):
    """The kernels hold cosine and sine times the factor in fp32: beyond it 0 would have turned to NaN."""
    from paper_2607_27692_b200 import build, paged
    build.build()
    with pytest.raises(paged._rt.RetopkError):
        paged.Rope(64, attn_factor=factor)
    assert paged.Rope(64, attn_factor=1e30).frequencies()[1] == 1e30
