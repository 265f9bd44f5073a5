"""Copies of a rotation (no GPU needed: the handle is host memory)."""
import copy
import gc
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
