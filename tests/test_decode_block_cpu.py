"""What a decoder block takes unless told otherwise: rows in front of the projections as bf16 (codes of 8 bits are turned back into bf16 by
the product, cost four mantissa bits and save no time)."""
import inspect

import pytest

import paper_2604_23108_amd as M
from paper_2604_23108_amd.decode_block import DecodeBlock, random_block


def test_rows_are_bf16_by_default():
    for f in (DecodeBlock.__init__, random_block):
        assert inspect.signature(f).parameters["norm_8bit"].default is False


@pytest.mark.gpu
def test_types_of_the_rows():
    for kw, dtype in (({}, M.BF16), (dict(norm_8bit=True), M.E4M3)):
        block = random_block(2, longest=64, **kw)
        assert block.attention_norm.cfg.y_dtype == block.qkv.cfg.x_dtype == dtype
