"""The decoding example end to end: packed linears, the 4-bit cache written from slices of the stacked projection, attention over it, steps replayed from a graph."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("decode_with_4bit_cache", os.path.join(ROOT, "examples", "decode_with_4bit_cache.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_prompts_then_tokens_through_two_layers():
    ex = load()
    args = ex.parser().parse_args("--layers 2 --hidden 512 --inter 1024 --head-dim 64 --kv-heads 2 --vocab 512 --group 64 --kv-group 32 --page 32 --tokens 9 "
                                  "--prompts 70 3 33 129".split())
    layers, batch, table, lens, out = ex.run(args)
    assert lens.tolist() == [79, 12, 42, 138] and out.shape == (9, 4)
    # out is rounded to bf16 (2^-9 at the most, of every element) and so are the values read back, which the kernel does not round; p and its products to 11 bits
    assert ex.check(args, layers, table, lens) <= 2.0 ** -6
    again = ex.run(args)[-1]
    assert torch.equal(out, again)
