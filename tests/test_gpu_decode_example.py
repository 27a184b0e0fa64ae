"""The example that serves a layer from compressed memory: its steps, captured once and replayed, do what
the same steps do call by call.

Bar of its attention against fp64 over the cached values (fp32 queries, heads of 64): a score is off by at
most 2^-23 shake, shake = 80 scale sum |q||k| <= 2^10 for entries of unit size, a weight by e^x of that, twice it,
in the sum and in the product: 2^-11 of sum p |V|, which is at most 2^5 times the largest output over 300 tokens.
"""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_example_steps(fmt):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import decode_step as E
    err, lens, x = E.main(["--tokens", "9", "--format", fmt])
    assert lens == [310, 51, 138]                       # 9 replays and the step before them
    assert err <= 2.0 ** -6
    again = E.main(["--tokens", "9", "--format", fmt])
    assert torch.equal(x, again[2]) and bool(torch.isfinite(x).all())
