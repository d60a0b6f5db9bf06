"""The example's block, all operators together, forward and backward against plain torch in 64 bits.

Tolerance.  Along the longest path a value is rounded to bf16 about six times (the norm's output, pre-activations, activations, experts'
rows, the combine, and the same on the way back), each with a relative error of at most 2^-8, at random: 0.02 is above five such errors in
a row all at their largest."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("sizes", [dict(), dict(N=1), dict(N=700, H=136, I=72, E=12, k=2, D=3, keep_groups=1), dict(N=520, H=512, I=256, E=8, k=4, D=2, keep_groups=2)])
def test_block(sizes):
    spec = importlib.util.spec_from_file_location("moe_block", os.path.join(ROOT, "examples", "moe_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    far = example.check(**sizes)
    assert max(far.values()) < 0.02, far
