"""The example examples/train_tokens.py: the embedding, the gated scan, the DendSN layer and
the cross entropy together learn a Markov chain of tokens."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import train_tokens  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_lowers_the_loss(dtype):
    if not torch.cuda.is_available():
        pytest.fail("needs a CUDA device")
    losses = train_tokens.train(steps=60, V=128, N=128, T=32, B=16, dtype=dtype)
    assert abs(losses[0] - math.log(128)) < 0.5 * math.log(128)      # starts near the uniform guess
    assert all(math.isfinite(v) for v in losses)
    assert sum(losses[-5:]) / 5 < 0.75 * losses[0]
