"""The example sequence model: training through the operators' gradients lowers its loss, and rolling
out one action at a time gives the predictions of the whole-sequence pass (in float32 up to the
order of sums: 1e-4 of the largest; in bfloat16 every layer boundary rounds to 2^-9: 2^-5)."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype,tol", [("float32", 1e-4), ("bfloat16", 2.0 ** -5)])
def test_training_and_rollout(dtype, tol):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import schedule_sequence_model as m
    losses, diff = m.run(programs=3, per_program=11, T=13, d=32, train_steps=8, dtype=getattr(torch, dtype))
    assert losses[-1] < 0.9 * losses[0], losses
    assert diff <= tol
