"""The example of the sampler and the distillation: it learns, and both ways to the gradient take it the same way."""
import pytest

pytestmark = pytest.mark.gpu


def test_the_student_learns_what_the_teacher_lists():
    from examples.distill_constrained import train
    small = dict(vocab=1024, batch=32, steps=8, rounds=12, report=lambda text: None)
    losses = train(**small)
    assert losses[-1] < 0.8 * losses[0]
    # (the gradients are the same numbers, so the first rounds are)
    assert train(one_pass=True, **small)[0] == losses[0]
