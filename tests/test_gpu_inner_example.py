"""The inner step's operators and the outer step together: workers that train, compress and meet."""
import pytest

pytestmark = pytest.mark.gpu


def test_workers_learn_together():
    """The loss starts near the variance of the targets (tanh of a standard normal: 0.39) and falls well below half of it."""
    from paper_2508_15706_amd import inner_example
    losses, model, teacher = inner_example.train(workers=2, rounds=5, inner_steps=15)
    assert losses[-1] < 0.5 * losses[0] and losses[-1] < 0.2
    import torch
    x = torch.randn(200, teacher.shape[1], device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    target = torch.tanh(x @ teacher.t())
    for rows in (1, 200):
        y = model.predict(x[:rows].bfloat16()).float()
        assert float((y - target[:rows]).square().mean()) < 0.3


def test_the_same_seeds_give_the_same_parameters():
    import torch
    from paper_2508_15706_amd import inner_example
    a = inner_example.train(workers=2, rounds=2, inner_steps=3)[1]
    b = inner_example.train(workers=2, rounds=2, inner_steps=3)[1]
    assert torch.equal(a.theta, b.theta) and torch.equal(a.v, b.v) and torch.equal(a.m, b.m)
