"""ps_soft's losses and torch's autograd, without a GPU: a table whose gradient would be lost is refused by name, before anything
else is looked at."""
import pytest
import torch

from paper_1410_8043_amd import ps_soft


def calls(h, X, W, weight=None, score=None, value=None, tlse=None):
    item = torch.zeros(4, dtype=torch.int32)
    if score is None and tlse is None:
        yield lambda: h.xent(X, W, item, value=value, weight=weight)
        yield lambda: h.xent(X, W, item, value=value, weight=weight, grad=False)
    if value is None:
        yield lambda: h.distill(X, W, item[:, None], torch.zeros(4, 1) if score is None else score, tlse=tlse, weight=weight)


@pytest.mark.parametrize("name", ["X", "W", "weight", "value", "score", "tlse"])
def test_tensors_that_require_gradients_are_refused(name):
    shapes = {"X": (4, 8), "W": (10, 8), "score": (4, 1)}
    wanted = {k: torch.zeros(shapes.get(k, (4,))) for k in {"X", "W", name}}
    wanted[name].requires_grad_()
    with ps_soft.PsSoft(10, 8) as h:
        some = list(calls(h, **wanted))
        assert some
        for call in some:
            with pytest.raises(ValueError, match=f"{name} requires a gradient"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="GPU"):  # past this check, to the next
                call()
        plain = {k: v.detach() for k, v in wanted.items()}
        for call in calls(h, **plain):
            with pytest.raises(ValueError, match="GPU"):
                call()


def test_the_search_takes_trained_tables():
    X, W = torch.zeros(4, 8, requires_grad=True), torch.zeros(10, 8, requires_grad=True)
    with ps_soft.PsSoft(10, 8) as h, pytest.raises(ValueError, match="GPU"):
        h.top(X, W, 2)
