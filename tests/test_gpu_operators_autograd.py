"""Token lookups, their gradients, norm and clipping beside autograd, which does not record them: what would be lost
is refused, and what is written counts as changed."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from paper_2511_08568_amd import embedding_backward, embedding_backward_rows, embedding_forward  # noqa: E402


def tensors():
    return (torch.ones(10, 8, device="cuda"), torch.tensor([1, 2, 2, 9], device="cuda"), torch.ones(4, 8, device="cuda"),
            torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"))


def recorded(t):
    """As a leaf, and as the result of a recorded operation."""
    leaf = t.clone().requires_grad_()
    return leaf, leaf * 1


def calls(table, tokens, g, number, count):
    """Each call with a place for a tensor that requires a gradient."""
    return [(table, lambda t: embedding_forward(t, tokens)), (g, lambda t: embedding_forward(table, tokens, out=t)),
            (g, lambda t: embedding_backward(t, tokens, 10)), (g, lambda t: embedding_backward_rows(t, tokens, 10)),
            (table, lambda t: embedding_backward(g, tokens, 10, grad=t)),
            (table, lambda t: embedding_backward(g, tokens, 10, grad=t, accumulate=True)),
            (g, lambda t: embedding_backward_rows(g, tokens, 10, out=(number, t, count)))]


def test_recorded_tensors_are_refused():
    for k, (like, call) in enumerate(calls(*tensors())):
        for t in recorded(like):
            with pytest.raises(ValueError, match="requires a gradient"):
                call(t)
                pytest.fail(f"call {k} was taken")
            with torch.no_grad():  # as in the backward pass of a torch.autograd.Function
                call(t)
