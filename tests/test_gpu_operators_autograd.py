"""Token lookups, their gradients, norm and clipping beside autograd, which does not record them: what would be lost
is refused, and what is written counts as changed."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from paper_2511_08568_amd import (GradientList, clip_grad_norm, clip_grads, embedding_backward,  # noqa: E402
                                  embedding_backward_rows, embedding_forward, grad_norm)


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


def writes():
    """Each call that writes a given tensor, and the tensor."""
    table, tokens, g, number, count = tensors()
    other, half, norm = torch.ones(50, device="cuda"), torch.ones(50, device="cuda").half(), torch.ones((), device="cuda")
    return [(g, lambda: embedding_forward(table, tokens, out=g)), (table, lambda: embedding_backward(g, tokens, 10, grad=table)),
            (table, lambda: embedding_backward(g, tokens, 10, grad=table, accumulate=True)),
            (g, lambda: embedding_backward_rows(g + 0, tokens, 10, out=(number, g, count))),
            (g, lambda: clip_grad_norm([other, g], 0.5)), (g, lambda: clip_grads(GradientList([other, g]), norm, 0.5)),
            (g, lambda: clip_grad_norm([other, table[:4]], 0.5, out=[half, g])),
            (g, lambda: clip_grad_norm([(g, count + 2)], 0.5, stream=torch.cuda.Stream()))]


@pytest.mark.parametrize("k", range(8))
def test_written_tensors_count_as_changed(k):
    """A backward pass that has kept one of them says so, instead of giving a wrong gradient."""
    t, call = writes()[k]
    w = torch.ones_like(t).requires_grad_()
    y = (w * t).sum()
    call()
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_read_tensors_do_not():
    table, tokens, g, number, count = tensors()
    w, v = torch.ones_like(table).requires_grad_(), torch.ones_like(g).requires_grad_()
    y = (w * table).sum() + (v * g).sum()
    embedding_forward(table, tokens)
    embedding_backward(g, tokens, 10)
    embedding_backward_rows(g, tokens, 10)
    grad_norm([table, g])
    clip_grad_norm([table, g], 0.5, out=[torch.ones_like(table), torch.ones_like(g)])
    y.backward()
    assert torch.equal(w.grad, table) and torch.equal(v.grad, g)


def test_inference_tensors_are_written():
    """They have no count of changes."""
    table, tokens, g, _, _ = tensors()
    with torch.inference_mode():
        out, grad = torch.zeros(4, 8, device="cuda"), torch.zeros(10, 8, device="cuda")
        embedding_forward(table, tokens, out=out)
    embedding_forward(table, tokens, out=out)
    embedding_backward(g, tokens, 10, grad=grad)
    clip_grad_norm([grad], 1e9)
    assert torch.equal(out, table[tokens]) and float(grad.sum()) == 32


def test_views_and_their_base_count_together():
    flat = torch.ones(300, device="cuda")
    parts = [flat[:100], flat[100:200].view(10, 10), flat[250:]]
    w = [torch.ones_like(t).requires_grad_() for t in parts + [flat]]
    y = [(a * t).sum() for a, t in zip(w, parts + [flat])]
    clip_grad_norm(GradientList(parts), 0.5)
    for a in y:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            a.backward()


def test_forward_mode_tangents_are_refused():
    from torch.autograd import forward_ad
    table, tokens, g, number, count = tensors()
    for no_grad in (False, True):
        with forward_ad.dual_level(), torch.set_grad_enabled(not no_grad):
            for k, (like, call) in enumerate(calls(table, tokens, g, number, count)):
                call(like.clone())  # others are taken inside a level too
                with pytest.raises(ValueError, match="has a tangent"):
                    call(forward_ad.make_dual(like.clone(), torch.ones_like(like)))
                    pytest.fail(f"call {k} was taken")
            dual = forward_ad.make_dual(g.clone(), torch.ones_like(g))
            for call in (lambda: grad_norm([table, dual]), lambda: clip_grad_norm([dual], 0.5),
                         lambda: clip_grad_norm([g], 0.5, out=[dual]), lambda: clip_grads([dual], torch.ones((), device="cuda"), 0.5)):
                with pytest.raises(ValueError, match="has a tangent"):
                    call()
            grad_norm([table, g])
    assert bool((g == 1).all())
