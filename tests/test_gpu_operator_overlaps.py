"""Tensors of one buffer: those that are apart are taken, those that share elements are refused."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from paper_2511_08568_amd import (GradientList, RecmgError, clip_grad_norm, clip_grads, embedding_backward,  # noqa: E402
                                  embedding_backward_rows, embedding_forward)

N, ROWS, DIM = 40, 30, 16


def given():
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    return (torch.randint(0, ROWS, (N,), generator=g, device="cuda"),
            torch.randint(-8, 9, (100, 50), generator=g, device="cuda").float())


def views(room):
    """(table or incoming gradient, output) of one matrix, apart."""
    return [(room[:N, :DIM], room[:N, DIM:2 * DIM]), (room[:N, 20:20 + DIM], room[:N, :DIM]), (room[:N, :DIM], room[N:2 * N, :DIM]),
            (room[1:2 * N:2, 5:5 + DIM], room[:2 * N:2, 5:5 + DIM]), (room[:N, :DIM], room[3:3 + N, 30:30 + DIM])]


def overlapping(room):
    return [(room[:N, :DIM], room[:N, :DIM]), (room[:N, :DIM], room[:N, DIM - 1:2 * DIM - 1]), (room[:N, :DIM], room[N - 1:2 * N - 1, :DIM]),
            (room[1:2 * N:2, :DIM], room[3:2 * N + 3:2, :DIM]), (room.view(-1)[:N * DIM].view(N, DIM), room[:N, 30:30 + DIM])]


@pytest.mark.parametrize("k", range(5))
def test_apart(k):
    tokens, room = given()
    a, b = views(room)[k]
    want = embedding_forward(a[:ROWS].clone(), tokens)
    assert torch.equal(embedding_forward(a[:ROWS], tokens, out=b), want)
    tokens, room = given()
    a, b = views(room)[k]
    want = embedding_backward(a.clone(), tokens, ROWS)
    assert torch.equal(embedding_backward(a, tokens, ROWS, grad=b[:ROWS]), want)
    tokens, room = given()
    a, b = views(room)[k]
    number, values, count = embedding_backward_rows(a.clone(), tokens, ROWS)
    got = (torch.empty_like(number), b[:ROWS], torch.empty_like(count))
    embedding_backward_rows(a, tokens, ROWS, out=got)
    m = int(count)
    assert all(torch.equal(x[:m], y[:m]) for x, y in zip(got, (number, values, count)))


@pytest.mark.parametrize("k", range(5))
def test_shared(k):
    tokens, room = given()
    old = room.clone()
    a, b = overlapping(room)[k]
    number, count = torch.empty(ROWS, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int64, device="cuda")
    for call in (lambda: embedding_forward(a, tokens, out=b), lambda: embedding_backward(a, tokens, N, grad=b),
                 lambda: embedding_backward(a, tokens, N, grad=b, accumulate=True),
                 lambda: embedding_backward_rows(a, tokens, N, out=(torch.empty(N, dtype=torch.int32, device="cuda"), b, count))):
        with pytest.raises(RecmgError, match="shares memory"):
            call()
    assert torch.equal(room, old)


def test_norms_and_counts_inside_an_output():
    t = torch.ones(1000, device="cuda")
    c = torch.ones(10, dtype=torch.int64, device="cuda")
    for call in (lambda: clip_grads([t], t[:1], 0.5), lambda: clip_grads([t], t[-1:], 0.5),
                 lambda: clip_grads(GradientList([t[:500], t[500:]]), t[500], 0.5),
                 lambda: clip_grad_norm([(c.view(torch.float32).view(10, 2), c[9:])], 0.5),
                 lambda: clip_grad_norm([t, (c.view(torch.float32).view(10, 2), c[:1])], 0.5)):
        with pytest.raises(ValueError):
            call()
    assert bool((t == 1).all()) and bool((c == 1).all())
    clip_grads([t[1:]], t[:1], 0.5)  # beside it is fine
    assert bool((t[1:] == 0.5).all() or (t[1:] - 0.5 / (1 + 1e-6)).abs().max() <= 1e-7)
