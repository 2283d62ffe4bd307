"""A GradientList that is kept while its tensors change under it: its calls take the memory that it was laid out
with, which nothing else comes to use, or are refused."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from paper_2511_08568_amd import GradientList, clip_grad_norm, clip_grads, grad_norm  # noqa: E402

U32 = 2.0 ** -24


def ones(n=1000):
    return torch.ones(n, device="cuda")


def listed(which):
    """A list, what it leaves alone, and its tensor that will change."""
    other, values, out = ones(), ones().view(10, 100), ones().view(10, 100)
    count = torch.tensor([10], device="cuda")
    return (GradientList([other, (values, count)], out=[other, out]), other,
            {"gradient": values, "output": out, "count": count}[which])


@pytest.mark.parametrize("resize", [lambda t: t.resize_(t.numel() * 1000), lambda t: t.untyped_storage().resize_(0),
                                    lambda t: t.untyped_storage().resize_(t.untyped_storage().nbytes() // 2)],
                         ids=["longer", "freed", "half"])
@pytest.mark.parametrize("which", ["gradient", "output", "count"])
def test_resized_memory_is_refused(resize, which):
    grads, other, t = listed(which)
    norm = grad_norm(grads)
    resize(t)
    for call in (lambda: grad_norm(grads), lambda: clip_grad_norm(grads, 0.5), lambda: clip_grads(grads, norm, 0.5)):
        with pytest.raises(ValueError, match="resized"):
            call()
    assert bool((other == 1).all())


@pytest.mark.parametrize("move", ["data", "set", "cpu", "half", "short"])
def test_dropped_memory_stays_with_the_list(move):
    """The calls take the former memory, and no other tensor lies there."""
    t = ones()
    where, former = t.data_ptr(), t.detach()
    grads = GradientList([t])
    if move == "set":
        t.set_(ones())
    else:
        t.data = {"data": ones(), "cpu": torch.ones(1000), "half": ones().half(), "short": ones(3)}[move]
    others = [ones() for _ in range(50)] + [ones(3) for _ in range(50)]
    assert all(o.data_ptr() != where for o in others)
    norm = clip_grad_norm(grads, 0.5)
    assert norm.is_cuda and abs(float(norm) - 1000 ** 0.5) <= 1.01 * U32 * 1000 ** 0.5
    assert bool(((former.double() - 0.5 * 1000 ** -0.5).abs() <= 1e-6).all())
    assert all(bool((o == 1).all()) for o in others + [t])


def test_first_clipping_after_a_move_checks_the_memory_that_it_writes():
    room = ones(2000)
    t, u = room[:1000], ones()
    grads = GradientList([t, room[500:1500], u])
    t.data = ones()  # apart from the second gradient now, but the list's memory is not
    with pytest.raises(ValueError, match="share memory"):
        clip_grad_norm(grads, 0.5)
    assert bool((room == 1).all()) and bool((u == 1).all())


def test_values_may_change():
    t = ones()
    grads = GradientList([t])
    for k in (1.0, 3.0):
        t.copy_(torch.full_like(t, k))
        assert abs(float(grad_norm(grads)) - k * 1000 ** 0.5) <= 1.01 * U32 * k * 1000 ** 0.5
