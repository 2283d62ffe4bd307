"""The norm of many gradients and their clipping against 64 bits, and a step of
training with lookups, their gradients, the norm and the clipping together.

Bounds.  The norm's squares and sums are in 64 bits (their error lies far below
the last bit of fp32), its rounding to fp32 is half a step.  A clipped value is
one fp32 product: the factor, rounded once from 64 bits of a norm that is off by
2^-24, is off by 2^-23, the product by 2^-24 more, and its type adds half a step.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from paper_2511_08568_amd import (GradientList, TieredEmbeddingCache, clip_grad_norm, clip_grads,  # noqa: E402
                                  embedding_backward, embedding_backward_rows, embedding_forward, grad_norm)

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
U32 = 2.0 ** -24


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def norm64(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


def check_norm(got, tensors):
    want = norm64(tensors)
    assert got.shape == () and got.dtype == F32 and abs(float(got) - want) <= U32 * 1.01 * want


def check_clipped(out, g, norm, max_norm, eps=1e-6):
    f = min(1.0, max_norm / (norm + eps))
    ref = g.double() * f
    tol = (torch.finfo(out.dtype).eps / 2 * (out.dtype != F32) + 3.01 * U32) * ref.abs()
    tol += torch.finfo(out.dtype).smallest_normal * torch.finfo(out.dtype).eps
    assert bool(((out.double() - ref).abs() <= tol).all())


SIZES = [0, 1, 2, 7, 8, 9, 63, 1000, 16_383, 16_384, 16_385, 50_001, 300_007]


def grads_of(sizes, dtypes, seed, scale=1.0):
    """Tensors that begin at any multiple of their element."""
    got = []
    for k, n in enumerate(sizes):
        room = (torch.randn(n + 16, generator=gen(seed + k), device="cuda") * scale).to(dtypes[k % len(dtypes)])
        got.append(room[k % 9:k % 9 + n])
    return got


@pytest.mark.parametrize("dtypes", [(F32,), (BF16,), (F16,), (F32, BF16, F16)])
def test_norm_and_clipping(dtypes):
    grads = grads_of(SIZES, dtypes, 1)
    old = [g.clone() for g in grads]
    want = norm64(grads)
    check_norm(grad_norm(grads), grads)
    for into in (F32, F16, BF16):
        outs = [torch.full_like(g, 9, dtype=into) for g in grads]
        check_norm(clip_grad_norm(grads, 0.25 * want, out=outs), old)
        for o, g in zip(outs, old):
            check_clipped(o, g, want, 0.25 * want)
    assert all(torch.equal(a, b) for a, b in zip(grads, old))
    check_norm(clip_grad_norm(grads, 0.25 * want), old)
    for g, b in zip(grads, old):
        check_clipped(g, b, want, 0.25 * want)


@pytest.mark.parametrize("count", [1, 159, 160, 161, 320, 500, 4_000])
def test_many_tensors(count):
    sizes = [(37 * k) % 701 for k in range(count + count % 2)]  # bf16 and fp32 in turn
    sizes[-1] = 40_000
    grads = grads_of(sizes, (BF16, F32), 2)
    old = [g.clone() for g in grads]
    check_norm(clip_grad_norm(grads, 1.0), old)
    check_clipped(torch.cat([g.float() for g in grads[1::2]]), torch.cat([b.float() for b in old[1::2]]), norm64(old), 1.0)
    check_clipped(torch.cat(grads[::2]), torch.cat(old[::2]), norm64(old), 1.0)


def test_one_long_tensor():
    """More than 2^31 elements."""
    n = 2 ** 31 + 12_345
    g = torch.empty(n, dtype=BF16, device="cuda").normal_(0.0, 1.0, generator=gen(3))
    want = float(torch.linalg.vector_norm(g, dtype=torch.float64))
    ends = [g[:999].clone(), g[-999:].clone(), g[2 ** 31 - 500:2 ** 31 + 500].clone()]
    got = clip_grad_norm([g], want / 2)
    assert abs(float(got) - want) <= U32 * 1.01 * want
    for now, was in zip((g[:999], g[-999:], g[2 ** 31 - 500:2 ** 31 + 500]), ends):
        check_clipped(now, was, want, want / 2)


def test_within_the_limit_nothing_changes():
    grads = grads_of(SIZES, (F32, BF16, F16), 4)
    old = [g.clone() for g in grads]
    clip_grad_norm(grads, 2 * norm64(grads))
    assert all(torch.equal(a, b) for a, b in zip(grads, old))
    outs = [torch.zeros_like(g, dtype=F32) for g in grads]
    clip_grad_norm(grads, float("inf"), out=outs)
    assert all(torch.equal(o, g.float()) for o, g in zip(outs, grads))


@pytest.mark.parametrize("value", [1e30, 1e-30, 3e38, 1e-40, 0.0])
def test_values_whose_squares_leave_fp32(value):
    g = torch.full((1000,), value, device="cuda")
    want = norm64([g])
    got = float(grad_norm([g]))
    assert got == float(np.float32(want)) or abs(got - want) <= U32 * 1.01 * want


def test_infinities_and_nan():
    for bad, norm_is, rest_is in ((float("inf"), float("inf"), 0.0), (float("nan"), float("nan"), float("nan"))):
        a, b = torch.ones(100, device="cuda"), torch.ones(20_000, device="cuda").to(BF16)
        b[12_345] = bad
        got = float(clip_grad_norm([a, b], 1.0))
        assert got == norm_is or (math.isnan(got) and math.isnan(norm_is))
        for t in (a, b[:12_345], b[12_346:]):
            assert bool((t == rest_is).all()) if rest_is == rest_is else bool(t.isnan().all())
        assert bool(b[12_345].isnan())


def test_rows_with_a_count():
    """Values behind the count take no part, and stay."""
    dim = 37
    for k, cap in ((0, 50), (1, 50), (49, 50), (50, 50), (999, 1000), (-3, 50), (70, 50)):
        values = torch.randn(cap, dim, generator=gen(5), device="cuda")
        values[max(k, 0):] = float("nan")
        old = values.clone()
        other = torch.randn(500, generator=gen(6), device="cuda").to(BF16)
        was = other.clone()
        live = old[:max(k, 0)]
        got = clip_grad_norm([(values, torch.tensor([k], device="cuda")), other], 0.5)
        check_norm(got, [live, was])
        check_clipped(values[:max(k, 0)], live, norm64([live, was]), 0.5)
        assert bool(values[max(k, 0):].isnan().all())
        check_clipped(other, was, norm64([live, was]), 0.5)


def test_many_tensors_with_counts():
    """More of them than one launch holds, between others."""
    grads, old = [], []
    for k in range(70):
        values = torch.randn(9, 5, generator=gen(300 + k), device="cuda")
        m = k % 11
        old.append((values[:m].clone(), values[m:].clone()))
        grads.append((values, torch.tensor([m], device="cuda")))
        if k % 3 == 0:
            t = torch.randn(20_000 * (k % 2) + 3, generator=gen(400 + k), device="cuda").to(F16)
            old.append((t.clone(), t[:0]))
            grads.append(t)
    want = norm64([a for a, _ in old])
    check_norm(clip_grad_norm(grads, 0.5), [a for a, _ in old])
    for g, (a, b) in zip(grads, old):
        g = g[0] if isinstance(g, tuple) else g
        check_clipped(g[:a.shape[0]], a, want, 0.5)
        assert torch.equal(g[a.shape[0]:], b)


def test_layouts():
    t = torch.randn(30, 40, generator=gen(7), device="cuda")
    p = torch.randn(4, 5, 6, 7, generator=gen(8), device="cuda").to(memory_format=torch.channels_last)
    grads, old = [t.t(), p], [t.clone(), p.clone()]
    check_norm(clip_grad_norm(grads, 1.0), old)
    check_clipped(t, old[0], norm64(old), 1.0)
    check_clipped(p, old[1], norm64(old), 1.0)


def test_norm_of_several_processes():
    """clip_grads takes a norm that was made of several lists' norms."""
    lists = [grads_of([5_000, 17], (F32,), s) for s in (10, 20)]
    old = [[g.clone() for g in x] for x in lists]
    both = torch.stack([grad_norm(x).double() ** 2 for x in lists]).sum().sqrt().float()
    for x, o in zip(lists, old):
        clip_grads(x, both, 3.0)
        for g, b in zip(x, o):
            check_clipped(g, b, float(both), 3.0)


def test_equal_calls_give_equal_bits():
    g = GradientList(grads_of([3_000_000, 5, 70_000], (BF16, F32), 9))
    first = grad_norm(g)
    assert all(torch.equal(first, grad_norm(g)) for _ in range(5))


def test_refusals():
    t = torch.ones(100, device="cuda")
    bad = [lambda: GradientList([t.double()]), lambda: GradientList([t[::2]]), lambda: GradientList([t], out=[]),
           lambda: GradientList([t], out=[t[:50]]), lambda: clip_grad_norm([t, t], 1.0),
           lambda: clip_grad_norm([t[:60], t[40:]], 1.0), lambda: clip_grad_norm([t[:50]], 1.0, out=[t[25:75]]),
           lambda: clip_grad_norm([t[:50], t[50:]], 1.0, out=[t[50:], t[:50]]),
           lambda: clip_grads([t], torch.ones(2, device="cuda"), 1.0), lambda: clip_grads([t], torch.ones(()), 1.0),
           lambda: clip_grad_norm(GradientList([t]), 1.0, out=[t]),
           lambda: GradientList([(t, torch.ones(1, dtype=torch.int64, device="cuda"))]),
           lambda: GradientList([(t.view(10, 10), torch.ones(1, device="cuda"))]),
           lambda: GradientList([t.expand(3, 100)]), lambda: GradientList([t.cpu()])]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")
    check_norm(grad_norm([t, t]), [t, t])  # reading one twice is fine
    from paper_2511_08568_amd import RecmgError
    for kw in (dict(max_norm=-1.0), dict(max_norm=1.0, eps=0.0)):
        with pytest.raises(RecmgError):
            clip_grad_norm([t], **kw)
    assert bool((t == 1).all())


def test_captured_clipping_replays_on_another_stream():
    a, b = torch.zeros(40_000, device="cuda"), torch.zeros(70_001, dtype=BF16, device="cuda")
    out = [torch.zeros_like(a), torch.zeros(70_001, device="cuda")]
    grads = GradientList([a, b], out=out)
    clip_grad_norm(grads, 1.0)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            norm = clip_grad_norm(grads, 2.0)
        graphs.append((graph, norm))
    side = torch.cuda.Stream()
    for k in range(6):
        a.normal_(generator=gen(100 + k))
        b.normal_(generator=gen(200 + k))
        torch.cuda.synchronize()
        graph, norm = graphs[k % 2]
        with torch.cuda.stream(side):
            graph.replay()
        side.synchronize()
        check_norm(norm, [a, b])
        got = [o.clone() for o in out]
        assert torch.equal(clip_grad_norm(grads, 2.0), norm)
        assert torch.equal(out[0], got[0]) and torch.equal(out[1], got[1])
        torch.cuda.synchronize()
        other = clip_grad_norm(grads, 2.0, stream=side)
        side.synchronize()
        assert torch.equal(other, norm)


# ---------------------------------------------------------------------------- together

def test_training_steps():
    """Steps of a token table with a linear layer behind it: lookup, gradients, norm, clipping and update, beside the same
    steps in 64 bits.  The lookup and the sums carry fp32, so values stay within a small multiple of the fp32 sums' bound:
    5 steps, sums of at most n = 600 values each, so (600 + 100) 2^-24 < 5e-5 of the largest values per step."""
    rows, dim, n = 400, 48, 600
    table = torch.randn(rows, dim, generator=gen(11), device="cuda")
    weight = torch.randn(dim, 10, generator=gen(12), device="cuda") * 0.1
    t64, w64 = table.double(), weight.double()
    scale = math.sqrt(dim)
    for step in range(5):
        tokens = torch.randint(0, rows // 2, (n,), generator=gen(13 + step), device="cuda")
        x = embedding_forward(table, tokens, scale=scale)
        gy = torch.randn(n, 10, generator=gen(30 + step), device="cuda")  # the gradient that a loss hands down
        grads = [embedding_backward(gy @ weight.t(), tokens, rows, scale=scale), x.t() @ gy]
        norm = clip_grad_norm(grads, 1.0)
        table -= 0.5 * grads[0]
        weight -= 0.5 * grads[1]
        x64 = t64[tokens] * float(np.float32(scale))
        g64 = [torch.zeros_like(t64).index_add(0, tokens, gy.double() @ w64.t()) * float(np.float32(scale)),
               x64.t() @ gy.double()]
        n64 = norm64(g64)
        f = min(1.0, 1.0 / (n64 + 1e-6))
        t64, w64 = t64 - 0.5 * f * g64[0], w64 - 0.5 * f * g64[1]
        assert abs(float(norm) - n64) <= 5e-5 * (step + 1) * n64
        assert float((table.double() - t64).abs().max()) <= 5e-5 * (step + 1) * float(t64.abs().max())
        assert float((weight.double() - w64).abs().max()) <= 5e-5 * (step + 1) * float(w64.abs().max())
    assert bool((table[rows // 2:].double() == t64[rows // 2:]).all())  # rows that no token named


def test_gradient_of_the_tiered_lookup():
    """Two host tables behind a cache: the pooled lookup's gradient as rows, clipped together with a dense gradient, written
    back to the host, and looked up again.  Whole numbers: the lookup's change is exactly what the gradient says."""
    rows, dim, bags, T = 3_000, 32, 40, 2
    r = np.random.default_rng(5)
    host = [torch.from_numpy(r.integers(-8, 9, (rows, dim)).astype(np.float32)).pin_memory() for _ in range(T)]
    counts = r.integers(0, 9, T * bags)
    counts[3] = 0
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
    idx = r.integers(0, rows, offsets[-1]).astype(np.int32)
    idx[: offsets[-1] // 3] = idx[0]
    d_idx, d_off = torch.from_numpy(idx).cuda(), torch.from_numpy(offsets).cuda()
    g = torch.randint(-4, 5, (T, bags, dim), generator=gen(14), device="cuda").float()
    outs = []
    for turn in range(2):
        cache = TieredEmbeddingCache(host, ["f32"] * T, [500] * T, max_bags_per_table=bags, max_indices=idx.size, max_prefetch=1)
        outs.append(cache.forward(d_idx, d_off, bags).view(T, bags, dim).clone())
        torch.cuda.synchronize()
        if turn == 1:
            cache.close()
            break
        grads = []
        for t in range(T):
            lo, hi = int(offsets[t * bags]), int(offsets[(t + 1) * bags])
            bag_ends = d_off[t * bags:(t + 1) * bags + 1]
            grads.append(cache.backward_rows(t, g[t], d_idx[lo:hi], bag_ends))
            same = embedding_backward_rows(g[t], d_idx[lo:hi], rows, offsets=bag_ends)
            k = int(same[2])
            assert int(grads[t][2]) == k and torch.equal(grads[t][0][:k], same[0][:k])
            assert torch.equal(grads[t][1][:k], same[1][:k])
        with pytest.raises(ValueError):
            cache.backward_rows(0, g[0][:, 1:], d_idx[lo:hi], bag_ends)
        cache.close()
        dense = torch.ones(7, device="cuda")
        clip_grad_norm([(v, c) for _, v, c in grads] + [dense], float("inf"))  # nothing is clipped: the values stay whole
        change = 0.0
        for t, (there, values, count) in enumerate(grads):
            k = int(count)
            host[t][there[:k].cpu().long()] += values[:k].cpu()
            change += float(values[:k].double().square().sum())
    # <g, F(E + G) - F(E)> = <G, G> where G is the gradient of <g, F(E)>
    assert float((g.double() * (outs[1] - outs[0]).double()).sum()) == change
