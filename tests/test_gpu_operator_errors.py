"""HIP errors of the calling thread's other calls: neither reported as these calls' own nor taken away from whoever
looks at them next."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from paper_2511_08568_amd import binding as bd  # noqa: E402


def runtime():
    """The HIP runtime that the process has loaded."""
    with open("/proc/self/maps") as f:
        path = next(line.split()[-1] for line in f if "libamdhip64" in line)
    return ctypes.CDLL(path)


def calls():
    t = lambda *shape, dtype=torch.float32: torch.ones(shape, dtype=dtype, device="cuda")  # noqa: E731
    mk = lambda c, *v: (c * len(v))(*v)  # noqa: E731
    made = []
    for n in (4, 3_000, 20_000):  # each sequence of kernels
        tokens, g, table, grad, values = t(n, dtype=torch.int64), t(n, 8), t(10, 8), t(10, 8), t(10, 8)
        number, count, out = t(10, dtype=torch.int32), t(1, dtype=torch.int64), t(n, 8)
        sizes = [max(1, bd.recmg_query_embedding_workspace(10, 8, n, form, 0)) for form in (0, 1)]
        works = [t(s, dtype=torch.uint8) for s in sizes]
        keep = (tokens, g, table, grad, values, number, count, out, works)
        p = lambda x: x.data_ptr()  # noqa: E731
        made += [(keep, bd.recmg_embedding_forward, (p(table), 0, 8, 10, 8, p(tokens), 1, n, 0, 1.0, p(out), 0, 8, None)),
                 (keep, bd.recmg_embedding_backward, (p(g), 0, 8, p(tokens), 1, n, None, 0, 10, 8, 0, -1, 1.0, p(grad), 0, 8, 0,
                                                      p(works[0]), sizes[0], None)),
                 (keep, bd.recmg_embedding_backward_rows, (p(g), 0, 8, p(tokens), 1, n, None, 0, 10, 8, 0, -1, 1.0, p(number),
                                                           p(values), 0, 8, p(count), p(works[1]), sizes[1], None))]
    g, norm, work = t(1000), t(1), t(bd.recmg_query_grad_workspace(1), dtype=torch.uint8)
    at, numel, f32 = mk(ctypes.c_void_p, g.data_ptr()), mk(ctypes.c_int64, 1000), mk(ctypes.c_int32, 0)
    keep = (g, norm, work)
    made += [(keep, bd.recmg_grad_norm, (1, at, numel, f32, None, None, norm.data_ptr(), work.data_ptr(), work.numel(), None)),
             (keep, bd.recmg_grad_clip, (1, at, at, numel, f32, f32, None, None, norm.data_ptr(), 1.0, 1e-6, None)),
             (keep, bd.recmg_grad_norm_clip, (1, at, at, numel, f32, f32, None, None, norm.data_ptr(), 1.0, 1e-6,
                                              work.data_ptr(), work.numel(), None))]
    return made


def test_pending_errors_stay():
    hip = runtime()
    made = calls()
    torch.cuda.synchronize()
    for _, call, args in made:
        hip.hipGetLastError()
        pending = hip.hipSetDevice(12_345)  # no such device
        assert pending != 0 and hip.hipPeekAtLastError() == pending
        status = call(*args)
        left = hip.hipGetLastError()
        assert (status, left) == (bd.RECMG_OK, pending), call.__name__
        assert hip.hipGetLastError() == 0
    torch.cuda.synchronize()
