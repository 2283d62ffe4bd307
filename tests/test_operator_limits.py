"""The first sizes behind the documented limits of the gradient norm and clipping: refused on the host, and by the check
of that size.  No address here is ever read."""
import ctypes

import pytest

from paper_2511_08568_amd import binding as bd

A = 4096
MOST_TENSORS, MOST_ELEMENTS = 1 << 16, 1 << 37


def _calls(n, numel):
    mk = lambda t, v: (t * n)(*([v] * n))  # noqa: E731
    at, numels, types = mk(ctypes.c_void_p, A), mk(ctypes.c_int64, numel), mk(ctypes.c_int32, 0)
    size = 1 << 40  # more than any call asks for
    return [lambda: bd.recmg_grad_norm(n, at, numels, types, None, None, A, A, size, None),
            lambda: bd.recmg_grad_clip(n, at, at, numels, types, types, None, None, A, 1.0, 1e-6, None),
            lambda: bd.recmg_grad_norm_clip(n, at, at, numels, types, types, None, None, A, 1.0, 1e-6, A, size, None)]


@pytest.mark.parametrize("k", range(3))
@pytest.mark.parametrize("n,numel,what", [(MOST_TENSORS + 1, 1, "num_tensors"), (1, MOST_ELEMENTS + 1, "numel"),
                                          (3, MOST_ELEMENTS + 1, "numel")])
def test_first_sizes_behind_the_limits(n, numel, what, k):
    assert _calls(n, numel)[k]() == bd.RECMG_E_INVALID
    assert what in bd.load_library().recmg_last_error().decode()


def test_workspace_of_most_tensors():
    assert bd.recmg_query_grad_workspace(MOST_TENSORS) >= bd.recmg_query_grad_workspace(MOST_TENSORS - 1)
    with pytest.raises(bd.RecmgError, match="num_tensors"):
        bd.recmg_query_grad_workspace(MOST_TENSORS + 1)
