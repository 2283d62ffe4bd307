"""Arguments that the lookup, its gradient, the gradient norm and the clipping
refuse.  The C entries check on the host before they enqueue anything, so these
run without a GPU; no address here is ever read."""
import ctypes

import pytest

import paper_2511_08568_amd as pk
from paper_2511_08568_amd import binding as bd

A = 4096  # stands for an address on the device


def _forward(**kw):
    a = dict(table=A, table_dtype=0, table_stride=8, rows=10, dim=8, tokens=A, index_type=1, num_tokens=5, first_row=0,
             scale=1.0, out=A, out_dtype=0, out_stride=8, stream=None)
    assert set(kw) <= set(a)
    return bd.recmg_embedding_forward(*{**a, **kw}.values())


def _backward(**kw):
    a = dict(grad_out=A, grad_out_dtype=0, grad_out_stride=8, tokens=A, index_type=1, num_tokens=5000, offsets=None, num_bags=0,
             rows=10, dim=8, first_row=0, padding_token=-1, scale=1.0, grad=A, grad_dtype=0, grad_stride=8, accumulate=0,
             workspace=A, workspace_bytes=1 << 30, stream=None)
    assert set(kw) <= set(a)
    return bd.recmg_embedding_backward(*{**a, **kw}.values())


def _rows(**kw):
    a = dict(grad_out=A, grad_out_dtype=0, grad_out_stride=8, tokens=A, index_type=1, num_tokens=5000, offsets=None, num_bags=0,
             rows=10, dim=8, first_row=0, padding_token=-1, scale=1.0, rows_out=A, values=A, values_dtype=0, values_stride=8,
             count=A, workspace=A, workspace_bytes=1 << 30, stream=None)
    assert set(kw) <= set(a)
    return bd.recmg_embedding_backward_rows(*{**a, **kw}.values())


COMMON = [dict(rows=0), dict(rows=1 << 31), dict(dim=0), dict(dim=65537), dict(index_type=2), dict(num_tokens=-1),
          dict(num_tokens=1 << 31), dict(first_row=-1), dict(tokens=None), dict(tokens=A + 4)]
GRAD = COMMON + [dict(grad_out=None), dict(grad_out=A + 2), dict(grad_out_dtype=3), dict(grad_out_stride=-1),
                 dict(offsets=A + 4, num_bags=2), dict(offsets=A, num_bags=-1), dict(offsets=A, num_bags=1 << 31),
                 dict(workspace=None), dict(workspace=A + 8)]


@pytest.mark.parametrize("kw", COMMON + [dict(table=None), dict(table=A + 2), dict(table_dtype=-1), dict(table_stride=7),
                                         dict(out=None), dict(out=A + 1, out_dtype=2), dict(out_dtype=3),
                                         dict(out_stride=7)], ids=str)
def test_forward_refuses(kw):
    assert _forward(**kw) == bd.RECMG_E_INVALID and pk.recmg_last_error()


@pytest.mark.parametrize("kw", GRAD + [dict(grad=None), dict(grad=A + 2), dict(grad_dtype=5), dict(grad_stride=7)], ids=str)
def test_backward_refuses(kw):
    assert _backward(**kw) == bd.RECMG_E_INVALID and pk.recmg_last_error()


@pytest.mark.parametrize("kw", GRAD + [dict(rows_out=None), dict(rows_out=A + 2), dict(values=None), dict(values=A + 2),
                                       dict(values_dtype=5), dict(values_stride=7), dict(count=None),
                                       dict(count=A + 4)], ids=str)
def test_backward_rows_refuses(kw):
    assert _rows(**kw) == bd.RECMG_E_INVALID and pk.recmg_last_error()


@pytest.mark.parametrize("call,form,bags", [(_backward, 0, 0), (_rows, 1, 0), (_backward, 0, 1), (_rows, 1, 1)])
@pytest.mark.parametrize("n", [3, 5_000, 70_000])
def test_small_workspaces_are_refused(call, form, bags, n):
    need = bd.recmg_query_embedding_workspace(10, 8, n, form, bags)
    if need == 0:
        assert (n, bags) == (3, 0)  # one kernel without a workspace
        return
    kw = dict(num_tokens=n, workspace_bytes=need - 1, **(dict(offsets=A, num_bags=4) if bags else {}))
    assert call(**kw) == bd.RECMG_E_NOMEM and "recmg_query_embedding_workspace" in pk.recmg_last_error()


@pytest.mark.parametrize("form,bags", [(0, 0), (0, 1), (1, 0), (1, 1)])
def test_workspace_query(form, bags):
    q = lambda rows, dim, n: bd.recmg_query_embedding_workspace(rows, dim, n, form, bags)  # noqa: E731
    assert q(10, 8, 0) == 0  # no ids: nothing to sort
    assert q(1 << 20, 8, 100_000) >= 16 * 100_000  # ids and their rows, twice
    # a workspace of more ids does for fewer
    for dim in (1, 64, 513, 5000, 65536):
        sizes = [q(1 << 17, dim, int(1.3 ** k)) for k in range(80)]
        assert sizes == sorted(sizes)
    # sizes that no call takes are refused, not computed
    for bad in ((0, 8, 5), (1 << 31, 8, 5), (10, 0, 5), (10, 65537, 5), (10, 8, -1), (10, 8, 1 << 31)):
        with pytest.raises(bd.RecmgError):
            q(*bad)
    # the largest call's size neither wraps nor overflows
    assert q((1 << 31) - 1, 65536, (1 << 31) - 1) > 40 * ((1 << 31) - 1)
    assert pk.load_library().recmg_query_embedding_workspace(10, 8, 5, form, bags, None) == bd.RECMG_E_INVALID


def _lists(n=2, grad=A, out=A, numel=100, dtype=0, out_dtype=0):
    mk = lambda t, v: (t * n)(*([v] * n))  # noqa: E731
    return dict(grads=mk(ctypes.c_void_p, grad), outs=mk(ctypes.c_void_p, out), numels=mk(ctypes.c_int64, numel),
                dtypes=mk(ctypes.c_int32, dtype), out_dtypes=mk(ctypes.c_int32, out_dtype))


def _norm(count=2, norm=A, workspace=A, size=1 << 20, live=None, lengths=None, **kw):
    d = {**_lists(), **{k: v for k, v in kw.items()}}
    return bd.recmg_grad_norm(count, d["grads"], d["numels"], d["dtypes"], live, lengths, norm, workspace, size, None)


def _clip(count=2, norm=A, max_norm=1.0, eps=1e-6, live=None, lengths=None, **kw):
    d = {**_lists(), **{k: v for k, v in kw.items()}}
    return bd.recmg_grad_clip(count, d["grads"], d["outs"], d["numels"], d["dtypes"], d["out_dtypes"], live, lengths, norm,
                              max_norm, eps, None)


def _norm_clip(count=2, norm=A, max_norm=1.0, eps=1e-6, workspace=A, size=1 << 20, live=None, lengths=None, **kw):
    d = {**_lists(), **kw}
    return bd.recmg_grad_norm_clip(count, d["grads"], d["outs"], d["numels"], d["dtypes"], d["out_dtypes"], live, lengths,
                                   norm, max_norm, eps, workspace, size, None)


BAD_LISTS = [dict(count=-1), dict(count=(1 << 20) + 1), dict(grads=None), dict(numels=None), dict(dtypes=None), dict(norm=None),
             dict(norm=A + 2), dict(numels=_lists(numel=-1)["numels"]), dict(numels=_lists(numel=(1 << 40) + 1)["numels"]),
             dict(dtypes=_lists(dtype=3)["dtypes"]), dict(grads=_lists(grad=None)["grads"]),
             dict(grads=_lists(grad=A + 2)["grads"]), dict(live=(ctypes.c_void_p * 2)(A, None)),
             dict(live=(ctypes.c_void_p * 2)(A, None), lengths=(ctypes.c_int32 * 2)(0, 0)),
             dict(live=(ctypes.c_void_p * 2)(A + 4, None), lengths=(ctypes.c_int32 * 2)(5, 5))]


BAD_WORK = [dict(workspace=None), dict(workspace=A + 16)]


@pytest.mark.parametrize("kw", BAD_LISTS + BAD_WORK, ids=lambda k: "-".join(k))
def test_norm_refuses(kw):
    assert _norm(**kw) == bd.RECMG_E_INVALID and pk.recmg_last_error()


BAD_CLIP = BAD_LISTS + [dict(outs=None), dict(out_dtypes=None), dict(outs=_lists(out=None)["outs"]),
                        dict(outs=_lists(out=A + 2)["outs"]), dict(out_dtypes=_lists(out_dtype=4)["out_dtypes"]),
                        dict(out_dtypes=_lists(out_dtype=1)["out_dtypes"]),  # in place, another type
                        dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=0.0), dict(eps=float("nan")),
                        dict(eps=float("inf"))]


@pytest.mark.parametrize("kw", BAD_CLIP, ids=lambda k: "-".join(k))
def test_clip_refuses(kw):
    assert _clip(**kw) == bd.RECMG_E_INVALID and pk.recmg_last_error()


@pytest.mark.parametrize("kw", BAD_CLIP + BAD_WORK, ids=lambda k: "-".join(k))
def test_norm_clip_refuses(kw):
    assert _norm_clip(**kw) == bd.RECMG_E_INVALID and pk.recmg_last_error()


def test_norm_refuses_small_workspaces():
    need = bd.recmg_query_grad_workspace(2)
    assert _norm(size=need - 1) == bd.RECMG_E_NOMEM == _norm_clip(size=need - 1)
    sizes = [bd.recmg_query_grad_workspace(n) for n in range(2000)]
    assert sizes == sorted(sizes)
    for n in (-1, (1 << 20) + 1):
        with pytest.raises(bd.RecmgError):
            bd.recmg_query_grad_workspace(n)


def test_cpu_tensors_are_refused():
    torch = pytest.importorskip("torch")
    t, ids = torch.zeros(4, 8), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        pk.embedding_forward(t, ids)
    with pytest.raises(ValueError):
        pk.embedding_backward(t[:3], ids, 4)
    with pytest.raises(ValueError):
        pk.embedding_backward_rows(t[:3], ids, 4)
    with pytest.raises(ValueError):
        pk.GradientList([t])
    with pytest.raises(ValueError):
        pk.grad_norm([])


def test_importing_the_package_does_not_import_torch():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = "import paper_2511_08568_amd, sys; assert 'torch' not in sys.modules"
    assert subprocess.run([sys.executable, "-c", code], cwd=root, timeout=120).returncode == 0
