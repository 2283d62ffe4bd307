"""Outputs of lookups and gradients that share memory with what the call reads, or with one another: refused on the
host, before anything is enqueued.  No address here is ever read."""
import pytest

from paper_2511_08568_amd import binding as bd

M = 1 << 20  # the arguments' addresses lie so far apart


def _refused(status, *names):
    assert status == bd.RECMG_E_INVALID
    message = bd.load_library().recmg_last_error().decode()
    assert "shares memory" in message and all(n in message for n in names), message


def _forward(**kw):
    """A table of 10 rows of 8 floats, 20 apart; 5 tokens; an output whose rows are 8 apart."""
    a = dict(table=M, table_dtype=0, table_stride=20, rows=10, dim=8, tokens=2 * M, index_type=1, num_tokens=5, first_row=0,
             scale=1.0, out=3 * M, out_dtype=0, out_stride=8, stream=None)
    assert set(kw) <= set(a)
    return bd.recmg_embedding_forward(*{**a, **kw}.values())


@pytest.mark.parametrize("kw,names", [
    (dict(out=M), ("out", "table")),
    (dict(out=M + 9 * 80 + 28), ("out", "table")),          # the last element of the last row
    (dict(out=M - 5 * 32 + 4), ("out", "table")),           # up to its first element
    (dict(out=M + 8 * 4, out_stride=20, table_stride=8), ("out", "table")),
    (dict(out=M + 7 * 4, out_stride=20), ("out", "table")),  # columns of the same rows
    (dict(out=M + 80 + 13 * 4, out_stride=20), ("out", "table")),
    (dict(out=M + 9 * 80 + 7 * 4, out_stride=20), ("out", "table")),
    (dict(out=M, out_dtype=2, out_stride=8), ("out", "table")),
    (dict(out=2 * M + 36), ("out", "tokens")),
    (dict(out=2 * M - 5 * 32 + 4), ("out", "tokens")),
    (dict(out=2 * M - 3 * 80 + 4, out_stride=20), ("out", "tokens")),
    (dict(out=2 * M + 16, index_type=0), ("out", "tokens")),
], ids=str)
def test_forward(kw, names):
    _refused(_forward(**kw), *names)


def _gradient(rows_form, **kw):
    a = dict(grad_out=M, grad_out_dtype=0, grad_out_stride=8, tokens=2 * M, index_type=1, num_tokens=5000, offsets=None, num_bags=0,
             rows=10, dim=8, first_row=0, padding_token=-1, scale=1.0)
    a.update(dict(rows_out=3 * M, grad=4 * M, grad_dtype=0, grad_stride=8, count=5 * M) if rows_form else
             dict(grad=4 * M, grad_dtype=0, grad_stride=8, accumulate=0))
    a.update(workspace=6 * M, workspace_bytes=1 << 30, stream=None)
    assert set(kw) <= set(a)
    return (bd.recmg_embedding_backward_rows if rows_form else bd.recmg_embedding_backward)(*{**a, **kw}.values())


@pytest.mark.parametrize("rows_form", [0, 1])
@pytest.mark.parametrize("kw,names", [
    (dict(grad=M), ("grad_out",)), (dict(grad=M + 5000 * 32 - 4), ("grad_out",)), (dict(grad=M - 10 * 32 + 4), ("grad_out",)),
    (dict(grad=M, num_tokens=4), ("grad_out",)),                       # without a workspace
    (dict(grad=M, grad_out_stride=0), ("grad_out",)), (dict(grad=M + 28, grad_out_stride=0), ("grad_out",)),
    (dict(grad=M + 4999 * 4, grad_out_stride=1), ("grad_out",)),       # rows that overlap one another
    (dict(grad=M + 7 * 4, grad_stride=16, grad_out_stride=16), ("grad_out",)),
    (dict(grad=2 * M + 39_996), ("tokens",)), (dict(grad=6 * M), ("workspace",)), (dict(workspace=M), ("workspace", "grad_out")),
    (dict(workspace=2 * M), ("workspace", "tokens")), (dict(grad=6 * M - 10 * 32 + 4), ("workspace",)),
    (dict(offsets=4 * M + 8, num_bags=4), ("offsets",)), (dict(offsets=4 * M - 32, num_bags=4), ("offsets",)),
    (dict(offsets=6 * M, num_bags=4), ("workspace", "offsets")),
], ids=str)
def test_gradients(rows_form, kw, names):
    _refused(_gradient(rows_form, **kw), *names)


@pytest.mark.parametrize("kw,names", [
    (dict(rows_out=4 * M + 4), ("rows_out", "values")), (dict(rows_out=4 * M - 36), ("rows_out", "values")),
    (dict(count=3 * M), ("count", "rows_out")), (dict(count=3 * M + 32), ("count", "rows_out")),
    (dict(count=4 * M), ("count", "values")), (dict(count=2 * M + 8), ("count", "tokens")), (dict(count=6 * M), ("count", "workspace")),
    (dict(rows_out=M), ("rows_out", "grad_out")), (dict(rows_out=2 * M), ("rows_out", "tokens")),
    (dict(rows_out=6 * M), ("rows_out", "workspace")), (dict(count=4 * M, num_tokens=3), ("count", "values")),
], ids=str)
def test_rows_form(kw, names):
    _refused(_gradient(1, **kw), *names)
