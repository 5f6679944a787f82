"""Limits of the quantized cache's batches that the host sees: no GPU needed."""
import ctypes as C

import pytest

from paper_2506_13472_b200 import binding as rb
from tests.test_kv_arguments import CTX, INVALID, ROWS, SHAPE, batch, kv, rows_call


@pytest.mark.parametrize("name", ["rosaq_kv_write", "rosaq_kv_read", "rosaq_attend"])
def test_columns_of_a_table_refused(name):
    for change, want in ((dict(table_pages=-1), INVALID), (dict(table_pages=4), INVALID), (dict(ld_table=1 << 25, table_pages=(1 << 24) + 1), SHAPE)):
        assert rows_call(name, kv(), batch(**change), ROWS, 256, 2 * ROWS, 256, 5) == want, change
    for change in (dict(table_pages=3), dict(table_pages=1), dict(ld_table=1 << 25, table_pages=1 << 24)):
        assert rows_call(name, kv(), batch(**change), ROWS, 256, 2 * ROWS, 256, 0) == rb.ROSAQ_OK, change


def test_locate_in_columns_of_a_wider_table():
    """The first pages of each row belong to the batch: lengths past them do not fit, whatever stands there."""
    size = rb.kv_page_bytes(2, 64, 4, 32)
    table = [[1, 2, 3, 4], [5, 6, 0, 1]]
    where = lambda lens, pages: rb.kv_locate([0, 1, 2], lens, table, 2, 7, 2, 64, 4, 32, table_pages=pages)  # noqa: E731
    assert where([97, 33], 0) == (rb.ROSAQ_OK, [4 * size, 6 * size], [0, 0])
    assert where([64, 33], 2) == (rb.ROSAQ_OK, [2 * size + 4 * 64 * 4 + 128, 6 * size], [15, 0])
    assert where([65, 33], 2) == (INVALID, [-1, 6 * size], [-1, 0])
    assert where([1, 128], 2) == (INVALID, [size, -1], [0, -1])


def test_scales_refused():
    call = lambda scale: rb.lib().rosaq_attend(CTX, C.byref(kv()), C.byref(batch()), ROWS, 256, 2, scale, 2 * ROWS, 256, 0, None)  # noqa: E731
    for scale in (2.0 ** 58, -2.0 ** 58, 0.0, 1e-45):
        assert call(scale) == rb.ROSAQ_OK, scale
    for scale in (2.0 ** 58 * 1.001, -1e30, float("inf"), float("nan")):
        assert call(scale) == INVALID, scale


@pytest.mark.parametrize("name", ["rosaq_kv_write", "rosaq_kv_read", "rosaq_attend"])
def test_batches_of_no_sequences(name):
    none = dict(n_seqs=0, ld_table=0, row_start=None, kv_len=None, table=None)
    assert rows_call(name, kv(), batch(**none), None, 256, None, 256, 0) == rb.ROSAQ_OK
    assert rows_call(name, kv(), batch(n_seqs=0), ROWS, 256, 2 * ROWS, 256, 0) == rb.ROSAQ_OK
    for n in (1, -1):
        assert rows_call(name, kv(), batch(**none), ROWS, 256, 2 * ROWS, 256, n) == INVALID
    assert rows_call(name, kv(), batch(n_seqs=-1), None, 256, None, 256, 0) == INVALID
    offset, slot = C.c_int64(), C.c_int32()
    assert rb.lib().rosaq_kv_locate(C.byref(kv()), C.byref(batch(**none)), 0, C.byref(offset), C.byref(slot)) == rb.ROSAQ_OK
