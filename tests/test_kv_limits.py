"""Limits of the quantized cache's batches that the host sees: no GPU needed."""
import ctypes as C

import pytest

from paper_2506_13472_b200 import binding as rb
from tests import test_gpu_kv_attention as gpu
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


# ---------------------------------------------------------------------------- which kernel a call runs on
def form(heads, group, hd, bits, page, lens, new, prefix=0, pages_of_seq=None):
    need = pages_of_seq or max(max(1, -(-n // page)) for n in lens)
    return rb.attend_forms(len(lens), sum(new), heads * group, heads, hd, need, page, bits, prefix)


def test_few_and_many_rows():
    """The rule of the kernels: 64 query rows per sequence and key/value head, and 2^22 of (row, head, token with room in the table)."""
    of = lambda rows, seqs, heads, group, pages, prefix=0: rb.attend_forms(seqs, rows, heads * group, heads, 128, pages, 64, 4, prefix)  # noqa: E731
    assert of(63, 1, 8, 1, 4096) == 0 and of(64, 1, 8, 1, 4096) == 1 and of(16, 1, 8, 4, 4096) == 1 and of(15, 1, 8, 4, 4096) == 0
    assert of(64, 1, 1, 1, 1024) == 1 and of(64, 1, 1, 1, 1023) == 0
    assert of(65, 2, 8, 1, 4096) == 0 and of(127, 2, 8, 1, 4096) == 1            # rows of a sequence: rounded up
    assert of(64, 64, 8, 1, 64, 8192) == 2 and of(64, 64, 8, 1, 64, 8191) == 0   # behind a prefix all rows are one sequence's
    assert of(64, 1, 8, 1, 4096, 8192) == 3 and of(0, 1, 8, 1, 4096) == 0 and of(0, 0, 8, 1, 1) == 0
    for bad in ((64, 1, 8, 1, 0), (-1, 1, 8, 1, 4), (1, 0, 8, 1, 4), (1, 1, 8, 1, 4, -1)):
        with pytest.raises(rb.RosaqError):
            of(*bad)


def test_what_the_gpu_tests_run_on():
    """The cases of the GPU tests, by the kernel that they are there for: a rule that moves must not take their kernel from them."""
    assert [form(*c) for c in gpu.CASES] == [0] * len(gpu.CASES)
    for heads, group, hd, bits, page, lens, new in gpu.MANY:
        rows = -(-sum(new) // len(lens)) * group
        room = max(max(-(-n // page) for n in lens), -(-(1 << 22) // (rows * len(lens) * heads * page)))
        assert form(heads, group, hd, bits, page, lens, new, pages_of_seq=room) == 1
    prefixes = [p.args[1] for p in gpu.test_attend_prefix.pytestmark if p.name == "parametrize"][0]
    assert [form(*c[:5], c[6], c[7], c[5]) for c in prefixes] == [0, 0, 2, 0, 0, 2, 2, 2]
    # (calls of two graphs; waits, scales, sizes, infinities: one new row each, and the many that those tests take)
    assert [form(4, 4, 128, 4, 64, [5000, 9000], [n, n], p) for n, p in ((60, 0), (1, 0), (30, 8999))] == [1, 0, 3]
    for many in (0, 1):
        new = lambda n: n if many else 1  # noqa: E731
        assert form(2, 4, 128, 4, 64, [20000, 40], [new(20)] * 2) == form(2, 4, 128, 8, 64, [20000, 40], [new(20)] * 2) == many
        assert form(2, 2, 64, 8, 64, [33000], [new(40)]) == form(2, 4, 128, 4, 1024, [4000], [new(40)], pages_of_seq=40) == many
        assert form(2, 4, 128, 8, 64, [33000], [new(40)]) == form(4, 4, 128, 4, 64, [8200, 90], [new(40)] * 2) == many
        assert form(4, 1, 128, 4, 64, [8200, 90], [new(70)] * 2) == form(4, 4, 128, 4, 64, [8200], [new(40)]) == many
        assert form(4, 4, 128, 4, 1024, [2048] * 3, [new(48)] * 3) == many
