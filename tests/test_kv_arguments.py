"""What the operators around the quantized cache refuse, and where they find things for batches that do not fit: no GPU needed.

Refusals come before anything of the context is used, so a block of zeros stands in for one."""
import ctypes as C

import numpy as np
import pytest

from paper_2506_13472_b200 import binding as rb
from tests import kv_reference as ref

INVALID, SHAPE, ALIGN = rb.ROSAQ_ERR_INVALID_ARG, rb.ROSAQ_ERR_UNSUPPORTED_SHAPE, rb.ROSAQ_ERR_ALIGNMENT
CTX = C.create_string_buffer(1 << 16)
ROWS = 1 << 30          # an address that nothing reads


def kv(**change):
    a = dict(pages=1 << 20, n_pages=4, page_tokens=64, n_kv_heads=2, head_dim=128, bits=4)
    a.update(change)
    return rb._Kv(*a.values())


def batch(**change):
    a = dict(n_seqs=2, ld_table=3, row_start=4096, kv_len=8192, table=12288, prefix_table=None, prefix_tokens=0)
    a.update(change)
    return rb._KvBatch(*a.values())


BAD_KV = [(dict(pages=None), INVALID), (dict(n_pages=0), INVALID), (dict(bits=3), INVALID), (dict(bits=16), INVALID), (dict(n_kv_heads=0), INVALID),
          (dict(page_tokens=0), INVALID), (dict(page_tokens=8), SHAPE), (dict(page_tokens=48), SHAPE), (dict(page_tokens=2048), SHAPE),
          (dict(head_dim=96), SHAPE), (dict(head_dim=256), SHAPE), (dict(n_kv_heads=1 << 20), SHAPE), (dict(pages=(1 << 20) + 8), ALIGN)]
BAD_BATCH = [(dict(n_seqs=0), INVALID), (dict(ld_table=0), INVALID), (dict(row_start=None), INVALID), (dict(kv_len=None), INVALID),
             (dict(table=None), INVALID), (dict(row_start=4098), ALIGN), (dict(kv_len=8193), ALIGN), (dict(table=12290), ALIGN),
             (dict(ld_table=1 << 25), SHAPE)]
# (k or q, stride, v or out, stride, rows)
BAD_ROWS = [((None, 256, 2 * ROWS, 256, 5), INVALID), ((ROWS, 256, None, 256, 5), INVALID), ((ROWS, 248, 2 * ROWS, 256, 5), INVALID),
            ((ROWS, 256, 2 * ROWS, 128, 5), INVALID), ((ROWS, 256, 2 * ROWS, 256, -1), INVALID), ((ROWS + 8, 256, 2 * ROWS, 256, 5), ALIGN),
            ((ROWS, 256, 2 * ROWS + 2, 256, 5), ALIGN), ((ROWS, 260, 2 * ROWS, 256, 5), ALIGN), ((ROWS, 256, 2 * ROWS, 257, 5), ALIGN)]


def rows_call(name, k, b, x, ldx, y, ldy, n):
    f = getattr(rb.lib(), name)
    if name == "rosaq_attend":
        return f(CTX, C.byref(k) if k else None, C.byref(b) if b else None, x, ldx, k.n_kv_heads if k else 2, 0.1, y, ldy, n, None)
    return f(CTX, C.byref(k) if k else None, C.byref(b) if b else None, x, ldx, y, ldy, n, None)


@pytest.mark.parametrize("name", ["rosaq_kv_write", "rosaq_kv_read", "rosaq_attend"])
def test_rows_refused(name):
    good = (ROWS, 256, 2 * ROWS, 256, 5)
    for change, want in BAD_KV:
        assert rows_call(name, kv(**change), batch(), *good) == want, change
    for change, want in BAD_BATCH:
        assert rows_call(name, kv(), batch(**change), *good) == want, change
    for args, want in BAD_ROWS:
        assert rows_call(name, kv(), batch(), *args) == want, args
    assert rows_call(name, None, batch(), *good) == INVALID
    assert rows_call(name, kv(), None, *good) == INVALID
    assert rows_call(name, kv(), batch(), ROWS, 256, 2 * ROWS, 256, 0) == rb.ROSAQ_OK
    assert rows_call(name, kv(), batch(), None, 256, None, 256, 0) == rb.ROSAQ_OK
    # outputs in the pages; outputs over each other or over the queries
    assert rows_call(name, kv(), batch(), ROWS, 256, (1 << 20) + 4096, 256, 5) == INVALID
    if name != "rosaq_kv_write":
        assert rows_call(name, kv(), batch(), ROWS, 256, ROWS + 2 * 256 * 4, 256, 5) == INVALID
        assert rows_call(name, kv(), batch(), ROWS, 512, ROWS + 2 * 248, 512, 5) == INVALID
        assert rows_call(name, kv(), batch(), ROWS, 512, ROWS, 256, 5) == INVALID
    f = getattr(rb.lib(), name)
    assert f(None, *([C.byref(kv()), C.byref(batch()), ROWS, 256] + ([2, 0.1] if name == "rosaq_attend" else []) + [2 * ROWS, 256, 5, None])) == INVALID


def test_attend_refused():
    def call(hq=2, scale=0.1, **change):
        return rb.lib().rosaq_attend(CTX, C.byref(kv()), C.byref(batch(**change)), ROWS, 4096, hq, scale, 2 * ROWS, 4096, 5, None)
    assert call(hq=0) == INVALID and call(hq=3) == SHAPE
    assert call(scale=float("nan")) == INVALID and call(scale=float("inf")) == INVALID
    assert call(prefix_tokens=-1) == INVALID and call(prefix_tokens=5) == INVALID
    assert call(prefix_tokens=5, prefix_table=4098) == ALIGN and call(prefix_tokens=(1 << 30) + 1, prefix_table=4096) == SHAPE


def test_page_bytes():
    for heads, hd, bits, page in ((1, 64, 4, 16), (32, 128, 4, 64), (8, 128, 8, 256), (5, 64, 8, 1024)):
        assert rb.kv_page_bytes(heads, hd, bits, page) == heads * (page // 16) * (2 * 16 * hd * bits // 8 + 128)
    for args in ((0, 128, 4, 64), (1, 100, 4, 64), (1, 128, 5, 64), (1, 128, 4, 24)):
        with pytest.raises(rb.RosaqError):
            rb.kv_page_bytes(*args)


def rope_desc(**change):
    a = dict(head_dim=128, rot_dim=128, interleaved=0, scaling=0, base=10000.0, factor=1.0, low=1.0, high=32.0, context=4096.0, magnitude=1.0)
    a.update(change)
    return rb._RopeDesc(*a.values())


@pytest.mark.parametrize("change,want", [
    (dict(head_dim=0), INVALID), (dict(rot_dim=0), INVALID), (dict(rot_dim=7), INVALID), (dict(rot_dim=130), INVALID), (dict(interleaved=2), INVALID),
    (dict(scaling=4), INVALID), (dict(scaling=-1), INVALID), (dict(base=0.0), INVALID), (dict(base=float("inf")), INVALID),
    (dict(magnitude=float("nan")), INVALID), (dict(scaling=1, factor=0.0), INVALID), (dict(scaling=2, rot_dim=2), INVALID),
    (dict(scaling=3, low=32.0), INVALID), (dict(scaling=3, context=0.0), INVALID), (dict(scaling=3, high=float("nan")), INVALID),
    (dict(head_dim=512, rot_dim=258), SHAPE), (dict(head_dim=1 << 17), SHAPE)])
def test_rope_refused(change, want):
    h = C.c_void_p(5)
    assert rb.lib().rosaq_rope_create(CTX, C.byref(rope_desc(**change)), C.byref(h)) == want and not h.value


def test_rope_rows_refused():
    h = C.c_void_p()
    assert rb.lib().rosaq_rope_create(CTX, C.byref(rope_desc()), C.byref(h)) == rb.ROSAQ_OK
    def call(x=ROWS, ldx=256, heads=2, pos=4096, y=2 * ROWS, ldy=256, n=5, r=h):  # noqa: E306
        return rb.lib().rosaq_rope_apply(CTX, r, x, n, ldx, heads, pos, y, ldy, None)
    assert call(r=None) == INVALID and call(heads=0) == INVALID and call(heads=3) == INVALID and call(x=None) == INVALID
    assert call(pos=None) == INVALID and call(pos=4097) == ALIGN and call(x=ROWS + 8) == ALIGN and call(ldy=260) == ALIGN
    assert call(y=ROWS + 512) == INVALID and call(y=ROWS, ldy=512) == INVALID and call(n=-1) == INVALID and call(n=0) == rb.ROSAQ_OK
    assert rb.lib().rosaq_rope_free(h) == rb.ROSAQ_OK and rb.lib().rosaq_rope_free(None) == INVALID


# ---------------------------------------------------------------------------- where things are found
def locate(row_start, kv_len, table, rows, n_pages=7, heads=2, hd=64, bits=4, page=32):
    return rb.kv_locate(row_start, kv_len, table, rows, n_pages, heads, hd, bits, page)


def plain_places(row_start, kv_len, table, rows, n_pages, heads, hd, bits, page):
    """Row by row, by the header's words."""
    block, size = 4 * hd * bits + 128, rb.kv_page_bytes(heads, hd, bits, page)
    offset, slot = [-1] * rows, [-1] * rows
    for i, n in enumerate(kv_len):
        for row in range(row_start[i], min(row_start[i + 1], rows)):
            t = n - (row_start[i + 1] - row)
            p = table[i][t // page]
            offset[row], slot[row] = p * size + t % page // 16 * block, t % 16
    return offset, slot


@pytest.mark.parametrize("seed", range(6))
def test_locate(seed):
    rng = np.random.default_rng(seed)
    heads, hd, bits, page = int(rng.integers(1, 5)), int(rng.choice([64, 128])), int(rng.choice([4, 8])), int(rng.choice([16, 64, 256]))
    n, ld = int(rng.integers(1, 70)), 4
    new = rng.integers(0, 3 if seed % 2 else 50, n)
    lens = [int(rng.integers(a, ld * page + 1)) for a in np.minimum(new, ld * page)]
    new = np.minimum(new, lens)
    start = [0] + np.cumsum(new).tolist()
    table = rng.permutation(n * ld).reshape(n, ld).tolist()
    rows = start[-1] + 3
    st, offset, slot = rb.kv_locate(start, lens, table, rows, n * ld, heads, hd, bits, page)
    assert st == rb.ROSAQ_OK
    assert (offset, slot) == plain_places(start, lens, table, rows, n * ld, heads, hd, bits, page)


def test_locate_what_does_not_fit():
    size, block = rb.kv_page_bytes(2, 64, 4, 32), 4 * 64 * 4 + 128
    # a page past the cache, a negative one: the other blocks and sequences keep their places
    st, offset, slot = locate([0, 40, 42], [40, 2], [[1, 9], [-1, 0]], 42)
    assert st == INVALID and offset[:32] == [size + block * (i // 16) for i in range(32)] and offset[32:] == [-1] * 10 and slot[:2] == [0, 1]
    st, offset, _ = locate([0, 2, 4], [2, 2], [[7, 0], [6, 0]], 4)
    assert st == INVALID and offset == [-1, -1, 6 * size, 6 * size]
    # more new rows than tokens, a length past the page list, a negative length
    for lens in ([3, 5], [65, 5], [-4, 5]):
        st, offset, _ = locate([0, 4, 5], lens, [[0, 1], [2, 3]], 5)
        assert st == INVALID and offset == [-1] * 4 + [2 * size]
    # rows past the buffers are cut, rows in front of the first sequence belong to none
    st, offset, slot = locate([2, 9], [40], [[0, 1]], 5)
    assert st == INVALID and offset[:2] == [-1, -1] and slot[2:] == [1, 2, 3]
    # not ascending, which not every walk comes across: nothing out of bounds
    for start in ([0, 4, 2], [3, 1, 5], [0, -5, 5], [-3, 2, 5], [2 ** 31 - 1, 0, 5]):
        st, offset, _ = locate(start, [30, 30], [[0, 1], [2, 3]], 5)
        assert all(-1 <= o <= 7 * size - 2 * block for o in offset) and st in (INVALID, rb.ROSAQ_OK)
    st, offset, _ = locate([0, 2 ** 31 - 1], [2 ** 31 - 1], [[0, 1]], 5)
    assert st == INVALID and offset == [-1] * 5


def test_reference_layout_is_a_bijection():
    t, ch = np.meshgrid(np.arange(16), np.arange(128), indexing="ij")
    for hd in (64, 128):
        for bits in (4, 8):
            for value in (False, True):
                at, shift = ref.code_place(t[:, :hd], ch[:, :hd], hd, bits, value)
                assert len(set(zip((8 * at + shift).ravel().tolist()))) == 16 * hd and at.max() < 2 * hd * bits
                for byte in range(2 * hd * bits):           # no byte is shared by two tokens
                    assert len(set(t[:, :hd][at == byte].tolist())) == 1
