"""Rotary positions, the quantized paged cache and the attention that reads it, against plain 64-bit implementations (kv_reference), with the
bounds derived there."""
import math

import numpy as np
import pytest
import torch

from paper_2506_13472_b200 import binding as rb
from tests import kv_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = rb.Context(0)
    yield c
    c.close()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def same(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


def inside(got, want, bound, where=""):
    got = got.double() if torch.is_tensor(got) else np.asarray(got, np.float64)
    ratio = abs(got - want) / bound
    worst = float(ratio.max()) if ratio.shape[0] else 0.0
    assert worst <= 1.0, f"{where}: {worst:.2f} bounds"
    return worst


# ---------------------------------------------------------------------------------------------- rotary positions
def frequencies(rot, scaling, base=10000.0, factor=4.0, low=1.0, high=32.0, context=4096.0):
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if scaling == "linear":
        return f / factor
    if scaling == "by_parts":
        keep = np.clip((context * f / (2 * math.pi) - low) / (high - low), 0, 1)
        return f * (keep + (1 - keep) / factor)
    return f


@pytest.mark.parametrize("rows,heads,hd,rot,interleaved,scaling,far", [
    (1, 1, 128, 128, False, "plain", 1),              # position 0: as it was
    (1, 64, 128, 128, False, "plain", 1 << 30),       # one token, far away
    (64, 40, 128, 128, True, "plain", 4096),
    (777, 3, 64, 64, False, "linear", 1 << 20),
    (50, 5, 128, 32, True, "ntk", 100000),            # part of the head
    (333, 2, 128, 64, False, "by_parts", 131072),
    (9, 7, 80, 24, False, "plain", 9000),             # pairs that no 16-byte access holds
    (9, 7, 72, 6, True, "by_parts", 9000),
    (31, 9, 2 * 8, 2, True, "plain", 9000),
    (5, 2, 256, 256, False, "plain", 9000),
    (3, 8, 136, 130, True, "linear", 1 << 24),
])
def test_rope(ctx, rows, heads, hd, rot, interleaved, scaling, far):
    rng = np.random.default_rng(rows + hd)
    wide = (heads * hd + 7) // 8 * 8 + 8
    x = rng.standard_normal((rows, wide)).astype(np.float16)
    pos = rng.integers(0, far, rows).astype(np.int32)
    magnitude = 1.25 if scaling == "by_parts" else 1.0
    r = ctx.rope_create(hd, rot, interleaved=interleaved, scaling=scaling, factor=4.0, low=1.0, high=32.0, context=4096.0, magnitude=magnitude)
    xs = dev(x)
    buf = torch.full((rows + 1, wide), 7.0, dtype=torch.float16, device="cuda")
    out = buf[:rows, :heads * hd]
    ctx.rope(xs[:, :heads * hd], dev(pos), r, out=out)
    want, bound = ref.rope(x[:, :heads * hd].reshape(rows, heads, hd), pos, frequencies(rot, scaling), rot, interleaved, magnitude)
    inside(out.cpu().numpy().reshape(rows, heads, hd), want, bound)
    assert torch.all(buf[rows:] == 7.0) and torch.all(buf[:, heads * hd:] == 7.0)
    got = out.reshape(rows, heads, hd)
    assert same(got[..., rot:], xs[:, :heads * hd].reshape(rows, heads, hd)[..., rot:])          # the rest of the head, bit for bit
    ctx.rope(xs[:, :heads * hd], dev(pos), r, out=xs[:, :heads * hd])                            # in place
    assert same(xs[:, :heads * hd], out) and same(xs[:, heads * hd:], dev(x)[:, heads * hd:])


def test_rope_negative_positions_turn_back(ctx):
    x = torch.randn((40, 4 * 128), device="cuda").half()
    pos = ints(list(range(0, 40000, 1000)))
    r = ctx.rope_create(128)
    back = ctx.rope(ctx.rope(x, pos, r), -pos, r)
    # two roundings of values no larger than the pair's length
    size = x.double().view(40, 4, 2, 64).pow(2).sum(2, keepdim=True).sqrt().expand(40, 4, 2, 64).reshape(40, 512)
    inside(back, x.double(), 2 * 2.0 ** -11 * 2 * size + 1e-6)
    far = ctx.rope(x, ints([-2 ** 31] * 40), r)
    want, bound = ref.rope(x.cpu().numpy().reshape(40, 4, 128), [-2 ** 31] * 40, frequencies(128, "plain"), 128, False, 1.0)
    inside(far.cpu().numpy().reshape(40, 4, 128), want, bound)


# ---------------------------------------------------------------------------------------------- the cache
def layout(rng, lens, page, extra=2):
    """(table as lists, number of pages): pages in no order, some of the cache unused."""
    need = [max(1, (n + page - 1) // page) for n in lens]
    order = rng.permutation(sum(need) + extra)
    table, at = np.full((len(lens), max(need)), -5, np.int64), 0           # entries behind a sequence's pages are never looked at
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, sum(need) + extra


@pytest.mark.parametrize("heads,hd,bits,page,old,new", [
    (1, 128, 4, 16, [0], [1]),
    (5, 128, 4, 64, [0, 63, 64, 15, 31], [1, 1, 1, 1, 1]),                     # decoding, at all sides of a page and of a block
    (3, 64, 8, 32, [0, 1, 15, 16, 17, 100], [16, 15, 1, 16, 33, 0]),           # blocks that begin and end inside
    (2, 128, 8, 16, [5, 0, 250], [300, 0, 7]),
    (9, 64, 4, 256, [3, 200], [40, 500]),
    (4, 128, 4, 128, [0] * 40, [i % 3 for i in range(40)]),
])
@pytest.mark.parametrize("kind", ["normal", "odd"])
def test_write_and_read(ctx, heads, hd, bits, page, old, new, kind):
    rng = np.random.default_rng(heads * hd + bits + len(old))
    lens = [a + b for a, b in zip(old, new)]
    table, n_pages = layout(rng, lens, page)
    rows = sum(new)
    k, v = (rng.standard_normal((rows, heads, hd)).astype(np.float16) for _ in range(2))
    if kind == "odd":
        # one value for all, ranges of one step and of everything, ties, signs of zero, no numbers
        k[0::7] = np.float16(1.5)
        k[1::7] *= np.float16(6e-8) / np.float16(1e-1)
        k[2::7] = rng.choice(np.array([-65504, 65504, 0], np.float16), k[2::7].shape)
        k[3::7] = rng.integers(0, 31, k[3::7].shape) / np.float16(2)
        k[4::7] = rng.choice(np.array([0.0, -0.0], np.float16), k[4::7].shape)
        k[5::7, :, 3::11], k[5::7, :, 4::13], k[5::7, :, 7] = np.nan, np.inf, -np.inf
        k[6::7] = np.nan
        v[0::3] += np.float16(100)
        v[1::3, :, :hd - 1] = np.nan
        v[2::3] = rng.choice(np.array([np.inf, -np.inf], np.float16), v[2::3].shape)
    cache = ref.Cache(heads, hd, bits, page, n_pages, rng)
    before = cache.pages.copy()
    start, at = [0] + np.cumsum(new).tolist(), 0
    for i, n in enumerate(new):
        cache.put(table[i], old[i], k[at:at + n], v[at:at + n])
        at += n
    wide = heads * hd + 24
    kv = torch.full((rows + 5, 2 * wide), float("nan"), dtype=torch.float16, device="cuda")      # rows behind the last sequence
    kd, vd = kv[:, 8:8 + heads * hd], kv[:, wide:wide + heads * hd]
    kd[:rows], vd[:rows] = dev(k.reshape(rows, -1)), dev(v.reshape(rows, -1))
    pages = dev(before.reshape(n_pages, -1))
    held = rb.KvCache(pages, heads, hd, bits, page)
    batch = rb.KvBatch(ints(start), ints(lens), ints(table.tolist()))
    ctx.kv_write(held, batch, kd, vd)
    assert ctx.last_status() == rb.ROSAQ_OK
    got = pages.cpu().numpy().reshape(before.shape)
    assert np.array_equal(got, cache.pages)
    back = torch.full((rows + 5, 2 * wide), 7.0, dtype=torch.float16, device="cuda")
    kb, vb = back[:, :heads * hd], back[:, wide + 8:wide + 8 + heads * hd]
    ctx.kv_read(held, batch, rows + 5, k=kb, v=vb)
    assert ctx.last_status() == rb.ROSAQ_OK
    for x, b in ((k, kb), (v, vb)):
        assert np.array_equal(b[:rows].cpu().numpy(),
                              ref.held(*ref.quantize(x, bits)).reshape(rows, -1))
    assert torch.all(back[rows:] == 7.0) and torch.all(back[:, heads * hd:wide + 8] == 7.0) and torch.all(back[:, wide + 8 + heads * hd:] == 7.0)


def test_write_matches_the_formula_at_every_quotient(ctx):
    """Codes of all fp16 numbers of [0, 1] over many scales: the corrected quotient is the IEEE one."""
    rng = np.random.default_rng(5)
    heads, hd, rows = 8, 128, 800
    x = rng.integers(0, 0x3c01, (rows, heads, hd)).astype(np.uint16).view(np.float16)
    x[..., 0] = 0
    x[..., 1] = rng.integers(0x0001, 0x7c00, (rows, heads)).astype(np.uint16).view(np.float16)
    for bits in (4, 8):
        pages = torch.zeros((50, rb.kv_page_bytes(heads, hd, bits, 16)), dtype=torch.uint8, device="cuda")
        held = rb.KvCache(pages, heads, hd, bits, 16)
        batch = rb.KvBatch(ints([0, rows]), ints([rows]), ints([list(range(50))]))
        d = dev(x.reshape(rows, -1))
        ctx.kv_write(held, batch, d, d)
        k, v = ctx.kv_read(held, batch, rows)
        want = ref.held(*ref.quantize(x, bits)).reshape(rows, -1)
        assert np.array_equal(k.cpu().numpy(), want) and np.array_equal(v.cpu().numpy(), want)


# ---------------------------------------------------------------------------------------------- attention
def filled(rng, heads, hd, bits, page, lens, extra=2, loud=1.0, v_size=1.0, offset=0.0):
    """Pages (torch) with quantized normal keys and values for sequences of those lengths, whatever bytes elsewhere; and the table."""
    table, n_pages = layout(rng, lens, page, extra)
    pages = torch.from_numpy(rng.integers(0, 256, (n_pages, rb.kv_page_bytes(heads, hd, bits, page)), dtype=np.uint8)).cuda()
    held = rb.KvCache(pages, heads, hd, bits, page)
    return held, table


def fill(ctx, rng, held, table, lens, loud=1.0, v_size=1.0, offset=0.0):
    rows, d = sum(lens), held.width
    if rows == 0:
        return
    g = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30)))
    k = torch.randn((rows, d), device="cuda", generator=g)
    k[:, ::17] *= loud
    v = torch.randn((rows, d), device="cuda", generator=g) * v_size + offset
    batch = rb.KvBatch(ints([0] + np.cumsum(lens).tolist()), ints(lens), ints(table.tolist()))
    ctx.kv_write(held, batch, (k + offset).half(), v.half())
    assert ctx.last_status() == rb.ROSAQ_OK


def expect(held, table, lens, new, q, scale, prefix=None):
    """(out, bound) of all rows."""
    outs, bounds, at = [], [], 0
    hd, hq = held.head_dim, q.shape[1] // held.head_dim
    args = (held.pages, held.n_kv_heads, hd, held.bits, held.page_tokens)
    pre, np_ = (ref.values(*args, prefix[0], prefix[1]), prefix[1]) if prefix else (None, 0)
    for i, (n, m) in enumerate(zip(lens, new)):
        if m == 0:
            continue
        kv = ref.values(*args, ints(table[i].tolist()), n)
        if pre:
            kv = [[torch.cat([a, b]) for a, b in zip(x, y)] for x, y in zip(pre, kv)]
        seen = torch.arange(np_ + n, device="cuda")[None, :] < np_ + n - m + 1 + torch.arange(m, device="cuda")[:, None]
        o, b = ref.attention(q[at:at + m].double().view(m, hq, hd), kv, seen, scale)
        outs.append(o.reshape(m, -1)), bounds.append(b.reshape(m, -1))
        at += m
    return torch.cat(outs), torch.cat(bounds)


CASES = [
    # heads, group, hd, bits, page, lengths, new
    (1, 1, 128, 4, 16, [1], [1]),                                       # one token sees itself
    (2, 1, 128, 4, 64, [15, 16, 17, 64, 65, 1], [1] * 6),               # ends of blocks and pages
    (32, 1, 128, 4, 64, [333], [1]),
    (8, 4, 128, 8, 64, [1000, 3, 129], [1, 1, 1]),
    (2, 8, 64, 4, 32, [700, 20], [1, 1]),
    (1, 5, 64, 8, 128, [257, 2049], [1, 1]),
    (3, 13, 128, 4, 64, [100], [1]),                                    # more query heads than a tile of rows
    (2, 4, 128, 4, 64, [40, 7, 9, 100], [7, 7, 0, 33]),                 # several new rows, none, all of them new
    (2, 1, 64, 8, 16, [150], [150]),                                    # a prompt
    (2, 2, 128, 4, 256, [5000, 1, 900], [130, 1, 64]),
    (40, 1, 128, 4, 64, [50] * 70, [1] * 70),                           # more tiles than CTAs
    (1, 1, 128, 8, 64, [i + 1 for i in range(300)], [1] * 300),
    (1, 4, 128, 4, 1024, [70000], [1]),                                 # one tile over all CTAs
]


MANY = [
    # many query rows per sequence and key/value head, in a table with room for long sequences (which is what the choice of the kernel goes by)
    (2, 1, 64, 8, 16, [150], [150]),                                    # a prompt
    (2, 2, 128, 4, 256, [5000, 1, 900], [130, 1, 64]),
    (1, 64, 128, 4, 64, [1], [1]),                                      # one token that all rows see
    (3, 16, 128, 8, 16, [15, 16, 17, 64, 65, 0, 700], [4, 4, 4, 4, 17, 0, 4]),   # ends of blocks and pages
    (1, 7, 64, 4, 32, [63, 64, 65, 129, 200], [40, 64, 20, 8, 30]),     # chunks, odd groups, tiles that end anywhere
    (5, 2, 64, 4, 128, [300] * 40, [37] * 40),                          # more tiles than CTAs
    (1, 2, 128, 4, 1024, [70000], [100]),                               # one tile over all CTAs
    (2, 3, 128, 8, 64, [600, 600], [600, 100]),                         # rows that see next to nothing beside rows that see all
]


@pytest.mark.parametrize("heads,group,hd,bits,page,lens,new,wide", [(*c, False) for c in CASES] + [(*c, True) for c in MANY])
def test_attend(ctx, heads, group, hd, bits, page, lens, new, wide):
    rng = np.random.default_rng(heads + 10 * group + sum(lens))
    held, table = filled(rng, heads, hd, bits, page, lens)
    if wide:
        rows = -(-sum(new) // len(lens)) * group
        assert rows >= 64
        room = -(-(1 << 22) // (rows * len(lens) * heads * page))
        table = np.pad(table, ((0, 0), (0, max(0, room - table.shape[1]))), constant_values=-5)
    fill(ctx, rng, held, table, lens, loud=5.0)
    rows, d = sum(new), heads * group * hd
    wide = d + 16
    q = torch.from_numpy(rng.standard_normal((rows + 3, wide)).astype(np.float16)).cuda()
    q[rows:] = float("nan")
    buf = torch.full((rows + 3, wide), 7.0, dtype=torch.float16, device="cuda")
    out = buf[:, 8:8 + d]
    batch = rb.KvBatch(ints([0] + np.cumsum(new).tolist()), ints(lens), ints(table.tolist()))
    ctx.attend(q[:, :d], held, batch, out=out)
    assert ctx.last_status() == rb.ROSAQ_OK
    want, bound = expect(held, table, lens, new, q[:rows, :d], hd ** -0.5)
    inside(out[:rows], want, bound)
    assert torch.all(buf[rows:] == 7.0) and torch.all(buf[:, :8] == 7.0) and torch.all(buf[:, 8 + d:] == 7.0)
    for _ in range(3):
        again = torch.full((rows + 3, d), 7.0, dtype=torch.float16, device="cuda")
        ctx.attend(q[:, :d], held, batch, out=again)
        assert same(again, out)
    # the queries' own memory
    mine = q[:, :d].clone()
    ctx.attend(mine, held, batch, out=mine)
    assert same(mine[:rows], out[:rows])


@pytest.mark.parametrize("heads,group,hd,bits,page,prefix,lens,new", [
    (2, 1, 128, 4, 64, 1, [1, 0, 5], [1, 0, 1]),
    (1, 4, 128, 4, 64, 777, [3, 100, 64], [1, 1, 1]),
    (8, 4, 128, 4, 64, 2500, [i % 40 + 1 for i in range(64)], [1] * 64),
    (2, 8, 64, 8, 16, 333, [30, 9, 400], [3, 9, 20]),
    (1, 3, 128, 8, 32, 4096, [40], [40]),
    (1, 3, 128, 8, 32, 40000, [40], [40]),                              # many rows behind the prefix from here on
    (2, 8, 64, 4, 16, 9001, [3, 1, 0, 70, 9], [3, 1, 0, 30, 9]),
    (8, 4, 128, 4, 64, 4100, [i % 40 + 1 for i in range(33)], [1] * 33),
])
def test_attend_prefix(ctx, heads, group, hd, bits, page, prefix, lens, new):
    rng = np.random.default_rng(prefix + sum(lens))
    held, table = filled(rng, heads, hd, bits, page, [prefix] + lens)
    fill(ctx, rng, held, table, [prefix] + lens, loud=4.0)
    rows = sum(new)
    q = torch.from_numpy(rng.standard_normal((rows, heads * group * hd)).astype(np.float16)).cuda()
    pre = (ints(table[0].tolist()), prefix)
    batch = rb.KvBatch(ints([0] + np.cumsum(new).tolist()), ints(lens), ints(table[1:].tolist()), prefix=pre)
    out = ctx.attend(q, held, batch, scale=0.2)
    assert ctx.last_status() == rb.ROSAQ_OK
    want, bound = expect(held, table[1:], lens, new, q, 0.2, pre)
    inside(out, want, bound)
    assert same(ctx.attend(q, held, batch, scale=0.2), out)
    mine = q.clone()
    assert same(ctx.attend(mine, held, batch, scale=0.2, out=mine), out)


@pytest.mark.parametrize("v_size,offset,q_size,loud", [
    (1e-4, 0.0, 1.0, 1.0),          # values whose scales are subnormal
    (3000.0, 0.0, 1.0, 1.0),
    (1.0, 50.0, 0.05, 1.0),         # least values far from zero
    (1.0, 0.0, 30.0, 6.0),          # scores in the hundreds: one token takes all
    (1.0, 0.0, 1e-6, 1.0),          # subnormal queries
    (1.0, 0.0, 0.0, 1.0),           # all tokens alike
])
@pytest.mark.parametrize("bits", [4, 8])
def test_attend_sizes_of_values(ctx, bits, v_size, offset, q_size, loud):
    rng = np.random.default_rng(3)
    lens, new = [600, 31], [2, 1]
    held, table = filled(rng, 2, 128, bits, 64, lens)
    fill(ctx, rng, held, table, lens, loud=loud, v_size=v_size, offset=offset)
    q = torch.from_numpy((q_size * rng.standard_normal((3, 6 * 128))).astype(np.float16)).cuda()
    batch = rb.KvBatch(ints([0, 2, 3]), ints(lens), ints(table.tolist()))
    out = ctx.attend(q, held, batch)
    want, bound = expect(held, table, lens, new, q, 128 ** -0.5)
    inside(out, want, bound)


def test_attend_rows_that_are_no_numbers(ctx):
    """A NaN or an infinity in a query reaches its own head and row only; so does one behind the last token of a sequence."""
    rng = np.random.default_rng(9)
    lens, new = [100, 90], [3, 1]
    held, table = filled(rng, 2, 128, 4, 64, lens)
    fill(ctx, rng, held, table, lens)
    raw = held.pages.view(held.pages.shape[0], 2, 4, -1)
    for i, n in enumerate(lens):                              # pairs behind the last token: infinities and NaNs
        block = raw[table[i, n // 64], :, n % 64 // 16]
        pairs = block[:, 2048:].clone().view(torch.int16).view(2, 2, 16, 2)
        pairs[:, :, n % 16:] = ints([0x7c00, 0x7e00]).to(torch.int16)
        block[:, 2048:] = pairs.view(2, 64).view(torch.uint8).view(2, 128)
    q = torch.from_numpy(rng.standard_normal((4, 4 * 128)).astype(np.float16)).cuda()
    batch = rb.KvBatch(ints([0, 3, 4]), ints(lens), ints(table.tolist()))
    clean = ctx.attend(q, held, batch)
    want, bound = expect(held, table, lens, new, q, 128 ** -0.5)
    inside(clean, want, bound)
    q[1, 5], q[2, 128], q[3, 300] = float("nan"), float("inf"), float("-inf")
    got = ctx.attend(q, held, batch)
    bad = torch.zeros((4, 4), dtype=torch.bool, device="cuda")
    bad[1, 0] = bad[2, 1] = bad[3, 2] = True
    assert torch.equal(torch.isnan(got.view(4, 4, 128)).any(-1), bad) and torch.equal(torch.isnan(got.view(4, 4, 128)).all(-1), bad)
    assert same(got.view(4, 4, 128)[~bad], clean.view(4, 4, 128)[~bad])


def test_attend_sees_nothing(ctx):
    """Sequences without a token: zeros, or the prefix alone."""
    rng = np.random.default_rng(2)
    held, table = filled(rng, 2, 64, 4, 16, [33, 5])
    fill(ctx, rng, held, table, [33, 5])
    q = torch.randn((3, 4 * 64), device="cuda").half()
    lens = ints([0, 0])
    out = ctx.attend(q, held, rb.KvBatch(ints([0, 2, 3]), lens, ints(table.tolist())))
    # more rows than tokens: the first rows see nothing
    assert torch.all(out == 0)
    pre = (ints(table[0].tolist()), 33)
    out = ctx.attend(q, held, rb.KvBatch(ints([0, 2, 3]), lens, ints(table.tolist()), prefix=pre))
    want, bound = ref.attention(q.double().view(3, 4, 64), ref.values(held.pages, 2, 64, 4, 16, pre[0], 33),
                                torch.ones((3, 33), dtype=torch.bool, device="cuda"), 0.125)
    inside(out, want.reshape(3, -1), bound.reshape(3, -1))
    out = torch.full((3, 256), 7.0, device="cuda").half()
    ctx.attend(q, held, rb.KvBatch(ints([0, 0, 0]), lens, ints(table.tolist())), out=out)           # no rows at all
    assert torch.all(out == 7.0) and ctx.last_status() == rb.ROSAQ_OK


def test_batches_that_do_not_fit_are_reported(ctx):
    """What the arrays say wrongly is cut, reported, and costs other sequences nothing."""
    rng = np.random.default_rng(4)
    held, table = filled(rng, 2, 64, 8, 16, [40, 40, 40])
    fill(ctx, rng, held, table, [40, 40, 40])
    q = torch.randn((3, 2 * 64), device="cuda").half()
    start, lens = ints([0, 1, 2, 3]), ints([40, 40, 40])
    good = ctx.attend(q, held, rb.KvBatch(start, lens, ints(table.tolist())))
    kept = held.pages.clone()
    for what in ("page", "negative", "length", "rows"):
        t, n, s = table.copy(), [40, 40, 40], [0, 1, 2, 3]
        if what == "page":
            t[1, 1] = held.pages.shape[0]
        elif what == "negative":
            t[1, 0] = -1
        elif what == "length":
            n[1] = 49
        else:
            s[3] = 9
        b = rb.KvBatch(ints(s), ints(n), ints(t.tolist()))
        got = ctx.attend(q, held, b)
        assert ctx.last_status() == rb.ROSAQ_ERR_INVALID_ARG and ctx.last_status() == rb.ROSAQ_OK, what
        rest = [0, 2] if what != "rows" else [0, 1]
        assert same(got[rest], good[rest]), what
        if what == "page":
            continue                                          # (the new row lies in another page)
        k, v = ctx.kv_read(held, b, 3)
        assert ctx.last_status() == rb.ROSAQ_ERR_INVALID_ARG or what == "negative", what
    b = rb.KvBatch(start, ints([40, 17, 40]), ints([table[0].tolist(), [table[1][0], -7, 0], table[2].tolist()]))
    x = torch.randn((3, 2 * 64), device="cuda").half()
    ctx.kv_write(held, b, x, x)
    assert ctx.last_status() == rb.ROSAQ_ERR_INVALID_ARG
    same_pages = [p for p in range(held.pages.shape[0]) if p not in (table[0][2], table[2][2])]
    assert torch.equal(held.pages[same_pages], kept[same_pages])


# ---------------------------------------------------------------------------------------------- as they are used
def step(ctx, x, w, r, held, batch, positions, rope, heads, kv_heads, hd):
    """A decoding step of the attention half of a layer."""
    d, dk = heads * hd, kv_heads * hd
    qkv = torch.empty((x.shape[0], d + 2 * dk), dtype=torch.float16, device="cuda")
    ctx.linear_multi(x, w[:3], outs=[qkv[:, :d], qkv[:, d:d + dk], qkv[:, d + dk:]])
    ctx.rope(qkv[:, :d + dk], positions, rope, out=qkv[:, :d + dk])
    ctx.kv_write(held, batch, qkv[:, d:d + dk], qkv[:, d + dk:])
    ctx.attend(qkv[:, :d], held, batch, out=qkv[:, :d])
    return ctx.linear(qkv[:, :d], w[3], r)


def test_a_decoding_step(ctx):
    """q/k/v linears, positions, cache, attention, rotated o_proj: by calls, captured and replayed as the sequences grow, on a stream of its
    own, and in other streams' contexts."""
    rng = np.random.default_rng(11)
    heads, kv_heads, hd, n = 4, 2, 128, 9
    d, dk = heads * hd, kv_heads * hd
    mat = lambda a, b: torch.from_numpy((0.05 * rng.standard_normal((a, b))).astype(np.float16)).cuda()  # noqa: E731
    blocks = np.stack([np.linalg.qr(rng.standard_normal((hd, hd)))[0] for _ in range(heads)]).astype(np.float32)
    w = [ctx.quantize(mat(d, m), None, bits=4, k_salient=128) for m in (d, dk, dk)]
    w.append(ctx.quantize(mat(d, d), dev(blocks), bits=4, k_salient=128))
    r = ctx.rotation_create(dev(blocks.astype(np.float16)))
    rope = ctx.rope_create(hd)
    lens0 = [int(a) for a in rng.integers(0, 200, n)]
    held, table = filled(rng, kv_heads, hd, 4, 64, [a + 12 for a in lens0])
    fill(ctx, rng, held, table, lens0)
    first = held.pages.clone()
    xs = [mat(n, d) for _ in range(3)]
    lens, start = ints([a + 1 for a in lens0]), ints(list(range(n + 1)))
    positions = ints(lens0)
    batch = rb.KvBatch(start, lens, ints(table.tolist()))
    want = []
    for x in xs:
        want.append(step(ctx, x, w, r, held, batch, positions, rope, heads, kv_heads, hd).clone())
        lens += 1
        positions += 1
    assert ctx.last_status() == rb.ROSAQ_OK
    last = held.pages.clone()
    # the first step piece by piece against the plain forms
    q, k, v = ctx.linear_multi(xs[0], w[:3])
    f = frequencies(hd, "plain")
    qr, qb = ref.rope(q.cpu().numpy().reshape(n, heads, hd), lens0, f, hd, False, 1.0)
    q1 = ctx.rope(q, ints(lens0), rope)
    inside(q1.cpu().numpy().reshape(n, heads, hd), qr, qb)
    held2 = rb.KvCache(first.clone(), kv_heads, hd, 4, 64)
    b1 = rb.KvBatch(start, ints([a + 1 for a in lens0]), ints(table.tolist()))
    ctx.kv_write(held2, b1, ctx.rope(k, ints(lens0), rope), v)
    o = ctx.attend(q1, held2, b1)
    ow, ob = expect(held2, table, [a + 1 for a in lens0], [1] * n, q1, hd ** -0.5)
    inside(o, ow, ob)
    assert same(ctx.linear(o, w[3], r), want[0])
    # captured
    x = xs[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = step(ctx, x, w, r, held, batch, positions, rope, heads, kv_heads, hd)
        lens += 1
        positions += 1
    held.pages.copy_(first)
    lens.copy_(ints([a + 1 for a in lens0]))
    positions.copy_(ints(lens0))
    for i in range(3):
        x.copy_(xs[i])
        graph.replay()
        assert same(y, want[i]), i
    torch.cuda.synchronize()
    assert torch.equal(held.pages, last) and ctx.last_status() == rb.ROSAQ_OK


def test_two_contexts_at_once(ctx):
    """Calls that overlap on the GPU need a context each."""
    rng = np.random.default_rng(12)
    lens = [3000, 1, 700]
    held, table = filled(rng, 2, 128, 4, 64, lens)
    fill(ctx, rng, held, table, lens)
    q = [torch.randn((3, 8 * 128), device="cuda").half() for _ in range(2)]
    batch = rb.KvBatch(ints([0, 1, 2, 3]), ints(lens), ints(table.tolist()))
    want = [ctx.attend(x, held, batch).clone() for x in q]
    other = rb.Context(0)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i, c in enumerate((ctx, other)):
            with torch.cuda.stream(streams[i]):
                outs[i].append(c.attend(q[i], held, batch))
    torch.cuda.synchronize()
    assert all(same(o, want[i]) for i in range(2) for o in outs[i])
    other.close()


@pytest.mark.parametrize("new,bits", [(1, 4), (20, 4), (20, 8)])
def test_attend_gives_up_in_time(ctx, new, bits):
    """A wait limit of one poll: whatever the launch makes of it, it ends, says so or is right, and the next call is as ever."""
    rng = np.random.default_rng(13)
    lens = [20000, 40]
    held, table = filled(rng, 2, 128, bits, 64, lens)
    fill(ctx, rng, held, table, lens)
    q = torch.randn((2 * new, 8 * 128), device="cuda").half()
    batch = rb.KvBatch(ints([0, new, 2 * new]), ints(lens), ints(table.tolist()))
    want = ctx.attend(q, held, batch).clone()
    limit = ctx.set_wait_limit(1)
    got = ctx.attend(q, held, batch)
    status = ctx.last_status()
    ctx.set_wait_limit(limit)
    assert status == rb.ROSAQ_ERR_TIMEOUT or (status == rb.ROSAQ_OK and same(got, want))
    assert same(ctx.attend(q, held, batch), want) and ctx.last_status() == rb.ROSAQ_OK


def test_calls_of_two_graphs_share_a_context(ctx):
    """A prompt's graph and a decoding step's, captured apart, replayed in turn with calls in between: one context's workspaces, outgrown ones among them."""
    rng = np.random.default_rng(14)
    own = rb.Context(0)
    lens = [5000, 9000]
    held, table = filled(rng, 4, 128, 4, 64, lens)
    fill(ctx, rng, held, table, lens)
    tab, n, pre = ints(table.tolist()), ints(lens), (ints(table[1].tolist()), 8999)
    calls = [(60, rb.KvBatch(ints([0, 60, 120]), n, tab)), (1, rb.KvBatch(ints([0, 1, 2]), n, tab)),
             (30, rb.KvBatch(ints([0, 30, 60]), n, tab, prefix=pre))]
    qs = [torch.randn((2 * m, 16 * 128), device="cuda").half() for m, _ in calls]
    want = [ctx.attend(q, held, b).clone() for q, (_, b) in zip(qs, calls)]
    side, graphs, outs = torch.cuda.Stream(), [], []
    for i in (1, 0, 2):                                       # the smallest workspaces first
        q, b = qs[i], calls[i][1]
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            own.attend(q, held, b)
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            outs.append((i, own.attend(q, held, b)))
        graphs.append(g)
    for turn in range(3):
        for (i, out), g in zip(outs, graphs):
            out.zero_()
            g.replay()
            assert same(own.attend(qs[turn], held, calls[turn][1]), want[turn])
            assert same(out, want[i]), (turn, i)
    assert own.last_status() == rb.ROSAQ_OK
    own.close()


@pytest.mark.parametrize("new", [2, 40])
@pytest.mark.parametrize("scale", [-0.11, 0.0, 1e-30])
def test_attend_scales(ctx, new, scale):
    """Scales below zero, at it and next to it, on both kernels."""
    rng = np.random.default_rng(15)
    lens = [33000]
    held, table = filled(rng, 2, 64, 8, 64, lens)
    fill(ctx, rng, held, table, lens)
    q = torch.randn((new, 4 * 64), device="cuda").half()
    batch = rb.KvBatch(ints([0, new]), ints(lens), ints(table.tolist()))
    out = ctx.attend(q, held, batch, scale=scale)
    want, bound = expect(held, table, lens, [new], q, scale)
    inside(out, want, bound)


def test_many_rows_that_are_no_numbers(ctx):
    """As above, where a row shares its tile with others; and pairs behind the last token."""
    rng = np.random.default_rng(16)
    lens, new = [8200, 90], [70, 70]
    held, table = filled(rng, 4, 128, 4, 64, lens)
    fill(ctx, rng, held, table, lens)
    raw = held.pages.view(held.pages.shape[0], 4, 4, -1)
    for i, n in enumerate(lens):
        block = raw[table[i, n // 64], :, n % 64 // 16]
        pairs = block[:, 2048:].clone().view(torch.int16).view(4, 2, 16, 2)
        pairs[:, :, n % 16:] = ints([0x7c00, 0x7e00]).to(torch.int16)
        block[:, 2048:] = pairs.view(4, 64).view(torch.uint8).view(4, 128)
    q = torch.from_numpy(rng.standard_normal((140, 4 * 128)).astype(np.float16)).cuda()
    batch = rb.KvBatch(ints([0, 70, 140]), ints(lens), ints(table.tolist()))
    clean = ctx.attend(q, held, batch)
    want, bound = expect(held, table, lens, new, q, 128 ** -0.5)
    inside(clean, want, bound)
    q[1, 5], q[69, 128], q[139, 300] = float("nan"), float("inf"), float("-inf")
    got = ctx.attend(q, held, batch).view(140, 4, 128)
    bad = torch.zeros((140, 4), dtype=torch.bool, device="cuda")
    bad[1, 0] = bad[69, 1] = bad[139, 2] = True
    assert torch.equal(torch.isnan(got).any(-1), bad) and torch.equal(torch.isnan(got).all(-1), bad)
    inside(got[~bad], want.view(140, 4, 128)[~bad], bound.view(140, 4, 128)[~bad])


@pytest.mark.parametrize("new", [1, 40])
def test_attend_to_pages_of_zeros(ctx, new):
    """Tokens of a sequence that nothing was ever written for, in pages of zeros: values of zero that all rows see alike."""
    held = rb.KvCache(torch.zeros((40, rb.kv_page_bytes(2, 128, 4, 1024)), dtype=torch.uint8, device="cuda"), 2, 128, bits=4, page_tokens=1024)
    tab = ints([list(range(40))])
    k = torch.randn((20, 256), device="cuda").half()
    ctx.kv_write(held, rb.KvBatch(ints([0, 20]), ints([20]), tab), k, k)
    q = torch.randn((new, 8 * 128), device="cuda").half()
    out = ctx.attend(q, held, rb.KvBatch(ints([0, new]), ints([4000]), tab))
    want, bound = expect(held, np.arange(40)[None], [4000], [new], q, 128 ** -0.5)
    inside(out, want, bound)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("bits", [4, 8])
def test_attend_values_of_all_sizes(ctx, bits, new):
    """Values of thousands beside values of nothing, whose scale is 2^-24 and whose weights count all the same."""
    rng = np.random.default_rng(17)
    lens = [33000]
    held, table = filled(rng, 2, 128, bits, 64, lens)
    size = torch.tensor(rng.choice([0.0, 1e-6, 1.0, 3000.0], lens[0]), device="cuda", dtype=torch.float32)[:, None]
    k, v = (torch.randn((lens[0], 256), device="cuda") for _ in range(2))
    batch = rb.KvBatch(ints([0, lens[0]]), ints(lens), ints(table.tolist()))
    ctx.kv_write(held, batch, k.half(), (size * v).half())
    q = torch.randn((new, 8 * 128), device="cuda").half()
    for n in (lens[0], 40):
        out = ctx.attend(q, held, rb.KvBatch(ints([0, new]), ints([n]), ints(table.tolist())))
        want, bound = expect(held, table, [n], [new], q, 128 ** -0.5)
        inside(out, want, bound)
    assert ctx.last_status() == rb.ROSAQ_OK
