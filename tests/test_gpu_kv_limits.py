"""The quantized cache and its attention where they could go wrong unnoticed: lost parts, errors by norm, queries of very different sizes, waits that run out."""
import numpy as np
import pytest
import torch

from paper_2506_13472_b200 import binding as rb
from tests import kv_reference as ref, test_gpu_kv_attention as gpu
from tests.test_gpu_kv_attention import expect, fill, filled, inside, ints, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = rb.Context(0)
    yield c
    c.close()


def starts(new):
    return ints([0] + np.cumsum(new).tolist())


@pytest.mark.parametrize("new", [1, 40])
def test_long_wait_limits(ctx, new):
    """A limit that nothing reaches, and that 64 bits do not hold 32 times."""
    rng = np.random.default_rng(24)
    lens = [8200]
    held, table = filled(rng, 4, 128, 4, 64, lens)
    fill(ctx, rng, held, table, lens)
    q = torch.randn((new, 16 * 128), device="cuda").half()
    batch = rb.KvBatch(starts([new]), ints(lens), ints(table.tolist()))
    want = ctx.attend(q, held, batch).clone()
    limit = ctx.set_wait_limit(2 ** 60)
    got = ctx.attend(q, held, batch)
    status = ctx.last_status()
    ctx.set_wait_limit(limit)
    assert status == rb.ROSAQ_OK and same(got, want)


@pytest.mark.parametrize("new", [1, 48])                                    # the second one: many rows
def test_columns_of_a_wider_table(ctx, new):
    """The pages of a sequence are those of the table, not what its rows go on with in memory: lengths past them are cut and reported."""
    rng = np.random.default_rng(25)
    lens = [2048, 1024, 2048]
    held, table = filled(rng, 4, 128, 4, 1024, [4096] * 3)
    fill(ctx, rng, held, table, [4096] * 3)
    q = torch.randn((3 * new, 16 * 128), device="cuda").half()
    wide = ints(table.tolist())
    assert wide.shape[1] == 4
    want = ctx.attend(q, held, rb.KvBatch(starts([new] * 3), ints(lens), wide[:, :2].contiguous())).clone()
    assert same(ctx.attend(q, held, rb.KvBatch(starts([new] * 3), ints(lens), wide[:, :2])), want) and ctx.last_status() == rb.ROSAQ_OK
    want = ctx.attend(q, held, rb.KvBatch(starts([new] * 3), ints([2048] * 3), wide[:, :2])).clone()
    kept = held.pages.clone()
    long = rb.KvBatch(starts([new] * 3), ints([2048, 2049, 2048]), wide[:, :2])
    got = ctx.attend(q, held, long)
    assert ctx.last_status() == rb.ROSAQ_ERR_INVALID_ARG
    for i in (0, 2):
        assert same(got[i * new:i * new + new], want[i * new:i * new + new])
    x = torch.randn((3 * new, 4 * 128), device="cuda").half()
    ctx.kv_write(held, long, x, x)
    assert ctx.last_status() == rb.ROSAQ_ERR_INVALID_ARG and torch.equal(held.pages[table[1]], kept[table[1]])
    ctx.kv_read(held, long, 3 * new)
    assert ctx.last_status() == rb.ROSAQ_ERR_INVALID_ARG


def test_short_page_lists_of_a_prefix_refused(ctx):
    """A list of fewer pages than the prefix has tokens for is refused before anything is launched; one of exactly as many is not."""
    rng = np.random.default_rng(26)
    held, table = filled(rng, 2, 64, 4, 16, [100, 40])
    fill(ctx, rng, held, table, [100, 40])
    q = torch.randn((1, 2 * 64), device="cuda").half()
    call = lambda pages, n: ctx.attend(q, held, rb.KvBatch(ints([0, 1]), ints([40]), ints(table[1:].tolist()), prefix=(pages, n)))  # noqa: E731
    pages = ints(table[0].tolist())
    assert pages.shape[0] == 7
    want = call(pages, 96).clone()
    assert same(call(pages[:6], 96), want) and ctx.last_status() == rb.ROSAQ_OK
    for short, n in ((pages[:6], 97), (pages[:1], 100), (pages[:0], 1)):
        with pytest.raises(AssertionError):
            call(short, n)
    assert same(call(pages.view(1, 7), 96), want)             # a row of a table is a list too, columns of several rows are none
    with pytest.raises(AssertionError):
        call(ints([table[0].tolist()] * 2)[:, :6], 96)
    call(pages[:0], 0)
    assert ctx.last_status() == rb.ROSAQ_OK


def test_reads_between_writes(ctx):
    """Writes and reads of the same tokens in turn, captured, none waiting for the host: each read returns what was written last."""
    rng = np.random.default_rng(27)
    lens, turns = [700, 90], 8
    held, table = filled(rng, 8, 128, 8, 64, lens)
    batch = rb.KvBatch(starts(lens), ints(lens), ints(table.tolist()))
    xs = [torch.randn((790, 8 * 128), device="cuda").half() for _ in range(turns)]
    want = []
    for x in xs:
        ctx.kv_write(held, batch, x, -x)
        torch.cuda.synchronize()
        want.append([t.clone() for t in ctx.kv_read(held, batch, 790)])
        torch.cuda.synchronize()
    outs = [[torch.empty_like(x) for _ in range(2)] for x in xs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x, (k, v) in zip(xs, outs):
            ctx.kv_read(held, batch, 790, k=k, v=v)
            ctx.kv_write(held, batch, x, -x)
            ctx.kv_read(held, batch, 790, k=k, v=v)
    for _ in range(20):
        graph.replay()
    torch.cuda.synchronize()
    for (k, v), (kw, vw) in zip(outs, want):
        assert same(k, kw) and same(v, vw)
    assert ctx.last_status() == rb.ROSAQ_OK


@pytest.mark.parametrize("new,prefix", [(1, 0), (1, 2000), (40, 0)])     # the last one: many rows
@pytest.mark.parametrize("bits,sign", [(4, 1.0), (4, -1.0), (8, 1.0)])
def test_infinite_queries_over_keys_of_one_sign(ctx, new, prefix, bits, sign):
    """Every score of such a row is minus infinity: NaN, and not the zeros of a row that sees nothing."""
    rng = np.random.default_rng(21)
    lens = [prefix or 16, 8200, 90]
    held, table = filled(rng, 4, 128, bits, 64, lens)
    k, v = (torch.randn((sum(lens), 512), device="cuda") for _ in range(2))
    k = 10 + k.clamp(-4, 4)
    k[:, 5::128] = 30.0                                       # the greatest of every head, whose codes are the greatest too
    ctx.kv_write(held, rb.KvBatch(starts(lens), ints(lens), ints(table.tolist())), k.half(), v.half())
    q = torch.randn((2 * new, 4 * 4 * 128), device="cuda").half()
    batch = rb.KvBatch(starts([new, new]), ints(lens[1:]), ints(table[1:].tolist()), prefix=(ints(table[0].tolist()), prefix) if prefix else None)
    clean = ctx.attend(q, held, batch, scale=sign * 0.1)
    q[new - 1, 5], q[2 * new - 1, 7 * 128 + 5] = -sign * float("inf"), -sign * float("inf")
    got = ctx.attend(q, held, batch, scale=sign * 0.1).view(2 * new, 16, 128)
    bad = torch.zeros((2 * new, 16), dtype=torch.bool, device="cuda")
    bad[new - 1, 0] = bad[2 * new - 1, 7] = True
    assert torch.isnan(got[bad]).all() and not torch.isnan(got[~bad]).any()
    assert same(got[~bad], clean.view(2 * new, 16, 128)[~bad])


@pytest.mark.parametrize("quiet,loud,key", [(2.0 ** -11, 60000.0, 60000.0), (2.0 ** -7, 30000.0, 4000.0), (0.1, 100.0, 300.0), (2.0 ** -20, 1.0, 60000.0)])
@pytest.mark.parametrize("bits,prefix", [(4, 0), (8, 0), (4, 900)])
def test_queries_of_very_different_sizes(ctx, bits, prefix, quiet, loud, key):
    """A row's result does not depend on how large the rows beside it are."""
    rng = np.random.default_rng(22)
    lens = [prefix or 16, 600, 31, 300]
    held, table = filled(rng, 2, 128, bits, 64, lens)
    k, v = (torch.randn((sum(lens), 256), device="cuda") for _ in range(2))
    ctx.kv_write(held, rb.KvBatch(starts(lens), ints(lens), ints(table.tolist())), (key * k / 4.5).half(), v.half())
    q = torch.randn((3, 8, 128), device="cuda").clamp(-4, 4) / 4
    size = torch.full((3, 8, 1), quiet, device="cuda")
    size[0, 1] = size[0, 6] = size[2, 4] = loud
    size[1, 3] = 0.0
    q = (q * size).half().view(3, -1)
    pre = (ints(table[0].tolist()), prefix) if prefix else None
    out = ctx.attend(q, held, rb.KvBatch(starts([1, 1, 1]), ints(lens[1:]), ints(table[1:].tolist()), prefix=pre))
    few = (size < loud).view(3, 8)
    args = (held.pages, 2, 128, bits, 64)
    for i in range(3):
        kv = ref.values(*args, ints(table[i + 1].tolist()), lens[i + 1])
        if pre:
            kv = [[torch.cat([a, b]) for a, b in zip(x, y)] for x, y in zip(ref.values(*args, *pre), kv)]
        seen = torch.ones((1, kv[0][0].shape[0]), dtype=torch.bool, device="cuda")
        want, bound = ref.attention_norm(q[i:i + 1].double().view(1, 8, 128), kv, seen, 128 ** -0.5)
        off = (out[i:i + 1].double().view(1, 8, 128) - want).norm(dim=-1)
        assert bool((off <= bound)[0, few[i]].all()), (off / bound)[0, few[i]].max()


@pytest.mark.parametrize("new,prefix", [(1, 0), (1, 500), (40, 0)])
@pytest.mark.parametrize("bits", [4, 8])
def test_results_at_the_end_of_fp16(ctx, bits, new, prefix):
    """Heads from -65504 to 65504: what a code stands for may lie past 65504, a result does not."""
    rng = np.random.default_rng(23)
    lens = [prefix or 16, 8200]
    held, table = filled(rng, 4, 128, bits, 64, lens)
    k, v = (torch.randn((sum(lens), 512), device="cuda").half() for _ in range(2))
    v[:, 3::128], v[:, 4::128] = 65504.0, -65504.0
    ctx.kv_write(held, rb.KvBatch(starts(lens), ints(lens), ints(table.tolist())), k, v)
    q = torch.randn((new, 16 * 128), device="cuda").half()
    pre = (ints(table[0].tolist()), prefix) if prefix else None
    out = ctx.attend(q, held, rb.KvBatch(starts([new]), ints(lens[1:]), ints(table[1:].tolist()), prefix=pre))
    want, bound = expect(held, table[1:], lens[1:], [new], q, 128 ** -0.5, pre)
    assert bool((want > 65520).any())
    inside(out, want.clamp(max=65504), bound)
    assert torch.all(out.view(new, 16, 128)[..., 3] == 65504)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("scale", [2.0 ** 58, 1e12])
def test_scores_far_below_zero(ctx, new, scale):
    """The greatest scale over the greatest queries and keys, every score negative: the token of the least of them has the whole weight."""
    rng = np.random.default_rng(28)
    lens = [8200]
    held, table = filled(rng, 4, 128, 4, 64, lens)
    k = torch.full((8200, 512), -65504.0, device="cuda").half()
    k[7] = -60000.0
    v = torch.randn((8200, 512), device="cuda").half()
    batch = rb.KvBatch(starts(lens), ints(lens), ints(table.tolist()))
    ctx.kv_write(held, batch, k, v)
    v = ctx.kv_read(held, batch, 8200)[1]
    q = torch.full((new, 16 * 128), 65504.0, device="cuda").half()
    out = ctx.attend(q, held, rb.KvBatch(starts([new]), ints(lens), ints(table.tolist())), scale=scale)
    want = v[7].double().view(4, 1, 128).expand(4, 4, 128).reshape(1, -1).expand(new, -1)
    # (a read is rounded to fp16 too: half a step each, and what a scale's logarithm and reciprocal are off by)
    inside(out, want, 2 * 2.0 ** -11 * want.abs() + 2.0 ** -19 * 16)


def test_a_step_of_no_sequences(ctx):
    held, _ = filled(np.random.default_rng(29), 2, 64, 4, 16, [5])
    kept = held.pages.clone()
    empty = torch.empty((0, 2 * 64), dtype=torch.float16, device="cuda")
    batch = rb.KvBatch(ints([0]), ints([]), torch.empty((0, 4), dtype=torch.int32, device="cuda"))
    ctx.kv_write(held, batch, empty, empty)
    assert ctx.kv_read(held, batch, 0)[1].shape == (0, 128) and ctx.attend(empty, held, batch).shape == (0, 128)
    assert ctx.rope(empty, ints([]), ctx.rope_create(64)).shape == (0, 128)
    assert ctx.last_status() == rb.ROSAQ_OK and torch.equal(held.pages, kept)


def updates(heads, group, lens, new, prefix=0):
    """Additions to one accumulator, at most: one per sixteen tokens of a CTA's share, which is an equal one or 16 chunks of 64 tokens."""
    return 128 + sum((n + prefix) // 16 * -(-m * group // 8) for n, m in zip(lens, new)) * heads // 148


@pytest.mark.parametrize("heads,group,hd,bits,page,lens,new,prefix,room", [(*c, 0, False) for c in gpu.CASES] + [(*c, 0, True) for c in gpu.MANY] + [
    (8, 4, 128, 4, 64, [i % 40 + 1 for i in range(64)], [1] * 64, 2500, False),
    (2, 8, 64, 8, 16, [30, 9, 400], [3, 9, 20], 333, False),
    (1, 3, 128, 8, 32, [40], [40], 40000, False),
    (2, 8, 64, 4, 16, [3, 1, 0, 70, 9], [3, 1, 0, 30, 9], 9001, False),
    (2, 2, 64, 8, 64, [33000], [2], 0, False),
    (2, 2, 64, 8, 64, [33000], [40], 0, False),
])
def test_errors_by_norm(ctx, heads, group, hd, bits, page, lens, new, prefix, room):
    """Every row and head of long contexts, whose results are small beside the values that they are made of."""
    rng = np.random.default_rng(30)
    all_lens = [prefix] + lens
    held, table = filled(rng, heads, hd, bits, page, all_lens)
    fill(ctx, rng, held, table, all_lens, loud=3.0)
    pre, table = ints(table[0].tolist()), table[1:]
    if room:
        width = -(-(1 << 22) // (-(-sum(new) // len(lens)) * group * len(lens) * heads * page))
        table = np.pad(table, ((0, 0), (0, max(0, width - table.shape[1]))), constant_values=-5)
    q = torch.from_numpy(rng.standard_normal((sum(new), heads * group * hd)).astype(np.float16)).cuda()
    out = ctx.attend(q, held, rb.KvBatch(starts(new), ints(lens), ints(table.tolist()), prefix=(pre, prefix) if prefix else None))
    assert ctx.last_status() == rb.ROSAQ_OK
    args, at = (held.pages, heads, hd, bits, page), 0
    shared = ref.values(*args, pre, prefix) if prefix else None
    for i, (n, m) in enumerate(zip(lens, new)):
        if m == 0:
            continue
        kv = ref.values(*args, ints(table[i].tolist()), n)
        if shared:
            kv = [[torch.cat([a, b]) for a, b in zip(x, y)] for x, y in zip(shared, kv)]
        seen = torch.arange(prefix + n, device="cuda")[None, :] < prefix + n - m + 1 + torch.arange(m, device="cuda")[:, None]
        want, bound = ref.attention_norm(q[at:at + m].double().view(m, -1, hd), kv, seen, hd ** -0.5, updates(heads, group, lens, new, prefix))
        off = (out[at:at + m].double().view(m, -1, hd) - want).norm(dim=-1)
        assert bool((off <= bound).all()), (i, float((off / bound).max()))
        at += m


@pytest.mark.parametrize("heads,group,hd,bits,page,lens,new,prefix,many", [
    (1, 4, 128, 4, 1024, [70000], [1], 0, 0),                               # one tile over all CTAs
    (2, 1, 128, 8, 64, [9000, 5000, 20000], [1, 1, 1], 0, 0),
    (8, 1, 64, 4, 64, [6000] * 5, [2] * 5, 0, 0),
    (1, 2, 128, 4, 1024, [70000], [100], 0, 1),
    (4, 4, 128, 8, 64, [9000, 20000], [30, 50], 0, 1),
    (2, 2, 64, 4, 64, [40000], [300], 0, 1),
    (2, 4, 128, 4, 64, [4500] * 30, [3] * 30, 16001, 2),
    (2, 4, 128, 8, 64, [5000, 4200], [1, 1], 9001, 0),
])
def test_no_part_is_lost(ctx, heads, group, hd, bits, page, lens, new, prefix, many):
    """Every 32 tokens have a value of 3 in one channel and nothing elsewhere, about alike in weight: a part that is missing or counts twice is a seventeenth
    or more of that channel's result, where roundings are a 300th."""
    rng = np.random.default_rng(31)
    all_lens = [prefix or 16] + lens
    held, table = filled(rng, heads, hd, bits, page, all_lens)
    assert rb.attend_forms(len(lens), sum(new), heads * group, heads, hd, table.shape[1], page, bits, prefix) == many
    k = torch.randn((sum(all_lens), heads * hd), device="cuda").half()
    at = torch.cat([torch.arange(n, device="cuda") for n in all_lens]) // 32 % hd
    v = 3.0 * (at[:, None, None] == torch.arange(hd, device="cuda")).half().expand(-1, heads, -1).reshape(-1, heads * hd)
    ctx.kv_write(held, rb.KvBatch(starts(all_lens), ints(all_lens), ints(table.tolist())), k, v)
    q = (0.3 * torch.randn((sum(new), heads * group * hd), device="cuda")).half()
    pre = (ints(table[0].tolist()), prefix) if prefix else None
    out = ctx.attend(q, held, rb.KvBatch(starts(new), ints(lens), ints(table[1:].tolist()), prefix=pre))
    assert ctx.last_status() == rb.ROSAQ_OK
    want, _ = expect(held, table[1:], lens, new, q, hd ** -0.5, pre)
    # All terms of a channel have one sign: the weights' 11 bits in product and sum, the result's rounding, and, of codes about their middle, what accumulators that hold up to the
    # middle times a scale cut off
    middle = 3.0 / ref.QMAX[bits] * (10 if bits == 4 else 128)
    inside(out, want, 3 * 2.0 ** -11 * want + updates(heads, group, lens, new, prefix) * 2.0 ** -23 * middle + 2.0 ** -20)


@pytest.mark.parametrize("new,bits", [(1, 4), (1, 8), (16, 4), (16, 8)])
def test_waits_that_run_out(ctx, new, bits):
    """One poll per wait, and more chunks than any warp has slots for: the launch ends and says so, and the next call is as ever."""
    rng = np.random.default_rng(32)
    lens = [70000]
    held, table = filled(rng, 8, 128, bits, 64, lens)
    fill(ctx, rng, held, table, lens)
    assert rb.attend_forms(1, new, 32, 8, 128, table.shape[1]) == (1 if new > 1 else 0)
    q = torch.randn((new, 32 * 128), device="cuda").half()
    batch = rb.KvBatch(starts([new]), ints(lens), ints(table.tolist()))
    want = ctx.attend(q, held, batch).clone()
    limit = ctx.set_wait_limit(1)
    status = []
    for _ in range(5):
        ctx.attend(q, held, batch)
        status.append(ctx.last_status())
    ctx.set_wait_limit(limit)
    assert rb.ROSAQ_ERR_TIMEOUT in status and set(status) <= {rb.ROSAQ_OK, rb.ROSAQ_ERR_TIMEOUT}
    for _ in range(2):
        assert same(ctx.attend(q, held, batch), want) and ctx.last_status() == rb.ROSAQ_OK


@pytest.mark.parametrize("lens,new,prefix,many", [([3], [20], 0, 0), ([3], [20], 40, 0), ([10, 600, 0], [700, 640, 5], 0, 1), ([0, 300], [600, 400], 4100, 3)])
def test_more_rows_than_tokens(ctx, lens, new, prefix, many):
    """The first rows of such a sequence see nothing but the prefix, whole tiles of them too: zeros, or the prefix alone."""
    rng = np.random.default_rng(33)
    held, table = filled(rng, 2, 128, 4, 64, [max(prefix, 16)] + lens)
    fill(ctx, rng, held, table, [max(prefix, 16)] + lens)
    pre, table = (ints(table[0].tolist()), prefix) if prefix else None, np.pad(table[1:], ((0, 0), (0, 60 if many else 0)), constant_values=-5)
    assert rb.attend_forms(len(lens), sum(new), 4, 2, 128, table.shape[1], 64, 4, prefix) == many
    q = torch.randn((sum(new), 4 * 128), device="cuda").half()
    out = torch.full_like(q, 7.0)
    ctx.attend(q, held, rb.KvBatch(starts(new), ints(lens), ints(table.tolist()), prefix=pre), out=out)
    assert ctx.last_status() == rb.ROSAQ_OK
    args, at = (held.pages, 2, 128, 4, 64), 0
    for i, (n, m) in enumerate(zip(lens, new)):
        kv = [[x[:n] for x in y] for y in ref.values(*args, ints(table[i].tolist()), max(n, 1))]
        if pre:
            kv = [[torch.cat([a, b]) for a, b in zip(x, y)] for x, y in zip(ref.values(*args, *pre), kv)]
        # (the prefix is seen by all: a sequence that is too short takes nothing away from it)
        t = torch.arange(prefix + n, device="cuda")[None, :]
        seen = (t < prefix) | (t - prefix < n - m + 1 + torch.arange(m, device="cuda")[:, None])
        want, bound = ref.attention(q[at:at + m].double().view(m, 4, 128), kv, seen, 128 ** -0.5)
        if prefix + n:                                        # (of nothing: zeros, seen to below)
            inside(out[at:at + m].view(m, 4, 128), want, bound, i)
        at += m
    if not prefix:
        blind = torch.cat([torch.arange(m) < m - n for n, m in zip(lens, new)]).cuda()
        assert blind.any() and torch.all(out[blind] == 0)


def test_caches_past_four_gigabytes(ctx):
    """Pages whose bytes lie past 32 bits, and a table of pages in no order over all of them: as in a small cache of the same pages."""
    rng = np.random.default_rng(34)
    heads, lens = 32, [700, 333, 64]
    size = rb.kv_page_bytes(heads, 128, 8, 64)
    n_pages = (9 << 30) // size
    small = rb.KvCache(torch.zeros((22, size), dtype=torch.uint8, device="cuda"), heads, 128, 8, 64)
    big = rb.KvCache(torch.empty((n_pages, size), dtype=torch.uint8, device="cuda"), heads, 128, 8, 64)
    places = rng.choice(n_pages, 22, replace=False)
    places[:3] = n_pages - 1, (1 << 32) // size, (1 << 33) // size
    table = np.full((3, 11), -5)
    at = 0
    for i, n in enumerate(lens):
        need = -(-n // 64)
        table[i, :need], at = np.arange(at, at + need), at + need
    pre = np.arange(at, at + 3)
    far = np.where(table < 0, -5, places[table])
    big.pages[torch.tensor(places, device="cuda")] = small.pages
    k, v = (torch.randn((sum(lens) + 150, heads * 128), device="cuda").half() for _ in range(2))
    q = torch.randn((sum(lens), heads * 128), device="cuda").half()
    outs = []
    for held, t, p in ((small, table, pre), (big, far, places[pre])):
        p = ints(p.tolist())
        ctx.kv_write(held, rb.KvBatch(ints([0, 150]), ints([150]), p[None]), k[:150], v[:150])
        tab = ints(t.tolist())
        batch = rb.KvBatch(starts(lens), ints(lens), tab)
        ctx.kv_write(held, batch, k[150:], v[150:])
        got = list(ctx.kv_read(held, batch, sum(lens)))
        for rows in (1, 64):                                  # decoding and many rows, behind a prefix
            got.append(ctx.attend(q[:3 * rows], held, rb.KvBatch(starts([rows] * 3), ints(lens), tab, prefix=(p, 150))))
        outs.append(got)
        assert ctx.last_status() == rb.ROSAQ_OK
    assert torch.equal(big.pages[torch.tensor(places, device="cuda")], small.pages)
    for a, b in zip(*outs):
        assert same(a, b)
    assert float(outs[0][2].abs().max()) > 0.1
