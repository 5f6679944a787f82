"""The quantized cache and its attention where they could go wrong unnoticed: lost parts, errors by norm, queries of very different sizes, waits that run out."""
import numpy as np
import pytest
import torch

from paper_2506_13472_b200 import binding as rb
from tests.test_gpu_kv_attention import fill, filled, ints, same

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
