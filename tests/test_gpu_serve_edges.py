"""GPU tests of the 8-bit serving operators at the edges of what their calls
accept: bounds that are loose, tables that start late or end early, buffers
that are replaced, operands at the ends of their types."""
import numpy as np
import pytest

from tests.test_gpu_serve import Pages, attend, dev, gen, i32, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bt", [16, 128])
@pytest.mark.parametrize("first", [1, 63, 64, 1000])
def test_read_into_rows_that_start_late(bt, first):
    """kv_start need not begin at 0: the rows before it are left alone, the others are those of a
    read that begins at 0."""
    import torch
    say("read late", bt, first)
    lens = [70, 0, 5, 200]
    pg = Pages(gen(31), lens, bt, 2, 64)
    start = np.concatenate([[0], np.cumsum(lens)])
    total = int(start[-1])
    want = [torch.empty((total, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pg.cache.read(dev(pg.table), i32(start), *want)
    got = [torch.full((first + total + 3, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pg.cache.read(dev(pg.table), i32(start + first), *got)
    for x, y in zip(got, want):
        assert torch.equal(x[first:first + total], y)
        assert (x[:first] == 9).all() and (x[first + total:] == 9).all()


@pytest.mark.parametrize("max_q", [2 ** 29, 2 ** 29 + 1, 2 ** 31 - 1])
def test_a_loose_max_q(max_q):
    """max_q only bounds a request's new tokens: times the heads of a group it may pass 32 bits."""
    say("loose max_q", max_q)
    pg = Pages(gen(32), [5000, 9, 2600], 64, 1, 128)
    attend(pg, [1, 1, 0], [5000, 9, 2600], 8, max_q=max_q)
    attend(pg, [1, 2, 4], [5000, 9, 2600], 8, max_q=max_q)
    attend(pg, [40, 2, 3], [5000, 9, 2600], 8, max_q=max_q)
