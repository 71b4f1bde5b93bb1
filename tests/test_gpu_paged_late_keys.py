"""Attention over an 8-bit paged cache where a late key scores far above all before it.

Each lane of a row's pair holds half of a block's keys, four and four in turn.  A key whose score lies 15 (base 2) and more above the row's reference raises it
for both lanes, wherever in a group of eight it lies."""
import pytest
import torch

import paper_2507_11978_amd as nt
from test_gpu_paged import Batch, normal

pytestmark = pytest.mark.gpu


def raise_keys(b, size, dt, positions, heads=1):
    """Queries share a large first element; the keys at `positions` of sequence 0 score 25.6 and a little less, the others a few units."""
    b.q[..., 0] = 8.0
    for i, at in enumerate(positions):
        k = normal((1, heads, size), dt, 70 + i)
        k[..., 0] = (3.2 - 0.05 * i) * size ** 0.5
        slot = torch.tensor([int(b.table[0, at // b.page]) * b.page + at % b.page]).cuda()
        nt.cache_write(k.cuda(), normal((1, heads, size), dt, 80 + i).cuda(), slot, *b.c)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("kind", ["same", "e4m3", "i8"])
@pytest.mark.parametrize("size", [64, 128, 256])
def test_a_late_key_above_all_others(dt, kind, size):
    for seqs, at, shared in (([(60, 300)], 200, False), ([(40, 2000)], 1500, True)):
        for j in range(8):
            b = Batch(seqs, 1, 1, size, 16, dt, kind, seed=j)
            raise_keys(b, size, dt, (at + j, at + j + 72))           # (both in the same half of their groups)
            got = b.run()
            torch.cuda.synchronize()
            p = nt.last_paged_plan()
            assert p.rows == 128 and (p.shares > 1) == shared
            b.check(got, f"{seqs} key {at + j}")
