"""Lengths far beyond what the page table has room for: tokens that see such a position get NaN, soon, and nothing else changes."""
import pytest
import torch

import paper_2507_11978_amd as nt
from test_gpu_paged import KINDS, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt,kind", KINDS)
@pytest.mark.parametrize("seqs,hints", [([(1, 40), (2, 33), (1, 64)], (2, 64)), ([(70, 150), (3, 40), (130, 131)], (0, 0)), ([(1, 3000), (1, 2900)], (1, 3000)), ([(40, 2000), (9, 1800)], (40, 2000))])
@pytest.mark.parametrize("window", [0, 5, 100])
def test_lengths_that_no_cache_has(dt, kind, seqs, hints, window):
    b = Batch(seqs, 4, 2, 64, 16, dt, kind)
    more = dict(window=window, max_queries=hints[0], max_length=hints[1])
    want = b.run(**more).clone()
    torch.cuda.synchronize()
    shares = nt.last_paged_plan().shares
    for length in (2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 4096, 2 ** 31 - 4097, 0x7f7f7f7f, 10 ** 9):
        b.lengths[0] = length
        got = b.run(**more)
        torch.cuda.synchronize()
        assert torch.isnan(got[:b.starts[1]]).all() and torch.equal(got[b.starts[1]:], want[b.starts[1]:])
    assert shares > 1 or hints[1] < 1000 or window or (hints[0] == 1 and kind != "same")          # (375 KB of codes to a head are not shared)
    # an end just behind the table's: the tokens whose window lies before it are what they are
    reach = 16 * b.table.shape[1]
    b.lengths[0] = reach + 1
    got = b.run(**more)
    assert torch.isnan(got[b.starts[1] - 1]).all()
    assert torch.equal(got[b.starts[1]:], want[b.starts[1]:])
    assert torch.isnan(b.run(**more, causal=False)[:b.starts[1]]).all()


@pytest.mark.parametrize("window,sees", [(0, True), (2 ** 30, False), (2 ** 30 + 2 ** 19, False), (2 ** 30 + 2 ** 20, True), (2 ** 31 - 1, True), (2 ** 40, True)])
def test_windows_longer_than_two_to_the_30(window, sees):
    """A table that names one page again and again, and another at its beginning, whose keys outweigh all the rest."""
    size, page, length = 8, 4096, 2 ** 30 + 2 ** 20
    k, v = torch.zeros(2, page, 1, size, dtype=torch.int8, device="cuda"), torch.ones(2, page, 1, size, dtype=torch.int8, device="cuda")
    k[1, :, :, 0], v[1] = 100, 7
    scale = torch.ones(2, page, 1, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.zeros(1, length // page, dtype=torch.int32, device="cuda")
    table[0, 0] = 1
    q = torch.zeros(1, 1, size, dtype=torch.float16, device="cuda")
    q[..., 0] = 1.0
    out = nt.sdpa_paged(q, k, v, table, i32([0, 1]), i32([length]), torch.empty_like(q), scale, scale, scale=0.5, window=window, max_queries=1, max_length=length)
    torch.cuda.synchronize()
    assert torch.equal(out, torch.full_like(q, 7.0 if sees else 1.0)), out


def test_shares_that_do_not_fit_the_workspace():
    """64 sequences of 131072: their shares' partial results would take more than the library's 256 MB.  Tables that name one page again and again: the result is that
    over the page."""
    size, page, heads, group, count, length = 128, 16, 8, 4, 64, 131072
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(1, page, heads, size, generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(count, heads * group, size, generator=g, device="cuda").bfloat16()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lengths = [length - 16 * 1000 * (b % 5) for b in range(count)]
    out = nt.sdpa_paged(q, k, v, torch.zeros(count, length // page, dtype=torch.int32, device="cuda"), i32(list(range(count + 1))), i32(lengths), torch.empty_like(q),
                        max_queries=1, max_length=length)
    torch.cuda.synchronize()
    K, V = (t[0].double().cpu().permute(1, 0, 2).repeat_interleave(group, 0) for t in (k, v))           # [query heads, keys, size]
    p = torch.softmax((q.double().cpu()[:, :, None] * K).sum(-1) / size ** 0.5, -1)
    want, A = ((p[..., None] * x).sum(2) for x in (V, V.abs()))
    # the result's rounding; sums of 131072 fp32 numbers, and scores' (size + 8 roundings of at most 4 sqrt(size) (1 + largest score))
    tol = 2.0 ** -8 * want.abs() + A * 2.0 ** -24 * (length + 2 * (size + 8) * 4 * size ** 0.5 * 6)
    assert ((out.double().cpu() - want).abs() <= tol).all()
