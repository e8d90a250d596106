"""The gate's mean probabilities where they are exact: a row that can take 1, 2, 4,
... heads with equal logits has p of 1, 1/2, 1/4, ..., whose sums lose no digit in
FP32 (a block's rows times 1,024 stay below 2^24), so that share is the exact mean
rounded once.  A row that is lost or counted twice shows, however many there are."""
import pytest
import torch

from test_gpu_gate import DTYPES, SHAPES

pytestmark = pytest.mark.gpu

LARGE = [(140001, 7, 3), (66000, 16, 9), (4200, 1000, 5), (4100, 1024, 12), (131072, 64, 4), (65502, 16, 2), (2048, 4, 1),
         (2049, 4, 1), (513, 13, 9)]


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", SHAPES + LARGE)
def test_share_counts_every_row(rt, dtype, shape):
    rows, heads, k = shape
    gen = torch.Generator().manual_seed(rows + heads)
    most = heads.bit_length() - 1
    take = torch.where(torch.rand(rows, generator=gen) < 0.05, 0, 2 ** torch.randint(0, most + 1, (rows,), generator=gen))
    place = torch.rand(rows, heads, generator=gen).argsort(1).argsort(1)
    on = place < take[:, None]
    x = torch.where(on, 3.0 * torch.randint(-1, 2, (rows, 1), generator=gen), -torch.inf)
    got = rt.gate(x.to(DTYPES[dtype]).cuda(), k)
    some = take > 0
    n = max(1, int(some.sum()))
    p = on.double() / take.clamp_min(1)[:, None]
    share = p.sum(0) / n
    assert int(got.totals[-1]) == int(some.sum())
    assert torch.equal(got.share.cpu(), share.float())
    counts = got.counts.cpu().double()
    assert int(counts.sum()) == int(take.clamp_max(k).sum())
    loss = heads * (counts / counts.sum().clamp_min(1) * share).sum()
    # (sums of 1,024 in FP64, one rounding)
    assert abs(float(got.loss) - float(loss)) <= 1.001 * 2.0 ** -24 * float(loss)
