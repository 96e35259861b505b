"""The balance loss where a thread adds up more than 256 rows, which takes a second turn of its outer loop.

Tolerance (u = 2^-24): a thread has at most n = rows / (slices * rows at a time) rows of a column; they are added 256 at a time, then those sums: at
most min(n, 256) + n / 256 + 1 additions in float32, and at most 44 more in the CTA, one rounding of the result, float64 above: that many u
relative to the mean itself (the weights are not negative).  Rows that are left out show from a 50 000th part of the sum on."""
import pytest
import torch

from paper_2308_14711_b200.binding import FFFLayer

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
THREADS, COLUMNS, SLICES = 512, 128, 296                   # of a CTA; columns of a tile; CTAs


def rows_of_a_thread(depth, B):
    L = 1 << depth
    cols, tiles = min(L, COLUMNS), max(1, L // COLUMNS)
    at_a_time = THREADS // (cols // 4 if cols >= 4 else cols)
    slices = min(max(1, SLICES // tiles), -(-B // (8 * at_a_time)))
    return -(-(-(-B // slices)) // at_a_time)


@pytest.mark.parametrize("masked", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("depth,B", [(0, 39_000_001), (1, 19_500_003), (5, 4_900_001), (6, 2_440_001), (13, 17_001), (14, 8_501), (15, 8_200)])
def test_more_rows_than_are_added_at_a_time(depth, B, masked):
    L = 1 << depth
    n = rows_of_a_thread(depth, B)
    assert n > 256
    g = torch.Generator("cuda").manual_seed(depth)
    mix = torch.rand(B, L, device="cuda", generator=g)
    leaf = torch.randint(0, L, (B,), device="cuda", generator=g, dtype=torch.int32)
    mask = torch.rand(B, device="cuda", generator=g) < 0.9 if masked else None
    counted = torch.ones(B, dtype=torch.bool, device="cuda") if mask is None else mask
    total = torch.zeros(L, dtype=torch.float64, device="cuda")
    for rows, keep in zip(mix.split(max(1, (1 << 24) // L)), counted.split(max(1, (1 << 24) // L))):
        total += rows.double()[keep].sum(0)
    if masked:
        mix[~mask] = float("nan")
    z = lambda *s: torch.zeros(s, device="cuda")
    layer = FFFLayer(1, 1, depth, 1, "relu", "f32", z(L - 1, 1) if depth else None, None, z(L, 1, 1), None, z(L, 1, 1), None)
    loss, counts, mean = layer.balance_loss(mix, leaf, token_mask=mask)
    kept = int(counted.sum())
    ref = total / kept
    want = torch.bincount(leaf[counted].long(), minlength=L)
    assert torch.equal(counts.long(), want)
    bound = (min(n, 256) + n // 256 + 1 + 45) * U
    assert ((mean.double() - ref).abs() <= bound * ref).all()
    loss_ref = float(L * (want.double() / kept * ref).sum())
    assert abs(float(loss) - loss_ref) <= (bound + U) * loss_ref
    layer.close()
