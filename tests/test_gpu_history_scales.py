"""Appending to a block whose scale is not the append's own: any positive number, as a cache has that was filled elsewhere
(the largest value over 448 is the usual choice there).  A row is its bytes times its block's scale before and after: the new
scale is a power of two at or above the old one, the older rows are rounded to it from what they stand for.  Bytes and
scales have to be equal to the oracle's, value for value."""
import numpy as np
import pytest
import torch

from oracle import history_operators as ho
from paper_2603_02561_b200 import solar

pytestmark = pytest.mark.gpu
BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def f64(x):
    return x.double().cpu().numpy() if x.dtype is not E4 else x.float().double().cpu().numpy()


def held(scale, B, H, N, d, seed=0):
    """A cache with arbitrary bytes and this scale in every block (a number, or one per user)."""
    g = torch.Generator().manual_seed(seed)
    c = solar.history_cache(B, H, N, d)
    for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x.copy_((torch.randn(x.shape, generator=g) * 60).clamp(-448, 448).to(E4))
        s.copy_(torch.as_tensor(scale, dtype=F32).reshape(-1, 1, 1).expand(s.shape))
    return c


SCALES = [3.0, 1.5, 1.0000001, 123.4 / 448, 0.1, 2.0 ** -110, 3.0 * 2.0 ** -101, 2.0 ** -149, 1.75 * 2.0 ** 119, 1.5 * 2.0 ** 123]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("size", [1.0, 100.0, 4000.0, 1e-20, 0.0])
def test_older_rows_keep_what_they_stand_for(dt, d, size):
    B, H, N, T = len(SCALES), 2, 128, 5
    c = held(SCALES, B, H, N, d)
    g = torch.Generator().manual_seed(3)
    k, v = ((torch.randn(B, T, H, d, generator=g) * size).to(dt).cuda() for _ in range(2))
    want = [f64(x) for x in c]
    start = [30, 61, 1, 63, 30, 30, 62, 30, 30, 30]
    ho.append(want[0], want[2], f64(k), start)
    ho.append(want[1], want[3], f64(v), start)
    solar.history_cache_append(k, v, c, torch.tensor(start, dtype=torch.int32, device="cuda"))
    for got, w in zip(c, want):
        assert np.array_equal(f64(got), w)


def test_the_rows_of_a_block_with_scale_three():
    """Rows of 30 (10 times 3); a new one of 96, then one of 4000."""
    c = solar.history_cache(1, 1, 64, 32)
    for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x.copy_(torch.full(x.shape, 10.0).to(E4))
        s.fill_(3.0)
    one = torch.ones(1, 1, 1, 32, device="cuda")
    solar.history_cache_append(96 * one, 96 * one, c, torch.full((1,), 2, dtype=torch.int32, device="cuda"))
    rows = f64(c.k)[0, 0, :, 0] * f64(c.k_scale)[0, 0, 0]
    assert float(c.k_scale) == 4.0 and list(rows[:3]) == [30.0, 30.0, 96.0]
    solar.history_cache_append(4000 * one, 4000 * one, c, torch.full((1,), 3, dtype=torch.int32, device="cuda"))
    rows = f64(c.v)[0, 0, :, 0] * f64(c.v_scale)[0, 0, 0]
    assert float(c.v_scale) == 16.0 and list(rows[:4]) == [30.0, 30.0, 96.0, 4096.0]      # 250 units of 16: 256 is nearer than 240


def test_a_call_without_new_rows_writes_nothing():
    c = held(3.0, 2, 1, 64, 64)
    want = [x.clone() for x in c]
    rows = torch.ones(2, 4, 1, 64, device="cuda")
    t = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    solar.history_cache_append(rows, rows, c, t(10, 63), counts=t(0, -3))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(c, want))


def test_an_unwritten_scale_of_zero_is_replaced():
    """A block that the caller says holds rows, its scale still zero: the rows stand for zeros, the new ones for themselves."""
    c = solar.history_cache(1, 1, 64, 32)
    for x in (c.k, c.v):
        x.copy_(torch.full(x.shape, 7.0).to(E4))
    rows = torch.full((1, 2, 1, 32), 1e-29, device="cuda")
    solar.history_cache_append(rows, rows, c, torch.full((1,), 5, dtype=torch.int32, device="cuda"))
    assert float(c.k_scale) == 2.0 ** -100 and (f64(c.k)[0, 0, :5] == 0).all() and (f64(c.k)[0, 0, 5:7] == 13.0).all()     # 12.68 units
