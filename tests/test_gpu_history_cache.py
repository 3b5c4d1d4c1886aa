"""The 8-bit history cache against its definition in double precision.

The rows in 8 bits and their scales have to be equal, value for value.  Attention: with W = sum p |v| (the same weights with
|v|), a score's error dz moves the output by at most 2 dz W.  fp32 sums of up to 128 products of exact terms: dz <=
scale sum |q k| 2^-20; bf16 storage rounds the weights to fp16 (2^-11 W) and the output to bf16 (2^-8 |o|).  fp32 storage:
q and p as 22 bits (2^-21).  Sums over up to 1200 rows in fp32: 2^-14 W at most, seen far below."""
import numpy as np
import pytest
import torch

from oracle import history_operators as ho
from paper_2603_02561_b200 import solar

pytestmark = pytest.mark.gpu
BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def f64(x):
    return x.double().cpu().numpy() if x.dtype is not E4 else x.float().double().cpu().numpy()


def filled(B, H, N, d, seed=0):
    """A cache whose bytes and scales are arbitrary (no NaN)."""
    g = torch.Generator().manual_seed(seed)
    c = solar.history_cache(B, H, N, d)
    for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x.copy_((torch.randn(x.shape, generator=g) * 60).clamp(-448, 448).to(E4))
        s.copy_(torch.exp2(torch.randint(-8, -3, s.shape, generator=g).float()))
    return c


def values(c):
    return [f64(x) for x in c]


def near(got, q, c, lengths, scale, causal, dt):
    k8, v8, ks, vs = values(c)
    want, size = ho.attention(f64(q), k8, v8, ks, vs, lengths, scale, causal)
    got = f64(got)
    assert np.isfinite(got).all()
    top = np.nanmax(np.abs(k8 * np.repeat(ks, 64, axis=2)[..., None])) * np.abs(f64(q)).sum(-1).max() * abs(scale)
    dz = 2 * top * 2.0 ** -20
    out, rest = (2.0 ** -8, 2.0 ** -10 + 2.0 ** -14) if dt is BF else (2.0 ** -24, 2.0 ** -20 + 2.0 ** -16)
    err = np.abs(got - want)
    assert np.all(err <= out * np.abs(want) + (rest + dz) * size + 1e-30), (err / (size + 1e-30)).max()
    if np.linalg.norm(want):
        assert np.linalg.norm(err) <= (2.0 ** -8 if dt is BF else 2.0 ** -16) * np.linalg.norm(want)


def queries(dt, B, M, Hq, d, seed=1):
    return torch.randn(B, M, Hq, d, generator=torch.Generator().manual_seed(seed)).to(dt).cuda()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("M,Hq,H,lengths,causal", [
    (1, 1, 1, [1, 64], False), (1, 8, 2, [1200, 0], False), (1, 4, 4, [65, 127], False), (37, 2, 1, [300, 1], False),
    (17, 3, 3, [640, 129], False), (100, 2, 1, [100, 513], True), (66, 4, 2, [7, 66], True), (5, 16, 1, [70, 4], True)])
def test_attention(dt, d, M, Hq, H, lengths, causal):
    c = filled(2, H, 1280, d)
    q = queries(dt, 2, M, Hq, d)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got = solar.history_cache_attention(q, c, n, 0.05, flags=solar.FLAG_CAUSAL if causal else 0)
    near(got, q, c, lengths, 0.05, causal, dt)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("M,Hq,H,lengths,causal", [(200, 1, 1, [1200, 0], False), (300, 2, 1, [300, 1100], True), (129, 2, 2, [129, 640], False)])
def test_attention_of_many_queries(dt, d, M, Hq, H, lengths, causal):
    c = filled(2, H, 1280, d)
    q = queries(dt, 2, M, Hq, d)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got = solar.history_cache_attention(q, c, n, 0.05, flags=solar.FLAG_CAUSAL if causal else 0)
    near(got, q, c, lengths, 0.05, causal, dt)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("strided", [False, True])
def test_append(dt, d, strided):
    B, H, N, T = 4, 3, 512, 150
    c = filled(B, H, N, d)
    g = torch.Generator().manual_seed(5)
    x = torch.randn(B, T, 2, H, d, generator=g) * torch.exp2(torch.randint(-9, 9, (B, T, 1, H, 1), generator=g).float())
    x[0, :, 0] *= 2.0 ** -30
    x = x.to(dt).cuda()
    k, v = (x[:, :, i] if strided else x[:, :, i].contiguous() for i in range(2))
    want = values(c)
    start, counts = [0, 70, 500, 63], [150, 150, 150, 2]
    ho.append(want[0], want[2], f64(k), start, counts)
    ho.append(want[1], want[3], f64(v), start, counts)
    t = [torch.tensor(y, dtype=torch.int32, device="cuda") for y in (start, counts)]
    solar.history_cache_append(k, v, c, t[0], counts=t[1])
    for got, w in zip(values(c), want):
        assert np.array_equal(got, w)


def test_append_one_by_one_moves_older_rows_to_a_larger_scale():
    B, H, N, d = 2, 2, 128, 64
    c = solar.history_cache(B, H, N, d)
    c.k.view(torch.uint8).fill_(0x7f)
    c.v.view(torch.uint8).fill_(0x7f)
    want = [np.full((B, H, N, d), np.nan), np.full((B, H, N, d), np.nan), np.zeros((B, H, 2)), np.zeros((B, H, 2))]
    g = torch.Generator().manual_seed(2)
    for t in range(80):
        k, v = ((torch.randn(B, 1, H, d, generator=g) * 2.0 ** (t % 23 - 11)).cuda() for _ in range(2))
        if t == 30:
            k[0, 0, 0, 5] = float("inf")
        start = torch.full((B,), t, dtype=torch.int32, device="cuda")
        solar.history_cache_append(k, v, c, start)
        ho.append(want[0], want[2], f64(k), [t] * B)
        ho.append(want[1], want[3], f64(v), [t] * B)
    for got, w in zip(values(c), want):
        assert np.array_equal(got, w, equal_nan=True)


def test_starts_outside_the_cache_write_nothing_and_rows_past_its_end_are_dropped():
    c = filled(4, 1, 128, 32)
    before = values(c)
    k = queries(F32, 4, 70, 1, 32)
    start = torch.tensor([-1, 128, 100, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    solar.history_cache_append(k, k, c, start, counts=torch.tensor([70, 70, 1000, 5], dtype=torch.int32, device="cuda"))
    ho.append(before[0], before[2], f64(k), [-1, 128, 100, 128], [70, 70, 70, 5])
    ho.append(before[1], before[3], f64(k), [-1, 128, 100, 128], [70, 70, 70, 5])
    for got, w in zip(values(c), before):
        assert np.array_equal(got, w)


def test_largest_and_smallest_values():
    c = solar.history_cache(1, 1, 64, 32)
    x = torch.zeros(1, 4, 1, 32, device="cuda")
    x[0, 0, 0, :4] = torch.tensor([3.4e38, -3.4e38, 1e-45, 1e38])
    want = [np.zeros((1, 1, 64, 32)), np.zeros((1, 1, 64, 32)), np.zeros((1, 1, 1)), np.zeros((1, 1, 1))]
    start = torch.zeros(1, dtype=torch.int32, device="cuda")
    for rows in (x, torch.zeros_like(x)):
        solar.history_cache_append(rows, rows, c, start)
        ho.append(want[0], want[2], f64(rows), [0])
        assert np.array_equal(f64(c.k)[:, :, :4], want[0][:, :, :4]) and np.array_equal(f64(c.k_scale), want[2])
    assert float(c.k_scale) == 2.0 ** -100


@pytest.mark.parametrize("dt,d,M", [(BF, 64, 1), (BF, 64, 200), (BF, 128, 200), (F32, 64, 1), (F32, 32, 200)])
def test_what_lies_behind_a_length_does_not_matter(dt, d, M):
    c = filled(2, 1, 256, d)
    q = queries(dt, 2, M, 2, d)
    lengths = torch.tensor([65, 128], dtype=torch.int32, device="cuda")
    want = solar.history_cache_attention(q, c, lengths, 0.1)
    for b, n in ((0, 65), (1, 128)):
        c.k.view(torch.uint8)[b, :, n:] = 0x7f
        c.v.view(torch.uint8)[b, :, n:] = 0xff
    c.k_scale[:, :, 3:] = float("nan")
    c.v_scale[:, :, 3:] = float("inf")
    assert torch.equal(solar.history_cache_attention(q, c, lengths, 0.1), want)


@pytest.mark.parametrize("dt,d", [(BF, 64), (BF, 128), (BF, 32), (F32, 64)])
@pytest.mark.parametrize("what", ["k", "v"])
def test_a_row_that_is_not_finite_reaches_only_those_that_see_it(dt, d, what):
    M = n = 200
    c = filled(1, 1, 256, d)
    q = queries(dt, 1, M, 1, d)
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    want = solar.history_cache_attention(q, c, lengths, 0.1, flags=solar.FLAG_CAUSAL)
    getattr(c, what).view(torch.uint8)[0, 0, 150, 7] = 0x7f
    got = solar.history_cache_attention(q, c, lengths, 0.1, flags=solar.FLAG_CAUSAL)
    assert torch.isnan(got[0, 150:, 0, 7]).all()
    assert torch.equal(got[0, :150], want[0, :150])


@pytest.mark.parametrize("dt,d", [(BF, 64), (BF, 128), (F32, 64)])
@pytest.mark.parametrize("M", [3, 700])
@pytest.mark.parametrize("scale", [-0.05, 0.0])
def test_scales_of_any_sign_and_groups_of_three(dt, d, M, scale):
    c = filled(2, 2, 320, d)
    q = queries(dt, 2, M, 6, d)
    lengths = torch.tensor([300, 64], dtype=torch.int32, device="cuda")
    near(solar.history_cache_attention(q, c, lengths, scale), q, c, [300, 64], scale, False, dt)


@pytest.mark.parametrize("dt,d,T", [(BF, 64, 40), (BF, 64, 400), (BF, 128, 400), (F32, 32, 40)])
def test_a_padded_batch_of_new_histories(dt, d, T):
    """Queries padded as the appended rows were, the cache behind those rows never written, one user's padding past its end."""
    B, H, Hq, N = 3, 2, 4, 512
    start, counts = [10, 120, 0], [T, min(13, T), 0]
    c = filled(B, H, N, d)
    for b in range(B):
        for x in (c.k, c.v):
            x.view(torch.uint8)[b, :, start[b]:] = 0x7f
    k, v, q = queries(dt, B, T, H, d, 3), queries(dt, B, T, H, d, 4), queries(dt, B, T, Hq, d, 5)
    st, n = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (start, counts))
    solar.history_cache_append(k, v, c, st, counts=n)
    got = solar.history_cache_attention(q, c, st + T, 0.05, flags=solar.FLAG_CAUSAL)
    for b in range(B - 1):
        one = solar.HistoryCache(*(x[b:b + 1] for x in c))
        near(got[b:b + 1, :counts[b]], q[b:b + 1, :counts[b]], one, [start[b] + counts[b]], 0.05, True, dt)


def test_scores_of_any_size():
    """Weights that vanish, and scores far outside what fp16 holds."""
    for dt in (BF, F32):
        c = filled(1, 1, 640, 64)
        q = queries(dt, 1, 130, 1, 64)
        q[0, ::3] *= 2.0 ** 40
        q[0, 1::3] *= 2.0 ** -60
        lengths = torch.tensor([600], dtype=torch.int32, device="cuda")
        k8, v8, ks, vs = values(c)
        want, _ = ho.attention(f64(q), k8, v8, ks, vs, [600], 0.1)
        got = f64(solar.history_cache_attention(q, c, lengths, 0.1))
        # rows 0, 3, ..: one key takes all the weight (its lead is 2^20 and more); rows 1, 4, ..: the mean of all values
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * np.abs(v8).max() * vs.max())


def test_strides_of_queries_and_outputs():
    B, M, Hq, H, d = 2, 70, 4, 2, 64
    c = filled(B, H, 256, d)
    buf = torch.randn(B, Hq, M, 2, d, generator=torch.Generator().manual_seed(4)).to(BF).cuda()
    q = buf[:, :, :, 0].transpose(1, 2)
    lengths = torch.tensor([200, 129], dtype=torch.int32, device="cuda")
    want = solar.history_cache_attention(q.contiguous(), c, lengths, 0.1)
    out = torch.full((B, Hq, M, 2, d), 7.0, dtype=BF, device="cuda")
    solar.history_cache_attention(q, c, lengths, 0.1, O=out[:, :, :, 1].transpose(1, 2))
    assert torch.equal(out[:, :, :, 1].transpose(1, 2), want) and (out[:, :, :, 0] == 7).all()


def test_no_queries_no_users_no_rows():
    c = filled(2, 1, 64, 64)
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert solar.history_cache_attention(queries(BF, 2, 0, 1, 64), c, n, 0.1).numel() == 0
    assert (solar.history_cache_attention(queries(BF, 2, 3, 1, 64), c, n, 0.1) == 0).all()
    assert (solar.history_cache_attention(queries(BF, 2, 300, 1, 64), c, n, 0.1) == 0).all()
    empty = solar.history_cache(2, 1, 0, 64)
    assert (solar.history_cache_attention(queries(BF, 2, 3, 1, 64), empty, n + 5, 0.1) == 0).all()
    assert (solar.history_cache_attention(queries(BF, 2, 300, 1, 64), empty, n + 5, 0.1) == 0).all()
    solar.history_cache_append(queries(BF, 2, 0, 1, 64), queries(BF, 2, 0, 1, 64), c, n)


@pytest.mark.parametrize("d", [64, 128])
def test_a_captured_serving_step_and_another_stream(d):
    B, H, Hq = 2, 2, 4
    k, v = queries(BF, B, 2, H, d, 7), queries(BF, B, 2, H, d, 8)
    q1, q2 = queries(BF, B, 1, Hq, d), queries(BF, B, 300, Hq, d)
    start = torch.tensor([100, 63], dtype=torch.int32, device="cuda")
    lengths = start + 2

    def step(c, o1, o2):
        solar.history_cache_append(k, v, c, start)
        solar.history_cache_attention(q1, c, lengths, 0.1, O=o1)
        solar.history_cache_attention(q2, c, lengths, 0.1, O=o2)
    want_c, want = filled(B, H, 256, d), [torch.empty_like(q1), torch.empty_like(q2)]
    step(want_c, *want)
    c, out = filled(B, H, 256, d), [torch.empty_like(q1), torch.empty_like(q2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(c, *out)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(c, *out)
    for x, y in zip(c, filled(B, H, 256, d)):
        x.copy_(y)
    for x in out:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(c, want_c))


def test_offsets_beyond_32_bits():
    """Users far into a cache of more than 2^32 bytes a tensor."""
    B, H, N, d = 260, 2, 65536, 128
    c = solar.history_cache(B, H, N, d)
    one = filled(1, H, 256, d)
    for x, y in zip(c, one):
        x[-1:, :, :y.shape[2]].copy_(y)
    q = queries(BF, 1, 1, 4, d).expand(B, -1, -1, -1)
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    lengths[-1] = 200
    got = solar.history_cache_attention(q, c, lengths, 0.1)
    n1 = torch.tensor([200], dtype=torch.int32, device="cuda")
    want = solar.history_cache_attention(q[:1], one, n1, 0.1)
    assert (got[:-1] == 0).all()
    assert (got[-1:].float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()
    many = solar.history_cache_attention(queries(BF, 1, 130, 4, d).expand(B, -1, -1, -1), c, lengths, 0.1)
    want = solar.history_cache_attention(queries(BF, 1, 130, 4, d), one, n1, 0.1)
    assert (many[-1:].float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()


def test_linear_state_and_cache_together():
    """A user's history is taken in once, then events come one by one: both forms of it are kept and both are asked."""
    B, T, H, d, more = 2, 150, 2, 64, 5
    g = torch.Generator().manual_seed(9)
    k, v, q = (torch.randn(B, T + more, H, d, generator=g).to(BF).cuda() for _ in range(3))
    ld = torch.tensor([-0.01, -0.2], device="cuda")
    c = solar.history_cache(B, H, T + more, d)
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    solar.history_cache_append(k[:, :T], v[:, :T], c, zero)
    _, S = solar.linear_attention_fwd(q[:, :T], k[:, :T], v[:, :T], ld, 0.125)
    for t in range(T, T + more):
        solar.history_cache_append(k[:, t:t + 1], v[:, t:t + 1], c, zero + t)
        soft = solar.history_cache_attention(q[:, t:t + 1], c, zero + t + 1, 0.125)
        lin = solar.linear_attention_step(q[:, t], k[:, t], v[:, t], ld, 0.125, S)
    o, last = ho.linear_attention(f64(q), f64(k), f64(v), f64(ld), 0.125)
    assert np.linalg.norm(f64(lin) - o[:, -1]) <= 2.0 ** -8 * np.linalg.norm(o[:, -1])
    assert np.linalg.norm(f64(S) - last) <= 2.0 ** -15 * np.linalg.norm(last)
    near(soft, q[:, -1:], c, [T + more] * B, 0.125, False, BF)
    # against the rows before they were rounded to 8 bits (half a step, 2^-4, of a value; the weights' own change twice that)
    full, size = ho.attention(f64(q[:, -1:]), f64(k).transpose(0, 2, 1, 3), f64(v).transpose(0, 2, 1, 3), np.ones((B, H, 3)), np.ones((B, H, 3)), [T + more] * B, 0.125)
    assert np.linalg.norm(f64(soft) - full) <= 2.0 ** -2 * np.linalg.norm(size)
