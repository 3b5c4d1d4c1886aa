"""Attention over the 8-bit cache at sizes that reach either of its kernels, which every call here is asserted to do: the one
of 256 query rows on tcgen05 (512 threads a CTA) and the one of 16 (128 threads).

Tolerance, component by component.  With p the softmax in 64 bits, W = sum p |v| and dz the error of a score: fp32 sums of exact
products, 2^-20 of sum |q k| at most (a product's rounding and the exponential's 2^-22 among them), which moves p by 2 dz.
A weight times its value scale is rounded to fp16, 2^-11 of it, or 2^-28 of the row's largest such product where that is more;
the sum of the weights is good to 2^-14; the output is rounded to bf16, half a step being 2^-8:
  |err| <= 2^-8 |o| + (2^-11 + 2^-14 + 2 dz) W + 2^-28 max(p vs) sum |v8|
The other kernel holds the weights alone, to 2^-40 of the largest where that is more than 2^-11 of them: 2^-40 max(p) sum |v| in
the place of the last term."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_02561_b200 import solar

pytestmark = pytest.mark.gpu
BF, E4, I32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32
FLASH, FEW = 512, 128


class _Node(ctypes.Structure):
    _fields_ = [("func", ctypes.c_void_p)] + [(n, ctypes.c_uint) for n in ("gx", "gy", "gz", "bx", "by", "bz", "smem")] + \
        [(n, ctypes.c_void_p) for n in ("params", "extra", "kern", "ctx")]


def launched(call):
    """Threads of a CTA and the grid's x of the one kernel that `call` launches (captured, not run)."""
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(g):
        call()
    cu, graph, n = ctypes.CDLL("libcuda.so.1"), ctypes.c_void_p(g.raw_cuda_graph()), ctypes.c_size_t(0)
    assert cu.cuGraphGetNodes(graph, None, ctypes.byref(n)) == 0 and n.value == 1
    nodes, p = (ctypes.c_void_p * 1)(), _Node()
    assert cu.cuGraphGetNodes(graph, nodes, ctypes.byref(n)) == 0
    assert cu.cuGraphKernelNodeGetParams_v2(ctypes.c_void_p(nodes[0]), ctypes.byref(p)) == 0
    return p.bx, p.gx


def attend(q, c, lengths, scale, causal=False, kernel=None, splits=None):
    n = torch.tensor(lengths, dtype=I32, device="cuda")
    out = torch.full_like(q, 7.0)
    call = lambda: solar.history_cache_attention(q, c, n, scale, flags=solar.FLAG_CAUSAL if causal else 0, O=out)  # noqa: E731
    if kernel is not None:
        threads, gx = launched(call)
        assert threads == kernel
        if splits is not None:
            assert gx == splits * -(-q.shape[1] * (q.shape[2] // c.k.shape[1]) // 256)
    call()
    return out


def filled(B, H, N, d, seed=0, spread=5):
    g = torch.Generator().manual_seed(seed)
    c = solar.history_cache(B, H, N, d)
    for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x.copy_((torch.randn(x.shape, generator=g) * 60).clamp(-448, 448).to(E4))
        s.copy_(torch.exp2(torch.randint(-3 - spread, -3, s.shape, generator=g).float()))
    return c


def queries(B, M, Hq, d, seed=1):
    return torch.randn(B, M, Hq, d, generator=torch.Generator().manual_seed(seed)).to(BF).cuda()


def wide(x):
    return x.float().double().cpu().numpy()


def near(got, q, c, lengths, scale, causal, rows, kernel=FLASH):
    """`rows`: the queries that are looked at (the definition in 64 bits takes its time)."""
    B, M, Hq, d = q.shape
    H, N = c.k.shape[1], c.k.shape[2]
    ks, vs = wide(c.k_scale).repeat(64, 2), wide(c.v_scale).repeat(64, 2)
    qw, gw = wide(q), wide(got)
    for b in range(B):
        n = min(max(lengths[b], 0), N)
        for h in range(H):
            k8, v8 = wide(c.k[b, h, :n]), wide(c.v[b, h, :n])
            K, V = k8 * ks[b, h, :n, None], v8 * vs[b, h, :n, None]
            for hq in range(h * (Hq // H), (h + 1) * (Hq // H)):
                for m in rows:
                    see = max(min(n, lengths[b] - M + m + 1), 0) if causal else n
                    o = gw[b, m, hq]
                    if see == 0:
                        assert (o == 0).all()
                        continue
                    z = scale * (K[:see] @ qw[b, m, hq])
                    p = np.exp(z - z.max())
                    p /= p.sum()
                    want, W = p @ V[:see], p @ np.abs(V[:see])
                    dz = 2.0 ** -20 * abs(scale) * (np.abs(K[:see]) @ np.abs(qw[b, m, hq])).max()
                    if kernel == FLASH:
                        floor = 2.0 ** -28 * (p * vs[b, h, :see]).max() * np.abs(v8[:see]).sum(0)
                    else:
                        floor = 2.0 ** -40 * p.max() * np.abs(V[:see]).sum(0)
                    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -14 + 2 * dz) * W + floor
                    err = np.abs(o - want)
                    assert (err <= bound).all(), (b, m, hq, see, (err / bound).max())


# which kernel a call gets, and in how many ranges of the cache, is the library's rule; the sizes are such that it takes this one
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,M,Hq,H,N,lengths,splits", [
    (2, 1300, 8, 2, 1088, [1088, 0], 1), (1, 2500, 1, 1, 10304, [10250], 8), (3, 1000, 4, 2, 2112, [2111, 64, 1], 2),
    (3, 700, 6, 2, 1984, [1984, 127, 1921], 2)])
@pytest.mark.parametrize("causal", [False, True])
def test_many_queries(d, B, M, Hq, H, N, lengths, splits, causal):
    c, q = filled(B, H, N, d), queries(B, M, Hq, d)
    got = attend(q, c, lengths, 0.05, causal, FLASH, splits)
    near(got, q, c, lengths, 0.05, causal, [0, 1, 63, 127, 128, 255, 256, M // 2, M - 65, M - 2, M - 1])
    assert torch.isfinite(got).all()
    assert torch.equal(got, attend(q, c, lengths, 0.05, causal))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [-0.05, 0.0])
def test_scales_of_any_sign(d, scale):
    B, M, Hq, H, N = 3, 700, 6, 2, 1984
    c, q = filled(B, H, N, d), queries(B, M, Hq, d)
    near(attend(q, c, [1984, 300, 64], scale, False, FLASH), q, c, [1984, 300, 64], scale, False, [0, 5, 200, M - 1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("down", [False, True])
@pytest.mark.parametrize("causal", [False, True])
def test_a_maximum_that_rises_from_tile_to_tile(d, down, causal):
    """Scores from -150 to 150 along the cache (or back): the reference is raised again and again, and weights vanish."""
    B, M, Hq, H, N = 3, 700, 6, 2, 1984
    c, q = filled(B, H, N, d), queries(B, M, Hq, d)
    q[..., 0], q[..., 1:] = 1.0, q[..., 1:] * 2.0 ** -5
    ramp = torch.linspace(448, -448, N) if down else torch.linspace(-448, 448, N)
    c.k[..., 0] = ramp.to(E4).cuda()
    c.k_scale.fill_(2.0 ** -3)
    lengths = [1984, 1000, 700]
    near(attend(q, c, lengths, 2.7, causal, FLASH), q, c, lengths, 2.7, causal, [0, 1, 130, 300, 511, M - 1])


@pytest.mark.parametrize("d", [64, 128])
def test_scores_of_any_size(d):
    """Rows 0, 3, ..: one key takes all the weight; rows 1, 4, ..: the mean of all values."""
    B, M, Hq, H, N = 3, 700, 6, 2, 1984
    c, q = filled(B, H, N, d), queries(B, M, Hq, d)
    q[:, ::3] *= 2.0 ** 40
    q[:, 1::3] *= 2.0 ** -60
    got = attend(q, c, [1984, 300, 64], 0.05, False, FLASH)
    near(got, q, c, [1984, 300, 64], 0.05, False, [1, 2, 4, 5, 400, 698])
    K, V = wide(c.k) * wide(c.k_scale).repeat(64, 2)[..., None], wide(c.v) * wide(c.v_scale).repeat(64, 2)[..., None]
    for b, n in ((0, 1984), (1, 300), (2, 64)):
        for m in (0, 3, 300, 699):
            z = K[b, 1, :n] @ wide(q[b, m, 4])
            lead = np.sort(z)[-1] - np.sort(z)[-2]
            assert lead > 2.0 ** -18 * (np.abs(K[b, 1, :n]) @ np.abs(wide(q[b, m, 4]))).max()       # more than rounding
            want = V[b, 1, z.argmax()]
            assert (np.abs(wide(got[b, m, 4]) - want) <= 2.0 ** -8 * np.abs(want)).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", ["k", "v"])
def test_a_row_that_is_not_finite_reaches_only_those_that_see_it(d, what):
    B, M, H, N = 1, 6000, 1, 6080
    clean, q = filled(B, H, N, d), queries(B, M, 1, d)
    c = solar.HistoryCache(*(x.clone() for x in clean))
    for row in (5000, 700):
        getattr(c, what).view(torch.uint8)[0, 0, row, 7] = 0x7f
        got = attend(q, c, [M], 0.1, True, FLASH)
        assert torch.isnan(got[0, row:, 0, 7]).all() and torch.isfinite(got[0, :row]).all()
        near(got, q, clean, [M], 0.1, True, [0, 200, 640, row - 60, row - 2, row - 1])


@pytest.mark.parametrize("d", [64, 128])
def test_what_lies_behind_a_length_does_not_matter(d):
    B, M, Hq, H, N = 3, 1000, 4, 2, 2112
    lengths = [2049, 65, 0]
    c, q = filled(B, H, N, d), queries(B, M, Hq, d)
    want = attend(q, c, lengths, 0.1, False, FLASH)
    for b, n in enumerate(lengths):
        c.k.view(torch.uint8)[b, :, n:] = 0x7f
        c.v.view(torch.uint8)[b, :, n:] = 0xff
        c.k_scale[b, :, -(-n // 64):] = float("nan")
        c.v_scale[b, :, -(-n // 64):] = float("inf")
    assert torch.equal(attend(q, c, lengths, 0.1), want) and (want[2] == 0).all()


@pytest.mark.parametrize("d", [64, 128])
def test_a_padded_batch_of_new_histories(d):
    """Queries padded as the appended rows were, one user's padding past the cache's end, one user without rows."""
    B, H, Hq, N, T = 3, 2, 4, 2112, 1200
    start, counts = [10, 1000, 0], [1200, 13, 0]
    c = filled(B, H, N, d)
    for b in range(B):
        for x in (c.k, c.v):
            x.view(torch.uint8)[b, :, start[b]:] = 0x7f
    k, v, q = queries(B, T, H, d, 3), queries(B, T, H, d, 4), queries(B, T, Hq, d, 5)
    st, n = (torch.tensor(x, dtype=I32, device="cuda") for x in (start, counts))
    solar.history_cache_append(k, v, c, st, counts=n)
    got = attend(q, c, [x + T for x in start], 0.05, True, FLASH)
    for b, rows in ((0, [0, 1, 53, 54, 118, 500, 1199]), (1, [0, 1, 12])):
        one = solar.HistoryCache(*(x[b:b + 1] for x in c))
        m = counts[b]
        near(got[b:b + 1, :m], q[b:b + 1, :m], one, [start[b] + m], 0.05, True, rows)


@pytest.mark.parametrize("d", [64, 128])
def test_a_captured_call_another_stream_and_strides(d):
    B, M, Hq, H, N = 3, 1000, 4, 2, 2112
    c = filled(B, H, N, d)
    buf = queries(B, Hq * 2, M, d).view(B, Hq, 2, M, d)
    q = buf[:, :, 0].transpose(1, 2)
    n = torch.tensor([2112, 1001, 3], dtype=I32, device="cuda")
    want = attend(q.contiguous(), c, [2112, 1001, 3], 0.1, True, FLASH)
    out = torch.full((B, Hq, 2, M, d), 7.0, dtype=BF, device="cuda")
    call = lambda: solar.history_cache_attention(q, c, n, 0.1, flags=solar.FLAG_CAUSAL, O=out[:, :, 1].transpose(1, 2))  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert torch.equal(out[:, :, 1].transpose(1, 2), want) and (out[:, :, 0] == 7).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    out.fill_(7.0)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[:, :, 1].transpose(1, 2), want) and (out[:, :, 0] == 7).all()


@pytest.mark.parametrize("d", [64, 128])
def test_few_queries(d):
    B, M, Hq, H, N = 3, 1000, 4, 2, 2112
    c, q = filled(B, H, N, d), queries(B, M, Hq, d)
    near(attend(q[:, :8].contiguous(), c, [2112, 65, 1], 0.1, False, FEW), q[:, :8], c, [2112, 65, 1], 0.1, False, [0, 7], FEW)


SIZES = {FLASH: (3, 1000, 4, 2, 2112), FEW: (3, 5, 4, 2, 2112)}


def test_queries_may_be_overwritten():
    """The output in the queries' own place."""
    for kernel, (B, M, Hq, H, N) in SIZES.items():
        c, q = filled(B, H, N, 64), queries(B, M, Hq, 64)
        n = torch.tensor([2112, 1500, 0], dtype=I32, device="cuda")
        want = attend(q, c, [2112, 1500, 0], 0.1, False, kernel)
        solar.history_cache_attention(q, c, n, 0.1, O=q)
        assert torch.equal(q, want)


# ---- values of very different size ----------------------------------------------------------------------
def spread_values(c, exponents, rise):
    """Value blocks of 2^e in turn, zeros where e is the smallest of all; `rise`: how much larger (in log2 units) the scores of the zero
    blocks are, by component 0 of the keys."""
    B, H, N, d = c.k.shape
    at = torch.arange(N // 64) % len(exponents)
    e = torch.tensor(exponents)[at]
    zero = (e == min(exponents)).cuda()
    c.v_scale.copy_(torch.exp2(e.double()).float().expand(B, H, N // 64))
    c.v.view(torch.uint8).view(B, H, N // 64, 64, d)[:, :, zero] = 0
    c.k_scale.fill_(2.0 ** -6)
    one = int(torch.tensor([64.0 if rise > 0 else -64.0]).to(E4).view(torch.uint8))
    k = c.k.view(torch.uint8).view(B, H, N // 64, 64, d)
    k[..., 0] = 0
    if rise:
        k[:, :, zero, :, 0] = one


@pytest.mark.parametrize("kernel", [FLASH, FEW])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("exponents", [[-100, 31], [31, -100, 0], [-100, 60, 0], [60, -100], [0, -100], [20, 5, -100], [0, 0, 0, 0, 0, 0, -100, 31, 31]])
@pytest.mark.parametrize("rise", [0, 20, 130, -20])
def test_value_scales_far_apart(kernel, d, exponents, rise):
    """Blocks of zeros (their scale is 2^-100) beside blocks of large values count in the softmax as any others do."""
    B, M, Hq, H, N = SIZES[kernel]
    c, q = filled(B, H, N, d), queries(B, M, Hq, d)
    spread_values(c, exponents, rise)
    q[..., 0] = 1.0
    scale = abs(rise) * np.log(2.0) if rise else 0.05        # component 0 of the zero blocks' keys is 1 (or -1)
    if rise:
        q[..., 1:] *= 2.0 ** -6
    lengths = [2112, 1500, 70]
    near(attend(q, c, lengths, scale, False, kernel), q, c, lengths, scale, False, [0, 1, M - 1], kernel)


@pytest.mark.parametrize("kernel", [FLASH, FEW])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e", [90, 105])
def test_largest_values(kernel, d, e):
    """Values of up to 448 * 2^105, and zeros: the weighted mean is far inside of what bf16 holds."""
    B, M, Hq, H, N = SIZES[kernel]
    c, q = filled(B, H, N, d), queries(B, M, Hq, d)
    spread_values(c, [e, -100, 0], 0)
    lengths = [2112, 1500, 70]
    near(attend(q, c, lengths, 0.05, False, kernel), q, c, lengths, 0.05, False, [0, 1, M - 1], kernel)


# ---- a cache whose memory was never set -----------------------------------------------------------------
@pytest.mark.parametrize("kernel", [FLASH, FEW])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("left", [float("nan"), float("inf"), -float("inf"), 3e38, 0.0])
def test_scales_that_were_never_written_are_not_read_as_numbers(kernel, d, left):
    """A padded batch in a cache of arbitrary memory: the padding's queries see blocks that hold nothing yet, in tiles that a
    user's own queries share."""
    B, H, Hq, N = 3, 2, 4, 2112
    T = 1200 if kernel == FLASH else 13
    start, counts = [60, 125, 0], [2, 7, 0]
    c = filled(B, H, N, d)
    clean = solar.HistoryCache(*(x.clone() for x in c))
    for b in range(B):
        at = -(-(start[b] + counts[b]) // 64)
        for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
            s[b, :, at:] = left
            x.view(torch.uint8)[b, :, start[b]:] = 0x7f
    k, v, q = queries(B, T, H, d, 3), queries(B, T, H, d, 4), queries(B, T, Hq, d, 5)
    st, n = (torch.tensor(x, dtype=I32, device="cuda") for x in (start, counts))
    solar.history_cache_append(k, v, clean, st, counts=n)
    solar.history_cache_append(k, v, c, st, counts=n)
    out = attend(q, c, [y + T for y in start], 0.05, True, kernel)
    for b in (0, 1):
        one, m = solar.HistoryCache(*(x[b:b + 1] for x in clean)), counts[b]
        assert torch.isfinite(out[b:b + 1, :m]).all()
        near(out[b:b + 1, :m], q[b:b + 1, :m], one, [start[b] + m], 0.05, True, range(m), kernel)
