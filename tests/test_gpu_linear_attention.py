"""Linear attention with a decay per head against its definition in double precision.

Tolerances.  Let A be the same sums with absolute values in the place of all factors.  bf16 storage rounds, by half a step
each (2^-8 of the value): the decayed scores or the state as an operand (2^-8 A in all, the two parts making up A),
and the output (2^-8 |o|); fp32 sums of some hundreds of terms add 2^-14 A at most (two hundred additions of 2^-22, an
MMA's additions being truncated).  So |err| <= 2^-8 (|o| + A) + 2^-14 A; and, the three roundings being independent of
one another, the error's norm is at most the output's times 2^-8 (each alone has an rms of 2^-8 / sqrt(3), a bf16
mantissa being on average well above its smallest).  fp32 storage: 2^-15 A and a norm of 2^-17.  States: keys with their
decay enter as 16 bits (bf16: 2^-16 A on top)."""
import numpy as np
import pytest
import torch

from oracle import history_operators as ho
from paper_2603_02561_b200 import solar

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
DECAYS = [-0.02, 0.0, -5.0, -float("inf"), -0.3]


def make(dt, B, T, H, d, seed=0, strided=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, T, 3, H, d, generator=g).to(dt).cuda()
    q, k, v = (x[:, :, i] for i in range(3)) if strided else (x[:, :, i].contiguous() for i in range(3))
    do = torch.randn(B, T, H, d, generator=g).to(dt).cuda()
    s0, ds = (torch.randn(B, H, d, d, generator=g).cuda() for _ in range(2))
    ld = torch.tensor([DECAYS[h % len(DECAYS)] for h in range(H)], device="cuda")
    return q, k, v, do, s0, ds, ld


def f64(x):
    return x.double().cpu().numpy() if x is not None else None


def near(got, want, size, dt, name):
    got = f64(got)
    assert got.shape == want.shape and np.isfinite(got).all(), name
    u, acc, norm = (2.0 ** -8, 2.0 ** -14, 2.0 ** -8) if dt is BF else (2.0 ** -24, 2.0 ** -15, 2.0 ** -17)
    out_bits = 2.0 ** -24 if name in ("state", "dstate0") else u
    part = 2.0 ** -16 if name in ("state", "dstate0") and dt is BF else u
    err = np.abs(got - want)
    assert np.all(err <= out_bits * np.abs(want) + (part + acc) * size + 1e-30), (name, (err / (size + 1e-30)).max())
    if np.linalg.norm(want):
        assert np.linalg.norm(err) <= (2.0 ** -15 if name in ("state", "dstate0") else norm) * np.linalg.norm(want) * 1.0001, name


def check(dt, B, T, H, d, lengths, states, scale=0.3, strided=True, seed=0):
    q, k, v, do, s0, ds, ld = make(dt, B, T, H, d, seed, strided)
    if not states:
        s0 = ds = None
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    O, S = solar.linear_attention_fwd(q, k, v, ld, scale, state0=s0, lengths=n)
    dq, dk, dv, d0 = solar.linear_attention_bwd(q, k, v, ld, scale, do, state0=s0, dstate=ds, lengths=n)
    a = [f64(x) for x in (q, k, v, do, s0, ds)]
    p = [None if x is None else np.abs(x) for x in a]
    lds = f64(ld)
    want = (*ho.linear_attention(a[0], a[1], a[2], lds, scale, a[4], lengths),
            *ho.linear_attention_backward(a[0], a[1], a[2], lds, scale, a[3], a[4], a[5], lengths))
    size = (*ho.linear_attention(p[0], p[1], p[2], lds, abs(scale), p[4], lengths),
            *ho.linear_attention_backward(p[0], p[1], p[2], lds, abs(scale), p[3], p[4], p[5], lengths))
    for x, w, s, name in zip((O, S, dq, dk, dv, d0), want, size, ("O", "state", "dq", "dk", "dv", "dstate0")):
        near(x, w, s, dt, name)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("T,lengths", [(1, None), (63, None), (64, [64, 0]), (65, [1, 65]), (200, [137, 200])])
def test_against_the_definition(dt, d, T, lengths):
    check(dt, 2, T, 5, d, lengths, True)


@pytest.mark.parametrize("dt,d", [(BF, 32), (BF, 64), (BF, 128), (F32, 32), (F32, 64), (F32, 128)])
def test_segments_of_a_long_history(dt, d):
    check(dt, 2, 1100, 2, d, [1100, 259], True, scale=-0.1, strided=False)


@pytest.mark.parametrize("dt,d", [(BF, 64), (BF, 128), (F32, 64)])
def test_one_head_in_sixteen_segments(dt, d):
    check(dt, 1, 7000, 1, d, [6999], True, scale=0.1)


def test_states_left_out():
    check(BF, 1, 130, 3, 64, None, False)
    check(F32, 1, 130, 3, 64, [77], False)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_events_one_by_one_are_the_history(dt, d):
    B, T, H = 3, 9, 5
    q, k, v, _, s0, _, ld = make(dt, B, T, H, d)
    S = s0.clone()
    O = torch.stack([solar.linear_attention_step(q[:, t], k[:, t], v[:, t], ld, 0.3, S) for t in range(T)], dim=1)
    a = [f64(x) for x in (q, k, v, s0)]
    p = [np.abs(x) for x in a]
    want, size = ho.linear_attention(*a[:3], f64(ld), 0.3, a[3]), ho.linear_attention(*p[:3], f64(ld), 0.3, p[3])
    near(O, want[0], size[0], dt, "O")
    near(S, want[1], size[1], dt, "state")


def test_continuing_a_history():
    """Half of the events, then the other half from the state that the first call left."""
    q, k, v, _, s0, _, ld = make(F32, 2, 150, 5, 64)
    whole, last = solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0)
    a, mid = solar.linear_attention_fwd(q[:, :70], k[:, :70], v[:, :70], ld, 0.3, state0=s0)
    b, end = solar.linear_attention_fwd(q[:, 70:], k[:, 70:], v[:, 70:], ld, 0.3, state0=mid)
    for x, y in ((torch.cat([a, b], 1), whole), (end, last)):
        assert (x - y).norm() <= 2.0 ** -16 * y.norm()


def test_what_lies_behind_a_length_is_not_read_and_comes_out_zero():
    for dt in (BF, F32):
        for d in (32, 64, 128):
            q, k, v, do, s0, ds, ld = make(dt, 3, 140, 2, d)
            lengths = torch.tensor([0, 65, 139], dtype=torch.int32, device="cuda")
            first = [*solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0, lengths=lengths),
                     *solar.linear_attention_bwd(q, k, v, ld, 0.3, do, state0=s0, dstate=ds, lengths=lengths)]
            for b, n in enumerate([0, 65, 139]):
                for x in (q, k, v, do):
                    x[b, n:] = float("nan")
            out = [torch.full_like(first[0], 7.0) for _ in range(4)]
            again = [*solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0, lengths=lengths, O=out[0]),
                     *solar.linear_attention_bwd(q, k, v, ld, 0.3, do, state0=s0, dstate=ds, lengths=lengths, dq=out[1], dk=out[2], dv=out[3])]
            for x, y in zip(first, again):
                assert torch.equal(x, y)
            for b, n in enumerate([0, 65, 139]):
                assert all((x[b, n:] == 0).all() for x in out)
            assert torch.equal(first[1][0], s0[0])


def test_no_events_and_no_users():
    q, k, v, do, s0, ds, ld = make(BF, 2, 0, 2, 64)
    O, S = solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0)
    assert O.numel() == 0 and torch.equal(S, s0)
    assert torch.equal(solar.linear_attention_bwd(q, k, v, ld, 0.3, do, state0=s0, dstate=ds)[3], ds)
    q, k, v, do, s0, ds, ld = make(BF, 0, 5, 2, 64)
    assert solar.linear_attention_fwd(q, k, v, ld, 0.3)[0].shape == (0, 5, 2, 64)


def test_outputs_into_strided_buffers():
    B, T, H, d = 2, 70, 3, 64
    q, k, v, do, s0, ds, ld = make(BF, B, T, H, d)
    want = solar.linear_attention_bwd(q, k, v, ld, 0.3, do, state0=s0, dstate=ds)
    buf = torch.full((B, T, 4, H, d), 7.0, dtype=BF, device="cuda")
    solar.linear_attention_bwd(q, k, v, ld, 0.3, do, state0=s0, dstate=ds, dq=buf[:, :, 0], dk=buf[:, :, 1], dv=buf[:, :, 2])
    for i in range(3):
        assert torch.equal(buf[:, :, i], want[i])
    assert (buf[:, :, 3] == 7).all()


def test_repeated_rows_as_input():
    """A head's keys for every head (stride 0): reading is all that happens to an input."""
    q, k, v, _, _, _, ld = make(BF, 2, 70, 3, 64)
    one = k[:, :, :1].expand(-1, -1, 3, -1)
    a = solar.linear_attention_fwd(q, one, v, ld, 0.3)[0]
    assert torch.equal(a, solar.linear_attention_fwd(q, one.contiguous(), v, ld, 0.3)[0])


def test_a_captured_step_and_another_stream():
    q, k, v, do, s0, ds, ld = make(BF, 2, 600, 2, 64)
    want = [*solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0), *solar.linear_attention_bwd(q, k, v, ld, 0.3, do, state0=s0, dstate=ds)]
    state = s0.clone()
    want_step = solar.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], ld, 0.3, state)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = [torch.empty_like(x) for x in want]
    state2, o2 = s0.clone(), torch.empty_like(want_step)

    def step():
        solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0, O=out[0], state=out[1])
        solar.linear_attention_bwd(q, k, v, ld, 0.3, do, state0=s0, dstate=ds, dq=out[2], dk=out[3], dv=out[4], dstate0=out[5])
        solar.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], ld, 0.3, state2, O=o2)
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.equal(state2, state) and torch.equal(o2, want_step)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x in out:
        x.zero_()
    state2.copy_(s0)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_inputs_written_just_before_the_call():
    B, T, H, d = 4, 2000, 4, 64
    src = make(BF, B, T, H, d, strided=False)
    want = solar.linear_attention_fwd(*src[:3], src[6], 0.3, state0=src[4])
    q, k, v, s0 = (torch.zeros_like(x) for x in (*src[:3], src[4]))
    for x, y in ((q, src[0]), (k, src[1]), (v, src[2]), (s0, src[4])):
        x.copy_(y)
    got = solar.linear_attention_fwd(q, k, v, src[6], 0.3, state0=s0)
    for x in (q, k, v, s0):
        x.zero_()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_what_is_not_finite_stays_with_its_head():
    q, k, v, _, s0, _, ld = make(BF, 2, 100, 3, 64, strided=False)
    want = solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0)[0]
    k[1, 50, 2, 3] = float("inf")
    got = solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0)[0]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1, :, :2], want[1, :, :2])
    assert not torch.isfinite(got[1, 50:, 2]).any()          # inf where the definition has it, NaN from the states on
