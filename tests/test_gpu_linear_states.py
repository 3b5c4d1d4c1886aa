"""How exact what ends in fp32 is: states of either storage, outputs of fp32 storage, in the norm.

Tolerance 2^-20 (9.5e-7) of the norm.  Operands enter with 24 bits (2^-24 each); a power of the decay is good to 2 ulp, 2^-22, and
2^-23 |n log2 g| for its rounded argument, which stays below 8 where the weight counts; a tile's sum in the tensor cores is
cut off at 2^-23 of it up to twelve times, half of that on average, 2^-21 in all but toward zero of sums that are a few per
cent of a long state's; sums of up to 63 chunks are rounded, 2^-25 rms of a sum that grows, 2^-22 rms in all.  Terms that add up to less than
2^-20 together.  (Two bf16 terms of a key are 16 bits, 2^-18.4 of a state of random events; sums that stay in the tensor cores' accumulators
over a whole history 2^-18.3.)"""
import numpy as np
import pytest
import torch

from oracle import history_operators as ho
from paper_2603_02561_b200 import solar

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def make(dt, B, T, H, d, seed=0):
    g = torch.Generator().manual_seed(seed)
    q, k, v, do = (torch.randn(B, T, H, d, generator=g).to(dt).cuda() for _ in range(4))
    s0, ds = (torch.randn(B, H, d, d, generator=g).cuda() for _ in range(2))
    return q, k, v, do, s0, ds


def f64(x):
    return x.double().cpu().numpy()


def close(got, want, name):
    err = np.linalg.norm(f64(got) - want) / np.linalg.norm(want)
    assert err <= 2.0 ** -20, (name, err)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("T", [64, 1, 33, 65, 200])
def test_states_of_heads_that_forget_soon(dt, d, T):
    """The last chunk's (in reversed time the first events') weights are the state."""
    q, k, v, do, s0, ds = make(dt, 2, T, 3, d)
    decays = [-2.5, -2.09, -6.0]
    ld = torch.tensor(decays, device="cuda")
    S = solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0)[1]
    ds0 = solar.linear_attention_bwd(q, k, v, ld, 0.3, do, state0=s0)[3]
    a = [f64(x) for x in (q, k, v, do, s0)]
    want = ho.linear_attention(*a[:3], f64(ld), 0.3, a[4])[1]
    back = ho.linear_attention_backward(*a[:3], f64(ld), 0.3, a[3], a[4])[3]
    for h in range(3):
        close(S[:, h], want[:, h], ("state", decays[h]))
        close(ds0[:, h], back[:, h], ("dstate0", decays[h]))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_a_long_history(dt, d):
    B, T, decays = 2, 4000, [0.0, -0.02, -0.2]
    lengths = [4000, 2999]
    q, k, v, do, s0, ds = make(dt, B, T, 3, d)
    ld, n = torch.tensor(decays, device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    O, S = solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0, lengths=n)
    grads = solar.linear_attention_bwd(q, k, v, ld, 0.3, do, state0=s0, dstate=ds, lengths=n)
    a = [f64(x) for x in (q, k, v, do, s0, ds)]
    want = ho.linear_attention(*a[:3], f64(ld), 0.3, a[4], lengths)
    back = ho.linear_attention_backward(*a[:3], f64(ld), 0.3, a[3], a[4], a[5], lengths)
    for h in range(3):
        close(S[:, h], want[1][:, h], ("state", decays[h]))
        close(grads[3][:, h], back[3][:, h], ("dstate0", decays[h]))
        if dt is F32:
            for x, y, name in ((O, want[0], "O"), *zip(grads[:3], back[:3], ("dq", "dk", "dv"))):
                close(x[:, :, h], y[:, :, h], (name, decays[h]))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_one_head_in_sixteen_segments(dt, d):
    q, k, v, do, s0, ds = make(dt, 1, 7000, 1, d)
    ld, n = torch.tensor([-0.02], device="cuda"), torch.tensor([6999], dtype=torch.int32, device="cuda")
    O, S = solar.linear_attention_fwd(q, k, v, ld, 0.3, state0=s0, lengths=n)
    d0 = solar.linear_attention_bwd(q, k, v, ld, 0.3, do, state0=s0, dstate=ds, lengths=n)[3]
    a = [f64(x) for x in (q, k, v, do, s0, ds)]
    want = ho.linear_attention(*a[:3], f64(ld), 0.3, a[4], [6999])
    close(S, want[1], "state")
    close(d0, ho.linear_attention_backward(*a[:3], f64(ld), 0.3, a[3], a[4], a[5], [6999])[3], "dstate0")
    if dt is F32:
        close(O, want[0], "O")
