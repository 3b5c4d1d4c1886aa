"""What the history operators refuse, before anything reaches a GPU: the C ABI with addresses that are never read, and
the binding with tensors that say they are on a GPU."""
import ctypes

import pytest
import torch

from paper_2603_02561_b200 import build as solar_build
from paper_2603_02561_b200 import solar

P, vp = ctypes.c_void_p(0x1000), ctypes.c_void_p
P2, P3, P4 = (ctypes.c_void_p(0x2000 + 0x1000 * i) for i in range(3))          # outputs
S3 = lambda *x: (ctypes.c_longlong * 3)(*x)  # noqa: E731
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
INVALID, UNSUPPORTED = solar.ERR_INVALID_ARG, solar.ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    solar_build.build()
    return solar.lib()


def fwd(L, B=2, T=5, H=3, d=64, dt=1, Q=P, qs=None, K=P, V=P, ld=P, lengths=None, s0=None, O=P2, os=None, S=P):
    return L.solar_linear_attention_fwd(B, T, H, d, dt, Q, qs, K, None, V, None, ld, 0.1, lengths, s0, O, os, S, None)


def bwd(L, B=2, T=5, H=3, d=64, dt=1, dO=P, s0=None, ds=None, dQ=P2, dqs=None, dK=P3, dV=P4, d0=None):
    return L.solar_linear_attention_bwd(B, T, H, d, dt, P, None, P, None, P, None, P, 0.1, None, s0, dO, None, ds, dQ, dqs, dK, None, dV,
                                        None, d0, None)


def step(L, B=2, H=3, d=64, dt=1, Q=P, ld=P, S=P, O=P2, os=None):
    return L.solar_linear_attention_step(B, H, d, dt, Q, None, P, None, P, None, ld, 0.1, S, O, os, None)


def append(L, B=2, T=5, H=3, N=128, d=64, dt=1, K=P, ks=None, start=P, counts=None, k8=P, v8=P, s=P):
    return L.solar_history_cache_append(B, T, H, N, d, dt, K, ks, P, None, start, counts, k8, v8, s, P, None)


def attend(L, B=2, M=5, Hq=6, H=3, N=128, d=64, dt=1, Q=P, k8=P, s=P, lengths=P, flags=0, O=P, os=None):
    return L.solar_history_cache_attention(B, M, Hq, H, N, d, dt, Q, None, k8, P, s, P, lengths, 0.1, flags, O, os, None)


@pytest.mark.parametrize("call", [fwd, bwd, step, append, attend])
def test_sizes_and_types(L, call):
    assert call(L, d=48) == UNSUPPORTED
    assert call(L, d=0) == UNSUPPORTED
    assert call(L, dt=2) == UNSUPPORTED
    assert call(L, B=-1) == INVALID
    assert call(L, H=0) == INVALID
    assert call(L, B=65536) == UNSUPPORTED
    assert call(L, H=30000) == UNSUPPORTED
    assert call(L, B=0) == solar.OK


def test_pointers(L):
    for call, names in ((fwd, ("Q", "K", "V", "O")), (bwd, ("dO", "dQ", "dK", "dV")), (step, ("Q", "S", "O")), (append, ("K", "k8", "v8")),
                        (attend, ("Q", "k8", "O"))):
        for n in names:
            assert call(L, **{n: vp(0)}) == INVALID, (call.__name__, n)
            assert call(L, **{n: vp(0x1008)}) == INVALID, (call.__name__, n)
    for call, names in ((fwd, ("ld",)), (step, ("ld",)), (append, ("start", "s")), (attend, ("lengths", "s"))):
        for n in names:
            assert call(L, **{n: vp(0)}) == INVALID and call(L, **{n: vp(0x1002)}) == INVALID, (call.__name__, n)
    assert fwd(L, lengths=vp(0x1002)) == INVALID and fwd(L, s0=vp(0x1004)) == INVALID and fwd(L, S=vp(0x1004)) == INVALID
    assert append(L, counts=vp(0x1001)) == INVALID


def test_a_state_is_not_read_and_written_in_one_call(L):
    assert fwd(L, s0=P, S=P) == INVALID
    assert bwd(L, ds=P, d0=P) == INVALID and bwd(L, s0=P, d0=P) == INVALID


def test_outputs_over_inputs_and_over_one_another(L):
    assert fwd(L, O=P) == INVALID and step(L, O=P) == INVALID
    for n in ("dQ", "dK", "dV"):
        assert bwd(L, **{n: P}) == INVALID
    assert bwd(L, dQ=P3) == INVALID and bwd(L, dQ=P4) == INVALID and bwd(L, dK=P4) == INVALID


def test_lengths_past_what_is_counted(L):
    for call in (fwd, bwd, append):
        assert call(L, T=(1 << 30) + 1) == UNSUPPORTED
    assert attend(L, M=(1 << 30) + 1) == UNSUPPORTED


def test_strides(L):
    assert fwd(L, qs=S3(5 * 3 * 64, 3 * 64 + 4, 64)) == INVALID           # 8 bytes past a 16-byte piece
    assert fwd(L, qs=S3(-960, 192, 64)) == INVALID
    for os in (S3(960, 192, 0), S3(960, 0, 64), S3(0, 192, 64), S3(960, 192, 32), S3(192, 192, 64), S3(800, 192, 64)):
        assert fwd(L, os=os) == INVALID and bwd(L, dqs=os) == INVALID and attend(L, Hq=3, os=os) == INVALID
    assert step(L, os=(ctypes.c_longlong * 2)(64, 64)) == INVALID


def test_cache_sizes_heads_and_flags(L):
    assert append(L, N=100) == INVALID and attend(L, N=100) == INVALID and append(L, N=-64) == INVALID
    assert attend(L, N=(1 << 30) + 64) == UNSUPPORTED
    assert attend(L, Hq=4) == INVALID and attend(L, Hq=0) == INVALID
    assert attend(L, flags=1) == UNSUPPORTED and attend(L, flags=4) == UNSUPPORTED
    assert attend(L, M=0) == solar.OK and append(L, T=0) == solar.OK and append(L, T=-1) == INVALID


# ---- the binding ----------------------------------------------------------------------------------
class Gpu:
    def __init__(self, *shape, dtype=BF, cuda=True, strided=False, device="cuda:0"):
        self.t = torch.zeros(*shape[:-1], 2 * shape[-1], dtype=dtype)[..., ::2] if strided else torch.zeros(shape, dtype=dtype)
        self.dtype, self.shape, self.is_cuda, self.device = dtype, self.t.shape, cuda, torch.device(device)

    def get_device(self): return self.device.index if self.is_cuda else -1
    def dim(self): return self.t.dim()
    def new_empty(self, shape, dtype=None): return Gpu(*shape, dtype=dtype or self.dtype)
    def numel(self): return self.t.numel()
    def is_contiguous(self): return self.t.is_contiguous()
    def data_ptr(self): return self.t.data_ptr()
    def stride(self, *a): return self.t.stride(*a)


@pytest.fixture
def calls(monkeypatch):
    made = []

    class Recorder:
        def __getattr__(self, name):
            if not name.startswith("solar_"):
                raise AttributeError(name)
            return lambda *a: (made.append((name, a)), 0)[1]
    monkeypatch.setattr(solar, "_lib", Recorder())
    monkeypatch.setattr(solar, "_stream", lambda stream=None: 0)
    monkeypatch.setattr(solar, "_current_device", lambda: 0)
    return made


B, T, H, d, N = 2, 5, 3, 64, 128


def tensors(call):
    tok, st, small = ((B, T, H, d), BF), ((B, H, d, d), F32), ((B,), I32)
    if call == "step":
        return {**{n: ((B, H, d), BF) for n in ("q", "k", "v", "O")}, "log_decay": ((H,), F32), "state": st}
    if call == "append":
        return {"k": tok, "v": tok, "start": small, "counts": small}
    if call == "attend":
        return {"q": ((B, T, 2 * H, d), BF), "O": ((B, T, 2 * H, d), BF), "lengths": small}
    x = {**{n: tok for n in ("q", "k", "v")}, "log_decay": ((H,), F32), "state0": st, "lengths": small}
    return {**x, "O": tok, "state": st} if call == "fwd" else {**x, "dO": tok, "dstate": st, "dq": tok, "dk": tok, "dv": tok, "dstate0": st}


def cache():
    E = torch.float8_e4m3fn
    return {"k": ((B, H, N, d), E), "v": ((B, H, N, d), E), "k_scale": ((B, H, N // 64), F32), "v_scale": ((B, H, N // 64), F32)}


def run(call, t, c):
    if call in ("append", "attend"):
        c = solar.HistoryCache(*(c[n] for n in ("k", "v", "k_scale", "v_scale")))
    if call == "append":
        solar.history_cache_append(t["k"], t["v"], c, t["start"], counts=t["counts"])
    elif call == "attend":
        solar.history_cache_attention(t["q"], c, t["lengths"], 0.1, O=t["O"])
    elif call == "step":
        solar.linear_attention_step(t["q"], t["k"], t["v"], t["log_decay"], 0.1, t["state"], O=t["O"])
    elif call == "fwd":
        solar.linear_attention_fwd(t["q"], t["k"], t["v"], t["log_decay"], 0.1, **{n: t[n] for n in ("state0", "lengths", "O", "state")})
    else:
        solar.linear_attention_bwd(t["q"], t["k"], t["v"], t["log_decay"], 0.1, t["dO"],
                                   **{n: t[n] for n in ("state0", "dstate", "lengths", "dq", "dk", "dv", "dstate0")})


@pytest.mark.parametrize("call", ["fwd", "bwd", "step", "append", "attend"])
def test_the_binding_looks_at_every_tensor(calls, call):
    want, held = tensors(call), cache()
    make = lambda w, **kw: {n: Gpu(*s, dtype=t, **kw) for n, (s, t) in w.items()}  # noqa: E731
    run(call, make(want), make(held))
    assert len(calls) == 1
    for name, (shape, dt) in want.items():
        other = torch.float16 if dt is BF else torch.float64 if dt is F32 else torch.int64
        wrong = [Gpu(*shape, dtype=other), Gpu(*shape, dtype=dt, cuda=False), Gpu(*shape[:-1], shape[-1] + 64, dtype=dt),
                 Gpu(*shape, dtype=dt, device="cuda:1"), Gpu(*shape, dtype=dt, strided=True)]
        for w in wrong:
            with pytest.raises((ValueError, TypeError)):
                run(call, {**make(want), name: w}, make(held))
    if call in ("append", "attend"):
        for name, (shape, dt) in held.items():
            for w in (Gpu(*shape, dtype=torch.int8), Gpu(*shape, dtype=dt, cuda=False), Gpu(*shape, 1, dtype=dt), Gpu(*shape, dtype=dt, device="cuda:1")):
                with pytest.raises((ValueError, TypeError)):
                    run(call, make(want), {**make(held), name: w})
    assert len(calls) == 1


def test_strides_go_to_the_library(calls):
    t = {n: Gpu(*s, dtype=x) for n, (s, x) in tensors("fwd").items()}
    t["k"].t = torch.zeros(B, T, 2, H, d, dtype=BF)[:, :, 1]
    run("fwd", t, {})
    args = calls[0][1]
    assert args[6] is None and list(args[8]) == [T * 2 * H * d, 2 * H * d, d]


@pytest.mark.parametrize("call", ["fwd", "bwd", "step", "append", "attend"])
def test_another_device_than_the_current_one_is_refused(calls, monkeypatch, call):
    monkeypatch.setattr(solar, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        run(call, {n: Gpu(*s, dtype=t) for n, (s, t) in tensors(call).items()}, {n: Gpu(*s, dtype=t) for n, (s, t) in cache().items()})
    assert not calls


@pytest.mark.parametrize("call", ["fwd", "bwd", "step", "append", "attend"])
def test_outputs_that_are_not_given_are_made(calls, call):
    t = {n: Gpu(*s, dtype=x) for n, (s, x) in tensors(call).items()}
    for n in ("O", "dq", "dk", "dv", "dstate0", "lengths", "counts", "state0", "dstate") + (() if call == "step" else ("state",)):
        if n in t and (n != "lengths" or call != "attend"):
            t[n] = None
    run(call, t, {n: Gpu(*s, dtype=x) for n, (s, x) in cache().items()})
    assert len(calls) == 1
