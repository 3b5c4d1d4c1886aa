"""The operators that keep a history, several at once: on streams of their own beside each other and beside the fused pass, and as
captured graphs that are replayed together.  None of them has a workspace; every result has to equal, bit for bit, that of the
call made alone."""
import pytest
import torch

from paper_2603_02561_b200 import solar

pytestmark = pytest.mark.gpu
BF, E4, I32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32


def calls(d, seed):
    """Closures over inputs and outputs of their own, and those outputs."""
    g = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g).to(BF).cuda()  # noqa: E731
    B, H, Hq, N, T = 3, 2, 4, 2112, 1300
    k, v, q, one, do = rn(B, T, H, d), rn(B, T, H, d), rn(B, T, Hq, d), rn(B, 1, Hq, d), rn(B, T, H, d)
    ld = torch.tensor([-0.01, -0.3], device="cuda")
    s0 = torch.randn(B, H, d, d, generator=g).cuda()
    cache = solar.history_cache(B, H, N, d)
    held = solar.history_cache(B, H, N, d)
    start = torch.tensor([100, 63, 0], dtype=I32, device="cuda")
    for x in (*cache[:2], *held[:2]):
        x.copy_(torch.randn(x.shape, generator=g).to(E4))
    for x in (*cache[2:], *held[2:]):
        x.fill_(0.25)
    state = s0.clone()
    n = torch.full((B,), N, dtype=I32, device="cuda")
    lens = start + T
    Hx, C = rn(4, 2000, d) / 8, rn(4, 300, d) / 8
    W = [rn(d, d) / 8 for _ in range(3)]
    ws = solar.alloc_fused_workspace(4, 300, 2000, d, 16, BF)
    out = {"many": torch.empty_like(q), "few": torch.empty_like(one), "O": torch.empty_like(k), "S": torch.empty_like(s0), "dq": torch.empty_like(k),
           "dk": torch.empty_like(k), "dv": torch.empty_like(k), "ds": torch.empty_like(s0), "o1": torch.empty_like(k[:, 0]), "state": state,
           "k8": cache.k.view(torch.uint8), "v8": cache.v.view(torch.uint8), "ks": cache.k_scale, "own": torch.empty_like(C)}
    sv = torch.empty(4, 16, device="cuda"), torch.empty(4, d, 16, device="cuda"), torch.zeros(4, dtype=I32, device="cuda")

    def serve():
        solar.history_cache_append(k, v, cache, start)
        solar.history_cache_attention(q, cache, lens, 0.1, flags=solar.FLAG_CAUSAL, O=out["many"])

    def ask():
        solar.history_cache_attention(one, held, n, 0.1, O=out["few"])

    def linear():
        solar.linear_attention_fwd(k, k, v, ld, 0.1, state0=s0, O=out["O"], state=out["S"])
        solar.linear_attention_bwd(k, k, v, ld, 0.1, do, state0=s0, dq=out["dq"], dk=out["dk"], dv=out["dv"], dstate0=out["ds"])

    def step():
        state.copy_(s0)
        solar.linear_attention_step(k[:, 0], k[:, 1], v[:, 2], ld, 0.1, state, O=out["o1"])

    def fused():
        solar.svd_attention_fused(Hx, C, *W, 16, 0.1, S=sv[0], V=sv[1], O=out["own"], info=sv[2], workspace=ws)
    return [serve, ask, linear, step, fused], out, sv[2]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("graphs", [False, True])
def test_at_once(d, graphs):
    lanes = [calls(d, seed) for seed in range(3)]
    want = []
    for todo, out, _ in lanes:
        for call in todo:
            call()
            torch.cuda.synchronize()
        want.append({n: x.clone() for n, x in out.items()})
    todo = [call for lane in lanes for call in lane[0]]
    streams = [torch.cuda.Stream() for _ in todo]
    made = []
    if graphs:
        for call in todo:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                call()
            made.append(g)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, call, i in zip(streams, todo, range(len(todo))):
            with torch.cuda.stream(s):
                made[i].replay() if graphs else call()
    torch.cuda.synchronize()
    for (_, out, info), w in zip(lanes, want):
        assert (info == 0).all()
        for name, x in out.items():
            assert torch.equal(x.view(torch.uint8), w[name].view(torch.uint8)), name
