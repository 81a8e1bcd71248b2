"""The sequence operators (include/luna_seq.h) at the ends of what they take: values, sizes and forms of a call that
choose between kernels."""
import pytest
import torch

from gpu_util import say
from paper_2512_08061_amd import luna
from seq_util import device, rand, unit

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    luna.load_library()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("H,Hk,d,dtype", [(2, 2, 64, "bf16"), (4, 2, 128, "bf16"), (2, 1, 32, "bf16"), (2, 1, 64, "f32")])
@pytest.mark.parametrize("size", [1000.0, 5000.0])
def test_gradients_of_very_large_scores(H, Hk, d, dtype, size):
    """Scores of 10^6 to 5 10^8, of which fp32 sums and lse hold 2^-24: a weight may come out too small, but none is above 1,
    so that gradients stay below the sums over weights of 1 (four roundings: P, dS, out and the result)."""
    say(f"very large scores: H={H} d={d} {dtype} {size}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device=device()).manual_seed(21)
    n, group, scale = 300, H // Hk, d ** -0.5
    K, V = (rand((1, Hk, n, d), dt, gen) for _ in range(2))
    K = (size * K.float()).to(dt)
    Q = K.repeat_interleave(group, 1)  # (the largest score of a row is mostly its own token's)
    dO = rand(Q.shape, dt, gen)
    out, lse = luna.softmax_attn(Q, K, V)
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all() and lse.max() > 1e5
    grads = luna.softmax_attn_bwd(Q, K, V, out, lse, dO)
    q, k, v, g, o = (t[0].double().abs() for t in (Q, K, V, dO, out))
    k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    seen = torch.ones((n, n), dtype=torch.float64, device=device()).tril()
    size_s = scale * seen * (g @ v.transpose(-1, -2).contiguous() + (g * o).sum(-1, keepdim=True))
    shared = lambda x: x.reshape(Hk, group, n, d).sum(1)  # noqa: E731
    most = (size_s @ k, shared(size_s.transpose(-1, -2).contiguous() @ q), shared(seen.t().contiguous() @ g))
    for got, bound, name in zip(grads, most, ("dQ", "dK", "dV")):
        assert torch.isfinite(got.float()).all(), name
        over = (got[0].double().abs() / bound).max().item()
        assert over <= 1 + 4 * unit(torch.bfloat16), f"{name}: {over} of the sum over weights of 1"
