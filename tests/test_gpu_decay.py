"""Linear attention with a decay for each head (luna_decay_fwd, _step, _bwd) against plain 64-bit forms."""
import math

import pytest
import torch

from gpu_util import say
from paper_2512_08061_amd import luna
from seq_util import (U32, assert_norm, assert_within, cut, cut_num, decay_grads, decay_ref, device, packed_offsets, rand,
                      unit)

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    luna.load_library()
    yield
    torch.cuda.synchronize()


def decays(H):
    """Factors from a half per token to none."""
    return torch.tensor([-(0.7 * 4.0 ** -h) if h < 6 else 0.0 for h in range(H)], device=device())


def make(layout, lens, H, D, d, dtype, norm, seed=0, extra=0, first=0):
    gen = torch.Generator(device=device()).manual_seed(seed)
    if layout == "packed":
        shape = lambda w: (first + sum(lens) + extra, H, w)  # noqa: E731
    else:
        shape = lambda w: (len(lens), H, max(lens) + extra, w)  # noqa: E731
    Q, K = (rand(shape(D), dtype, gen, norm) for _ in range(2))
    return Q, K, rand(shape(d), dtype, gen), gen


def kw(layout, lens, first=0, padded=False):
    if layout == "packed":
        return {"offsets": packed_offsets(lens, first)}
    return {"lens": torch.tensor(lens, dtype=torch.int32, device=device())} if padded else {}


def check_forward(Q, K, V, g, out, den, layout, lens, norm, scale, S0=None, z0=None, S=None, z=None, first=0, what=""):
    """bf16: weights, state, (without a returned state) discounted values and out are rounded to U each; fp32
    sums of n + D terms.  The norm of independent roundings stays below a plain sum of four."""
    u = unit(out.dtype) if out.dtype == torch.bfloat16 else 0.0
    for i, n in enumerate(lens):
        q, k, v = (cut(t, layout, lens, i, first) for t in (Q, K, V))
        s0 = None if S0 is None else S0[i].double()
        zz = None if z0 is None else z0[i].double()
        ref, rden, rS, rz = decay_ref(q, k, v, g, s0, zz, norm, scale, EPS)
        size, dsize, sS, sz = decay_ref(q.abs(), k.abs(), v.abs(), g, None if s0 is None else s0.abs(),
                                        None if zz is None else zz.abs(), False, abs(scale), EPS)
        sums = (n + Q.shape[-1] + 16) * U32
        got = cut(out, layout, lens, i, first)
        w = 1.0 / (rden + EPS)[..., None] if norm else 1.0
        bound = (3 * u + (2 if norm else 1) * sums) * size * w + u * ref.abs()
        if norm and n:
            bound = bound + sums * dsize[..., None] * w * ref.abs()
        assert_within(got, ref, bound + 1e-30, f"{what} out[{i}]")
        assert_norm(got, ref, 4 * u + 8 * math.sqrt(n + Q.shape[-1]) * U32 * (4 if norm else 8), f"{what} out[{i}]")
        if norm and den is not None:
            assert_within(cut_num(den, layout, lens, i, first), rden, sums * dsize + 1e-30, f"{what} den[{i}]")
        if S is not None:
            assert_within(S[i], rS, (n + 16) * U32 * sS + 1e-30, f"{what} S[{i}]")
            if norm:
                assert_within(z[i], rz, (n + 16) * U32 * sz + 1e-30, f"{what} z[{i}]")


CASES = [  # layout, lens, H, D, d, dtype, norm, state
    ("batch", [1], 1, 32, 32, "bf16", False, False),
    ("batch", [64, 64], 3, 128, 128, "bf16", False, True),
    ("batch", [65], 2, 64, 64, "bf16", True, True),
    ("batch", [300, 300], 2, 256, 128, "bf16", True, True),
    ("batch", [517], 1, 256, 64, "bf16", False, True),
    ("batch", [1999], 2, 128, 128, "bf16", False, True),
    ("batch", [1100], 2, 32, 128, "bf16", True, False),
    ("packed", [1, 63, 64, 0, 65, 700], 2, 128, 128, "bf16", False, True),
    ("packed", [0, 257, 1, 513, 0], 3, 64, 128, "bf16", True, True),
    ("packed", [30, 1300], 1, 256, 128, "bf16", True, False),
    ("packed", [129, 31], 5, 32, 32, "bf16", False, False),
    ("batch", [1], 2, 128, 64, "f32", True, True),
    ("batch", [33], 2, 64, 32, "f32", False, True),
    ("batch", [700], 2, 128, 128, "f32", False, True),
    ("packed", [1, 32, 31, 0, 600], 2, 256, 128, "f32", True, True),
    ("packed", [77, 290], 3, 32, 64, "f32", False, False),
]


@pytest.mark.parametrize("layout,lens,H,D,d,dtype,norm,state", CASES)
def test_forward(layout, lens, H, D, d, dtype, norm, state):
    say(f"decay forward {layout} {lens} H={H} D={D} d={d} {dtype} norm={norm} state={state}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    Q, K, V, gen = make(layout, lens, H, D, d, dt, norm)
    g, S, z, S0, z0 = decays(H), None, None, None, None
    if state:
        S = torch.randn((len(lens), H, D, d), generator=gen, device=device())
        S0 = S.clone()
        if norm:
            z = torch.rand((len(lens), H, D), generator=gen, device=device()) + 1.0
            z0 = z.clone()
    scale = 1.0 / math.sqrt(D)
    out, den = luna.decay_attn(Q, K, V, g, S=S, z=z, normalize=norm, scale=scale, eps=EPS, **kw(layout, lens))
    check_forward(Q, K, V, g, out, den, layout, lens, norm, scale, S0, z0, S, z)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batch_and_packed_gap(dtype):
    """Unused rows hold NaN: they are not read, and out keeps what it held there."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    lens, H, D, d = [70, 0, 129, 1], 2, 64, 64
    Q, K, V, _ = make("batch", lens, H, D, d, dt, True, extra=9)
    for t in (Q, K, V):
        for i, n in enumerate(lens):
            t[i, :, n:] = float("nan")
    out = torch.full_like(V, 7.0)
    luna.decay_attn(Q, K, V, decays(H), normalize=True, eps=EPS, out=out, **kw("batch", lens, padded=True))
    check_forward(Q, K, V, decays(H), out, None, "batch", lens, True, 1.0)
    assert all((out[i, :, n:] == 7.0).all() for i, n in enumerate(lens))
    Q, K, V, _ = make("packed", lens, H, D, d, dt, True, extra=9, first=5)
    for t in (Q, K, V):
        t[:5] = float("nan")
        t[5 + sum(lens):] = float("nan")
    out = torch.full_like(V, 7.0)
    luna.decay_attn(Q, K, V, decays(H), normalize=True, eps=EPS, out=out, **kw("packed", lens, 5))
    check_forward(Q, K, V, decays(H), out, None, "packed", lens, True, 1.0, first=5)
    assert (out[:5] == 7.0).all() and (out[5 + sum(lens):] == 7.0).all()


def test_strides_and_shared_heads():
    """Slices of one projection [T, 2 H D + H d], a [B, n, H, *] batch, and keys that all heads share."""
    gen = torch.Generator(device=device()).manual_seed(3)
    lens, H, D, d = [100, 31], 3, 64, 64
    x = rand((131, H * (2 * D + d)), torch.bfloat16, gen)
    Q, K, V = (x[:, a:b].unflatten(1, (H, -1)) for a, b in ((0, H * D), (H * D, 2 * H * D), (2 * H * D, H * (2 * D + d))))
    g = decays(H)
    out, _ = luna.decay_attn(Q, K, V, g, scale=0.125, **kw("packed", lens))
    check_forward(Q, K, V, g, out, None, "packed", lens, False, 0.125)
    Q, K, V = (rand((2, 200, H, w), torch.bfloat16, gen).transpose(1, 2) for w in (D, D, d))
    K = K[:, :1].expand(-1, H, -1, -1)
    out, _ = luna.decay_attn(Q, K, V, g, scale=0.125)
    check_forward(Q, K, V, g, out, None, "batch", [200, 200], False, 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_factors_at_their_ends(dtype):
    """No decay, none remembered (-infinity), nearly none, and above 0 (counts as 0)."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.tensor([0.0, -math.inf, -200.0, -1e-6, 0.5], device=device())
    Q, K, V, gen = make("batch", [400], 5, 64, 64, dt, True)
    S = torch.randn((1, 5, 64, 64), generator=gen, device=device())
    z = torch.rand((1, 5, 64), generator=gen, device=device()) + 1.0
    S0, z0 = S.clone(), z.clone()
    out, den = luna.decay_attn(Q, K, V, g, S=S, z=z, normalize=True, eps=EPS)
    check_forward(Q, K, V, g, out, den, "batch", [400], True, 1.0, S0, z0, S, z)
    S, z = S0.clone(), z0.clone()
    o1 = luna.decay_attn_step(Q[:, :, :1], K[:, :, :1], V[:, :, :1], g, S, z, normalize=True, eps=EPS)
    check_forward(Q[:, :, :1], K[:, :, :1], V[:, :, :1], g, o1, None, "batch", [1], True, 1.0, S0, z0, S, z)


def test_empty_calls():
    z3 = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=device())  # noqa: E731
    S = torch.ones((2, 1, 32, 32), device=device())
    out, _ = luna.decay_attn(z3(0, 1, 32), z3(0, 1, 32), z3(0, 1, 32), decays(1), S=S, offsets=packed_offsets([0, 0]))
    assert out.shape == (0, 1, 32) and (S == 1).all()
    g = luna.decay_attn_bwd(z3(0, 1, 32), z3(0, 1, 32), z3(0, 1, 32), z3(0, 1, 32), decays(1), offsets=packed_offsets([0]))
    assert all(t.shape[0] == 0 for t in g)


@pytest.mark.parametrize("B,H,m,D,d,dtype,norm", [
    (1, 1, 1, 32, 32, "bf16", False), (3, 2, 1, 128, 128, "bf16", False), (2, 3, 5, 256, 128, "bf16", True),
    (2, 2, 9, 64, 64, "bf16", True), (1, 2, 4, 128, 32, "f32", True), (5, 1, 1, 256, 64, "f32", False),
    (1, 3, 17, 32, 128, "f32", True)])
def test_step(B, H, m, D, d, dtype, norm):
    say(f"decay step B={B} H={H} m={m} D={D} d={d} {dtype} norm={norm}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    Q, K, V, gen = make("batch", [m] * B, H, D, d, dt, norm)
    S = torch.randn((B, H, D, d), generator=gen, device=device())
    z = torch.rand((B, H, D), generator=gen, device=device()) + 1.0 if norm else None
    S0, z0 = S.clone(), z.clone() if norm else None
    g = decays(H)
    out = luna.decay_attn_step(Q, K, V, g, S, z, normalize=norm, scale=0.5, eps=EPS)
    check_forward(Q, K, V, g, out, None, "batch", [m] * B, norm, 0.5, S0, z0, S, z)


def test_prompt_then_steps_is_the_whole_sequence():
    """Prefill, a further chunk from its state and single tokens against one call over all of them."""
    H, D, d, n = 2, 128, 64, 400
    Q, K, V, _ = make("batch", [n, n], H, D, d, torch.float32, True)
    g = decays(H)
    S, z = torch.zeros((2, H, D, d), device=device()), torch.zeros((2, H, D), device=device())
    parts = [luna.decay_attn(*(t[:, :, a:b] for t in (Q, K, V)), g, S=S, z=z, normalize=True, eps=EPS)[0]
             for a, b in ((0, 290), (290, 395))]
    parts += [luna.decay_attn_step(*(t[:, :, a:a + 1] for t in (Q, K, V)), g, S, z, normalize=True, eps=EPS)
              for a in range(395, n)]
    check_forward(Q, K, V, g, torch.cat(parts, 2), None, "batch", [n, n], True, 1.0, S=S, z=z)


BWD = [("batch", [1], 1, 32, 32, "bf16", False), ("batch", [130, 130], 2, 128, 128, "bf16", False),
       ("batch", [600], 2, 256, 128, "bf16", True), ("packed", [65, 0, 1, 300], 2, 64, 64, "bf16", True),
       ("packed", [700, 3], 1, 128, 64, "bf16", False), ("batch", [333], 3, 64, 64, "f32", True),
       ("packed", [40, 290, 1], 2, 256, 128, "f32", True), ("batch", [90], 2, 32, 64, "f32", False)]


@pytest.mark.parametrize("layout,lens,H,D,d,dtype,norm", BWD)
def test_backward(layout, lens, H, D, d, dtype, norm):
    """As the forward pass, four roundings of operands and terms (the row's dO.out from the rounded out among
    them), one of the result."""
    say(f"decay backward {layout} {lens} H={H} D={D} d={d} {dtype} norm={norm}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    Q, K, V, gen = make(layout, lens, H, D, d, dt, norm)
    dO = rand(V.shape, dt, gen)
    g, k = decays(H), kw(layout, lens)
    scale = 1.0 / math.sqrt(D)
    out, den = luna.decay_attn(Q, K, V, g, normalize=norm, scale=scale, eps=EPS, **k)
    grads = luna.decay_attn_bwd(Q, K, V, dO, g, out=out, den=den, normalize=norm, scale=scale, eps=EPS, **k)
    u = unit(dt) if dt == torch.bfloat16 else 0.0
    for i, n in enumerate(lens):
        refs, sizes = decay_grads(*(cut(t, layout, lens, i) for t in (Q, K, V, dO)), g, norm, scale, EPS)
        for got, ref, size, name in zip(grads, refs, sizes, ("dQ", "dK", "dV")):
            sums = (2 * n + D + d + 32) * U32 * (4 if norm else 1)
            assert_within(cut(got, layout, lens, i), ref, (5 * u + sums) * size + u * ref.abs() + 1e-30, f"{name}[{i}]")
            if n > 1:
                assert_norm(cut(got, layout, lens, i), ref, 8 * u + 32 * math.sqrt(2 * n + D + d) * U32, f"{name}[{i}]")


def test_backward_against_differences():
    """fp32 gradients against central differences of the 64-bit form along random directions."""
    Q, K, V, gen = make("batch", [50], 2, 32, 32, torch.float32, True)
    dO = rand(V.shape, torch.float32, gen)
    g = decays(2)
    out, den = luna.decay_attn(Q, K, V, g, normalize=True, eps=EPS)
    grads = luna.decay_attn_bwd(Q, K, V, dO, g, out=out, den=den, normalize=True, eps=EPS)
    x = [t[0].double() for t in (Q, K, V)]
    for i, name in enumerate("QKV"):
        u = torch.randn(x[i].shape, generator=gen, device=device(), dtype=torch.float64)
        h = 1e-5
        f = lambda s: (decay_ref(*[t + s * h * u if j == i else t for j, t in enumerate(x)], g, normalize=True,  # noqa: E731
                                 eps=EPS)[0] * dO[0].double()).sum()
        want = ((f(1) - f(-1)) / (2 * h)).item()
        got = (grads[i][0].double() * u).sum().item()
        size = (grads[i][0].double() * u).abs().sum().item()
        assert abs(got - want) <= 1e-5 * size + 1e-6, (name, got, want)  # (differences: h^2 and 1e-16 / h of the sum)


def test_same_bits_streams_and_graph():
    """Two calls, a call on another stream and replays of a captured call give the same bits."""
    H, D, d, lens = 2, 128, 128, [300, 1, 700]
    Q, K, V, gen = make("packed", lens, H, D, d, torch.bfloat16, True)
    dO, g, k = rand(V.shape, torch.bfloat16, gen), decays(H), kw("packed", lens)

    def call(S, z):
        out, den = luna.decay_attn(Q, K, V, g, S=S, z=z, normalize=True, eps=EPS, **k)
        return (out, den) + luna.decay_attn_bwd(Q, K, V, dO, g, out=out, den=den, normalize=True, eps=EPS, **k)

    S0 = torch.randn((3, H, D, d), generator=gen, device=device())
    z0 = torch.rand((3, H, D), generator=gen, device=device()) + 1.0
    S, z = S0.clone(), z0.clone()
    want = call(S, z) + (S, z)
    S1, z1 = S0.clone(), z0.clone()
    assert all(torch.equal(a, b) for a, b in zip(call(S1, z1) + (S1, z1), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        S1, z1 = S0.clone(), z0.clone()
        got = call(S1, z1) + (S1, z1)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    S1, z1 = S0.clone(), z0.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = call(S1, z1)
        step = luna.decay_attn_step(*(t[:1].transpose(0, 1)[None] for t in (Q, K, V)), g, S1[:1], z1[:1], normalize=True, eps=EPS)
    for _ in range(3):
        S1.copy_(S0)
        z1.copy_(z0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[:5]))
        S2, z2 = S[:1].clone(), z[:1].clone()
        again = luna.decay_attn_step(*(t[:1].transpose(0, 1)[None] for t in (Q, K, V)), g, S2, z2, normalize=True, eps=EPS)
        assert torch.equal(step, again) and torch.equal(S1[:1], S2) and torch.equal(S1[1:], S[1:])
