"""Linear attention by the gated delta rule (luna_delta_fwd, _step, _bwd) against the recurrence in 64 bits."""
import math

import pytest
import torch

from delta_util import check_backward, check_forward, delta_grads, sums
from gpu_util import say
from paper_2512_08061_amd import luna
from seq_util import U32, assert_norm, device, packed_offsets, rand, unit

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    luna.load_library()
    yield
    torch.cuda.synchronize()


def make(layout, lens, H, Hk, D, d, dtype, seed=0, extra=0, first=0):
    """Q, K (of norm 1), V, dO, log_decay (heads that forget within a token to heads that do not) and beta in [0, 1]."""
    gen = torch.Generator(device=device()).manual_seed(seed)
    if layout == "packed":
        shape = lambda h, w: (first + sum(lens) + extra, h, w)  # noqa: E731
        num = (H, first + sum(lens) + extra)
    else:
        shape = lambda h, w: (len(lens), h, max(lens) + extra, w)  # noqa: E731
        num = (len(lens), H, max(lens) + extra)
    unit_rows = lambda: torch.nn.functional.normalize(rand(shape(Hk, D), torch.float32, gen), dim=-1).to(dtype)  # noqa: E731
    Q, K = unit_rows(), unit_rows()
    V, dO = rand(shape(H, d), dtype, gen), rand(shape(H, d), dtype, gen)
    rate = torch.tensor([2.0 * 4.0 ** -h for h in range(H)], device=device())[:, None]
    g = -rate * rand(num, torch.float32, gen).abs()
    return Q, K, V, dO, g, torch.sigmoid(rand(num, torch.float32, gen)), gen


def kw(layout, lens, first=0, padded=False):
    if layout == "packed":
        return {"offsets": packed_offsets(lens, first)}
    return {"lens": torch.tensor(lens, dtype=torch.int32, device=device())} if padded else {}


def of(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


CASES = [  # layout, lens, H, Hk, D, d, dtype, state
    ("batch", [1], 1, 1, 32, 32, "bf16", False),
    ("batch", [64, 64], 3, 3, 128, 128, "bf16", True),
    ("batch", [65], 2, 1, 64, 64, "bf16", True),
    ("batch", [17], 4, 2, 128, 64, "bf16", True),
    ("batch", [700], 2, 2, 128, 128, "bf16", False),
    ("batch", [300], 1, 1, 32, 128, "bf16", True),
    ("packed", [1, 63, 64, 0, 65, 300], 4, 2, 128, 128, "bf16", True),
    ("packed", [0, 129, 1, 200, 0], 3, 3, 64, 128, "bf16", True),
    ("packed", [130, 31], 6, 2, 64, 32, "bf16", False),
    ("packed", [77, 12], 2, 2, 128, 32, "bf16", False),
    ("batch", [1], 2, 2, 128, 64, "f32", True),
    ("batch", [33], 2, 1, 64, 32, "f32", False),
    ("batch", [200, 200], 2, 2, 128, 128, "f32", True),
    ("packed", [1, 32, 31, 0, 260], 2, 2, 128, 128, "f32", True),
    ("packed", [77, 90], 3, 1, 32, 64, "f32", False),
]


@pytest.mark.parametrize("layout,lens,H,Hk,D,d,dtype,state", CASES)
def test_forward(layout, lens, H, Hk, D, d, dtype, state):
    say(f"delta forward {layout} {lens} H={H} Hk={Hk} D={D} d={d} {dtype} state={state}")
    Q, K, V, _, g, beta, gen = make(layout, lens, H, Hk, D, d, of(dtype))
    S = torch.randn((len(lens), H, D, d), generator=gen, device=device()) if state else None
    S0 = S.clone() if state else None
    scale = D ** -0.5
    out = luna.delta_attn(Q, K, V, g, beta, S=S, scale=scale, **kw(layout, lens))
    check_forward(Q, K, V, g, beta, out, layout, lens, scale, S0, S)


@pytest.mark.parametrize("layout,lens,H,Hk,D,d,dtype,state", CASES)
def test_backward(layout, lens, H, Hk, D, d, dtype, state):
    say(f"delta backward {layout} {lens} H={H} Hk={Hk} D={D} d={d} {dtype}")
    Q, K, V, dO, g, beta, _ = make(layout, lens, H, Hk, D, d, of(dtype), seed=1)
    grads = luna.delta_attn_bwd(Q, K, V, dO, g, beta, scale=D ** -0.5, **kw(layout, lens))
    check_backward(Q, K, V, dO, g, beta, grads, layout, lens, D ** -0.5)


@pytest.mark.parametrize("Hk,D,d,dtype,state", [(32, 128, 128, "bf16", True), (16, 64, 64, "bf16", False), (32, 32, 128, "bf16", False),
                                                (16, 128, 128, "f32", True), (32, 32, 128, "f32", False)])
def test_many_heads(Hk, D, d, dtype, state):
    """Heads and sequences that fill the device, where workgroups take 64 columns of d instead of 32."""
    say(f"delta, many heads: Hk={Hk} D={D} d={d} {dtype} state={state}")
    lens, H = [70, 1, 130, 64, 65], 32
    Q, K, V, dO, g, beta, gen = make("packed", lens, H, Hk, D, d, of(dtype), seed=12)
    S = torch.randn((len(lens), H, D, d), generator=gen, device=device()) if state else None
    S0 = S.clone() if state else None
    out = luna.delta_attn(Q, K, V, g, beta, S=S, scale=D ** -0.5, **kw("packed", lens))
    check_forward(Q, K, V, g, beta, out, "packed", lens, D ** -0.5, S0, S)
    grads = luna.delta_attn_bwd(Q, K, V, dO, g, beta, scale=D ** -0.5, **kw("packed", lens))
    check_backward(Q, K, V, dO, g, beta, grads, "packed", lens, D ** -0.5)


@pytest.mark.parametrize("H,Hk,D,d,dtype,lens", [
    (6, 2, 128, 128, "bf16", [70] * 60), (6, 2, 128, 128, "f32", [70] * 60), (4, 2, 64, 64, "bf16", [3] * 66), (8, 1, 32, 128, "f32", [1] * 250),
    (6, 2, 128, 128, "bf16", [70, 1]), (6, 2, 128, 128, "f32", [70, 0, 1]), (8, 1, 32, 64, "bf16", [65]), (5, 1, 64, 128, "f32", [129, 64])])
def test_gradients_of_shared_heads(H, Hk, D, d, dtype, lens):
    """Value heads one after another in a workgroup, and with few chunks in workgroups of their own, whose sums are joined."""
    say(f"delta backward, shared heads: H={H} Hk={Hk} D={D} d={d} {dtype} {len(lens)} sequences")
    Q, K, V, dO, g, beta, _ = make("packed", lens, H, Hk, D, d, of(dtype), seed=61)
    run = lambda: luna.delta_attn_bwd(Q, K, V, dO, g, beta, scale=D ** -0.5, **kw("packed", lens))  # noqa: E731
    grads = run()
    check_backward(Q, K, V, dO, g, beta, grads, "packed", lens, D ** -0.5)
    assert all(torch.equal(x, y) for x, y in zip(grads, run()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_shared_heads_with_chunks_for_every_unit(dtype):
    """More chunks and key heads than compute units, and value heads in workgroups of their own all the same (260 of a group of 4: 8
    turns one after another, 5 apart)."""
    lens, H, Hk, D, d = [20] * 130, 8, 2, 64, 64
    say(f"delta backward, shared heads, 260 chunks {dtype}")
    Q, K, V, dO, g, beta, _ = make("batch", lens, H, Hk, D, d, of(dtype), seed=63)
    grads = luna.delta_attn_bwd(Q, K, V, dO, g, beta, scale=D ** -0.5)
    check_backward(Q, K, V, dO, g, beta, grads, "batch", lens, D ** -0.5)


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (32, "bf16"), (64, "f32"), (32, "f32")])
def test_equal_lengths_of_more_columns_than_units(D, dtype):
    """320 workgroups of 32 columns of equal sequences (64 columns each then), and the same sequences packed (32)."""
    n, H, d = 70, 8, 64
    for B in (10, 20):  # (both serial passes; the forward one)
        Q, K, V, dO, g, beta, _ = make("batch", [n] * B, H, H, D, d, of(dtype), seed=64)
        say(f"delta, {B} equal sequences D={D} {dtype}")
        out = luna.delta_attn(Q, K, V, g, beta, scale=D ** -0.5)
        grads = luna.delta_attn_bwd(Q, K, V, dO, g, beta, scale=D ** -0.5)
        check_forward(Q, K, V, g, beta, out, "batch", [n] * B, D ** -0.5)
        check_backward(Q, K, V, dO, g, beta, grads, "batch", [n] * B, D ** -0.5)
        flat = lambda t: t.transpose(1, 2).flatten(0, 1).contiguous() if t.dim() == 4 else t.transpose(0, 1).flatten(1).contiguous()  # noqa: E731
        Q, K, V, dO, g, beta = (flat(t) for t in (Q, K, V, dO, g, beta))
        opt = kw("packed", [n] * B)
        check_forward(Q, K, V, g, beta, luna.delta_attn(Q, K, V, g, beta, scale=D ** -0.5, **opt), "packed", [n] * B, D ** -0.5)
        check_backward(Q, K, V, dO, g, beta, luna.delta_attn_bwd(Q, K, V, dO, g, beta, scale=D ** -0.5, **opt), "packed", [n] * B, D ** -0.5)


def test_captured_gradients_of_shared_heads():
    """Sums of value heads that are joined by a second launch: from a graph replayed between eager calls, and over a padded batch."""
    lens, n, H, Hk, D, d = [70, 0, 33], 70, 6, 2, 64, 64
    gen = torch.Generator(device=device()).manual_seed(62)
    Q, K, V, dO, g, beta, _ = make("batch", [n] * 3, H, Hk, D, d, torch.bfloat16, seed=62)
    used = torch.tensor(lens, dtype=torch.int32, device=device())
    call = lambda: luna.delta_attn_bwd(Q, K, V, dO, g, beta, scale=D ** -0.5, lens=used)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call()
    for _ in range(3):
        V.copy_(rand(V.shape, torch.bfloat16, gen))
        for t in outs:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        eager = call()
        assert all(torch.equal(x[i, :, :k], y[i, :, :k]) for x, y in zip(got, eager) for i, k in enumerate(lens))
    single = lambda i, k: [t[i:i + 1, :, :k].contiguous() for t in (Q, K, V, dO, g, beta)]  # noqa: E731
    for i, k in enumerate(lens):
        if k:
            check_backward(*single(i, k), [t[i:i + 1, :, :k] for t in eager], "batch", [k], D ** -0.5)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_not_finite_with_many_heads(bad):
    """The forward call's rules for 64 columns a workgroup: a value's column, a key's and a gate's heads, each from its token on."""
    lens, H, D, d = [100, 140, 30], 32, 64, 128
    Q, K, V, _, g, beta, gen = make("packed", lens, H, H, D, d, torch.bfloat16, seed=13)
    S = torch.randn((len(lens), H, D, d), generator=gen, device=device())
    want, WS = luna.delta_attn(Q, K, V, g, beta, S=(S0 := S.clone()), offsets=packed_offsets(lens)), S0
    V[40, 3, 77], K[100 + 90, 5, 9], g[7, 100 + 20], Q[70, 9, 2] = bad, bad, math.nan, bad
    out = luna.delta_attn(Q, K, V, g, beta, S=S, offsets=packed_offsets(lens))
    lost = torch.zeros(out.shape, dtype=torch.bool, device=device())
    lost[40:100, 3, 77] = lost[190:240, 5] = lost[120:240, 7] = True
    lost[70, 9] = True
    assert torch.isnan(out.float()[lost & (torch.arange(out.shape[0], device=device()) != 70)[:, None, None]]).all()
    assert not torch.isfinite(out[70, 9].float()).any() and torch.equal(out[~lost], want[~lost])
    gone = torch.zeros(S.shape, dtype=torch.bool, device=device())
    gone[0, 3, :, 77] = gone[1, 5] = gone[1, 7] = True
    assert torch.isnan(S[gone]).all() and torch.equal(S[~gone], WS[~gone])


def test_more_sequences_than_lanes():
    gen = torch.Generator(device=device()).manual_seed(14)
    lens = torch.randint(0, 90, (70,), generator=gen, device=device()).tolist()
    lens[33] = 200
    for dtype in (torch.bfloat16, torch.float32):
        Q, K, V, dO, g, beta, _ = make("packed", lens, 2, 1, 32, 64, dtype, seed=15)
        out = luna.delta_attn(Q, K, V, g, beta, offsets=packed_offsets(lens))
        check_forward(Q, K, V, g, beta, out, "packed", lens, 1.0)
        grads = luna.delta_attn_bwd(Q, K, V, dO, g, beta, offsets=packed_offsets(lens))
        check_backward(Q, K, V, dO, g, beta, grads, "packed", lens, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batch_and_packed_gap(dtype):
    """Unused rows hold NaN, in the gates too: they are not read, and what is written keeps what it held there."""
    lens, H, Hk, D, d = [70, 0, 129, 1], 2, 1, 64, 64
    for layout, first, extra in (("batch", 0, 9), ("packed", 5, 9)):
        Q, K, V, dO, g, beta, _ = make(layout, lens, H, Hk, D, d, of(dtype), seed=2, extra=extra, first=first)
        used = torch.zeros(g.shape, dtype=torch.bool, device=device())
        for i, n in enumerate(lens):
            if layout == "batch":
                used[i, :, :n] = True
            else:
                used[:, first + sum(lens[:i]):first + sum(lens[:i + 1])] = True
        rows = used if layout == "batch" else used.t()
        for t in (Q, K, V, dO):
            t[~rows[:, :t.shape[1]]] = math.nan
        g[~used], beta[~used] = math.nan, math.nan
        opt = kw(layout, lens, first, padded=True)
        out = torch.full_like(V, 7.0)
        luna.delta_attn(Q, K, V, g, beta, out=out, **opt)
        check_forward(Q, K, V, g, beta, out, layout, lens, 1.0, first=first)
        grads = [torch.full_like(t, 7.0) for t in (Q, K, V, g, beta)]
        luna.delta_attn_bwd(Q, K, V, dO, g, beta, grads=grads, **opt)
        check_backward(Q, K, V, dO, g, beta, grads, layout, lens, 1.0, first=first)
        for t in [out] + grads[:3]:
            assert (t[~rows[:, :t.shape[1]]] == 7).all()
        assert all((t[~used] == 7).all() for t in grads[3:])
    new = luna.delta_attn_bwd(*(t.transpose(0, 1)[None].contiguous() for t in (Q, K, V, dO)), g[None], beta[None],
                              lens=torch.tensor([3], dtype=torch.int32, device=device()))
    assert all((t[:, :, 3:] == 0).all() for t in new), "unused rows of new gradients"


def test_strides_and_shared_heads():
    """[B, n, H, width] storage, keys and queries that all heads or sequences share, and rows wider than their width."""
    B, n, H, D, d = 2, 150, 4, 64, 128
    gen = torch.Generator(device=device()).manual_seed(3)
    _, _, _, _, g, beta, _ = make("batch", [n] * B, H, H, D, d, torch.bfloat16)
    wide = rand((B, n, H, d + D + 8), torch.bfloat16, gen).transpose(1, 2)
    V, Q = wide[..., :d], 0.1 * wide[..., d:d + D]
    K = torch.nn.functional.normalize(rand((1, 1, n, D), torch.float32, gen), dim=-1).to(torch.bfloat16).expand(B, H, n, D)
    Q = Q.to(torch.bfloat16)
    out = torch.empty((B, n, H, d), dtype=torch.bfloat16, device=device()).transpose(1, 2)
    luna.delta_attn(Q, K, V, g, beta, out=out)
    check_forward(Q, K, V, g, beta, out, "batch", [n] * B, 1.0)
    dO = rand((B, n, H, d), torch.bfloat16, gen).transpose(1, 2)
    grads = luna.delta_attn_bwd(Q, K, V, dO, g, beta, grads=[torch.empty(t.shape, dtype=t.dtype, device=device()) for t in
                                                             (Q, K, V, g, beta)])
    check_backward(Q, K, V, dO, g, beta, grads, "batch", [n] * B, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gates_at_their_ends(dtype):
    """Tokens that forget everything (minus infinity, and a sequence of its own then begins), that forget nothing, log decays above
    0 (counted as 0, without a gradient), beta 0 and 2."""
    n, H, D, d = 200, 2, 64, 64
    Q, K, V, dO, g, beta, gen = make("batch", [n], H, H, D, d, of(dtype), seed=4)
    g[:, :, 40], g[:, :, 100:104] = -math.inf, -1e30
    g[:, 0, 150:] = 0.0
    g[:, 1, 160:170] = 3.0
    beta[:, :, 10:20], beta[:, 0, 30] = 0.0, 2.0
    S = torch.randn((1, H, D, d), generator=gen, device=device())
    S0 = S.clone()
    out = luna.delta_attn(Q, K, V, g, beta, S=S)
    check_forward(Q, K, V, g, beta, out, "batch", [n], 1.0, S0, S)
    grads = luna.delta_attn_bwd(Q, K, V, dO, g, beta)
    check_backward(Q, K, V, dO, g, beta, grads, "batch", [n], 1.0)
    assert (grads[3][:, 1, 160:170] == 0).all()
    tail = [t[:, :, 40:].contiguous() for t in (Q, K, V, g, beta)]
    assert_norm(luna.delta_attn(*tail)[0], out[0, :, 40:], 8 * unit(torch.bfloat16) if dtype == "bf16" else 2 * sums(n, D), "after a reset")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_key_again_and_again(dtype):
    """One key for all tokens with beta near 1 and no decay: each token overwrites what the one before wrote."""
    n, H, D, d = 130, 2, 32, 32
    Q, K, V, dO, g, beta, _ = make("batch", [n], H, H, D, d, of(dtype), seed=5)
    K = K[:, :, :1].expand(1, H, n, D).contiguous()
    g.zero_()
    beta = 1.0 - 0.01 * beta
    out = luna.delta_attn(Q, K, V, g, beta)
    check_forward(Q, K, V, g, beta, out, "batch", [n], 1.0)
    check_backward(Q, K, V, dO, g, beta, luna.delta_attn_bwd(Q, K, V, dO, g, beta), "batch", [n], 1.0)


@pytest.mark.parametrize("B,H,Hk,m,D,d,dtype", [(1, 1, 1, 1, 32, 32, "bf16"), (3, 4, 2, 1, 128, 128, "bf16"), (2, 3, 3, 9, 64, 128, "bf16"),
                                                (2, 2, 1, 4, 128, 32, "f32"), (1, 2, 2, 5, 32, 64, "f32")])
def test_step(B, H, Hk, m, D, d, dtype):
    say(f"delta step B={B} H={H} Hk={Hk} m={m} D={D} d={d} {dtype}")
    Q, K, V, _, g, beta, gen = make("batch", [m] * B, H, Hk, D, d, of(dtype), seed=6)
    S = torch.randn((B, H, D, d), generator=gen, device=device())
    S0 = S.clone()
    out = luna.delta_attn_step(Q, K, V, g, beta, S, scale=D ** -0.5)
    check_forward(Q, K, V, g, beta, out, "batch", [m] * B, D ** -0.5, S0, S)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("B,H,Hk,m,D,d,dtype", [(2, 2, 2, 9, 128, 128, "bf16"), (1, 4, 2, 5, 64, 32, "bf16"), (2, 3, 1, 6, 32, 64, "f32")])
def test_step_with_what_is_not_finite(B, H, Hk, m, D, d, dtype, bad):
    """As in the call over sequences: a value makes its column NaN from its token on, a key or a gate its heads, in out and in S;
    the tokens before, the other columns and heads keep their bits.  A query reaches its own row alone."""
    say(f"delta step, not finite: B={B} H={H} Hk={Hk} m={m} D={D} d={d} {dtype} {bad}")
    Q, K, V, _, g, beta, gen = make("batch", [m] * B, H, Hk, D, d, of(dtype), seed=21)
    S0 = torch.randn((B, H, D, d), generator=gen, device=device())

    def call(q, k, v, gg, b):
        S = S0.clone()
        return luna.delta_attn_step(q, k, v, gg, b, S, scale=D ** -0.5), S

    want, wS = call(Q, K, V, g, beta)
    for at in (0, 4, m - 1):  # (tokens pass through in groups of four)
        v2 = V.clone()
        v2[0, 0, at, 5] = bad
        out, S = call(Q, K, v2, g, beta)
        assert torch.isnan(out[0, 0, at:, 5].float()).all() and torch.isnan(S[0, 0, :, 5]).all()
        out[0, 0, at:, 5], S[0, 0, :, 5] = want[0, 0, at:, 5], wS[0, 0, :, 5]
        assert torch.equal(out, want) and torch.equal(S, wS)
        for which in ("key", "log_decay", "beta"):
            k2, g2, b2 = K.clone(), g.clone(), beta.clone()
            heads = H // Hk if which == "key" else 1  # the value heads that it reaches, the first ones
            if which == "key":
                k2[0, 0, at, D - 3] = bad
            elif which == "log_decay":
                g2[0, 0, at] = math.nan
            else:
                b2[0, 0, at] = bad
            out, S = call(Q, k2, V, g2, b2)
            assert torch.isnan(out[0, :heads, at:].float()).all() and torch.isnan(S[0, :heads]).all(), which
            out[0, :heads, at:], S[0, :heads] = want[0, :heads, at:], wS[0, :heads]
            assert torch.equal(out, want) and torch.equal(S, wS), which
        q2 = Q.clone()
        q2[0, 0, at, 3] = bad
        out, S = call(q2, K, V, g, beta)
        assert not torch.isfinite(out[0, :H // Hk, at].float()).any()
        out[0, :H // Hk, at] = want[0, :H // Hk, at]
        assert torch.equal(out, want) and torch.equal(S, wS)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_then_steps_is_the_whole_sequence(dtype):
    n, cut, H, Hk, D, d = 140, 101, 4, 2, 64, 64
    Q, K, V, _, g, beta, _ = make("batch", [n], H, Hk, D, d, of(dtype), seed=7)
    S = torch.zeros((1, H, D, d), device=device())
    part = lambda a, b: [t[:, :, a:b].contiguous() for t in (Q, K, V, g, beta)]  # noqa: E731
    outs = [luna.delta_attn(*part(0, 70), S=S), luna.delta_attn(*part(70, cut), S=S)]
    outs += [luna.delta_attn_step(*part(t, t + 3), S) for t in range(cut, n, 3)]
    check_forward(Q, K, V, g, beta, torch.cat(outs, 2), "batch", [n], 1.0, None, S)


@pytest.mark.parametrize("H,Hk", [(2, 2), (4, 2)])
def test_backward_against_differences(H, Hk):
    """Central differences of the fp32 forward call along random directions of each input.  out is within sums(n, D) of its norm, so
    that a difference over 2 h is within sums |out| |dO| / h; the cubic term is below h of the directions' size here."""
    n, D, d, h = 90, 32, 32, 1e-2
    Q, K, V, dO, g, beta, gen = make("batch", [n], H, Hk, D, d, torch.float32, seed=8)
    g = g - 0.1  # (away from the border at 0)
    ins = [Q, K, V, g, beta]
    grads = luna.delta_attn_bwd(Q, K, V, dO, g, beta)
    loss = lambda x: (luna.delta_attn(*x).double() * dO.double()).sum().item()  # noqa: E731
    noise = sums(n, D) * luna.delta_attn(*ins).double().norm().item() * dO.double().norm().item()
    for i, grad in enumerate(grads):
        way = rand(grad.shape, torch.float32, gen)
        way *= 0.02 if i < 2 else 0.1
        at = lambda s: loss([t + s * way if j == i else t for j, t in enumerate(ins)])  # noqa: E731
        diff, want = (at(h) - at(-h)) / (2 * h), (grad.double() * way.double()).sum().item()
        size = grad.double().norm().item() * way.double().norm().item()
        assert abs(diff - want) <= noise / h + h * size, (i, diff, want)


def test_same_bits_streams_and_graph():
    """The same call gives the same bits, on a stream of its own and from a captured graph replayed with other work between."""
    lens, H, Hk, D, d = [70, 1, 300, 64], 4, 2, 128, 128
    Q, K, V, dO, g, beta, gen = make("packed", lens, H, Hk, D, d, torch.bfloat16, seed=9)
    S0 = torch.randn((len(lens), H, D, d), generator=gen, device=device())
    S, opt = S0.clone(), kw("packed", lens)
    tok = [t[None, :, :2].contiguous() for t in (Q.transpose(0, 1), K.transpose(0, 1), V.transpose(0, 1), g, beta)]

    def call():
        return (luna.delta_attn(Q, K, V, g, beta, S=S, **opt), luna.delta_attn_step(*tok, S[:1]),
                *luna.delta_attn_bwd(Q, K, V, dO, g, beta, **opt))

    want = [t.clone() for t in call()] + [S.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        S.copy_(S0)
        got = call()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(list(got) + [S], want))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(3):
        S.copy_(S0)
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(list(got) + [S], want))


def test_two_graphs_and_an_eager_call():
    """Two captured backward passes of different inputs and eager calls between their replays do not share workspaces."""
    made = [make("batch", [n], 2, 2, 64, 64, torch.bfloat16, seed=s)[:6] for n, s in ((130, 10), (200, 11), (90, 12))]
    call = lambda Q, K, V, dO, g, b: luna.delta_attn_bwd(Q, K, V, dO, g, b) + (luna.delta_attn(Q, K, V, g, b),)  # noqa: E731
    want = [[t.clone() for t in call(*x)] for x in made]
    torch.cuda.synchronize()
    graphs, got = [], []
    for x in made[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(call(*x))
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        eager = call(*made[2])
        torch.cuda.synchronize()
        for a, b in zip(got + [eager], want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("H,Hk,D,d,dtype,lens", [(2, 2, 128, 128, "bf16", [300, 65]), (4, 2, 64, 32, "bf16", [90]),
                                                 (2, 1, 64, 64, "f32", [100, 33])])
@pytest.mark.parametrize("bad", [math.nan, -math.inf])
def test_later_tokens_do_not_reach_earlier_rows(H, Hk, D, d, dtype, lens, bad):
    """Values that are not finite from one token on (in some columns), a key, a gate: rows before, and columns without, are as
    without them; the others are NaN, and so is the state.  A query reaches its own row alone."""
    say(f"later tokens, delta: H={H} D={D} d={d} {dtype} {lens} {bad}")
    Q, K, V, _, g, beta, _ = make("batch", lens, H, Hk, D, d, of(dtype), seed=13)
    B, opt = len(lens), kw("batch", lens, padded=True)

    def call(q, k, v, gg, b):
        S = torch.zeros((B, H, D, d), device=device())
        return luna.delta_attn(q, k, v, gg, b, S=S, **opt), S

    want, wS = call(Q, K, V, g, beta)
    first, key = [x // 3 for x in lens], [x - 3 for x in lens]
    V2 = V.clone()
    for i in range(B):
        V2[i, :, first[i]:, 1::4] = bad
    out, S = call(Q, K, V2, g, beta)
    for i in range(B):
        a, m = first[i], lens[i]
        assert torch.equal(out[i, :, :a], want[i, :, :a]), "rows before"
        for c in (0, 2, 3):
            assert torch.equal(out[i, :, a:m, c::4], want[i, :, a:m, c::4]), "columns without"
            assert torch.equal(S[i, :, :, c::4], wS[i, :, :, c::4])
        assert torch.isnan(out[i, :, a:m, 1::4].float()).all() and torch.isnan(S[i, :, :, 1::4]).all()
    for which in ("key", "log_decay", "beta"):
        k2, g2, b2 = K.clone(), g.clone(), beta.clone()
        heads = range(H // Hk) if which == "key" else [0]  # the value heads that it reaches
        for i in range(B):
            if which == "key":
                k2[i, 0, key[i], 5] = bad
            elif which == "log_decay":
                g2[i, 0, key[i]] = math.nan
            else:
                b2[i, 0, key[i]] = bad
        out, S = call(Q, k2, V, g2, b2)
        for i in range(B):
            assert torch.equal(out[i, :, :key[i]], want[i, :, :key[i]]), which
            for h in range(H):
                if h in heads:
                    assert torch.isnan(out[i, h, key[i]:lens[i]].float()).all() and torch.isnan(S[i, h]).all(), which
                else:
                    assert torch.equal(out[i, h], want[i, h]) and torch.equal(S[i, h], wS[i, h]), which
    q2 = Q.clone()
    for i in range(B):
        q2[i, 0, first[i], 3] = bad
    out, S = call(q2, K, V, g, beta)
    keep = torch.ones(out.shape[:3], dtype=torch.bool, device=device())
    for i in range(B):
        keep[i, :H // Hk, first[i]] = False
        assert not torch.isfinite(out[i, :H // Hk, first[i]].float()).any()
    assert torch.equal(out[keep], want[keep]) and torch.equal(S, wS)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_finite_stays_in_its_sequence(dtype):
    """One sequence's second key head with NaN everywhere: rows, states and gradients of the others are the same bits."""
    lens, first, H, Hk, D, d = [70, 130, 5, 200], 3, 4, 2, 64, 64
    Q, K, V, dO, g, beta, _ = make("packed", lens, H, Hk, D, d, of(dtype), seed=14, first=first, extra=9)
    opt = kw("packed", lens, first)

    def call():
        S = torch.zeros((len(lens), H, D, d), device=device())
        rows = [luna.delta_attn(Q, K, V, g, beta, S=S, **opt), *luna.delta_attn_bwd(Q, K, V, dO, g, beta, **opt)]
        rows[4:] = [t.t() for t in rows[4:]]
        return rows, S

    want, wS = call()
    a, b, T = first + 70, first + 200, first + sum(lens)
    for t in (Q, K, V, dO):
        t[a:b, t.shape[1] // 2:] = math.nan
    got, gS = call()
    for x, y in zip(got, want):
        h = x.shape[1] // 2
        assert torch.equal(x[first:a], y[first:a]) and torch.equal(x[b:T], y[b:T]) and torch.equal(x[a:b, :h], y[a:b, :h])
    assert torch.equal(gS[[0, 2, 3]], wS[[0, 2, 3]]) and torch.equal(gS[1, :2], wS[1, :2])


def test_many_packed_sequences():
    """Packed sequences by the thousand, empty ones among them: the same bits as the padded batch of the same rows."""
    count, H, Hk, D, d, most = 4500, 2, 1, 32, 32, 70
    gen = torch.Generator(device=device()).manual_seed(15)
    lens = torch.randint(0, 6, (count,), generator=gen, device=device(), dtype=torch.int32)
    lens[::61], lens[count // 2] = 0, most
    off = torch.cat([torch.zeros(1, dtype=torch.int32, device=device()), lens.cumsum(0).int()])
    pad = make("batch", [most] * count, H, Hk, D, d, torch.bfloat16, seed=16)[:6]
    used = torch.arange(most, device=device())[None, :] < lens[:, None]
    rows = lambda t: (t.transpose(1, 2)[used].contiguous() if t.dim() == 4 else t.transpose(1, 2)[used].t().contiguous())  # noqa: E731
    own = [rows(t) for t in pad]

    def call(Q, K, V, dO, g, b, **opt):
        S = torch.ones((count, H, D, d), device=device())
        return [luna.delta_attn(Q, K, V, g, b, S=S, **opt), *luna.delta_attn_bwd(Q, K, V, dO, g, b, **opt)], S

    got, S = call(*own, offsets=off)
    want, wS = call(*pad, lens=lens)
    for x, y in zip(got, want):
        assert torch.equal(x, rows(y))
    assert torch.equal(S, wS) and (S[lens == 0] == 1).all()


def test_offsets_beyond_32_bits():
    """Heads and sequences that lie more than 2^31 bytes apart."""
    n, H, D, d = 100, 2, 64, 64
    Q, K, V, dO, g, beta, _ = make("batch", [n, n], H, H, D, d, torch.bfloat16, seed=17)
    store = torch.empty(7 << 29, dtype=torch.bfloat16, device=device())  # 7 GiB
    far = lambda: torch.as_strided(store, (2, H, n, d), ((1 << 31) + (1 << 28), 1 << 30, d, 1))  # noqa: E731
    far().copy_(V)
    out = luna.delta_attn(Q, K, far(), g, beta)
    assert torch.equal(out, luna.delta_attn(Q, K, V, g, beta))
    luna.delta_attn(Q, K, V, g, beta, out=far())
    assert torch.equal(far(), out)


def test_empty_calls():
    dev = device()
    S = torch.randn((2, 2, 64, 32), device=dev)
    S0 = S.clone()
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=dev)  # noqa: E731
    n = torch.zeros((2, 0), device=dev)
    off = torch.zeros(3, dtype=torch.int32, device=dev)
    out = luna.delta_attn(z(0, 1, 64), z(0, 1, 64), z(0, 2, 32), n, n, S=S, offsets=off)
    assert out.shape == (0, 2, 32) and torch.equal(S, S0)
    assert [t.numel() for t in luna.delta_attn_bwd(z(0, 1, 64), z(0, 1, 64), z(0, 2, 32), z(0, 2, 32), n, n, offsets=off)] == [0] * 5
    n = torch.zeros((2, 2, 0), device=dev)
    luna.delta_attn(z(2, 1, 0, 64), z(2, 1, 0, 64), z(2, 2, 0, 32), n, n, S=S)
    assert torch.equal(S, S0)
