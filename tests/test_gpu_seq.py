"""The sequence operators (include/luna_seq.h) together, as a hybrid decoder uses them: learned features, linear
attention with decay and softmax attention over the same sequences, in training and in serving."""
import math

import pytest
import torch

from gpu_util import say
from paper_2512_08061_amd import luna
from paper_2512_08061_amd import workloads as wl
from seq_util import cut, decay_grads, device, packed_offsets, rand, assert_within, softmax_ref, unit, U32
from test_gpu_decay import EPS, check_forward as check_decay, decays
from test_gpu_softmax import check_backward, check_forward as check_softmax

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    luna.load_library()
    yield
    torch.cuda.synchronize()


def features(d, M=16, L=8):
    return luna.PhiVariant.from_arrays(wl.make_variant_params("mlp", M, d, L=L, hidden=16), device(), torch.bfloat16)


def packed_features(x, v):
    """The features of packed rows [T, H, d], as a strided [T, H, D] view."""
    return luna.featuremap_variant(x.transpose(0, 1)[None].contiguous(), v)[0].transpose(0, 1)


def test_training_step_of_two_layers():
    """Features, a linear layer with decay and a softmax layer (grouped heads) that reads it, forward and backward over packed
    sequences; each operator against its 64-bit form on what it was given."""
    lens, H, Hk, d = [70, 1, 0, 300, 129], 4, 2, 64
    gen = torch.Generator(device=device()).manual_seed(1)
    T, off, g, v = sum(lens), packed_offsets(lens), decays(H), features(d)
    X, Y, V1 = (rand((T, H, d), torch.bfloat16, gen) for _ in range(3))
    K2, V2 = (rand((T, Hk, d), torch.bfloat16, gen) for _ in range(2))
    dO = rand((T, H, d), torch.bfloat16, gen)
    Q1, K1 = packed_features(X, v), packed_features(Y, v)
    D = Q1.shape[-1]
    a, den = luna.decay_attn(Q1, K1, V1, g, normalize=True, eps=EPS, offsets=off)
    out, lse = luna.softmax_attn(a, K2, V2, offsets=off)
    da, dK2, dV2 = luna.softmax_attn_bwd(a, K2, V2, out, lse, dO, offsets=off)
    grads = luna.decay_attn_bwd(Q1, K1, V1, da, g, out=a, den=den, normalize=True, eps=EPS, offsets=off)
    check_decay(Q1, K1, V1, g, a, den, "packed", lens, True, 1.0)
    check_softmax(a, K2, V2, out, lse, "packed", lens)
    check_backward(a, K2, V2, dO, (da, dK2, dV2), "packed", lens)
    u = unit(torch.bfloat16)
    for i, n in enumerate(lens):  # (the bounds of the operator's own test)
        refs, sizes = decay_grads(*(cut(t, "packed", lens, i) for t in (Q1, K1, V1, da)), g, True, 1.0, EPS)
        for got, ref, size, name in zip(grads, refs, sizes, ("dQ", "dK", "dV")):
            sums = (2 * n + D + d + 32) * U32 * 4
            assert_within(cut(got, "packed", lens, i), ref, (5 * u + sums) * size + u * ref.abs() + 1e-30, f"{name}[{i}]")


def test_prompts_then_tokens_in_a_graph():
    """Padded prompts of different lengths into states and caches, then tokens one at a time by one captured step whose
    lengths move on the device; the replays' rows are those of the whole sequences."""
    prompts, H, Hk, d, steps, cap = [130, 1, 77], 4, 2, 64, 4, 160
    gen = torch.Generator(device=device()).manual_seed(2)
    B, g, v = len(prompts), decays(H), features(d)
    whole = [n + steps for n in prompts]
    Xq, Xk, Xv = (rand((B, H, cap, d), torch.bfloat16, gen) for _ in range(3))
    Q1, K1 = luna.featuremap_variant(Xq, v), luna.featuremap_variant(Xk, v)
    D = Q1.shape[-1]
    Q2 = rand((B, H, cap, d), torch.bfloat16, gen)
    K2, V2 = (rand((B, Hk, cap, d), torch.bfloat16, gen) for _ in range(2))
    lens = torch.tensor(prompts, dtype=torch.int32, device=device())
    S, z = torch.zeros((B, H, D, d), device=device()), torch.zeros((B, H, D), device=device())
    lin, _ = luna.decay_attn(Q1, K1, Xv, g, S=S, z=z, normalize=True, eps=EPS, lens=lens)
    soft, _ = luna.softmax_attn(Q2, K2, V2, lens=lens)
    cK, cV = (torch.full_like(t, math.nan) for t in (K2, V2))  # what no sequence has reached is never read
    for b, n in enumerate(prompts):
        cK[b, :, :n], cV[b, :, :n] = K2[b, :, :n], V2[b, :, :n]

    at = torch.arange(B, device=device())
    tq, tk, tv, t2 = (torch.zeros((B, H, 1, w), dtype=torch.bfloat16, device=device()) for w in (D, D, d, d))
    nk, nv = (torch.zeros((B, Hk, d), dtype=torch.bfloat16, device=device()) for _ in range(2))

    def step():
        where = lens.long()
        cK[at, :, where], cV[at, :, where] = nk, nv
        lens.add_(1)
        return (luna.decay_attn_step(tq, tk, tv, g, S, z, normalize=True, eps=EPS),) + luna.softmax_attn(t2, cK, cV, k_lens=lens)

    def feed(i):
        where = torch.tensor([n + i for n in prompts], device=device())
        for to, x in ((tq, Q1), (tk, K1), (tv, Xv), (t2, Q2)):
            to.copy_(x[at, :, where][:, :, None])
        nk.copy_(K2[at, :, where])
        nv.copy_(V2[at, :, where])

    feed(0)
    saved = [t.clone() for t in (S, z, cK, cV, lens)]
    eager = [t.clone() for t in step()]
    for t, x in zip((S, z, cK, cV, lens), saved):
        t.copy_(x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(steps):
        feed(i)
        graph.replay()
        torch.cuda.synchronize()
        if i == 0:
            assert all(torch.equal(x, y) for x, y in zip(got, eager))
        for b, n in enumerate(prompts):
            lin[b, :, n + i], soft[b, :, n + i] = got[0][b, :, 0], got[1][b, :, 0]
    assert lens.tolist() == whole
    say("prompts then tokens: replays done")
    check_decay(Q1, K1, Xv, g, lin, None, "batch", whole, True, 1.0, S=S, z=z)
    _, lse = luna.softmax_attn(Q2, K2, V2, lens=lens)
    check_softmax(Q2, K2, V2, soft, lse, "batch", whole)
    for b, n in enumerate(whole):  # behind the sequences: as they were
        assert (lin[b, :, n:] == 0).all() and torch.isnan(cK[b, :, n:].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_not_finite_stays_in_its_sequence(dtype, bad):
    """One sequence and one key head with NaN or infinity everywhere: the others' rows, states and gradients are the same
    bits.  Rows of no sequence hold NaN too."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    say(f"not finite: {dtype} {bad}")
    lens, first, H, Hk, d, D = [70, 130, 5, 300, 64], 3, 4, 2, 64, 64
    gen = torch.Generator(device=device()).manual_seed(4)
    T, off, g = first + sum(lens) + 9, packed_offsets(lens, first), decays(H)
    Q, dO, K1, V1 = (rand((T, H, d), dt, gen) for _ in range(4))
    K2, V2 = (rand((T, Hk, d), dt, gen) for _ in range(2))
    few = torch.tensor([first, first + 2, first + 3, first + 4, first + 6, first + 7], dtype=torch.int32, device=device())

    def call():
        S = torch.zeros((len(lens), H, D, d), device=device())
        a, _ = luna.decay_attn(Q, K1, V1, g, S=S, offsets=off)
        da = luna.decay_attn_bwd(Q, K1, V1, dO, g, offsets=off)
        out, lse = luna.softmax_attn(Q, K2, V2, offsets=off)
        db = luna.softmax_attn_bwd(Q, K2, V2, out, lse, dO, offsets=off)
        last, _ = luna.softmax_attn(Q, K2, V2, offsets=few, k_offsets=off)
        rows = [x.clone() for x in (a, *da, out, *db)]
        return rows, S, last

    want, wS, wlast = call()
    a, b = first + lens[0], first + lens[0] + lens[1]
    for t in (Q, dO, K1, V1, K2, V2):
        t[a:b, t.shape[1] // 2:] = bad  # the second half of the heads (one key head), sequence 1
        t[:first], t[first + sum(lens):] = math.nan, math.nan
    got, gS, glast = call()
    for x, y in zip(got, want):
        h = x.shape[1] // 2
        assert torch.equal(x[first:a], y[first:a]) and torch.equal(x[b:T - 9], y[b:T - 9])
        assert torch.equal(x[a:b, :h], y[a:b, :h]), "the other heads of the sequence"
    others = [i for i in range(len(lens)) if i != 1]
    assert torch.equal(gS[others], wS[others])
    assert torch.equal(gS[1, :2], wS[1, :2])
    assert torch.equal(glast[first:first + 2], wlast[first:first + 2])
    assert torch.equal(glast[first + 3:first + 7], wlast[first + 3:first + 7])


@pytest.mark.parametrize("H,Hk,d,dtype,lens,m", [(4, 2, 128, "bf16", [300, 1, 129], 0), (8, 8, 64, "bf16", [130] * 40 + [450], 0),
                                                 (2, 1, 32, "bf16", [200], 0), (2, 1, 64, "f32", [150, 70], 0),
                                                 (4, 2, 128, "bf16", [700, 20, 90], 9), (2, 2, 32, "f32", [600, 5, 33], 5)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_later_tokens_do_not_reach_earlier_rows(H, Hk, d, dtype, lens, m, bad):
    """Keys and values that are not finite from one token on: the rows before it are what they are without them (up to
    the rounding that either way of forming a row has), those that see NaN are NaN."""
    say(f"later tokens: H={H} d={d} {dtype} {lens} m={m} {bad}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device=device()).manual_seed(7)
    n = max(lens)
    qlens = [min(m, x) for x in lens] if m else lens
    K, V = (rand((len(lens), Hk, n, d), dt, gen) for _ in range(2))
    Q = rand((len(lens), H, m or n, d), dt, gen)
    opt = {"lens": torch.tensor(qlens, dtype=torch.int32, device=device())}
    if m:
        opt["k_lens"] = torch.tensor(lens, dtype=torch.int32, device=device())
    want, wl = luna.softmax_attn(Q, K, V, **opt)
    K2, V2 = K.clone(), V.clone()
    first = [max(x - (m // 2 + 1 if m else x // 3), 0) for x in lens]
    for i, a in enumerate(first):
        V2[i, :, a:, ::3] = bad
        K2[i, :, a + 1:] = math.nan
    out, lse = luna.softmax_attn(Q, K2, V2, **opt)
    u = unit(dt) if dt == torch.bfloat16 else 0.0
    for i, a in enumerate(first):
        rows = max(qlens[i] - (lens[i] - a), 0)  # that see none of it
        q, k, v = Q[i, :, :rows].double(), K[i, :, :a].double(), V[i, :, :a].double()
        ref, rlse, _, size, _ = softmax_ref(q, k, v, d ** -0.5, H // Hk)
        most = d ** -0.5 * (q.abs().amax((0, 1)) * k.abs().amax((0, 1))).sum().item() if rows and a else 0.0
        score, sums = (d + 8) * U32 * most, (lens[i] + 16) * U32
        assert_within(out[i, :, :rows], ref, (u + 2 * score + 2 * sums) * size + u * ref.abs() + 1e-30, f"out[{i}]")
        assert_within(lse[i, :, :rows], rlse, score + sums + 4 * U32 * rlse.abs() + 1e-30, f"lse[{i}]")
        assert torch.isnan(out[i, :, rows + 1:qlens[i]].float()).all(), "rows that see a NaN key"
        if rows < qlens[i]:  # sees the first bad values, through finite keys
            assert not torch.isfinite(out[i, :, rows, ::3].float()).any()


@pytest.mark.parametrize("H,D,d,dtype,norm,lens", [(2, 128, 128, "bf16", False, [300, 65]), (2, 256, 128, "bf16", True, [200, 700]),
                                                   (3, 256, 64, "bf16", True, [130]), (2, 64, 32, "bf16", False, [90]),
                                                   (2, 64, 64, "f32", True, [100, 33]), (1, 256, 64, "f32", False, [75])])
@pytest.mark.parametrize("bad", [math.nan, -math.inf])
def test_later_tokens_do_not_reach_earlier_rows_of_linear_attention(H, D, d, dtype, norm, lens, bad):
    """Values that are not finite from one token on (in some columns), later a key: rows before, and columns without, are as
    without them; the others are NaN, and so is the state."""
    say(f"later tokens, decay: H={H} D={D} d={d} {dtype} {norm} {lens} {bad}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device=device()).manual_seed(8)
    B, n, g = len(lens), max(lens), decays(H)
    Q, K = (rand((B, H, n, D), dt, gen, True) for _ in range(2))
    V = rand((B, H, n, d), dt, gen)
    opt = {"lens": torch.tensor(lens, dtype=torch.int32, device=device()), "normalize": norm, "eps": EPS}

    def call(k, v):
        S = torch.zeros((B, H, D, d), device=device())
        z = torch.zeros((B, H, D), device=device()) if norm else None
        return luna.decay_attn(Q, k, v, g, S=S, z=z, **opt) + (S, z)

    want, wden, wS, wz = call(K, V)
    V2, K2 = V.clone(), K.clone()
    first, key = [x // 3 for x in lens], [x - 3 for x in lens]
    for i in range(B):
        V2[i, :, first[i]:, 1::4] = bad
    out, den, S, z = call(K, V2)
    for i in range(B):
        a, m = first[i], lens[i]
        assert torch.equal(out[i, :, :a], want[i, :, :a]), "rows before"
        for c in (0, 2, 3):
            assert torch.equal(out[i, :, a:m, c::4], want[i, :, a:m, c::4]), "columns without"
        assert torch.isnan(out[i, :, a:m, 1::4].float()).all()
        assert torch.isnan(S[i, :, :, 1::4]).all() and torch.equal(S[i, :, :, ::4], wS[i, :, :, ::4])
        if norm:
            assert torch.equal(den[i, :, :m], wden[i, :, :m]) and torch.equal(z, wz)
        K2[i, :, key[i], 5] = math.nan
    out, _, S, _ = call(K2, V)
    for i in range(B):
        assert torch.equal(out[i, :, :key[i]], want[i, :, :key[i]]), "rows before the key"
        assert torch.isnan(out[i, :, key[i]:lens[i]].float()).all() and torch.isnan(S[i, :, 5]).all()


def test_more_sequences_than_lanes():
    """Packed sequences beyond 64, empty ones among them, in every pass."""
    lens = [(7 * i) % 5 if i % 3 else (13 * i) % 140 for i in range(150)]
    H, Hk, d = 4, 2, 64
    gen = torch.Generator(device=device()).manual_seed(11)
    T, off, g = sum(lens), packed_offsets(lens), decays(H)
    Q, dO, K1, V1 = (rand((T, H, d), torch.bfloat16, gen) for _ in range(4))
    K2, V2 = (rand((T, Hk, d), torch.bfloat16, gen) for _ in range(2))
    out, lse = luna.softmax_attn(Q, K2, V2, offsets=off)
    check_softmax(Q, K2, V2, out, lse, "packed", lens)
    check_backward(Q, K2, V2, dO, luna.softmax_attn_bwd(Q, K2, V2, out, lse, dO, offsets=off), "packed", lens)
    S = torch.zeros((len(lens), H, d, d), device=device())
    a, _ = luna.decay_attn(Q, K1, V1, g, S=S, offsets=off)
    check_decay(Q, K1, V1, g, a, None, "packed", lens, False, 1.0, S=S)
    u, grads = unit(torch.bfloat16), luna.decay_attn_bwd(Q, K1, V1, dO, g, offsets=off)
    for i, n in enumerate(lens):
        refs, sizes = decay_grads(*(cut(t, "packed", lens, i) for t in (Q, K1, V1, dO)), g)
        for got, ref, size, name in zip(grads, refs, sizes, ("dQ", "dK", "dV")):
            bound = (5 * u + (2 * n + 2 * d + 32) * U32) * size + u * ref.abs() + 1e-30
            assert_within(cut(got, "packed", lens, i), ref, bound, f"{name}[{i}]")


def test_offsets_beyond_32_bits():
    """Rows 2^20 elements apart and sequences more than 2^31, so that addresses pass 2^32 bytes within and between sequences."""
    H, d, n, row, seq = 2, 64, 2100, 1 << 20, 2101 << 20
    gen = torch.Generator(device=device()).manual_seed(12)
    store = torch.empty(2 * seq + 1024, dtype=torch.bfloat16, device=device())
    far = lambda at: store.as_strided((2, H, n, d), (seq, d, row, 1), at)  # noqa: E731
    Q, K, V, dO = (rand((2, H, n, d), torch.bfloat16, gen) for _ in range(4))
    Kf, Vf, out = far(0), far(H * d), far(2 * H * d)
    Kf.copy_(K)
    Vf.copy_(V)
    g = decays(H)
    say("offsets beyond 32 bits: store filled")
    luna.decay_attn(Q, Kf, Vf, g, out=out)
    want, _ = luna.decay_attn(Q, K, V, g)
    assert torch.equal(out, want)
    want, wl = luna.softmax_attn(Q, K, V)
    _, lse = luna.softmax_attn(Q, Kf, Vf, out=out)
    assert torch.equal(out, want) and torch.equal(lse, wl)
    lens = torch.tensor([n, n - 3], dtype=torch.int32, device=device())
    for m in (1, 5):
        a, _ = luna.softmax_attn(Q[:, :, :m], Kf, Vf, k_lens=lens)
        b, _ = luna.softmax_attn(Q[:, :, :m], K, V, k_lens=lens)
        assert torch.equal(a, b)
    grads = [far(i * H * d) for i in range(3, 6)]
    luna.softmax_attn_bwd(Q, Kf, Vf, want, wl, dO, grads=grads)
    assert all(torch.equal(a, b) for a, b in zip(grads, luna.softmax_attn_bwd(Q, K, V, want, wl, dO)))
    luna.decay_attn_bwd(Q, Kf, Vf, dO, g, grads=grads)
    assert all(torch.equal(a, b) for a, b in zip(grads, luna.decay_attn_bwd(Q, K, V, dO, g)))
