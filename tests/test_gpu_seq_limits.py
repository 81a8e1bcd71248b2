"""The sequence operators (include/luna_seq.h) at the ends of what they take: values, sizes and forms of a call that
choose between kernels."""
import ctypes

import pytest
import torch

from gpu_util import say
from paper_2512_08061_amd import luna
from seq_util import U32, assert_within, cut, decay_grads, device, packed_offsets, rand, unit
from test_gpu_decay import EPS, check_forward as check_decay, decays
from test_gpu_softmax import check_backward as check_softmax_grads, check_forward as check_softmax

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


@pytest.mark.parametrize("norm,dtype,D", [(True, "bf16", 64), (False, "bf16", 128), (True, "f32", 64)])
def test_long_sequences_among_many_short_ones(norm, dtype, D):
    """More packed sequences than states of pieces: only the long ones have states, wherever they lie."""
    say(f"long among many short: norm={norm} {dtype} D={D}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    lens = [(7 * i) % 19 if i % 4 else 0 for i in range(400)]
    for i, n in ((0, 1300), (57, 641), (58, 640), (200, 513), (399, 2100)):
        lens[i] = n
    H, d, T, off, g = 4, 64, sum(lens), packed_offsets(lens), decays(4)
    opt = {"normalize": norm, "eps": EPS, "offsets": off}
    at = lambda a: ctypes.addressof(a)  # noqa: E731
    rows = (ctypes.c_int64 * 4)(len(lens), T, off.data_ptr(), 0)
    nb = luna.load_library().luna_seq_workspace_bytes(luna.OP_DECAY_FWD, luna.LUNA_BF16 if dtype == "bf16" else luna.LUNA_F32, at(rows),
                                                      None, H, H, D, d)
    assert 0 < nb < len(lens) * H * (D * d + max(D, d)) * 4, "pieces, and fewer states than sequences"
    gen = torch.Generator(device=device()).manual_seed(22)
    Q, K = (rand((T, H, D), dt, gen, norm) for _ in range(2))
    V, dO = (rand((T, H, d), dt, gen) for _ in range(2))
    S = torch.randn((len(lens), H, D, d), generator=gen, device=device())
    z = torch.rand((len(lens), H, D), generator=gen, device=device()) + 1.0 if norm else None
    S0, z0 = S.clone(), None if z is None else z.clone()
    out, den = luna.decay_attn(Q, K, V, g, S=S, z=z, **opt)
    check_decay(Q, K, V, g, out, den, "packed", lens, norm, 1.0, S0, z0, S, z)
    out, den = luna.decay_attn(Q, K, V, g, **opt)
    grads = luna.decay_attn_bwd(Q, K, V, dO, g, out=out, den=den, **opt)
    u = unit(dt) if dt == torch.bfloat16 else 0.0
    for i, n in enumerate(lens):  # (the bounds of the operator's own test)
        refs, sizes = decay_grads(*(cut(t, "packed", lens, i) for t in (Q, K, V, dO)), g, norm, 1.0, EPS)
        for got, ref, size, name in zip(grads, refs, sizes, ("dQ", "dK", "dV")):
            sums = (2 * n + D + d + 32) * U32 * (4 if norm else 1)
            assert_within(cut(got, "packed", lens, i), ref, (5 * u + sums) * size + u * ref.abs() + 1e-30, f"{name}[{i}]")


@pytest.mark.parametrize("count", [65, 4097, 5000])
def test_thousands_of_packed_sequences(count):
    """Each packed sequence of thousands is found: the same bits as the padded batch of the same rows, forward and backward.
    (The sequence of two chunks may be one piece in one form and two in the other.  A piece hands dK the state of dV's
    product transposed, formed from other roundings than its own, so there dK is held to its bound instead.)"""
    say(f"packed sequences: {count}")
    H, Hk, d, most = 2, 1, 64, 70
    gen = torch.Generator(device=device()).manual_seed(23)
    lens = torch.randint(0, 6, (count,), generator=gen, device=device(), dtype=torch.int32)
    lens[::61] = 0
    lens[count // 2] = most
    off = torch.cat([torch.zeros(1, dtype=torch.int32, device=device()), lens.cumsum(0).int()])
    T, g = int(off[-1]), decays(H)
    used = torch.arange(most, device=device())[None, :] < lens[:, None]  # [count, most]: row by row as packed
    pad = {n: rand((count, h, most, d), torch.bfloat16, gen) for n, h in (("Q", H), ("K", H), ("V", H), ("dO", H), ("K2", Hk), ("V2", Hk))}
    rows = lambda t: t.transpose(1, 2)[used].contiguous()  # noqa: E731
    own = {n: rows(t) for n, t in pad.items()}
    assert own["Q"].shape[0] == T

    def call(x, **opt):
        a, _ = luna.decay_attn(x["Q"], x["K"], x["V"], g, **opt)
        out, lse = luna.softmax_attn(x["Q"], x["K2"], x["V2"], **opt)
        return (a, out, *luna.decay_attn_bwd(x["Q"], x["K"], x["V"], x["dO"], g, **opt),
                *luna.softmax_attn_bwd(x["Q"], x["K2"], x["V2"], out, lse, x["dO"], **opt))

    at, u = int(off[count // 2]), unit(torch.bfloat16)
    for i, (got, want) in enumerate(zip(call(own, offsets=off), call(pad, lens=lens))):
        want = rows(want)
        if i == 3:
            ref, size = (x[1] for x in decay_grads(*(own[n][at:at + most].double().transpose(0, 1) for n in ("Q", "K", "V", "dO")), g))
            for t in (got, want):
                assert_within(t[at:at + most].transpose(0, 1), ref, (5 * u + (2 * most + 2 * d + 32) * U32) * size + u * ref.abs() + 1e-30, "dK")
                t[at:at + most] = 0
        assert torch.equal(got, want), i


@pytest.mark.parametrize("H,d,layout", [(32, 64, "packed"), (32, 128, "packed"), (64, 64, "packed"), (48, 128, "batch")])
def test_gradients_of_shared_key_heads_without_parts(H, d, layout):
    """Enough key tiles that a workgroup takes all query heads of a key head, one after the other, instead of leaving fp32 parts."""
    say(f"shared key heads without parts: H={H} d={d} {layout}")
    Hk, lens = 16, [(29 * i) % 131 for i in range(70)]
    gen = torch.Generator(device=device()).manual_seed(24)
    shape = (lambda h: (sum(lens), h, d)) if layout == "packed" else (lambda h: (len(lens), h, max(lens), d))
    Q, dO = (rand(shape(H), torch.bfloat16, gen) for _ in range(2))
    K, V = (rand(shape(Hk), torch.bfloat16, gen) for _ in range(2))
    index = packed_offsets(lens) if layout == "packed" else torch.tensor(lens, dtype=torch.int32, device=device())
    opt = {"offsets" if layout == "packed" else "lens": index}
    rows = sum(lens) if layout == "packed" else max(lens)
    seqs = (ctypes.c_int64 * 4)(len(lens), rows, *((index.data_ptr(), 0) if layout == "packed" else (0, index.data_ptr())))
    nb = luna.load_library().luna_seq_workspace_bytes(luna.OP_SOFTMAX_BWD, luna.LUNA_BF16, ctypes.addressof(seqs), None, H, Hk, d, d)
    numbers = Q[..., 0].numel() * 4
    assert nb == (numbers + 255) // 256 * 256, "dO.out per row and nothing else"
    out, lse = luna.softmax_attn(Q, K, V, **opt)
    check_softmax(Q, K, V, out, lse, layout, lens)
    check_softmax_grads(Q, K, V, dO, luna.softmax_attn_bwd(Q, K, V, out, lse, dO, **opt), layout, lens)


@pytest.mark.parametrize("m,H,Hk", [(4, 6, 1), (11, 4, 2), (1, 48, 1), (16, 4, 1), (64, 1, 1), (8, 16, 2)])
@pytest.mark.parametrize("d,dtype", [(32, "bf16"), (64, "bf16"), (128, "bf16"), (32, "f32"), (64, "f32"), (128, "f32")])
def test_rows_of_a_key_head_over_a_cache(m, H, Hk, d, dtype):
    """24 to 64 query rows per key head (two and four tiles of rows), over caches of several pieces, short and empty ones."""
    say(f"rows of a key head over a cache: m={m} H={H} Hk={Hk} d={d} {dtype}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    klens = [1300, 129, 40, 3, 0, 512]
    gen = torch.Generator(device=device()).manual_seed(25)
    Q = rand((len(klens), H, m, d), dt, gen)
    K, V = (rand((len(klens), Hk, 1310, d), dt, gen) for _ in range(2))
    for t in (K, V):
        for i, n in enumerate(klens):
            t[i, :, n:] = float("nan")
    k_lens = torch.tensor(klens, dtype=torch.int32, device=device())
    out, lse = luna.softmax_attn(Q, K, V, k_lens=k_lens)
    check_softmax(Q, K, V, out, lse, "batch", [m] * len(klens), klens)
    few = [min(m, i) for i in (1, 0, m, 3, 2, m)]  # padded queries
    out, lse = luna.softmax_attn(Q, K, V, lens=torch.tensor(few, dtype=torch.int32, device=device()), k_lens=k_lens)
    check_softmax(Q, K, V, out, lse, "batch", few, klens)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f32")])
def test_many_query_heads_on_one_key_head(d, dtype):
    """128 query heads of one key head, a token and three over a cache: more rows than the split form takes."""
    say(f"many query heads on one: d={d} {dtype}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    klens = [700, 1, 130]
    gen = torch.Generator(device=device()).manual_seed(26)
    K, V = (rand((3, 1, 700, d), dt, gen) for _ in range(2))
    for m in (1, 3):
        Q = rand((3, 128, m, d), dt, gen)
        out, lse = luna.softmax_attn(Q, K, V, k_lens=torch.tensor(klens, dtype=torch.int32, device=device()))
        check_softmax(Q, K, V, out, lse, "batch", [m] * 3, klens)


@pytest.mark.parametrize("lens,klens,H,Hk,d,layout", [([512], None, 32, 4, 128, "batch"), ([1024, 700], None, 16, 2, 64, "packed"),
                                                      ([600], [1500], 16, 1, 128, "batch"), ([1100, 900], None, 12, 2, 128, "packed")])
def test_gradients_of_shared_key_heads_from_parts(lens, klens, H, Hk, d, layout):
    """Few key tiles and long chains: a workgroup per query head, whose fp32 parts are added up."""
    say(f"shared key heads from parts: {lens} {klens} H={H} Hk={Hk} d={d} {layout}")
    gen = torch.Generator(device=device()).manual_seed(27)
    shape = (lambda ls, h: (sum(ls), h, d)) if layout == "packed" else (lambda ls, h: (len(ls), h, max(ls), d))
    Q, dO = (rand(shape(lens, H), torch.bfloat16, gen) for _ in range(2))
    K, V = (rand(shape(klens or lens, Hk), torch.bfloat16, gen) for _ in range(2))
    opt = {"offsets": packed_offsets(lens)} if layout == "packed" else {}
    if klens:
        opt["k_lens"] = torch.tensor(klens, dtype=torch.int32, device=device())
    seqs = (ctypes.c_int64 * 4)(len(lens), sum(lens) if layout == "packed" else max(lens), 1 if layout == "packed" else 0, 0)
    keys = (ctypes.c_int64 * 4)(len(klens), max(klens), 0, 1) if klens else None
    nb = luna.load_library().luna_seq_workspace_bytes(luna.OP_SOFTMAX_BWD, luna.LUNA_BF16, ctypes.addressof(seqs),
                                                      None if keys is None else ctypes.addressof(keys), H, Hk, d, d)
    assert nb > Q[..., 0].numel() * 4 + K[..., 0].numel() * (H // Hk) * 2 * d * 4 - 1, "fp32 rows of every query head"
    out, lse = luna.softmax_attn(Q, K, V, **opt)
    grads = luna.softmax_attn_bwd(Q, K, V, out, lse, dO, **opt)
    check_softmax_grads(Q, K, V, dO, grads, layout, lens, klens)
    assert all(torch.equal(a, b) for a, b in zip(grads, luna.softmax_attn_bwd(Q, K, V, out, lse, dO, **opt)))


@pytest.mark.parametrize("n,D,d", [(200, 64, 64), (200, 128, 128), (250, 32, 64)])
def test_gradients_where_values_are_equal(n, D, d):
    """bf16, all values 1, so that out is 1 and dO.v - dO.out is 0 in every term: dQ and dK are 0 up to fp32 sums and the two
    parts of 2^-9 each in which dO.out meets the state.  (Queries and keys are small whole numbers and nothing decays, so that
    weights, sums of keys and the state are whole numbers up to 256: exact in bf16.)"""
    say(f"gradients where values are equal: n={n} D={D} d={d}")
    H, gen = 2, torch.Generator(device=device()).manual_seed(28)
    Q, K = (torch.randint(0, 2, (1, H, n, D), generator=gen, device=device()).to(torch.bfloat16) for _ in range(2))
    Q[..., 0], K[..., 0] = 1, 1
    V, dO = torch.ones((1, H, n, d), dtype=torch.bfloat16, device=device()), rand((1, H, n, d), torch.bfloat16, gen)
    g = torch.zeros(H, device=device())
    out, den = luna.decay_attn(Q, K, V, g, normalize=True, eps=EPS)
    assert (out == 1).all()
    dQ, dK, _ = luna.decay_attn_bwd(Q, K, V, dO, g, out=out, den=den, normalize=True, eps=EPS)
    q, k, do = (t[0].double() for t in (Q, K, dO))
    z, w = k.cumsum(1), 1 / den[0].double()
    total, size = do.sum(-1), do.abs().sum(-1)  # |dO.out| and the sum that forms it
    # two parts of both factors leave 3 2^-18 of a product; P's terms are 2^-24 sums, rounded once more
    each = 3 * 2.0 ** -18 * total.abs() + (n + 2 * d + 16) * U32 * size
    assert_within(dQ[0], torch.zeros_like(q), (each * w)[..., None] * z + 1e-30, "dQ")

    # dK behind one query with a weight of 2^-8: dO / 256 is exact in bf16 as the state, its sum is not
    Q = torch.zeros_like(Q)
    K = torch.zeros_like(K)
    K[..., 0] = 1
    at = 127
    Q[:, :, at, 0] = 2
    dO[:, :, at] = rand((1, H, d), torch.bfloat16, gen)
    out, den = luna.decay_attn(Q, K, V, g, normalize=True, eps=1e-30)
    assert (out[:, :, at] == 1).all() and (den[:, :, at] == 256).all()
    _, dK, _ = luna.decay_attn_bwd(Q, K, V, dO, g, out=out, den=den, normalize=True, eps=1e-30)
    do = dO[0, :, at].double()
    each = (3 * 2.0 ** -18 * do.sum(-1).abs() + (n + 2 * d + 16) * U32 * do.abs().sum(-1)) * 2 / 256
    assert_within(dK[0], torch.zeros_like(k), each[:, None, None].expand_as(k), "dK")
