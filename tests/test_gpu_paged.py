"""Softmax attention over a cache in pages (luna_paged_append, luna_paged_fwd) against plain 64-bit forms, and the layers of a
hybrid decoder (with luna_delta.h) together."""
import math

import pytest
import torch

from delta_util import check_forward as check_delta
from gpu_util import say
from paper_2512_08061_amd import luna
from seq_util import U32, assert_within, cut, cut_num, device, packed_offsets, rand, unit
from test_gpu_softmax import check_forward, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    luna.load_library()
    yield
    torch.cuda.synchronize()


def of(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def tables(lens, page, gen, spare=3, width=0):
    """(table, pages of the pool): the sequences' pages in no order; entries behind them name none."""
    counts = [-(-n // page) for n in lens]
    order = torch.randperm(sum(counts) + spare, generator=gen, device=device()).to(torch.int32)
    table = torch.full((len(lens), max(max(counts), 1) + width), -1, dtype=torch.int32, device=device())
    at = 0
    for i, n in enumerate(counts):
        table[i, :n] = order[at:at + n]
        at += n
    return table, sum(counts) + spare


def pages_of(K, lens, table, pool, page, by_token, fill=math.nan):
    """[pool, Hk, page, d] pages that hold the first lens rows of K [B, Hk, n, d], and `fill` elsewhere."""
    Hk, d = K.shape[1], K.shape[3]
    x = torch.full((pool, page, Hk, d) if by_token else (pool, Hk, page, d), fill, dtype=K.dtype, device=device())
    x = x.transpose(1, 2) if by_token else x
    for i, n in enumerate(lens):
        at = torch.arange(n, device=device())
        x[table[i].long()[at // page], :, at % page] = K[i, :, :n].transpose(0, 1)
    return x


def gathered(pages, lens, table, page):
    """[B, Hk, longest, d] of what the pages hold."""
    out = torch.zeros((len(lens), pages.shape[1], max(max(lens), 1), pages.shape[3]), dtype=pages.dtype, device=device())
    for i, n in enumerate(lens):
        at = torch.arange(n, device=device())
        out[i, :, :n] = pages[table[i].long()[at // page], :, at % page].transpose(0, 1)
    return out


def make(m, klens, H, Hk, d, dtype, page, by_token=False, seed=0):
    gen = torch.Generator(device=device()).manual_seed(seed)
    K, V = (rand((len(klens), Hk, max(max(klens), 1), d), dtype, gen) for _ in range(2))
    table, pool = tables(klens, page, gen, width=seed % 3)
    kp, vp = (pages_of(t, klens, table, pool, page, by_token) for t in (K, V))
    return rand((len(klens), H, m, d), dtype, gen), K, V, kp, vp, table, gen


CASES = [  # m, cached lengths, H, Hk, d, type, page
    (1, [1], 2, 1, 32, "bf16", 16), (1, [1, 777, 64], 8, 2, 128, "bf16", 16), (1, [4097, 130, 0], 4, 4, 64, "bf16", 64),
    (1, [300], 16, 1, 128, "bf16", 128), (1, [0, 0], 2, 2, 64, "bf16", 32), (5, [3, 0, 70], 2, 1, 32, "bf16", 16),
    (4, [500, 17, 2000], 16, 2, 128, "bf16", 32), (8, [900, 33], 8, 1, 64, "bf16", 256), (1, [2500] * 9 + [5], 64, 1, 128, "bf16", 64),
    (17, [17, 500], 4, 1, 64, "bf16", 16), (70, [450, 90, 1, 0, 64], 4, 2, 128, "bf16", 16), (200, [450, 170, 200], 4, 2, 64, "bf16", 32),
    (33, [33, 300], 4, 2, 32, "bf16", 64), (1, [900, 33], 6, 2, 32, "f32", 16), (9, [4, 300], 2, 2, 128, "f32", 16),
    (1, [3000, 1, 64], 8, 2, 128, "f32", 64), (40, [100, 350], 4, 2, 64, "f32", 32), (70, [100], 2, 1, 32, "f32", 16)]


@pytest.mark.parametrize("m,klens,H,Hk,d,dtype,page", CASES)
def test_attention(m, klens, H, Hk, d, dtype, page):
    """Rows of no token in the pages hold NaN, and table entries behind the last page name none."""
    say(f"paged attention m={m} {klens} H={H} Hk={Hk} d={d} {dtype} page={page}")
    Q, K, V, kp, vp, table, _ = make(m, klens, H, Hk, d, of(dtype), page, by_token=len(klens) % 2 == 0)
    out, lse = luna.paged_attn(Q, kp, vp, table, i32(klens))
    check_forward(Q, K, V, out, lse, "batch", [m] * len(klens), klens)
    q = torch.cat([Q[i].transpose(0, 1) for i in range(len(klens))])
    out, lse = luna.paged_attn(q, kp, vp, table, i32(klens), offsets=packed_offsets([m] * len(klens)))
    k, v = (torch.cat([t[i, :, :n].transpose(0, 1) for i, n in enumerate(klens)]) for t in (K, V))
    check_forward(q, k, v, out, lse, "packed", [m] * len(klens), klens)


@pytest.mark.parametrize("count,most,m", [(300, 700, 1), (700, 40, 2), (65, 3000, 1)])
def test_many_sequences(count, most, m):
    """More sequences than lanes and threads, empty ones among them: shares that hold many and sequences in many shares."""
    gen = torch.Generator(device=device()).manual_seed(20)
    klens = torch.randint(0, most, (count,), generator=gen, device=device()).tolist()
    klens[::7] = [0] * len(klens[::7])
    klens[count // 2] = 20 * most
    Q, K, V, kp, vp, table, _ = make(m, klens, 4, 2, 64, torch.bfloat16, 64, seed=21)
    out, lse = luna.paged_attn(Q, kp, vp, table, i32(klens))
    check_forward(Q, K, V, out, lse, "batch", [m] * count, klens)


@pytest.mark.parametrize("m,klens,H,Hk,d", [
    (130, [0, 1, 511, 512, 513, 3000, 1024, 9000], 2, 1, 128), (300, [512, 512, 512, 512], 4, 4, 64), (65, [20000, 130], 16, 4, 128),
    (500, [1536, 5], 32, 8, 64), (129, [4096], 1, 1, 128)])
def test_tiles_of_long_and_short_caches(m, klens, H, Hk, d):
    """Few tiles, whose keys are cut in shares: sequences of one share, of several, and none."""
    say(f"paged tiles m={m} {klens} H={H} Hk={Hk} d={d}")
    Q, K, V, kp, vp, table, _ = make(m, klens, H, Hk, d, torch.bfloat16, 64, seed=31)
    out, lse = luna.paged_attn(Q, kp, vp, table, i32(klens))
    check_forward(Q, K, V, out, lse, "batch", [m] * len(klens), klens)


@pytest.mark.parametrize("m,klens,H,Hk,d", [
    (2, [3], 32, 1, 128), (17, [700, 0, 5, 3001, 16], 32, 2, 64), (70, [2000, 69, 1], 8, 8, 128), (33, [1000, 33, 34], 6, 2, 32),
    (130, [1500], 4, 1, 128), (17, [300] * 30, 32, 2, 64), (3, [100, 40], 33, 1, 32), (65, [300] * 70, 8, 8, 32)])
def test_many_rows_in_fp32(m, klens, H, Hk, d):
    """Rows of a key head in groups of 32, the last of them not full, and (the last case) more tiles than that pays for."""
    say(f"paged rows m={m} {klens[:5]} H={H} Hk={Hk} d={d}")
    Q, K, V, kp, vp, table, _ = make(m, klens, H, Hk, d, torch.float32, 32, seed=51)
    out, lse = luna.paged_attn(Q, kp, vp, table, i32(klens))
    check_forward(Q, K, V, out, lse, "batch", [m] * len(klens), klens)


def test_captured_calls_of_many_rows_in_fp32():
    """Padded queries, some more than their cache holds, and lengths that change between the replays; rows behind q_lens stay."""
    m, room, H, d = 70, [2000, 300, 900], 4, 64
    Q, K, V, kp, vp, table, _ = make(m, room, H, 2, d, torch.float32, 32, seed=53)
    lens, q_lens = i32(room), i32([m] * 3)
    out, lse = torch.empty_like(Q), torch.empty(Q.shape[:3], device=device())
    call = lambda: luna.paged_attn(Q, kp, vp, table, lens, q_lens=q_lens, out=out, lse=lse)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for klens, qlens in ((room, [m, m - 1, 33]), ([1999, 40, 0], [1, 70, 70]), ([65, 1, 33], [64, 0, 40]), (room, [m] * 3)):
        lens.copy_(i32(klens))
        q_lens.copy_(i32(qlens))
        out.fill_(7.0)
        lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        check_forward(Q, K, V, out, lse, "batch", qlens, klens)
        assert all((t[i, :, n:] == 7).all() for t in (out, lse) for i, n in enumerate(qlens))
        replayed = [out.clone(), lse.clone()]
        call()
        assert torch.equal(out, replayed[0]) and torch.equal(lse, replayed[1])


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_values_behind_some_rows_in_fp32(bad):
    """A value that is not finite at a token which only the last rows see (m = 40: in another group of rows than the first)."""
    m, n, H, d = 40, 700, 4, 64
    Q, K, V, kp, vp, table, _ = make(m, [n], H, 1, d, torch.float32, 32, seed=52)
    want, want_lse = luna.paged_attn(Q, kp, vp, table, i32([n]))
    at = n - 7  # rows m - 7 and on
    vp[int(table[0, at // 32]), 0, at % 32, 3] = bad
    out, lse = luna.paged_attn(Q, kp, vp, table, i32([n]))
    keep = torch.arange(d, device=device()) != 3
    assert torch.equal(lse, want_lse)
    # both ways of forming a row: scores off by d + 4 steps of their terms' sum, weights by twice that, an exponential's 4 steps and
    # the 2 n of sums; a row by this share of the largest value, and two rows by twice as much
    terms = (Q[0].double().abs() @ K[0, 0, :n].double().abs().T).max().item() / math.sqrt(d)
    bound = 2 * (2 * (d + 4) * terms + 4 + 2 * n) * 2.0 ** -24 * V[0, 0, :n].abs().max().item()
    assert_within(out[:, :, :m - 7], want[:, :, :m - 7], bound, "rows before")
    assert not torch.isfinite(out[:, :, m - 7:, 3]).any()
    assert torch.isfinite(out[..., keep]).all()


def test_tiles_of_many_sequences():
    gen = torch.Generator(device=device()).manual_seed(32)
    klens = torch.randint(0, 1500, (200,), generator=gen, device=device()).tolist()
    klens[::9] = [0] * len(klens[::9])
    klens[77] = 9000
    Q, K, V, kp, vp, table, _ = make(66, klens, 2, 2, 64, torch.bfloat16, 32, seed=33)
    out, lse = luna.paged_attn(Q, kp, vp, table, i32(klens))
    check_forward(Q, K, V, out, lse, "batch", [66] * 200, klens)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_in_other_shares(bad):
    """A value of a later token reaches no earlier row, and one of an early token all of them, where they lie in other shares."""
    m, n = 140, 2600
    Q, K, V, _, _, table, _ = make(m, [n], 2, 1, 64, torch.bfloat16, 16, seed=34)
    V[0, 0, n - 3, 5] = bad
    kp, vp = (pages_of(t, [n], table, int(table.max()) + 4, 16, False) for t in (K, V))
    out, lse = luna.paged_attn(Q, kp, vp, table, i32([n]))
    assert torch.isfinite(out[:, :, :m - 3]).all() and torch.isfinite(lse).all()
    assert not torch.isfinite(out[:, :, m - 3:, 5]).any() and torch.isfinite(out[:, :, m - 3:, 6]).all()
    check_forward(Q[:, :, :m - 3], K[:, :, :n - 3], V[:, :, :n - 3], out[:, :, :m - 3], lse[:, :, :m - 3], "batch", [m - 3], [n - 3])
    V[0, 0, n - 3, 5], V[0, 0, 700, 5] = 0.0, bad
    vp = pages_of(V, [n], table, int(table.max()) + 4, 16, False)
    out, lse = luna.paged_attn(Q, kp, vp, table, i32([n]))
    assert not torch.isfinite(out[..., 5]).any() and torch.isfinite(out[..., 6]).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("m,H,d,dtype", [(3, 2, 64, "bf16"), (3, 2, 32, "bf16"), (90, 2, 128, "bf16"), (3, 2, 32, "f32")])
def test_padded_queries_keep_other_rows(m, H, d, dtype):
    qlens, klens = [m, 0, m - 1, 1], [m + 60, 90, m - 1, 300]
    Q, K, V, kp, vp, table, _ = make(m + 2, klens, H, 1, d, of(dtype), 16, seed=3)
    for i, n in enumerate(qlens):
        Q[i, :, n:] = math.nan
    out, lse = torch.full_like(Q, 7.0), torch.full(Q.shape[:3], 7.0, device=device())
    luna.paged_attn(Q, kp, vp, table, i32(klens), q_lens=i32(qlens), out=out, lse=lse)
    check_forward(Q, K, V, out, lse, "batch", qlens, klens)
    assert all((t[i, :, n:] == 7).all() for t in (out, lse) for i, n in enumerate(qlens))
    new, _ = luna.paged_attn(Q, kp, vp, table, i32(klens), q_lens=i32(qlens))
    assert all((new[i, :, n:] == 0).all() for i, n in enumerate(qlens))


@pytest.mark.parametrize("m", [1, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_that_are_none(m, dtype):
    """Tokens of table entries outside of the pool are seen by no row, lengths beyond the table end with it, and lengths below
    0 are 0: as the same call without these tokens, whatever a row then sees."""
    page, n, d = 16, 230, 64
    Q, K, V, kp, vp, table, _ = make(m, [n, n, n], 4, 2, d, of(dtype), page, seed=4)
    table = table[:, :15].contiguous()
    table[0, 3], table[0, 14], table[1, 0] = -1, kp.shape[0], 2 ** 31 - 1
    lens = i32([n, n, -5])
    out, lse = luna.paged_attn(Q, kp, vp, table, lens)
    assert (out[2] == 0).all() and (lse[2] == -math.inf).all()
    key, row = torch.arange(n, device=device()), torch.arange(m, device=device())[:, None] + n - m
    for i, gone in ((0, (key // page == 3) | (key // page == 14)), (1, key < page)):
        seen = (key <= row) & ~gone
        q, k, v = Q[i].double(), K[i].double().repeat_interleave(2, 0), V[i].double().repeat_interleave(2, 0)
        s = torch.where(seen, d ** -0.5 * (q @ k.transpose(-1, -2).contiguous()), -math.inf)
        some, want = seen.any(-1), torch.logsumexp(s, -1)
        P = torch.where(seen, torch.exp(s - want[..., None]), 0.0)
        u, sums = unit(of(dtype)) if dtype == "bf16" else 0.0, (n + 16 + d) * U32 * 8
        assert_within(out[i][:, some], (P @ v)[:, some], ((u + sums) * (P @ v.abs()) + u * (P @ v).abs() + 1e-30)[:, some], f"out[{i}]")
        assert_within(lse[i][:, some], want[:, some], torch.full_like(want[:, some], sums * 8), f"lse[{i}]")
        assert (out[i][:, ~some] == 0).all() and (lse[i][:, ~some] == -math.inf).all()
    lens = i32([10 ** 9, 2 ** 31 - 1, 15 * page])
    got = luna.paged_attn(Q, kp.nan_to_num(0), vp.nan_to_num(0), table, lens)
    same = luna.paged_attn(Q, kp.nan_to_num(0), vp.nan_to_num(0), table, i32([15 * page] * 3))
    assert all(torch.equal(x, y) for x, y in zip(got, same))


@pytest.mark.parametrize("H,Hk,d,dtype,m", [(4, 2, 128, "bf16", 5), (2, 1, 32, "bf16", 4), (4, 2, 64, "f32", 6), (4, 2, 128, "bf16", 150),
                                            (2, 1, 32, "bf16", 100), (2, 1, 64, "f32", 80)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_later_tokens_do_not_reach_earlier_rows(H, Hk, d, dtype, m, bad):
    """Keys and values that are not finite from one of the new tokens on: the rows before it are the same with finite ones."""
    say(f"later tokens, paged: H={H} Hk={Hk} d={d} {dtype} m={m} {bad}")
    klens, half = [1500, m, 333], m // 2
    Q, K, V, kp, vp, table, _ = make(m, klens, H, Hk, d, of(dtype), 32, seed=5)
    want, wl = luna.paged_attn(Q, kp, vp, table, i32(klens))
    for i, n in enumerate(klens):
        V[i, :, n - half:, ::3] = bad
        K[i, :, n - half + 1:] = math.nan
    kp, vp = (pages_of(t, klens, table, kp.shape[0], 32, False) for t in (K, V))
    out, lse = luna.paged_attn(Q, kp, vp, table, i32(klens))
    check_forward(Q[:, :, :m - half], K, V, out[:, :, :m - half], lse[:, :, :m - half], "batch", [m - half] * 3, [n - half for n in klens])
    assert torch.isnan(out[:, :, m - half + 1:].float()).all()
    assert not torch.isfinite(out[:, :, m - half, ::3].float()).any()


def rotated(x, pos, inv_freq, near):
    """[tokens, heads, d] in 64 bits and the size of each component's terms."""
    x, r = x.double().clone(), 2 * inv_freq.shape[0]
    a = pos.double()[:, None] * inv_freq.double()
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    size = x.abs()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if near else (slice(0, r // 2), slice(r // 2, r))
    u, v = x[..., first].clone(), x[..., second].clone()
    x[..., first], x[..., second] = u * c - v * s, u * s + v * c
    size[..., first] = size[..., second] = u.abs() + v.abs()
    return x, size


def check_rotated(got, x, pos, inv_freq, near, what):
    """Sine, cosine (2 ulp each), two products and a sum in fp32, and one rounding to the type."""
    ref, size = rotated(x, pos, inv_freq, near)
    u = unit(got.dtype) if got.dtype == torch.bfloat16 else 0.0
    assert_within(got, ref, u * ref.abs() + 8 * U32 * size * (1 + u) + 1e-30, what)


def frequencies(rot, base=10000.0):
    return (base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device()) / max(rot, 1))).float()


@pytest.mark.parametrize("layout,new,had,H,Hk,d,dtype,page,rot,near", [
    ("batch", [1], [0], 1, 1, 32, "bf16", 16, 32, False), ("batch", [1, 1, 1], [8191, 0, 63], 16, 4, 128, "bf16", 64, 128, False),
    ("batch", [5, 5], [100, 27], 4, 2, 64, "bf16", 16, 32, True), ("packed", [300, 1, 0, 65], [0, 70, 9, 200], 4, 2, 128, "bf16", 16, 64, False),
    ("packed", [4000, 700], [0, 100000], 2, 2, 64, "bf16", 128, 64, True), ("packed", [33, 100], [5, 0], 3, 1, 32, "f32", 32, 16, False),
    ("batch", [9, 9], [120000, 0], 2, 1, 128, "f32", 256, 128, True), ("padded", [7, 0, 3], [1, 2, 30], 4, 4, 64, "f32", 16, 64, False),
    ("packed", [40, 3], [0, 17], 2, 2, 64, "bf16", 16, 0, False)])
def test_append(layout, new, had, H, Hk, d, dtype, page, rot, near):
    """Keys and queries rotated, values as they are, all other rows of the pages as they were; far positions too."""
    say(f"append {layout} {new} behind {had} H={H} Hk={Hk} d={d} {dtype} page={page} rot={rot} near={near}")
    gen = torch.Generator(device=device()).manual_seed(6)
    shape = lambda h: (sum(new), h, d) if layout == "packed" else (len(new), h, max(new), d)  # noqa: E731
    Q, K, V = (rand(shape(h), of(dtype), gen) for h in (H, Hk, Hk))
    lens = [a + b for a, b in zip(new, had)]
    table, pool = tables(lens, page, gen)
    by_token = len(new) % 2 == 0
    kp, vp = (rand((pool, page, Hk, d) if by_token else (pool, Hk, page, d), of(dtype), gen) for _ in range(2))
    kp, vp = (t.transpose(1, 2) if by_token else t for t in (kp, vp))
    k0, v0, f = kp.clone(), vp.clone(), frequencies(rot) if rot else None
    opt = {"packed": {"offsets": packed_offsets(new)}, "padded": {"new_lens": i32(new)}, "batch": {}}[layout]
    q = luna.paged_append(K, V, kp, vp, table, i32(lens), Q=Q, inv_freq=f, interleaved=near, **opt)
    f = frequencies(0) if f is None else f
    written = torch.zeros((pool, page), dtype=torch.bool, device=device())
    for i, n in enumerate(new):
        pos = torch.arange(had[i], lens[i], device=device())
        at, row = table[i].long()[pos // page], pos % page
        written[at, row] = True
        part = lambda t: cut(t, "packed" if layout == "packed" else "batch", new, i).transpose(0, 1)  # noqa: E731
        check_rotated(kp[at, :, row], part(K), pos, f, near, f"K[{i}]")
        assert torch.equal(vp[at, :, row].double(), part(V))
        check_rotated(part(q).to(q.dtype), part(Q), pos, f, near, f"Q[{i}]")
    for t, t0 in ((kp, k0), (vp, v0)):
        assert torch.equal(t.transpose(1, 2)[~written], t0.transpose(1, 2)[~written])
    if layout == "padded":
        assert all((q[i, :, n:] == 0).all() for i, n in enumerate(new))
    # in place, and without queries
    same = Q.clone()
    assert luna.paged_append(K, V, kp, vp, table, i32(lens), Q=same, inv_freq=f if rot else None, interleaved=near, q_out=same, **opt) is same
    k1 = kp.clone()
    assert luna.paged_append(K, V, kp, vp, table, i32(lens), inv_freq=f if rot else None, interleaved=near, **opt) is None
    assert torch.equal(kp, k1)
    for i, n in enumerate(new):
        assert torch.equal(cut(same, "packed" if layout == "packed" else "batch", new, i), cut(q, "packed" if layout == "packed" else "batch", new, i))


def test_append_outside_of_the_pages():
    """More new tokens than lens says, a table that ends before the sequence, entries that name no page: what has no place is not
    written, what has one is, and queries are rotated by their positions all the same."""
    gen = torch.Generator(device=device()).manual_seed(7)
    page, m, d, pool = 16, 40, 32, 4
    Q, K, V = (rand((4, 1, m, d), torch.float32, gen) for _ in range(3))
    table = i32([0, 1]).repeat(4, 1).contiguous()
    table[1], table[2], table[3] = i32([2, -1]), i32([2 ** 31 - 1, 3]), i32([-7, pool])
    lens, f = [25, 40, 20, 10 ** 9], frequencies(d)
    kp, vp = (torch.full((pool, 1, page, d), 7.0, device=device()) for _ in range(2))
    q = luna.paged_append(K, V, kp, vp, table, i32(lens), Q=Q, inv_freq=f)
    for i, n in enumerate(lens):
        pos = torch.arange(n - m, n, device=device())
        check_rotated(q[i].transpose(0, 1), Q[i].transpose(0, 1).double(), pos, f, False, f"Q[{i}]")
        for t in range(m):
            p = n - m + t
            if 0 <= p < 2 * page and 0 <= table[i, p // page] < pool:
                assert torch.equal(vp[table[i, p // page], 0, p % page], V[i, 0, t])
    used = torch.zeros((pool, page), dtype=torch.bool, device=device())
    used[0], used[1, :9], used[2], used[3, :4] = True, True, True, True
    for t in (kp, vp):
        assert (t[:, 0][~used] == 7).all() and (t[:, 0][used] != 7).any(-1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_new_tokens_at_one_place(dtype):
    """Sequences that append to the same rows of a page, against the rules of a cache: each element comes from one of them (workgroups
    write side by side, and a row in several stores), and nothing else is written."""
    B, m, Hk, d, page = 40, 3, 2, 64, 16
    gen = torch.Generator(device=device()).manual_seed(31)
    K, V = (rand((B, Hk, m, d), of(dtype), gen) for _ in range(2))
    kp, vp = (torch.full((2, Hk, page, d), 9.0, dtype=of(dtype), device=device()) for _ in range(2))
    luna.paged_append(K, V, kp, vp, torch.zeros((B, 1), dtype=torch.int32, device=device()), i32([5] * B))
    for pages, rows in ((kp, K), (vp, V)):
        assert (pages[0, :, 2:5] == rows).any(0).all()
        assert (pages[0, :, :2] == 9).all() and (pages[0, :, 5:] == 9).all() and (pages[1] == 9).all()


def test_pages_beyond_32_bits():
    """Pages more than 2^32 bytes into the pool, for the tile kernel, the split one and appending."""
    page, Hk, d, far = 64, 2, 64, 300000
    Q, K, V, kp, vp, table, gen = make(3, [150, 70], 4, Hk, d, torch.bfloat16, page, seed=8)
    pool = torch.empty((far + kp.shape[0], Hk, page, d), dtype=torch.bfloat16, device=device())  # 4.9 GB
    assert far * Hk * page * d * 2 > 2 ** 32
    tab = torch.where(table >= 0, table + far, table)
    pool[far:] = kp
    vpool = pool.clone()
    vpool[far:] = vp
    for m in (3, 70):
        q = rand((2, 4, m, d), torch.bfloat16, gen)
        a, b = luna.paged_attn(q, kp, vp, table, i32([150, 70])), luna.paged_attn(q, pool, vpool, tab, i32([150, 70]))
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    f, new = frequencies(d), rand((2, Hk, 3, d), torch.bfloat16, gen)
    luna.paged_append(new, new, kp, vp, table, i32([150, 70]), inv_freq=f)
    luna.paged_append(new, new, pool, vpool, tab, i32([150, 70]), inv_freq=f)
    assert torch.equal(pool[far:].nan_to_num(9), kp.nan_to_num(9)) and torch.equal(vpool[far:].nan_to_num(9), vp.nan_to_num(9))


def test_shared_pages():
    """Two sequences that begin with the same pages see the same keys; one sequence's new token leaves the other as it was."""
    Q, K, V, kp, vp, table, gen = make(1, [100, 100], 4, 2, 64, torch.bfloat16, 16, seed=9)
    table[1, :6] = table[0, :6]  # 96 tokens
    K[1, :, :96], V[1, :, :96] = K[0, :, :96], V[0, :, :96]
    new = rand((2, 2, 1, 64), torch.bfloat16, gen)
    luna.paged_append(new, new, kp, vp, table, i32([101, 101]))
    out, lse = luna.paged_attn(Q, kp, vp, table, i32([101, 101]))
    K, V = torch.cat([K, new], 2), torch.cat([V, new], 2)
    check_forward(Q, K, V, out, lse, "batch", [1, 1], [101, 101])


def test_empty_calls():
    _, _, _, kp, vp, table, _ = make(1, [40, 5], 2, 1, 32, torch.bfloat16, 16)
    z = torch.zeros((0, 2, 32), dtype=torch.bfloat16, device=device())
    out, lse = luna.paged_attn(z, kp, vp, table, i32([40, 5]), offsets=i32([0, 0, 0]))
    assert out.shape == (0, 2, 32) and lse.shape == (2, 0)
    k0 = kp.clone()
    luna.paged_append(z[:, :1], z[:, :1], kp, vp, table, i32([40, 5]), offsets=i32([0, 0, 0]))
    assert torch.equal(kp.nan_to_num(9), k0.nan_to_num(9))


def test_a_decoder_of_both_layers_in_a_graph():
    """Packed prompts into pages and states (appended, attended and corrected chunk by chunk), then tokens one at a time by one captured
    step over both layers whose lengths move on the device: the rows are those of the whole sequences."""
    prompts, H, Hk, d, steps, page = [130, 1, 77], 4, 2, 64, 5, 16
    gen = torch.Generator(device=device()).manual_seed(10)
    B, T, whole, off = len(prompts), sum(prompts), [n + 5 for n in prompts], packed_offsets(prompts)
    n = max(whole)
    Q, Q2, V = (rand((B, H, n, d), torch.bfloat16, gen) for _ in range(3))
    K2, V2 = (rand((B, Hk, n, d), torch.bfloat16, gen) for _ in range(2))
    Kd = torch.nn.functional.normalize(rand((B, Hk, n, d), torch.float32, gen), dim=-1).to(torch.bfloat16)
    Qd = torch.nn.functional.normalize(rand((B, Hk, n, d), torch.float32, gen), dim=-1).to(torch.bfloat16)
    g, beta = -0.1 * rand((B, H, n), torch.float32, gen).abs(), torch.sigmoid(rand((B, H, n), torch.float32, gen))
    table, pool = tables(whole, page, gen)
    kp, vp = (torch.full((pool, Hk, page, d), math.nan, dtype=torch.bfloat16, device=device()) for _ in range(2))
    lens, f, S = i32(prompts), frequencies(d), torch.zeros((B, H, d, d), device=device())
    packed = lambda t: torch.cat([t[i, :, :p].transpose(0, 1) for i, p in enumerate(prompts)])  # noqa: E731
    nums = lambda t: torch.cat([t[i, :, :p] for i, p in enumerate(prompts)], 1)  # noqa: E731
    q = luna.paged_append(packed(K2), packed(V2), kp, vp, table, lens, Q=packed(Q2), inv_freq=f, offsets=off)
    soft, _ = luna.paged_attn(q, kp, vp, table, lens, offsets=off)
    lin = luna.delta_attn(packed(Qd), packed(Kd), packed(V), nums(g), nums(beta), S=S, offsets=off)
    outs = [torch.zeros((B, H, n, d), dtype=torch.bfloat16, device=device()) for _ in range(2)]
    at = 0
    for i, p in enumerate(prompts):
        for t, x in zip(outs, (soft, lin)):
            t[i, :, :p] = x[at:at + p].transpose(0, 1)
        at += p
    ins = [torch.zeros((B, t.shape[1], 1) + tuple(t.shape[3:]), dtype=t.dtype, device=device()) for t in (Q2, K2, V2, Qd, Kd, V, g, beta)]

    def step():
        q2, k2, v2, qd, kd, v, gg, bb = ins
        lens.add_(1)
        q2 = luna.paged_append(k2, v2, kp, vp, table, lens, Q=q2, inv_freq=f)
        return luna.paged_attn(q2, kp, vp, table, lens)[0], luna.delta_attn_step(qd, kd, v, gg, bb, S)

    def feed(i):
        where = torch.tensor([p + i for p in prompts], device=device())
        for to, x in zip(ins, (Q2, K2, V2, Qd, Kd, V, g, beta)):
            to.copy_(x[torch.arange(B, device=device()), :, where][:, :, None])

    feed(0)
    saved = [t.clone() for t in (S, kp, vp, lens)]
    eager = [t.clone() for t in step()]
    for t, x in zip((S, kp, vp, lens), saved):
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
        for b, p in enumerate(prompts):
            for t, x in zip(outs, got):
                t[b, :, p + i] = x[b, :, 0]
    assert lens.tolist() == whole
    check_delta(Qd, Kd, V, g, beta, outs[1], "batch", whole, 1.0, None, S)
    # what is in the pages against the rotation, and the rows of attention against what is in the pages
    k, v = gathered(kp, whole, table, page), gathered(vp, whole, table, page)
    rq = torch.zeros_like(Q2)
    for b, p in enumerate(whole):
        pos = torch.arange(p, device=device())
        check_rotated(k[b, :, :p].transpose(0, 1), K2[b, :, :p].transpose(0, 1), pos, f, False, f"K[{b}]")
        assert torch.equal(v[b, :, :p], V2[b, :, :p])
        rq[b, :, :p] = rotated(Q2[b, :, :p].transpose(0, 1), pos, f, False)[0].transpose(0, 1).to(torch.bfloat16)
    _, lse = luna.softmax_attn(rq, k, v, lens=i32(whole))
    check_forward(rq, k, v, outs[0], lse, "batch", whole)


def test_same_bits_streams_and_two_graphs():
    """The same call gives the same bits, on a stream of its own and from two captured graphs replayed in turn with eager calls between."""
    made = [make(m, klens, 8, 2, 128, torch.bfloat16, 64, seed=s) for m, klens, s in ((1, [3000, 50, 700], 11), (2, [900, 2000], 12), (80, [400, 90], 13))]
    args = [(x[0], x[3], x[4], x[5], i32(k)) for x, k in zip(made, ([3000, 50, 700], [900, 2000], [400, 90]))]
    want = [[t.clone() for t in luna.paged_attn(*a)] for a in args]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [luna.paged_attn(*a) for a in args]
    side.synchronize()
    assert all(torch.equal(x, y) for a, b in zip(got, want) for x, y in zip(a, b))
    graphs, outs = [], []
    for a in args[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(luna.paged_attn(*a))
    for _ in range(3):
        for o in outs:
            for t in o:
                t.zero_()
        for graph in graphs:
            graph.replay()
        eager = luna.paged_attn(*args[2])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(outs + [eager], want) for x, y in zip(a, b))


@pytest.mark.parametrize("m", [1, 130])
def test_a_captured_call_follows_the_lengths(m):
    """The shares of the keys are worked out on the device: a captured call over caches that grow and shrink between its replays."""
    room = [4000, 300, 2100]
    Q, K, V, kp, vp, table, _ = make(m, room, 4, 2, 64, torch.bfloat16, 32, seed=41)
    lens = i32(room)
    luna.paged_attn(Q, kp, vp, table, lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = luna.paged_attn(Q, kp, vp, table, lens)
    for klens in ([1, 300, 700], [4000, 0, 2100], [513, 299, 1024], [0, 0, 0], room):
        lens.copy_(i32(klens))
        want = luna.paged_attn(Q, kp, vp, table, lens)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        check_forward(Q, K, V, out, lse, "batch", [m] * 3, klens)


def test_tiles_on_a_stream_and_in_two_graphs():
    """The tile kernels with keys in shares: the same bits on another stream and from graphs replayed in turn with eager calls."""
    klens = ([3000, 50, 700], [900, 2000])
    args = [(x[0], x[3], x[4], x[5], i32(k)) for x, k in ((make(200, k, 8, 2, 128, torch.bfloat16, 64, seed=42 + len(k)), k) for k in klens)]
    want = [[t.clone() for t in luna.paged_attn(*a)] for a in args]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [luna.paged_attn(*a) for a in args]
    side.synchronize()
    assert all(torch.equal(x, y) for a, b in zip(got, want) for x, y in zip(a, b))
    graphs, outs = [], []
    for a in args:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(luna.paged_attn(*a))
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        eager = luna.paged_attn(*args[0])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(outs + [eager], want + want[:1]) for x, y in zip(a, b))
