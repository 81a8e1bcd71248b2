"""The two kinds of layer of a hybrid decoder over a paged cache and a corrected state, as cases to be timed and compared.

Operators, all reached through `paper_2512_08061_amd.luna`:

  append        paged_append: new keys and values into the pages of a cache, keys and queries rotated by their positions
  paged         paged_attn: causal softmax attention of new tokens over a paged cache, grouped heads
  delta         delta_attn: linear attention by the gated delta rule, chunked, over prompts
  delta_step    delta_attn_step: the next tokens of every sequence from its recurrent state
  delta_bwd     delta_attn_bwd: dQ, dK, dV and the gradients of both gates

Layouts: "batch" holds [B, H, n, width] tensors of equal lengths, "packed" [T, H, width] tensors of one sequence behind the
other with their offsets, "cache" [B, H, m, width] tensors of the m new tokens of sequences whose lengths (these tokens
included) are given, over pages of [pages, Hk, page, d] that a table assigns to the sequences.  Where `own` is false `run`
computes the operators in plain torch, in 32 bits (angles and sums of log decays in 64); `exact` goes token by token (delta)
or head by head (the others) in 64 bits.
"""
import math

import torch

own = False
CHUNK = 64  # tokens per chunk of the plain delta rule


def _case(kind, H, d, lens, Hk=0, D=0, layout="packed", dtype="bf16", m=0, page=0, rot=0, near=False, tokens=False, state=False):
    """lens: "B*n" (equal) or "n1,n2,..."; Hk: heads of the keys (delta: and queries); D: query and key width (delta);
    m: new tokens per sequence (cache and step); page: tokens per page; rot: rotated components; near: their pairs are
    neighbours, not halves; tokens: a page holds [token, head] rows, not [head, token]; state: from a state."""
    return {"kind": kind, "H": H, "d": d, "lens": lens, "Hk": Hk or H, "D": D or d, "layout": layout, "dtype": dtype, "m": m,
            "page": page, "rot": rot or d, "near": near, "tokens": tokens, "state": state}


def listed():
    def named(name, *a, **k):
        return dict(_case(*a, **k), name=name)

    served = ("8192,517,4096,1,7777,3001,2048,6500,333,5120,1999,8000,64,4500,7168,2750,"
              "6001,900,3600,8191,1500,4800,250,7400,3333,5555,1024,6666,2222,4097,128,7999")
    return [
        # a decode step's new token of 32 sequences into their pages
        named("append_token", "append", 16, 128, served, Hk=4, layout="cache", m=1, page=64),
        # prompts of different lengths into empty caches, small pages, half of the components rotated
        named("append_prompts", "append", 16, 128, "1999,4096,517,1,7001,2770", Hk=4, page=16, rot=64),
        # the next token of one user in the second half of a long dialogue
        named("paged_one", "paged", 16, 128, "3001", Hk=4, layout="cache", m=1, page=16),
        # the next token of 32 sequences served together
        named("paged_served", "paged", 16, 128, served, Hk=4, layout="cache", m=1, page=64),
        # a piece of 512 tokens of four long prompts that are prefilled piece by piece
        named("paged_prefill", "paged", 16, 128, "4096,1999,700,16384", Hk=4, layout="cache", m=512, page=64),
        # a short prompt of one user, continued from a state
        named("delta_short_prompt", "delta", 16, 128, "1*333", layout="batch", state=True),
        # prompts of different lengths prefilled together, pairs of heads with one key
        named("delta_packed_prompts", "delta", 32, 128, "1999,4096,517,1,7001,2770", Hk=16, state=True),
        # the forward pass of training on long sequences
        named("delta_long_batch", "delta", 16, 128, "8*16384", layout="batch"),
        # the next token of eight sequences
        named("delta_step_one", "delta_step", 16, 128, "8*1", layout="batch", m=1),
        # the next token of many sequences served together
        named("delta_step_many", "delta_step", 32, 128, "64*1", Hk=16, layout="batch", m=1),
        # a fine-tuning step's backward half
        named("delta_backward", "delta_bwd", 16, 128, "2*2048", layout="batch"),
        # fp32 training on packed sentences of a small 12-head model
        named("delta_f32_backward", "delta_bwd", 12, 64, "512,33,700,197,1021,64,1500,69", dtype="f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _ragged(rng, total, most, longest=1):
    """Up to 12 lengths from one token on, of `total` tokens at most; one has `longest` or more."""
    out = [] if longest == 1 else [_log(rng, longest, most)]
    for _ in range(rng.randint(1, 12)):
        n = _log(rng, 1, most)
        if sum(out) + n > total:
            break
        out.append(n)
    out = out or [_log(rng, 1, min(total, most))]
    rng.shuffle(out)
    return ",".join(str(n) for n in out)


def draw(rng):
    """One more case: head widths 32 to 128, one head to 32, key heads down to one, sequences of one token to 16384, pages of
    16 to 256 tokens, both types.  A training batch has a sequence of 64 tokens or more."""
    kind = rng.choice(["append", "paged", "paged", "paged", "delta", "delta", "delta_step", "delta_bwd"])
    H, d = rng.choice([1, 2, 4, 8, 12, 16, 32]), rng.choice([32, 64, 64, 128, 128])
    dtype = "bf16" if rng.random() < 0.75 else "f32"
    Hk = rng.choice([k for k in (1, 2, 4, 8, 16, 32) if H % k == 0] + [H])
    if kind.startswith("delta"):
        opt = {"D": rng.choice([d, d, 32, 64, 128]), "dtype": dtype, "Hk": rng.choice([H, H, Hk])}
        if kind == "delta_step":
            return _case(kind, H, d, "%d*1" % _log(rng, 1, 64), layout="batch", m=rng.choice([1, 1, 1, 2, 5, 8]), **opt)
        least = 64 if kind == "delta_bwd" else 1
        rows = (1 << 19 if kind == "delta" else 1 << 16) // (1 if dtype == "bf16" else 4)
        if kind == "delta":
            opt["state"] = rng.random() < 0.5
        if rng.random() < 0.4:
            n = _log(rng, least, min(16384, max(1, rows // H)))
            return _case(kind, H, d, "%d*%d" % (_log(rng, 1, max(1, min(16, rows // (n * H)))), n), layout="batch", **opt)
        return _case(kind, H, d, _ragged(rng, max(64, rows // H), min(8192, rows // H), least), **opt)
    opt = {"Hk": Hk, "dtype": dtype, "page": rng.choice([16, 32, 64, 128, 256]), "tokens": rng.random() < 0.4}
    if kind == "append":
        opt.update(rot=rng.choice([d, d, d // 2]), near=rng.random() < 0.4)
        if rng.random() < 0.5:
            return _case(kind, H, d, _ragged(rng, 16384, 8192), **opt)
    m = rng.choice([1, 1, 1, 2, 5, 17] + ([] if dtype == "f32" else [_log(rng, 18, 512)]))
    most = 8192 if m < 18 else 4096
    lens = ",".join(str(_log(rng, m if kind == "append" else 1, most)) for _ in range(_log(rng, 1, 24 if m < 18 else 4)))
    return _case(kind, H, d, lens, layout="cache", m=m, **opt)


def _lens(case):
    s = case["lens"]
    if "*" in s:
        B, n = s.split("*")
        return [int(n)] * int(B)
    return [int(n) for n in s.split(",")]


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------

def _dev():
    return torch.device("cuda:0")


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _scale(case):
    return 1.0 / math.sqrt(case["D"] if case["kind"].startswith("delta") else case["d"])


def prepare(case, seed):
    gen = torch.Generator(device=_dev()).manual_seed(1000003 * seed + 31)
    lens, H, Hk, D, d, m = _lens(case), case["H"], case["Hk"], case["D"], case["d"], case["m"]
    dt = _dtype(case)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=_dev())

    def rows(heads, width):
        """A tensor of the case's layout (in caches: of the new tokens)."""
        return randn(sum(lens), heads, width) if case["layout"] == "packed" else randn(len(lens), heads, m or max(lens), width)

    def numbers():
        """One number per row and head."""
        return randn(H, sum(lens)) if case["layout"] == "packed" else randn(len(lens), H, m or max(lens))

    x = {}
    if case["layout"] == "packed":
        at = [0]
        for n in lens:
            at.append(at[-1] + n)
        x["offsets"] = torch.tensor(at, dtype=torch.int32, device=_dev())
    if case["kind"].startswith("delta"):
        # keys and queries of norm 1, as such layers have them; gates as from a sigmoid and a softplus, with heads that forget
        # within a few tokens and heads that remember hundreds
        for c in "QK":
            x[c] = torch.nn.functional.normalize(rows(Hk, D), dim=-1).to(dt)
        x["V"] = rows(H, d).to(dt)
        rate = torch.exp(torch.rand(H, generator=gen, device=_dev()) * math.log(250.0)) * 0.002
        x["log_decay"] = -torch.nn.functional.softplus(numbers()) * rate[:, None]
        x["beta"] = torch.sigmoid(numbers())
        if case["kind"] == "delta_step" or case["state"]:
            x["S"] = randn(len(lens), H, D, d)
        if case["kind"] == "delta_bwd":
            x["dO"] = rows(H, d).to(dt)
        return {"case": case, "x": x}
    x["Q"], page = rows(H, d).to(dt), case["page"]
    if case["kind"] == "append":
        x["K"], x["V"] = rows(Hk, d).to(dt), rows(Hk, d).to(dt)
        x["inv_freq"] = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float32, device=_dev()) / case["rot"])
    # pages come from a pool in the order in which they became free
    counts = [-(-n // page) for n in lens]
    total = sum(counts) + 3
    order = torch.randperm(total, generator=gen, device=_dev()).to(torch.int32)
    x["table"] = torch.full((len(lens), max(counts) + 1), -1, dtype=torch.int32, device=_dev())
    at = 0
    for i, n in enumerate(counts):
        x["table"][i, :n] = order[at:at + n]
        at += n
    x["lens"] = torch.tensor(lens, dtype=torch.int32, device=_dev())
    for c in ("k_pages", "v_pages"):
        if case["tokens"]:
            x[c] = randn(total, page, Hk, d).to(dt).transpose(1, 2)
        else:
            x[c] = randn(total, Hk, page, d).to(dt)
    return {"case": case, "x": x}


def run(st):
    case, x = st["case"], st["x"]
    return _run_own(case, x) if own else _run_plain(case, x)


def _run_own(case, x):
    from paper_2512_08061_amd import luna

    kind, off, scale = case["kind"], x.get("offsets"), _scale(case)
    if kind == "append":
        q = luna.paged_append(x["K"], x["V"], x["k_pages"], x["v_pages"], x["table"], x["lens"], Q=x["Q"],
                              inv_freq=x["inv_freq"], interleaved=case["near"], offsets=off)
        return {"q": q, "k_pages": x["k_pages"], "v_pages": x["v_pages"]}
    if kind == "paged":
        out, lse = luna.paged_attn(x["Q"], x["k_pages"], x["v_pages"], x["table"], x["lens"], scale=scale)
        return {"out": out, "lse": lse}
    if kind == "delta":
        out = luna.delta_attn(x["Q"], x["K"], x["V"], x["log_decay"], x["beta"], S=x.get("S"), scale=scale, offsets=off)
        return {"out": out, "S": x.get("S")}
    if kind == "delta_step":
        out = luna.delta_attn_step(x["Q"], x["K"], x["V"], x["log_decay"], x["beta"], x["S"], scale=scale)
        return {"out": out, "S": x["S"]}
    grads = luna.delta_attn_bwd(x["Q"], x["K"], x["V"], x["dO"], x["log_decay"], x["beta"], scale=scale, offsets=off)
    return dict(zip(("dQ", "dK", "dV", "dlog_decay", "dbeta"), grads))


# ---------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------

def _padded(case, t):
    """[B, heads, chunks, CHUNK(, width)] in 32 bits, zeros behind the sequences, of rows or (packed [H, T]) of numbers."""
    lens, packed = _lens(case), case["layout"] == "packed"
    if not packed:
        lens = [t.shape[2]] * t.shape[0]
    elif t.dim() == 3:
        t = t.transpose(0, 1)
    n = -(-max(lens) // CHUNK) * CHUNK
    p = torch.zeros((len(lens), t.shape[0 if packed else 1], n) + tuple(t.shape[2 if packed else 3:]), device=t.device)
    if packed:
        at = 0
        for i, k in enumerate(lens):
            p[i, :, :k] = t[:, at:at + k]
            at += k
    else:
        p[:, :, :lens[0]] = t
    return p.unflatten(2, (n // CHUNK, CHUNK))


def _unpadded(case, p, numbers=False):
    """The tensor of the case's layout from [B, heads, chunks, CHUNK(, width)]."""
    lens, p = _lens(case), p.flatten(2, 3)
    if case["layout"] != "packed":
        return p[:, :, :lens[0]].contiguous()
    t = torch.cat([p[i, :, :k] for i, k in enumerate(lens)], 1)
    return t if numbers else t.transpose(0, 1).contiguous()


def _mm(a, b):
    return torch.matmul(a, b.contiguous())


def _plain_delta(q, k, v, g, beta, S, scale):
    """Padded [B, H, chunks, CHUNK, *] -> out, and the state behind the last token.  Rows behind a sequence change nothing:
    their keys and gates are zeros."""
    group = v.shape[1] // k.shape[1]
    q, k = q.repeat_interleave(group, 1), k.repeat_interleave(group, 1)
    kt = k.transpose(-1, -2)
    G = g.double().cumsum(-1)
    i = torch.arange(CHUNK, device=v.device)
    seen = i[:, None] >= i[None, :]
    decay = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(~seen, -math.inf)).float()
    # (I + A)^-1 of the strictly lower A as the product of (I + X^(2^j)), X = -A
    X = -(beta[..., None] * _mm(k, kt) * decay).masked_fill(i[:, None] <= i[None, :], 0.0)
    T = X + torch.eye(CHUNK, device=v.device)
    for _ in range(5):
        X = _mm(X, X)
        T = T + _mm(T, X)
    first, last = torch.exp(G).float()[..., None], torch.exp(G[..., -1:] - G).float()[..., None]
    U, W = _mm(T, beta[..., None] * v), _mm(T, beta[..., None] * first * k)
    P = scale * _mm(q, kt) * decay
    qs, ks = scale * first * q, (last * k).transpose(-1, -2)
    whole = torch.exp(G[..., -1]).float()[..., None, None]
    outs = []
    for c in range(v.shape[2]):
        u = U[:, :, c] - _mm(W[:, :, c], S)
        outs.append(_mm(qs[:, :, c], S) + _mm(P[:, :, c], u))
        S = whole[:, :, c] * S + _mm(ks[:, :, c], u)
    return torch.stack(outs, 2), S


def _rotated(x, pos, inv_freq, near):
    """[tokens, heads, d] in 32 bits, rotated by the angles of their positions."""
    a = pos.double()[:, None] * inv_freq.double()
    c, s = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]
    x, r = x.float().clone(), 2 * inv_freq.shape[0]
    u, v = (x[..., :r:2], x[..., 1:r:2]) if near else (x[..., :r // 2], x[..., r // 2:r])
    turned = torch.stack([u * c - v * s, u * s + v * c], -1 if near else -2)
    x[..., :r] = turned.flatten(-2)
    return x


def _run_plain(case, x):
    kind, scale, dt = case["kind"], _scale(case), _dtype(case)
    if kind == "append":
        K, V, Q, table, lens = x["K"], x["V"], x["Q"], x["table"].long(), x["lens"].long()
        if case["layout"] == "packed":
            t = torch.arange(K.shape[0], device=K.device)
            seq = torch.bucketize(t, x["offsets"][1:].long(), right=True)
            pos = t - x["offsets"].long()[seq]
        else:
            B, m = K.shape[0], K.shape[2]
            seq = torch.arange(B, device=K.device).repeat_interleave(m)
            pos = (lens[:, None] - m + torch.arange(m, device=K.device)).flatten()
            K, V, Q = (t.transpose(1, 2).flatten(0, 1) for t in (K, V, Q))
        at, row = table[seq, pos // case["page"]], pos % case["page"]
        x["k_pages"][at, :, row] = _rotated(K, pos, x["inv_freq"], case["near"]).to(dt)
        x["v_pages"][at, :, row] = V
        q = _rotated(Q, pos, x["inv_freq"], case["near"]).to(dt)
        if case["layout"] != "packed":
            q = q.unflatten(0, (B, m)).transpose(1, 2).contiguous()
        return {"q": q, "k_pages": x["k_pages"], "v_pages": x["v_pages"]}
    if kind == "paged":
        outs, lses = zip(*(_plain_paged(case, x, i, n) for i, n in enumerate(_lens(case))))
        return {"out": torch.stack(outs).to(dt), "lse": torch.stack(lses)}
    if kind == "delta_step":
        group, outs = case["H"] // case["Hk"], []
        q, k = (x[c].float().repeat_interleave(group, 1) for c in "QK")
        v, f, S = x["V"].float(), torch.exp(x["log_decay"]), x["S"]
        for t in range(case["m"]):
            S.mul_(f[:, :, t, None, None])
            u = x["beta"][:, :, t, None] * (v[:, :, t] - (k[:, :, t, :, None] * S).sum(-2))
            S.add_(k[:, :, t, :, None] * u[..., None, :])
            outs.append(scale * (q[:, :, t, :, None] * S).sum(-2))
        return {"out": torch.stack(outs, 2).to(dt), "S": S}
    ins = [_padded(case, x[c]) for c in ("Q", "K", "V", "log_decay", "beta")]
    if kind == "delta":
        S = x["S"] if "S" in x else torch.zeros((len(_lens(case)), case["H"], case["D"], case["d"]), device=_dev())
        out, S = _plain_delta(*ins, S, scale)
        if "S" in x:
            x["S"].copy_(S)
        return {"out": _unpadded(case, out).to(dt), "S": x.get("S")}
    for t in ins:
        t.requires_grad_(True)
    S = torch.zeros((len(_lens(case)), case["H"], case["D"], case["d"]), device=_dev())
    out, _ = _plain_delta(*ins, S, scale)
    grads = torch.autograd.grad(out, ins, _padded(case, x["dO"]))
    res = {n: _unpadded(case, t).to(dt) for n, t in zip(("dQ", "dK", "dV"), grads)}
    return {**res, "dlog_decay": _unpadded(case, grads[3], True), "dbeta": _unpadded(case, grads[4], True)}


def _plain_paged(case, x, i, n):
    """out [H, m, d] and the rows' log-sums [H, m] of sequence i, of n tokens in its pages."""
    H, Hk, d, m, page = case["H"], case["Hk"], case["d"], case["m"], case["page"]
    at = x["table"][i, :-(-n // page)].long()
    k, v = (x[c][at].transpose(0, 1).reshape(Hk, -1, d)[:, :n].float() for c in ("k_pages", "v_pages"))
    q = x["Q"][i].float().reshape(Hk, H // Hk * m, d)
    s = _scale(case) * _mm(q, k.transpose(-1, -2))
    last = n - m + torch.arange(m, device=q.device).repeat(H // Hk)
    s = s.masked_fill(torch.arange(n, device=q.device) > last[:, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    out = _mm(p, v) / total.clamp(min=1e-37)
    return out.reshape(H, m, d), (top + torch.log(total)).reshape(H, m)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    lens, H, Hk, D, d, m = _lens(case), case["H"], case["Hk"], case["D"], case["d"], case["m"]
    kind, rows = case["kind"], sum(lens) if case["layout"] != "cache" else len(lens) * m
    if kind == "append":
        return {"bytes": 2 * rows * (H + 2 * Hk) * d * e, "flops": 3 * rows * (H + Hk) * case["rot"]}
    if kind == "paged":
        pairs = sum(m * n - m * (m - 1) // 2 if n >= m else n * (n + 1) // 2 for n in lens)
        return {"bytes": (2 * rows * H + 2 * sum(lens) * Hk) * d * e + rows * H * 4, "flops": 4 * d * pairs * H}
    if kind == "delta_step":
        rows = len(lens) * m
    io, state = rows * (2 * Hk * D + 2 * H * d) * e + rows * H * 8, len(lens) * H * D * d * 4
    if kind == "delta_bwd":  # Q, K, V, dO and the gates read, their gradients written
        return {"bytes": rows * (4 * Hk * D + 3 * H * d) * e + rows * H * 16, "flops": 14 * rows * H * D * d}
    # per token the products with k, with q and of k and u
    return {"bytes": io + (2 * state if "step" in kind or case["state"] else 0), "flops": 6 * rows * H * D * d}


# ---------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------

def _aligned(case, t, numbers=False):
    """[n, B, heads(, width)] in 64 bits, the first tokens of all sequences first; zeros behind them."""
    lens = _lens(case)
    if case["layout"] != "packed":
        return t.double().movedim(2, 0).contiguous()
    if numbers:
        t = t.t()
    p = torch.zeros((max(lens), len(lens)) + tuple(t.shape[1:]), dtype=torch.float64, device=t.device)
    at = 0
    for i, n in enumerate(lens):
        p[:n, i] = t[at:at + n]
        at += n
    return p


def _placed(case, p, numbers=False):
    """Back in the case's layout."""
    if case["layout"] != "packed":
        return p.movedim(0, 2).contiguous()
    t = torch.cat([p[:n, i] for i, n in enumerate(_lens(case))])
    return t.t().contiguous() if numbers else t


def _exact_delta(case, x):
    scale, group, d = _scale(case), case["H"] // case["Hk"], case["d"]
    q, k = (_aligned(case, x[c]).repeat_interleave(group, 2)[..., None] for c in "QK")  # [n, B, H, D, 1]
    v = _aligned(case, x["V"])[..., None, :]
    a, beta = torch.exp(_aligned(case, x["log_decay"], True))[..., None, None], _aligned(case, x["beta"], True)[..., None, None]
    n = v.shape[0]
    S = x["S"].double() if "S" in x else torch.zeros(v.shape[1:3] + (case["D"], d), dtype=torch.float64, device=_dev())
    back = case["kind"] == "delta_bwd"
    if not back:
        out = torch.zeros_like(v)
        for t in range(n):
            S = S * a[t]
            S = S + k[t] * (beta[t] * (v[t] - (k[t] * S).sum(-2, keepdim=True)))
            out[t] = scale * (q[t] * S).sum(-2, keepdim=True)
        return {"out": _placed(case, out[..., 0, :]), "S": S if "S" in x else None}
    before, err = torch.zeros((n,) + S.shape, dtype=torch.float64, device=_dev()), torch.zeros_like(v)
    for t in range(n):
        before[t] = S
        S = S * a[t]
        err[t] = v[t] - (k[t] * S).sum(-2, keepdim=True)
        S = S + k[t] * (beta[t] * err[t])
    dS, dO = torch.zeros_like(S), _aligned(case, x["dO"])[..., None, :]
    dq, dk, dv, dg, db = (torch.zeros_like(t) for t in (q, k, v, a, beta))
    for t in reversed(range(n)):
        dq[t] = scale * (S * dO[t]).sum(-1, keepdim=True)
        dS = dS + scale * q[t] * dO[t]
        u = beta[t] * err[t]
        du = (k[t] * dS).sum(-2, keepdim=True)
        db[t] = (du * err[t]).sum(-1, keepdim=True)
        dv[t] = beta[t] * du
        was = before[t] * a[t]
        dk[t] = (dS * u).sum(-1, keepdim=True) - (was * dv[t]).sum(-1, keepdim=True)
        dS = dS - k[t] * dv[t]
        dg[t] = (dS * was).sum((-1, -2), keepdim=True)
        dS, S = dS * a[t], before[t]
    res = {"dV": _placed(case, dv[..., 0, :])}
    for c, t in (("dQ", dq), ("dK", dk)):
        res[c] = _placed(case, t[..., 0].unflatten(2, (case["Hk"], group)).sum(3))
    return {**res, "dlog_decay": _placed(case, dg[..., 0, 0], True), "dbeta": _placed(case, db[..., 0, 0], True)}


def exact(case, seed):
    x = prepare(case, seed)["x"]
    if case["kind"].startswith("delta"):
        return _exact_delta(case, x)
    H, Hk, d, m, page, dev = case["H"], case["Hk"], case["d"], case["m"], case["page"], _dev()
    lens, offsets = _lens(case), [0]
    for n in lens:
        offsets.append(offsets[-1] + n)
    if case["kind"] == "append":
        res = {"q": x["Q"].double(), "k_pages": x["k_pages"].double(), "v_pages": x["v_pages"].double()}
        half = torch.arange(case["rot"] // 2, device=dev)
        i, j = (2 * half, 2 * half + 1) if case["near"] else (half, half + case["rot"] // 2)
        for b, n in enumerate(lens):
            if case["layout"] == "packed":
                new = slice(offsets[b], offsets[b + 1])
                Q, K, V = (x[c][new].double() for c in "QKV")
                place = res["q"][new]
            else:
                Q, K, V = (x[c][b].transpose(0, 1).double() for c in "QKV")
                place = res["q"][b].transpose(0, 1)
            pos = torch.arange(n - K.shape[0], n, device=dev)
            w = torch.polar(torch.ones((), dtype=torch.float64, device=dev), pos[:, None] * x["inv_freq"].double())[:, None]
            for t in (Q, K):
                z = torch.complex(t[..., i], t[..., j]) * w
                t[..., i], t[..., j] = z.real, z.imag
            place.copy_(Q)
            for h in range(Hk):
                slot = x["table"][b].long()[pos // page], torch.full_like(pos, h), pos % page
                res["k_pages"].index_put_(slot, K[:, h])
                res["v_pages"].index_put_(slot, V[:, h])
        return res
    res = {"out": torch.zeros_like(x["Q"], dtype=torch.float64),
           "lse": torch.full(x["Q"].shape[:3], -math.inf, dtype=torch.float64, device=dev)}
    for b, n in enumerate(lens):
        key = torch.arange(n, device=dev)
        at, row = x["table"][b].long()[key // page], key % page
        for h in range(H):
            hk = h // (H // Hk)
            k, v = x["k_pages"][at, hk, row].double(), x["v_pages"][at, hk, row].double()
            s = torch.mv(k, x["Q"][b, h, 0].double())[None] if m == 1 else torch.matmul(x["Q"][b, h].double(), k.t())
            s = _scale(case) * s
            first = max(0, m - n)  # rows that see a key
            rows = torch.arange(first, m, device=dev)
            s = torch.where(key[None] <= rows[:, None] + n - m, s[first:], -math.inf)
            res["lse"][b, h, first:] = torch.logsumexp(s, -1)
            res["out"][b, h, first:] = torch.matmul(torch.softmax(s, -1), v)
    return res
