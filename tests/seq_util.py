"""Plain 64-bit forms of the operators over sequences (include/luna_seq.h) and the bounds that
their kernels have to keep, for the GPU tests.

Bounds.  A rounding to a type moves a value by at most U = finfo(type).eps / 2 of it.  A sum of
products is compared with the same sum over absolute values ("abs form"): roundings of its operands
or terms move it by at most U of that each, fp32 accumulation of N terms by at most
N 2^-24 of it."""
import math

import torch

U32 = 2.0 ** -24


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def device():
    return torch.device("cuda:0")


def rand(shape, dtype, gen, positive=False):
    x = torch.randn(shape, generator=gen, device=device())
    if positive:
        x = torch.relu(x + 0.5)
    return x.to(dtype)


def packed_offsets(lens, first=0):
    at = [first]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device=device())


def cut(t, layout, lens, i, first=0):
    """[heads, n, width] of sequence i in 64 bits."""
    if layout == "packed":
        a = first + sum(lens[:i])
        return t[a:a + lens[i]].double().transpose(0, 1)
    return t[i, :, :lens[i]].double()


def cut_num(t, layout, lens, i, first=0):
    """[heads, n] of the numbers per row of sequence i."""
    if layout == "packed":
        a = first + sum(lens[:i])
        return t[:, a:a + lens[i]].double()
    return t[i, :, :lens[i]].double()


def powers(log_decay, n):
    """f^(i - j) for j <= i, else 0: [H, n, n]."""
    g = log_decay.double().clamp(max=0.0).clamp(min=-1e30)
    i = torch.arange(n, device=g.device, dtype=torch.float64)
    far = i[:, None] - i[None, :]
    return torch.exp(g[:, None, None] * far.clamp(min=0)) * (far >= 0)


def decay_ref(q, k, v, log_decay, S=None, z=None, normalize=False, scale=1.0, eps=1e-6):
    """(out, den, S, z) of [H, n, *] in 64 bits."""
    n = q.shape[1]
    g = log_decay.double().clamp(max=0.0).clamp(min=-1e30)[:, None]
    P = torch.matmul(q, k.transpose(-1, -2)) * powers(log_decay, n)
    i = torch.arange(n, device=q.device, dtype=torch.float64)
    num, den = torch.matmul(P, v), P.sum(-1)
    f, r = torch.exp(g * (i + 1)), torch.exp(g * (n - 1 - i))
    S1, z1 = torch.matmul((k * r[..., None]).transpose(-1, -2), v), (k * r[..., None]).sum(1)
    if S is not None:
        num = num + f[..., None] * torch.matmul(q, S)
        S1 = S1 + torch.exp(g * n)[..., None] * S
    if z is not None:
        den = den + f * torch.matmul(q, z[..., None])[..., 0]
        z1 = z1 + torch.exp(g * n) * z
    out = scale * num
    if normalize:
        out = out / (scale * den + eps)[..., None]
    return out, scale * den, S1, z1


def decay_grads(q, k, v, dO, log_decay, normalize=False, scale=1.0, eps=1e-6):
    """dQ, dK, dV and the abs form of each, by the formulas in 64 bits."""
    F = powers(log_decay, q.shape[1])
    A = torch.matmul(q, k.transpose(-1, -2)) * F
    w = torch.ones_like(q[..., 0])
    D = torch.zeros_like(w)
    absD = torch.zeros_like(w)
    if normalize:
        den = scale * A.sum(-1)
        out = scale * torch.matmul(A, v) / (den + eps)[..., None]
        w = 1.0 / (den + eps)
        D = (dO * out).sum(-1)
        absD = (dO.abs() * out.abs()).sum(-1)
    dA = F * w[..., None] * (torch.matmul(dO, v.transpose(-1, -2)) - D[..., None])
    absA = F * w.abs()[..., None] * (torch.matmul(dO.abs(), v.abs().transpose(-1, -2)) + absD[..., None])
    absP = F * torch.matmul(q.abs(), k.abs().transpose(-1, -2)) * w.abs()[..., None]
    t = lambda x: x.transpose(-1, -2)  # noqa: E731
    grads = tuple(scale * x for x in (torch.matmul(dA, k), torch.matmul(t(dA), q), torch.matmul(t(A * w[..., None]), dO)))
    sizes = tuple(abs(scale) * x for x in (torch.matmul(absA, k.abs()), torch.matmul(t(absA), q.abs()),
                                           torch.matmul(t(absP), dO.abs())))
    return grads, sizes


def softmax_ref(q, k, v, scale, group):
    """(out, lse, P, sum P |v|, visible) of q [H, Lq, d], k and v [Hk, Lk, d] in 64 bits."""
    k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    nq, nk = q.shape[1], k.shape[1]
    row = torch.arange(nq, device=q.device)[:, None] + nk - nq
    seen = torch.arange(nk, device=q.device)[None, :] <= row
    s = scale * torch.matmul(q, k.transpose(-1, -2))
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, -1) if nk else torch.full(q.shape[:2], -math.inf, dtype=q.dtype, device=q.device)
    P = torch.where(seen, torch.exp(s - lse[..., None]), torch.zeros_like(s))
    return torch.matmul(P, v), lse, P, torch.matmul(P, v.abs()), seen


def softmax_grads(q, k, v, dO, scale, group):
    """dQ, dK, dV and the abs form of each, by the formulas in 64 bits."""
    out, _, P, _, _ = softmax_ref(q, k, v, scale, group)
    ke, ve = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    t = lambda x: x.transpose(-1, -2)  # noqa: E731
    dP = torch.matmul(dO, t(ve))
    D = (dO * out).sum(-1, keepdim=True)
    dS = scale * P * (dP - D)
    size = abs(scale) * P * (torch.matmul(dO.abs(), t(ve).abs()) + (dO.abs() * out.abs()).sum(-1, keepdim=True))
    shared = lambda x: x.reshape(k.shape[0], group, *x.shape[1:]).sum(1)  # noqa: E731
    grads = torch.matmul(dS, ke), shared(torch.matmul(t(dS), q)), shared(torch.matmul(t(P), dO))
    sizes = torch.matmul(size, ke.abs()), shared(torch.matmul(t(size), q.abs())), shared(torch.matmul(t(P), dO.abs()))
    return grads, sizes


def assert_within(got, want, bound, what):
    """|got - want| <= bound everywhere (and finite where want is)."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    if want.numel() == 0:
        return
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = ((got - want).abs() - bound).max().item()
    worst = ((got - want).abs() / (bound + 1e-300)).max().item()
    assert over <= 0, f"{what}: {worst:.2f} of the bound"


def assert_norm(got, want, rel, what):
    """The norm of the error of each head within rel of the head's norm."""
    if want.numel() == 0:
        return
    e = (got.double() - want.double()).flatten(1).norm(dim=1)
    n = want.double().flatten(1).norm(dim=1)
    assert (e <= rel * n + 1e-30).all(), f"{what}: {(e / (n + 1e-300)).max().item():.2e} > {rel:.2e}"
