"""The gated delta rule token by token in 64 bits (include/luna_delta.h) and the bounds that its kernels keep, for the tests.

Bounds are on the 2-norm of a head's error.  Each rounding moves a tensor by at most U = finfo(type).eps / 2 of its norm.  A
chunk's correction is formed from sums that are of the size of what they correct, and the recurrence does not amplify errors
where beta |k|^2 <= 2, so that roundings count once each: of bf16 out its own, that of the weights q.k and (without a
returned state) parts of 2^-17, together below four; of bf16 gradients their own, and parts.  In fp32 n tokens of D
products each leave sqrt(n + D) independent roundings, of which a chunk's factors, its correction and its sums are
counted eight times.

out_t = scale S_t^T q_t may be small where its terms are not (one token: scale (q.k) u): in fp32 the roundings of S_t and of the sum are
relative to scale |S_t| |q_t|, with the Frobenius norm of S_t, which bounds |out_t| by Cauchy's inequality.  Alike dq_t = scale S_t dO_t, dk_t = dS u_t - S dv_t and dv_t = beta k^T dS, whose terms
are scale |S| |dO_t|, |dS| |u_t| + |S| |dv_t| and beta |k_t| |dS|.

dlog_decay is bounded relative to its terms, not to itself.  With G_i the sum of a chunk's log decays up to token i, a loss
depends on log_decay_t through G_i, i >= t, alone, and dL/dG_i is a sum of inner products of q_i with what forms dq_i and of
k_i with what forms dk_i, from the tokens of the chunk (U dS^T, dR S^T, dO S^T restricted to them) and from the states at its
ends.  By Cauchy's inequality these are at most a_i = scale |q_i| |S| |dO_i| + |k_i| (|dS| |u_i| + |S| |dv_i|), with |S| and |dS|
the largest Frobenius norms of a state and a state's gradient in the chunk, once for the tokens' part and once for the ends';
the end itself adds |dS| |S|.  Where tokens overwrite each other's keys the sum is (1 - beta) of its terms or less: the
cancellation is in dS - k (k^T dS beta)^T and the like, in every form of the gradient, and their roundings stay.

dbeta_t = du_t.err_t is bounded by its terms alike: it may vanish where du and err do not (one token: scale (q.k) (dO.v)).  The
roundings of du_t = dS^T k_t are relative to |k_t| |dS|, those of err_t = v_t - S^T k_t to |v_t| + |k_t| |S|, and those of the sum itself to
|du_t| |err_t|, which is less: together |k_t| |dS| |err_t| + |du_t| (|v_t| + |k_t| |S|).  Both gradients have this accuracy in bf16 calls too,
whose operands are counted in parts of 2^-24."""
import math

import torch

from seq_util import U32, assert_norm, cut, cut_num, unit

PART = 2.0 ** -17


def delta_ref(q, k, v, g, beta, S=None, scale=1.0):
    """(out, S) of [H, n, *] (k, q of all value heads) in 64 bits, and the size of each token's terms of out."""
    H, n, D = k.shape
    a = torch.exp(g.clamp(max=0.0))
    S = torch.zeros((H, D, v.shape[-1]), dtype=torch.float64, device=v.device) if S is None else S.clone()
    out, sizes = torch.zeros_like(v), torch.zeros_like(g)
    for t in range(n):
        S = S * a[:, t, None, None]
        u = beta[:, t, None] * (v[:, t] - (k[:, t, :, None] * S).sum(1))
        S = S + k[:, t, :, None] * u[:, None]
        out[:, t] = scale * (q[:, t, :, None] * S).sum(1)
        sizes[:, t] = abs(scale) * q[:, t].norm(dim=1) * S.flatten(1).norm(dim=1)
    return out, S, sizes


def delta_grads(q, k, v, dO, g, beta, scale=1.0):
    """dQ, dK, dV, dlog_decay, dbeta of the value heads, by the recurrence's own adjoint in 64 bits, and the sizes of each token's
    terms of all five."""
    H, n, D = k.shape
    a = torch.exp(g.clamp(max=0.0))
    S = torch.zeros((n + 1, H, D, v.shape[-1]), dtype=torch.float64, device=v.device)
    err = torch.zeros_like(v)
    for t in range(n):
        W = S[t] * a[:, t, None, None]
        err[:, t] = v[:, t] - (k[:, t, :, None] * W).sum(1)
        S[t + 1] = W + k[:, t, :, None] * (beta[:, t, None] * err[:, t])[:, None]
    dS = torch.zeros_like(S[0])
    dq, dk, dv, dg, db, us, dus, *sizes = (torch.zeros_like(t) for t in (q, k, v, g, beta, v, v, g, g, g, g, g))
    norms = torch.zeros((2, H, n + 1), dtype=torch.float64, device=v.device)  # |S_t| and |dS_t|, of the state before token t
    norms[0] = S.flatten(2).norm(dim=2).t()
    for t in reversed(range(n)):
        dq[:, t] = scale * (S[t + 1] * dO[:, t, None]).sum(-1)
        dS = dS + scale * q[:, t, :, None] * dO[:, t, None]
        us[:, t] = u = beta[:, t, None] * err[:, t]
        norms[1, :, t + 1] = dS.flatten(1).norm(dim=1)
        dus[:, t] = du = (k[:, t, :, None] * dS).sum(1)
        db[:, t] = (du * err[:, t]).sum(-1)
        dv[:, t] = beta[:, t, None] * du
        W = S[t] * a[:, t, None, None]
        dk[:, t] = (dS * u[:, None]).sum(-1) - (W * dv[:, t, None]).sum(-1)
        dS = dS - k[:, t, :, None] * dv[:, t, None]
        dg[:, t] = (dS * W).sum((-1, -2))
        dS = dS * a[:, t, None, None]
        norms[1, :, t] = dS.flatten(1).norm(dim=1)
    for t0 in range(0, n, 64):
        c = slice(t0, min(t0 + 64, n))
        mS, mD = norms[:, :, t0:c.stop + 1].amax(-1)[..., None]
        x, y = scale * q[:, c].norm(dim=2) * mS * dO[:, c].norm(dim=2), mD * us[:, c].norm(dim=2) + mS * dv[:, c].norm(dim=2)
        terms = 2 * (x + k[:, c].norm(dim=2) * y)
        nk, ne, nd = k[:, c].norm(dim=2), err[:, c].norm(dim=2), dus[:, c].norm(dim=2)
        for size, x in zip(sizes, (scale * mS * dO[:, c].norm(dim=2), y, beta[:, c].abs() * nk * mD,
                                   terms.flip(1).cumsum(1).flip(1) + mS * mD, nk * mD * ne + nd * (v[:, c].norm(dim=2) + nk * mS))):
            size[:, c] = x
    return dq, dk, dv, torch.where(g > 0, 0.0, dg), db, sizes


def sums(n, D):
    return 8 * math.sqrt(n + D) * U32


def check_forward(Q, K, V, g, beta, out, layout, lens, scale, S0=None, S=None, first=0, what=""):
    group = V.shape[1] // K.shape[1]
    u = unit(out.dtype) if out.dtype == torch.bfloat16 else 0.0
    for i, n in enumerate(lens):
        q, k = (cut(t, layout, lens, i, first).repeat_interleave(group, 0) for t in (Q, K))
        gi, bi = (cut_num(t, layout, lens, i, first) for t in (g, beta))
        ref, rS, sizes = delta_ref(q, k, cut(V, layout, lens, i, first), gi, bi, None if S0 is None else S0[i].double(), scale)
        off = (cut(out, layout, lens, i, first) - ref).flatten(1).norm(dim=1)
        most = 4 * u * ref.flatten(1).norm(dim=1) + sums(n, K.shape[-1]) * sizes.norm(dim=1) + 1e-30
        assert (off <= most).all(), f"{what} out[{i}]: {(off / most).max().item():.2e} of its bound"
        if S is not None:
            assert_norm(S[i], rS, sums(n, K.shape[-1]), f"{what} S[{i}]")


def check_backward(Q, K, V, dO, g, beta, grads, layout, lens, scale, first=0, what=""):
    group = V.shape[1] // K.shape[1]
    bf16 = Q.dtype == torch.bfloat16
    for i, n in enumerate(lens):
        q, k = (cut(t, layout, lens, i, first).repeat_interleave(group, 0) for t in (Q, K))
        v, o = (cut(t, layout, lens, i, first) for t in (V, dO))
        gi, bi = (cut_num(t, layout, lens, i, first) for t in (g, beta))
        refs = delta_grads(q, k, v, o, gi, bi, scale)
        shared = lambda x: x.reshape(K.shape[1], group, *x.shape[1:]).sum(1)  # noqa: E731
        refs, sizes = (shared(refs[0]), shared(refs[1])) + refs[2:5], refs[5]
        sizes = [shared(sizes[0]), shared(sizes[1])] + sizes[2:]
        rows = 2 * unit(torch.bfloat16) if bf16 else 0.0
        for got, ref, size, name in zip(grads[:3], refs[:3], sizes[:3], ("dQ", "dK", "dV")):
            off = (cut(got, layout, lens, i, first) - ref).flatten(1).norm(dim=1)
            most = rows * ref.flatten(1).norm(dim=1) + sums(n, K.shape[-1]) * size.norm(dim=1) + 1e-30
            assert (off <= most).all(), f"{what} {name}[{i}]: {(off / most).max().item():.2e} of its bound"
        if n == 0:
            continue
        for got, ref, size, name in zip(grads[3:], refs[3:], sizes[3:], ("dlog_decay", "dbeta")):
            off = (cut_num(got, layout, lens, i, first) - ref).norm(dim=1) / (size.norm(dim=1) + 1e-300)
            assert off.max().item() <= 2 * sums(n, K.shape[-1]), f"{what} {name}[{i}]: {off.max().item():.2e}"
