"""The gated delta rule token by token in 64 bits, with PyTorch's own gradients of it, and what the kernels' results may be off by.

A product of operands in up to three parts is off by at most u = 2^-22 of its terms' 2-norms (2^-24 for the parts left out; 64 to 128 additions in fp32, whose errors are
independent of each other, as much again).  Keys no longer than one, betas and decays in 0 .. 1 make a token's map of the states a contraction, so that what is off stays
that far off: an output is six to nine products away from the inputs (forward and backward), whose errors are independent of each other.  A column j of the states is
at most R_j = max over its tokens of |S_j| and |v_j| in 2-norm, so states are off by 16 u R_j and y by that times the query's length; a gradient is counted by the
norms of the factors of its terms in the same way."""
import math

import torch

UNIT = 2.0 ** -22
COUNT = 16
CHUNK = {"f32": 32, "f16": 64, "bf16": 64}


def _normal(x, eps):
    return x / torch.sqrt((x * x).sum(-1, keepdim=True) + eps) if eps > 0 else x


def run(q, k, v, decay, beta, s0, starts, heads, key_heads, dk, dv, scale, eps, dy=None, ds_last=None, dtype="f32"):
    """{name: (value, slack)} of y, s_last and (dy given) the gradients; every tensor in 64 bits and shaped as the call has it."""
    N, nseq, u = q.shape[0], len(starts) - 1, COUNT * UNIT
    leaf = lambda t: t.detach().double().clone().requires_grad_(dy is not None)
    q, k, v, decay, beta = (leaf(t) for t in (q, k, v, decay, beta))
    s0 = leaf(s0 if s0 is not None else torch.zeros(nseq, heads, dk, dv, device=q.device))
    group = heads // key_heads
    qn = _normal(q.view(N, key_heads, dk), eps).repeat_interleave(group, 1)
    kn = _normal(k.view(N, key_heads, dk), eps).repeat_interleave(group, 1)
    vh, a = v.view(N, heads, dv), torch.exp(decay.clamp(min=-10000.0))
    ys, lasts, R, kept = [None] * N, [], [], {}
    for n in range(nseq):
        S = s0[n]
        size = S.detach().norm(dim=1)                                        # heads x dv
        for t in range(starts[n], starts[n + 1]):
            D = S * a[t, :, None, None]
            e = vh[t] - (kn[t][:, :, None] * D).sum(1)
            S = D + kn[t][:, :, None] * (beta[t][:, None] * e)[:, None, :]
            if dy is not None:
                S.retain_grad()
                D.retain_grad()
                kept[t] = S, D, e
            ys[t] = scale * (qn[t][:, :, None] * S).sum(1)
            size = torch.maximum(size, torch.maximum(S.detach().norm(dim=1), vh[t].detach().abs()))
        lasts.append(S)
        R.append(size)
    y = torch.stack(ys).reshape(N, heads * dv) if N else torch.zeros(0, heads * dv, dtype=torch.float64, device=q.device)
    s_last, R = torch.stack(lasts), torch.stack(R)
    of = torch.repeat_interleave(torch.arange(nseq, device=q.device), torch.tensor([b - a for a, b in zip(starts, starts[1:])], device=q.device))
    length = abs(scale) * qn.detach().norm(dim=2)                            # N x heads
    out = {"y": (y.detach(), u * (length[..., None] * R[of]).reshape(N, heads * dv)), "s_last": (s_last.detach(), u * R[:, :, None, :].expand_as(s_last))}
    if dy is None:
        return out
    total = (y * dy.double()).sum() + ((s_last * ds_last.double()).sum() if ds_last is not None else 0.0)
    wanted = [q, k, v, decay, beta, s0]
    held = [t for triple in kept.values() for t in triple[:2]]
    grads = torch.autograd.grad(total, wanted + held, allow_unused=True)
    grads = [g if g is not None else torch.zeros_like(t) for g, t in zip(grads, wanted + held)]
    dS = dict(zip(kept, grads[6::2]))
    dq, dkey, dvalue, ddecay, dbeta, ds0 = grads[:6]
    # sizes: of a sequence and head, the largest norm that its states and their gradients have
    zero = torch.zeros(nseq, heads, dtype=torch.float64, device=q.device)
    big_s, big_d = R.norm(dim=2), (ds_last.double().flatten(2).norm(dim=2) if ds_last is not None else zero.clone())
    big_u = zero.clone()
    for n in range(nseq):
        for t in range(starts[n], starts[n + 1]):
            big_d[n] = torch.maximum(big_d[n], torch.maximum(dS[t].flatten(1).norm(dim=1), length[t] * dy[t].double().view(heads, dv).norm(dim=1)))
            big_u[n] = torch.maximum(big_u[n], torch.maximum(kept[t][2].detach().norm(dim=1), vh[t].detach().norm(dim=1)))
    S_, D_, U_ = big_s[of], big_d[of], big_u[of]                             # N x heads
    klen, dyn = kn.detach().norm(dim=2), dy.double().view(N, heads, dv).norm(dim=2)
    joint = lambda x: x.view(N, key_heads, group).sum(2)
    back = lambda x, raw: (joint(x) / (torch.sqrt((raw.detach().view(N, key_heads, dk) ** 2).sum(2) + eps) if eps > 0 else 1.0))
    sq = back(abs(scale) * dyn * S_ * 2 * (1 + length), q)
    sk = back(D_ * (U_ + S_) * 2 * (1 + klen), k)
    wide = lambda x, d: x[..., None].expand(*x.shape, d).reshape(N, -1)
    sv = D_ * klen
    sb = D_ * klen * (U_ + S_ * klen)
    # a decay's gradient is a sum over what follows it in its chunk, and of the product of the states and their gradients at the chunk's end
    each = abs(scale) * dyn * S_ * length + 2 * D_ * (U_ + S_) * klen
    sd = torch.zeros_like(each)
    for n in range(nseq):
        for c in range(starts[n], starts[n + 1], CHUNK[dtype]):
            end = min(c + CHUNK[dtype], starts[n + 1])
            # (independent errors: the root of the sum of their squares)
            sd[c:end] = (each[c:end] ** 2).flip(0).cumsum(0).flip(0).sqrt() + D_[c:end] * S_[c:end]
    # (fp32 sums of 64 terms in the running sum of the decays' gradients)
    out.update(dq=(dq, u * wide(sq, dk)), dk=(dkey, u * wide(sk, dk)), dv=(dvalue, u * wide(sv, dv)), ddecay=(ddecay, u * sd), dbeta=(dbeta, u * sb),
               ds0=(ds0, u * (big_d[:, :, None, None].expand_as(ds0))))
    return {name: (value.detach(), slack.detach()) for name, (value, slack) in out.items()}
