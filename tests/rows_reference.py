"""The operators on rows of logits (draws from given numbers, log-probabilities, policy loss) in 64 bits, written from
their definitions with elementary torch operations, and the bounds that the fp32 kernels are held to.

Bounds count roundings (2^-24 relative each in fp32, half a step of the logits' type for a stored gradient).  For a
row of V logits with t = (x - m) / T:
  a weight 2^(t log2 e): the exponent is three roundings (difference, factor, product), which move the weight by at most
    3 * 2^-24 |t| relative, and the hardware's power of 2 is within one step (2^-23);
  a sum of V weights over at least 256 threads, at most V / 256 + 80 per thread one after the other and 10 levels of
    merging, each with a rescaling of at most 3 * 2^-24 |t| + 2^-23: (V / 256 + 80 + 60) * 2^-24 relative for all of it
    (positive terms; |t| e^t <= 0.37 bounds what the weights' own errors add).
"""
import math

import torch

U = 2.0 ** -24
MASKED = -1e30


def sum_bound(V):
    """Relative error of a row's softmax sum."""
    return (V / 256 + 140) * U


def used_rows(tokens, V):
    return (tokens >= 0) & (tokens < V)


def softmax_rows(x, temperature, tokens):
    """x [N, V] float64 on the CPU.  Returns per row t, ln pi, pi (0 where masked), logprob, entropy, S and used."""
    V = x.shape[1]
    used = used_rows(tokens, V)
    x = torch.where(used[:, None], x, 0.0)
    masked = x <= MASKED
    m = torch.where(masked, -math.inf, x).amax(1, keepdim=True)
    empty = torch.isinf(m)
    m = torch.where(empty, 0.0, m)
    T = float(torch.tensor(temperature, dtype=torch.float32))
    t = torch.where(masked, -math.inf, (x - m) / T)
    w = t.exp()
    S = torch.where(empty, 1.0, w.sum(1, keepdim=True))
    pi, logpi = w / S, t - S.log()
    token = torch.where(used, tokens, 0).long()
    logprob = torch.where(used, logpi.gather(1, token[:, None])[:, 0], 0.0)
    entropy = S.log()[:, 0] - torch.where(masked, 0.0, pi * t.clamp(min=-1e30)).sum(1)
    return dict(t=t, logpi=logpi, pi=pi, masked=masked, logprob=logprob, entropy=torch.where(used, entropy, 0.0), S=S[:, 0], used=used,
                token=token, T=T)


def logits_grad(f, g, h):
    """Gradient on the logits [N, V] from g on the log-probability and h on the entropy of each row."""
    g, h = torch.where(f["used"], g, 0.0)[:, None], torch.where(f["used"], h, 0.0)[:, None]
    at = torch.zeros_like(f["pi"])
    at.scatter_(1, f["token"][:, None], 1.0)
    lp = torch.where(f["masked"], 0.0, f["logpi"])
    d = g * (at - f["pi"]) - h * f["pi"] * (lp + f["entropy"][:, None])
    return torch.where(f["masked"] | ~f["used"][:, None], 0.0, d / f["T"])


def logprob_bound(f, V):
    # (m - x) / T: two roundings; ln S: the sum's error, the logarithm within two steps; their sum: one
    g = torch.where(f["used"], -f["t"].gather(1, f["token"][:, None])[:, 0], 0.0)
    ls = f["S"].log().abs()
    return torch.where(torch.isinf(g), 0.0, 2 * U * g + sum_bound(V) + 4 * U * ls + U * f["logprob"].abs())


def entropy_bound(f, V):
    # ln S and the quotient sum t e^t / S, whose terms share one sign: each sum within sum_bound, the terms' exponents
    # 3 * 2^-24 |t| (1 + |t|) relative to e^t (at most 5 at |t| = 2.6), a handful of roundings behind them
    ls = f["S"].log().abs()
    q = (f["entropy"] - f["S"].log()).abs()
    return sum_bound(V) * (1 + 2 * q) + 16 * U * (1 + q + ls)


def grad_bound(f, g, h, ref, half_step, V):
    """Bound on a stored gradient: half a step of its type, and the errors of pi, of H and of the factors.  `half_step`:
    finfo(type).eps / 2."""
    g, h = g.abs()[:, None], h.abs()[:, None]
    t = torch.where(f["masked"], 0.0, f["t"]).abs()
    size = g + h * (t + 2 * f["S"].log().abs()[:, None] + f["entropy"].abs()[:, None])
    rel = 2 * sum_bound(V) + (3 * t + 16) * U
    H = entropy_bound(f, V)[:, None] + sum_bound(V)
    err = f["pi"] / f["T"] * (size * rel + h * H)
    at = torch.zeros_like(f["pi"])
    at.scatter_(1, f["token"][:, None], 1.0)
    err = err + at * 4 * U * g / f["T"]
    # a weight below 2^-126, the least normal fp32 number, may count as 0: pi is then off by that over S, and so is what it multiplies
    floor = 2.0 ** -126 * (1 + size / (f["T"] * f["S"][:, None]))
    return half_step * (ref.abs() + err) + err + floor


def policy_terms(f, old, adv, weights, scale, lo, hi, coef):
    """g and h of each row, and the five sums of the result (float64)."""
    d = torch.where(f["used"], f["logprob"] - old, 0.0)
    A = torch.where(f["used"], adv, 0.0)
    r = d.clamp(max=88.0).exp()
    w = torch.where(f["used"], scale * weights, 0.0)
    clipped = r.clamp(1 - lo, 1 + hi)
    best = torch.minimum(r * A, clipped * A)
    cut = torch.where(A >= 0, r > 1 + hi, r < 1 - lo)
    g = torch.where(cut, 0.0, -w * r * A)
    h = -w * coef
    sums = [(w * (-best - coef * f["entropy"])).sum(), (-w * best).sum(), (w * f["entropy"]).sum(), (w * (r - 1 - d)).sum(),
            (w * cut).sum()]
    return g, h, sums, dict(r=r, cut=cut, w=w, A=A, d=d)


def sample_row(x, T, k, p, min_p, u):
    """espo_sample's definition for one row: x [V] float64 on the CPU, settings as the kernel reads them (fp32 values).
    Returns the token, its log-probability and how close u W comes to a running sum, relative to W."""
    V, k = x.numel(), int(k)
    index = torch.nonzero(x > MASKED)[:, 0]
    if index.numel() == 0:
        return -1, 0.0, 1.0
    v = x[index]
    if not T > 0:
        return int(index[torch.nonzero(v == v.max())[0, 0]]), 0.0, 1.0
    w = ((v - v.max()) / T).exp()
    keep = torch.ones_like(v, dtype=torch.bool)
    if 0 < k < V:
        kth = torch.sort(v, descending=True).values[min(k, v.numel()) - 1]
        keep &= v >= kth
    if 0 < p < 1:
        mass = torch.where(keep, w, 0.0)
        levels, member = torch.unique(v, sorted=True, return_inverse=True)
        per = torch.zeros_like(levels).index_add_(0, member, mass).flip(0)
        above = per.cumsum(0) - per
        keep &= (above < p * mass.sum()).flip(0)[member]
    keep &= w >= min(min_p, 1.0)
    index, v, w = index[keep], v[keep], w[keep]
    upto = w.cumsum(0)
    W = upto[-1]
    i = min(int((upto <= u * W).sum()), index.numel() - 1)
    return int(index[i]), float((v[i] - x.max()) / T - W.log()), float((upto - u * W).abs().min() / W)
