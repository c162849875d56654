"""The calls that the draw of given random numbers, the token log-probabilities and the policy loss are timed on.

Three operators follow the logits of a language-model head, on either side of what the rest of the
library does.  A serving or evaluation program draws a token per row from a random number that it
holds itself, every row with its own temperature, top-k, top-p and min-p (`espo_sample`).  The
policy update reads the logits of the tokens that were drawn: their log-probabilities and the
entropy, with the gradient that a loss of the caller's sends back (`espo_logprobs`,
`espo_logprobs_backward`), or the clipped objective of PPO and its gradient in one call
(`espo_policy_loss`), from the advantages and old log-probabilities that the library has produced.

`run` computes them from elementary torch operations where `own` is false and calls the library
where it is true.  Logits are shaped like a language-model head's: few tokens carry most of the mass, and
the bf16 grid makes many ties.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
QWEN_VOCAB = 152064         # the vocabulary of the paper's models
MASKED = -1e30              # logits at or below this are masked
MOST_BYTES = 2.5e9          # what a drawn case reads and writes at most

# A draw: B rows of V logits.  `mode`: "plain" (the whole vocabulary), "top_p" and "top_k" (that filter
# alone, for all rows), "mixed" (every row its own temperature and filters, greedy rows among them).
# `done`: share of rows that are done; `masked`: share of the vocabulary that a grammar rules out.
_SAMPLE = {"kind": "sample", "B": 1, "V": 1, "dtype": "bf16", "mode": "plain", "tau": 1.0, "top_p": 0.0, "top_k": 0, "done": 0.0, "masked": 0.0}
# Log-probabilities of N given tokens; `entropy`: the entropy too; `grad`: the backward pass as well;
# `unused`: share of rows that hold padding or prompt.
_LOGP = {"kind": "logprobs", "N": 1, "V": 1, "dtype": "bf16", "tau": 1.0, "entropy": False, "grad": False, "unused": 0.0}
# The policy loss of N tokens with its gradient, `bonus` the weight of the entropy.
_LOSS = {"kind": "loss", "N": 1, "V": 1, "dtype": "bf16", "tau": 1.0, "bonus": 0.0, "unused": 0.0}


def _case(base, name, **kw):
    return {"name": name, **base, **kw}


def listed():
    return [
        # One decode step of the four-row fp32 reference rollout: nothing but latency.
        _case(_SAMPLE, "sample_f32_b4", B=4, V=32768, dtype="f32"),
        # A serving step: 64 requests, each with its own settings, some of them greedy, some of the vocabulary
        # ruled out by a grammar.
        _case(_SAMPLE, "sample_mixed_b64", B=64, V=QWEN_VOCAB, mode="mixed", masked=0.3),
        # The rollout of 8 samples for each of 64 prompts at the training temperature, an eighth of the rows done.
        _case(_SAMPLE, "sample_plain_b512", B=512, V=QWEN_VOCAB, tau=0.6, done=0.13),
        # Evaluation as the paper runs it: nucleus 0.7 at temperature 1.
        _case(_SAMPLE, "sample_top_p_b512", B=512, V=QWEN_VOCAB, mode="top_p", top_p=0.7),
        # An engine that hands out fp32 logits of a small model with an odd vocabulary, settings per request.
        _case(_SAMPLE, "sample_mixed_f32_b100", B=100, V=50003, dtype="f32", mode="mixed"),
        # Log-probabilities of the reference rollout's tokens with their gradient: the smallest training step.
        _case(_LOGP, "logprobs_f32_n32", N=32, V=32768, dtype="f32", grad=True),
        # The reference policy's log-probabilities of a micro-batch: forward alone.
        _case(_LOGP, "logprobs_n1024", N=1024, V=QWEN_VOCAB, entropy=True, unused=0.1),
        # A micro-batch of a trainer with a loss of its own: forward, then the gradient from that loss.
        _case(_LOGP, "logprobs_grad_n2048", N=2048, V=QWEN_VOCAB, entropy=True, grad=True, unused=0.2),
        # The same for fp32 logits of an odd vocabulary.
        _case(_LOGP, "logprobs_grad_f32_n700", N=700, V=50003, dtype="f32", entropy=True, grad=True, tau=0.8),
        # The policy update of the reference rollout: 4 rows of 32 steps.
        _case(_LOSS, "loss_f32_n128", N=128, V=32768, dtype="f32"),
        # A micro-batch of the policy update, with an entropy bonus, odd vocabulary.
        _case(_LOSS, "loss_n1000", N=1000, V=150001, tau=0.6, bonus=0.01, unused=0.3),
        # The largest: a trajectory of 4096 tokens with the paper's vocabulary.
        _case(_LOSS, "loss_n4096", N=4096, V=QWEN_VOCAB, unused=0.1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        what = rng.random()
        V, dtype = _log_int(rng, 8000, 200000), rng.choice(("bf16", "bf16", "f32"))
        if what < 0.5:
            case = dict(_SAMPLE, B=_log_int(rng, 1, 1024), V=V, dtype=dtype, mode=rng.choice(("plain", "top_p", "top_k", "mixed")),
                        tau=rng.choice((0.6, 0.8, 1.0)), done=rng.choice((0.0, 0.0, 0.13, 0.5)), masked=rng.choice((0.0, 0.0, 0.3)))
            if case["mode"] == "top_p":
                case["top_p"] = rng.choice((0.7, 0.9, 0.95))
            elif case["mode"] == "top_k":
                case["top_k"] = rng.choice((1, 20, 50, 200))
        elif what < 0.75:
            case = dict(_LOGP, N=_log_int(rng, 1, 4096), V=V, dtype=dtype, tau=rng.choice((0.6, 1.0)), entropy=rng.random() < 0.6,
                        grad=rng.random() < 0.6, unused=rng.choice((0.0, 0.1, 0.5)))
        else:
            case = dict(_LOSS, N=_log_int(rng, 16, 4096), V=V, dtype=dtype, tau=rng.choice((0.6, 1.0)), bonus=rng.choice((0.0, 0.01)),
                        unused=rng.choice((0.0, 0.1, 0.5)))
        if work(case)["bytes"] <= MOST_BYTES:
            return case


# --------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _logits(case, rows, seed):
    """[rows, V] logits whose rows start at multiples of 16 bytes (a view if V does not fill them): normal noise plus
    the logarithm of a Zipf law over a random ranking of the vocabulary."""
    V, dt = case["V"], _dtype(case)
    pitch = 16 // (2 if dt == torch.bfloat16 else 4)
    x = torch.zeros(rows, (V + pitch - 1) // pitch * pitch, dtype=dt, device=DEVICE)
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    boost = -1.1 * torch.log(torch.randperm(V, generator=g, device=DEVICE).float() + 1.0)
    for part in x.split(1024):
        part[:, :V] = torch.randn(part.shape[0], V, generator=g, device=DEVICE).mul_(3.0).add_(boost)
    return x[:, :V]


def _out(n, dtype):
    return torch.zeros(n, dtype=dtype, device=DEVICE)


def _like(x):
    """An output of the layout of `x`: the rows' pitch too."""
    return torch.zeros(x.shape[0], x.stride(0), dtype=x.dtype, device=x.device)[:, :x.shape[1]]


def _prepare_sample(case, seed):
    B, V = case["B"], case["V"]
    g = torch.Generator().manual_seed(seed)
    x = _logits(case, B, seed)
    if case["masked"]:
        gone = torch.randperm(V, generator=g)[:int(V * case["masked"])].to(DEVICE)
        x[:, gone] = -math.inf
    s = {"case": case, "logits": x, "u": torch.rand(B, generator=g).to(DEVICE), "temperature": None, "top_k": None, "top_p": None,
         "min_p": None, "alive": None, "tokens": _out(B, torch.int32), "logprob": _out(B, torch.float32)}
    full = lambda v, dtype=torch.float32: torch.full((B,), v, dtype=dtype, device=DEVICE)
    pick = lambda values, dtype=torch.float32: torch.tensor(values, dtype=dtype)[torch.randint(len(values), (B,), generator=g)].to(DEVICE)
    if case["mode"] == "mixed":
        s["temperature"] = pick([0.0, 0.6, 0.7, 0.8, 1.0, 1.0, 1.3])
        s["top_k"] = pick([0, 0, 0, 20, 40, 50], torch.int32)
        s["top_p"] = pick([1.0, 0.7, 0.8, 0.9, 0.95])
        s["min_p"] = pick([0.0, 0.0, 0.02, 0.05, 0.1])
    else:
        if case["tau"] != 1.0:
            s["temperature"] = full(case["tau"])
        if case["mode"] == "top_k":
            s["top_k"] = full(case["top_k"], torch.int32)
        if case["mode"] == "top_p":
            s["top_p"] = full(case["top_p"])
    if case["done"]:
        s["alive"] = full(1, torch.uint8)
        s["alive"][torch.randperm(B, generator=g)[:int(round(B * case["done"]))].to(DEVICE)] = 0
    if own:
        import paper_2605_29860_amd as espo
        n = espo.espo_sample_workspace_bytes(B, V, _dtype(case))
        s["ws"] = torch.zeros(n, dtype=torch.uint8, device=DEVICE) if n else None
    return s


def _drawn(x, tau, seed):
    """A token per row from softmax(x / tau), and its log-probability."""
    g = torch.Generator(device=x.device).manual_seed(seed)
    tokens, logp = [], []
    for part in x.split(512):
        y = part.float() / tau
        e = torch.empty_like(y).exponential_(generator=g)
        t = (y - e.log()).argmax(1)
        tokens.append(t)
        logp.append(y.gather(1, t[:, None])[:, 0] - y.logsumexp(1))
    return torch.cat(tokens), torch.cat(logp)


def _prepare_update(case, seed):
    N, V = case["N"], case["V"]
    x = _logits(case, N, seed)
    tokens, logp = _drawn(x, case["tau"], seed)
    g = torch.Generator().manual_seed(seed)
    unused = torch.randperm(N, generator=g)[:int(round(N * case["unused"]))].to(DEVICE)
    tokens = tokens.to(torch.int32)
    tokens[unused] = -1
    randn = lambda: torch.randn(N, generator=g).to(DEVICE)
    s = {"case": case, "logits": x, "tokens": tokens, "logprob": _out(N, torch.float32), "entropy": _out(N, torch.float32)}
    used = max(N - unused.numel(), 1)
    if case["kind"] == "loss":
        # the policy has moved a little since the rollout: ratios around 1, some of them beyond the clip range
        s["old"], s["adv"], s["scale"], s["dlogits"] = logp + 0.15 * randn(), randn(), 1.0 / used, _like(x)
    elif case["grad"]:
        s["dlogprob"], s["dlogits"] = randn() / used, _like(x)
        s["dentropy"] = randn() * (0.01 / used) if case["entropy"] else None
    if own:
        import paper_2605_29860_amd as espo
        size = espo.espo_policy_loss_workspace_bytes if case["kind"] == "loss" else espo.espo_logprobs_workspace_bytes
        n = size(N, V, _dtype(case))
        s["ws"] = torch.zeros(n, dtype=torch.uint8, device=DEVICE) if n else None
        s["stats"] = torch.zeros(N, 2, device=DEVICE)
        if case["kind"] == "loss":
            s["out"] = torch.zeros(espo.POLICY_RESULT_BYTES, dtype=torch.uint8, device=DEVICE)
            s["sums"] = s["out"][:20].view(torch.float32)
    return s


def prepare(case, seed):
    return _prepare_sample(case, seed) if case["kind"] == "sample" else _prepare_update(case, seed)


# --------------------------------------------------------------------------- the plain forms
def _plain_sample(s):
    """In 64 bits: which tokens are kept and which one is drawn turn on sums over the whole vocabulary."""
    x, inf = s["logits"], math.inf
    B, V = x.shape
    col = lambda t, off: torch.full((B, 1), off, dtype=torch.float64, device=x.device) if t is None else t.double()[:, None]
    T, k, p, mp = col(s["temperature"], 1.0), col(s["top_k"], 0.0), col(s["top_p"], 1.0), col(s["min_p"], 0.0)
    masked = x <= MASKED
    m = x.float().amax(1, keepdim=True)
    y = (x.double() - m.double()) / torch.where(T > 0, T, 1.0)
    w = torch.where(masked, 0.0, y.exp())
    keep = ~masked & (w >= mp.clamp(max=1.0))
    if s["top_k"] is not None or s["top_p"] is not None:
        by, order = torch.sort(x.float(), dim=1, descending=True)
        kth = by.gather(1, (torch.where((k > 0) & (k < V), k, float(V)) - 1).long())
        keep &= x.float() >= kth
        ws = torch.where(by >= kth, w.gather(1, order), 0.0)
        upto = ws.cumsum(1)
        first = torch.ones_like(by, dtype=torch.bool)
        first[:, 1:] = by[:, 1:] != by[:, :-1]
        in_p = first & ((upto - ws < p * upto[:, -1:]) | (p <= 0) | (p >= 1))
        keep &= x.float() >= torch.where(in_p, by, inf).amin(1, keepdim=True)
    upto = torch.where(keep, w, 0.0).cumsum(1)
    total = upto[:, -1:]
    last = (keep * torch.arange(V, device=x.device)).amax(1)
    token = torch.minimum((upto <= s["u"].double()[:, None] * total).sum(1), last)
    logprob = (y.gather(1, token[:, None]) - total.log())[:, 0]
    greedy = T[:, 0] <= 0
    token = torch.where(greedy, (x.float() == m).int().argmax(1), token)
    logprob = torch.where(greedy, 0.0, logprob)
    gone = masked.all(1)
    if s["alive"] is not None:
        gone |= s["alive"] == 0
    return {"tokens": torch.where(gone, -1, token).int(), "logprob": torch.where(gone, 0.0, logprob).float()}


def _softmax_parts(s):
    """Log-softmax over temperature in 32 bits, and per row: used, token, log-probability and entropy (0 in unused rows)."""
    x = s["logits"]
    y = x.float() / s["case"]["tau"]
    y = y - y.amax(1, keepdim=True)
    e = y.exp()
    total = e.sum(1, keepdim=True)
    logpi, pi = y - total.log(), e / total
    used = (s["tokens"] >= 0) & (s["tokens"] < x.shape[1])
    token = torch.where(used, s["tokens"], 0).long()
    logprob = torch.where(used, logpi.gather(1, token[:, None])[:, 0], 0.0)
    entropy = torch.where(used, (total.log()[:, 0] - (pi * y).sum(1)), 0.0)
    return logpi, pi, used, token, logprob, entropy


def _plain_grad(s, parts, g, h):
    """Gradient on the logits from `g` on the log-probability and `h` (or None) on the entropy of each row."""
    logpi, pi, used, token, _, entropy = parts
    g = torch.where(used, g, 0.0)[:, None]
    d = -g * pi
    d.scatter_add_(1, token[:, None], g)
    if h is not None:
        d -= torch.where(used, h, 0.0)[:, None] * pi * (logpi + entropy[:, None])
    return (d / s["case"]["tau"]).to(s["logits"].dtype)


CLIP = 0.2


def _plain_logprobs(s):
    parts = _softmax_parts(s)
    out = {"logprob": parts[4]}
    if s["case"]["entropy"]:
        out["entropy"] = parts[5]
    if s["case"]["grad"]:
        out["dlogits"] = _plain_grad(s, parts, s["dlogprob"], s["dentropy"])
    return out


def _plain_loss(s):
    parts = _softmax_parts(s)
    _, _, used, _, logprob, entropy = parts
    A, scale, bonus = s["adv"], s["scale"], s["case"]["bonus"]
    d = logprob - s["old"]
    r = d.exp()
    clipped = r.clamp(1 - CLIP, 1 + CLIP)
    policy = torch.where(used, -torch.minimum(r * A, clipped * A), 0.0)
    through = torch.where(A >= 0, r <= 1 + CLIP, r >= 1 - CLIP)
    g = torch.where(through, -scale * r * A, 0.0)
    h = torch.full_like(g, -scale * bonus) if bonus else None
    each = (policy - bonus * entropy, policy, entropy, torch.where(used, r - 1 - d, 0.0), torch.where(used & ~through, 1.0, 0.0))
    return {"sums": torch.stack([scale * v.double().sum() for v in each]).float(), "logprob": logprob, "entropy": entropy,
            "dlogits": _plain_grad(s, parts, g, h)}


# --------------------------------------------------------------------------- one pass
def _own_sample(s):
    import paper_2605_29860_amd as espo
    espo.espo_sample(s["logits"], s["u"], s["tokens"], logprob=s["logprob"], temperature=s["temperature"], top_k=s["top_k"],
                     top_p=s["top_p"], min_p=s["min_p"], alive=s["alive"], workspace=s["ws"])
    return {"tokens": s["tokens"], "logprob": s["logprob"]}


def _own_logprobs(s):
    import paper_2605_29860_amd as espo
    c = s["case"]
    entropy = s["entropy"] if c["entropy"] else None
    espo.espo_logprobs(s["logits"], c["tau"], s["tokens"], s["logprob"], entropy=entropy, stats=s["stats"] if c["grad"] else None,
                       workspace=s["ws"])
    out = {"logprob": s["logprob"]}
    if c["entropy"]:
        out["entropy"] = entropy
    if c["grad"]:
        espo.espo_logprobs_backward(s["logits"], c["tau"], s["tokens"], s["stats"], s["dlogprob"], s["dlogits"], entropy=entropy,
                                    dentropy=s["dentropy"])
        out["dlogits"] = s["dlogits"]
    return out


def _own_loss(s):
    import paper_2605_29860_amd as espo
    c = s["case"]
    espo.espo_policy_loss(s["logits"], c["tau"], s["tokens"], s["old"], s["adv"], s["out"], s["ws"], dlogits=s["dlogits"],
                          logprob=s["logprob"], entropy=s["entropy"], clip_low=CLIP, clip_high=CLIP, entropy_coef=c["bonus"],
                          scale=s["scale"])
    return {"sums": s["sums"], "logprob": s["logprob"], "entropy": s["entropy"], "dlogits": s["dlogits"]}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"sample": _own_sample, "logprobs": _own_logprobs, "loss": _own_loss}[kind](state)
    return {"sample": _plain_sample, "logprobs": _plain_logprobs, "loss": _plain_loss}[kind](state)


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    es, V = (2 if case["dtype"] == "bf16" else 4), case["V"]
    if case["kind"] == "sample":
        B = case["B"]
        live = B - int(round(B * case["done"]))
        return {"bytes": live * (V * es + 20) + B * 9, "flops": live * V * 4}
    N = case["N"]
    used = N - int(round(N * case["unused"]))
    # the logits of used rows come in once, the gradient goes out once, zeros of unused rows included
    grad = case["kind"] == "loss" or case["grad"]
    return {"bytes": used * V * es + (N * V * es if grad else 0) + N * 20, "flops": used * V * (10 if grad else 5)}


# --------------------------------------------------------------------------- the definitions in 64 bits
def _exact_sample(s):
    """Row by row, by classes of equal logits from the largest down, then the inverse of the kept distribution."""
    tokens, logprobs = [], []
    x = s["logits"]
    row = lambda name, b, off: off if s[name] is None else float(s[name][b])
    for b in range(x.shape[0]):
        T, k, p, mp = (row(n, b, off) for n, off in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0)))
        index = torch.nonzero(x[b] > MASKED)[:, 0]
        if (s["alive"] is not None and not int(s["alive"][b])) or index.numel() == 0:
            tokens.append(-1)
            logprobs.append(0.0)
            continue
        v = x[b][index].double()
        if T <= 0:
            tokens.append(int(index[torch.nonzero(v == v.max())[0, 0]]))
            logprobs.append(0.0)
            continue
        level, member, count = torch.unique(v, sorted=True, return_inverse=True, return_counts=True)
        level, count, member = level.flip(0), count.flip(0), level.numel() - 1 - member
        weight = torch.exp((level - level[0]) / T)
        mass = weight * count
        above = count.cumsum(0) - count                     # tokens with a larger logit
        keep = torch.ones_like(level, dtype=torch.bool) if k <= 0 else above < k
        mass = torch.where(keep, mass, 0.0)
        if 0 < p < 1:
            keep = keep & (mass.cumsum(0) - mass < p * mass.sum())
        keep = keep & (weight >= min(mp, 1.0))
        kept = keep[member]
        index, each = index[kept], weight[member[kept]]
        upto = each.cumsum(0)
        i = min(int(torch.searchsorted(upto, float(s["u"][b]) * float(upto[-1]), right=True)), index.numel() - 1)
        tokens.append(int(index[i]))
        logprobs.append(math.log(float(each[i])) - math.log(float(upto[-1])))
    return {"tokens": torch.tensor(tokens, dtype=torch.int32, device=x.device),
            "logprob": torch.tensor(logprobs, dtype=torch.float64, device=x.device)}


def _exact_update(s):
    case, tau = s["case"], float(torch.tensor(s["case"]["tau"], dtype=torch.float32))
    N, V = s["logits"].shape
    dev, f64 = s["logits"].device, torch.float64
    loss = case["kind"] == "loss"
    grad = loss or case["grad"]
    logprob, entropy = torch.zeros(N, dtype=f64, device=dev), torch.zeros(N, dtype=f64, device=dev)
    dlogits = torch.zeros(N, V, dtype=f64, device=dev) if grad else None
    sums = torch.zeros(5, dtype=f64, device=dev)
    rows = torch.nonzero((s["tokens"] >= 0) & (s["tokens"] < V))[:, 0]
    for part in rows.split(256):
        y = s["logits"][part].double() / tau
        logpi = torch.log_softmax(y, 1)
        pi = logpi.exp()
        at = torch.zeros_like(pi)
        at[torch.arange(part.numel(), device=dev), s["tokens"][part].long()] = 1.0
        lp = (logpi * at).sum(1)
        H = -(pi * logpi).sum(1)
        logprob[part], entropy[part] = lp, H
        if loss:
            A, scale, bonus, lo, hi = s["adv"][part].double(), s["scale"], case["bonus"], 1 - CLIP, 1 + CLIP
            r = torch.exp(lp - s["old"][part].double())
            best = torch.minimum(r * A, r.clamp(lo, hi) * A)
            cut = ((A >= 0) & (r > hi)) | ((A < 0) & (r < lo))
            g, h = torch.where(cut, 0.0, -scale * r * A), torch.full_like(r, -scale * bonus)
            sums += scale * torch.stack([(-best - bonus * H).sum(), -best.sum(), H.sum(), (r - 1 - r.log()).sum(), cut.double().sum()])
        elif grad:
            g = s["dlogprob"][part].double()
            h = s["dentropy"][part].double() if case["entropy"] else torch.zeros_like(g)
        if grad:
            dlogits[part] = (g[:, None] * (at - pi) - h[:, None] * pi * (logpi + H[:, None])) / tau
    if loss:
        return {"sums": sums, "logprob": logprob, "entropy": entropy, "dlogits": dlogits}
    out = {"logprob": logprob}
    if case["entropy"]:
        out["entropy"] = entropy
    if grad:
        out["dlogits"] = dlogits
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_sample(s) if case["kind"] == "sample" else _exact_update(s)
