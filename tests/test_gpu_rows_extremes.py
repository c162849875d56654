"""espo_sample, espo_logprobs and espo_policy_loss where exponents leave the ordinary range: low temperatures, logits far from 0, masks
that hide the first tiles, weights of 0 (needs an MI355X).  The definitions are those of tests/rows_reference.py in 64 bits, and tokens have
to be equal."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import rows_reference as R  # noqa: E402
import paper_2605_29860_amd as espo  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def padded(x, fill=50.0):
    """x [B, V] of the CPU as a view of rows that start at multiples of 16 bytes, on the GPU; behind V lies `fill`."""
    E = 8 if x.dtype == BF16 else 4
    buf = torch.full((x.shape[0], -(-x.shape[1] // E) * E), fill, dtype=x.dtype)
    buf[:, :x.shape[1]] = x
    return buf.cuda()[:, :x.shape[1]]


def draw(x, u, T=None, k=None, p=None):
    """Draws from x [B, V] (on the CPU, settings [B]) with and without a workspace, and compares with the definition.  The sums' errors are below
    1e-9 of the total here, so a u that comes closer than that to a running sum would decide nothing, nor a p that
    does to the mass above a logit."""
    B, V = x.shape
    gpu = padded(x)
    dev = lambda t: None if t is None else t.cuda()
    n = espo.espo_sample_workspace_bytes(B, V, x.dtype)
    ws = torch.full((n,), 0xCD, dtype=torch.uint8, device="cuda") if n else None
    tokens, again = (torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    lp = torch.full((B,), math.nan, device="cuda")
    espo.espo_sample(gpu, u.cuda(), tokens, logprob=lp, temperature=dev(T), top_k=dev(k), top_p=dev(p), workspace=ws)
    espo.espo_sample(gpu, u.cuda(), again, temperature=dev(T), top_k=dev(k), top_p=dev(p))
    tokens, lp = tokens.cpu(), lp.cpu()
    at = lambda t, b, off: off if t is None else float(t[b])
    wrong = []
    for b in range(B):
        tok, want, near = R.sample_row(x[b].double(), at(T, b, 1.0), at(k, b, 0), at(p, b, 1.0), 0.0, float(u[b]))
        assert near > 1e-9, ("this input decides nothing", b, near)
        if int(tokens[b]) != tok or not abs(float(lp[b]) - want) <= 2.0 ** -24 * abs(want) + 1e-9:
            wrong.append((b, at(T, b, 1.0), at(p, b, 1.0), int(tokens[b]), tok, float(lp[b]), want))
    assert not wrong, (len(wrong), wrong[:4])
    assert torch.equal(tokens, again.cpu())


def settings(values, B, g, dtype=F32):
    return torch.tensor(values, dtype=dtype)[torch.randint(len(values), (B,), generator=g)]


def hot_rows(B, V, dtype, g):
    """Largest logits from 6 to 60, some hundred different ones below them."""
    x = torch.randn(B, V, generator=g) * 2.0
    top = torch.linspace(6.0, 60.0, B)[torch.randperm(B, generator=g)]
    for b in range(B):
        at = torch.randperm(V, generator=g)[:300]
        x[b, at] = top[b] * torch.rand(300, generator=g)
        x[b, at[:20]] = top[b] - 0.4 * torch.rand(20, generator=g)
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,V", [(200, 9001), (300, 9001), (30, 152064)])
def test_nuclei_at_low_temperatures(B, V, dtype):
    print(f"[case] low temperature nuclei B={B} V={V} {dtype}", flush=True)
    g = torch.Generator().manual_seed(B + V)
    x = hot_rows(B, V, dtype, g)
    T, p = settings([0.02, 0.05, 0.07, 0.1, 0.12, 0.15], B, g), settings([0.5, 0.7, 0.95], B, g)
    draw(x, torch.rand(B, generator=g), T=T, p=p)
    draw(x, torch.rand(B, generator=g), T=T, p=p, k=settings([0, 500, 2000, 30], B, g, torch.int32))


@pytest.mark.parametrize("B,V", [(5, 9001), (300, 9001), (3, 152064)])
@pytest.mark.parametrize("top", [-10.0, 0.0, 1.5, 12.0])
def test_unfiltered_bf16_rows_around_the_lowest_temperature_of_the_table(top, B, V):
    """Where (128 - the largest logit) log2 e / T crosses 1000 the weights are not taken from a table any more."""
    print(f"[case] table's lowest temperature, top {top}, B={B} V={V}", flush=True)
    g = torch.Generator().manual_seed(B + V)
    x = top - 3.0 * torch.rand(B, V, generator=g)
    edge = (128.0 - top) * math.log2(math.e) / 1000.0
    T = edge * settings([0.5, 0.9, 0.97, 0.99, 1.0, 1.01, 1.03, 1.2], B, g)
    draw(x.to(BF16), torch.rand(B, generator=g), T=T)


@pytest.mark.parametrize("T", [1e-3, 3e-4, 1e-4, 5e-5, 1e-5])
def test_fp32_nuclei_next_to_0(T):
    """Logits on both sides of 2^-10, the end of the bin of 0, at temperatures that tell them apart."""
    print(f"[case] nuclei next to 0, T={T}", flush=True)
    g = torch.Generator().manual_seed(int(1 / T))
    B, V = 40, 5001
    x = torch.full((B, V), -1.0)
    at = torch.randperm(V, generator=g)[:600]
    x[:, at] = (torch.rand(B, 600, generator=g) * 2.4 - 1.2) * 2.0 ** -10
    p = settings([0.3, 0.5, 0.7, 0.95], B, g)
    draw(x, torch.rand(B, generator=g), T=torch.full((B,), T), p=p)
    draw(x, torch.rand(B, generator=g), T=torch.full((B,), T), p=p, k=torch.full((B,), 550, dtype=torch.int32))


@pytest.mark.parametrize("T", [0.1, 0.02, 0.01, 1e-3, 1e-5])
def test_fp32_nuclei_of_negative_logits(T):
    """Rows with nothing above 0, as of log-probabilities, whose largest logit is up to 10^7 temperatures below it."""
    print(f"[case] nuclei of negative logits, T={T}", flush=True)
    g = torch.Generator().manual_seed(int(1 / T))
    B, V = 40, 5001
    top = -torch.logspace(-1, 2.09, B)
    x = top[:, None] * (1.5 + torch.rand(B, V, generator=g))
    for b in range(B):
        at = torch.randperm(V, generator=g)[:500]
        x[b, at] = top[b] - 6 * T * torch.rand(500, generator=g)
    x[0, :2], x[1, :2] = torch.tensor([-100.49, -100.5]), torch.tensor([-7.99, -8.0])
    x[:2, 2:] = -130.0
    p = settings([0.3, 0.5, 0.7, 0.95], B, g)
    draw(x, torch.rand(B, generator=g), T=torch.full((B,), T), p=p)
    draw(x, torch.rand(B, generator=g), T=torch.full((B,), T), p=p, k=torch.full((B,), 450, dtype=torch.int32))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,V", [(6, 9001), (300, 9001), (4, 152064)])
def test_masks_that_leave_low_logits_outside_the_first_tiles(B, V, dtype):
    """Nothing is left in the first quarter of every 2048 logits, and what is left lies on both sides of -128."""
    print(f"[case] low logits outside the first tiles B={B} V={V} {dtype}", flush=True)
    g = torch.Generator().manual_seed(B + V)
    x = torch.full((B, V), -math.inf)
    for b in range(B):
        at = 2048 * torch.randint(V // 2048, (8,), generator=g) + 600 + torch.randint(1400, (8,), generator=g)
        x[b, at] = -120.0 - 24.0 * torch.rand(8, generator=g)
    T = settings([1.0, 2.0, 5.0, 20.0], B, g)
    draw(x.to(dtype), torch.rand(B, generator=g), T=T)


def far_rows(V, dtype, g):
    """Rows whose largest logit is many temperatures away from 0, on either side, and rows with masks that are not masked for the kernels, each
    with the temperature to use: [(T, rows)]."""
    noise = lambda n, scale=1.0: scale * torch.randn(n, V, generator=g)
    rows = []
    for T, m in ((1e-6, 9999.0), (1e-6, -300.0), (1e-4, 777777.0), (1e-4, -777777.0), (1.0, -1e10), (1.0, 1e10), (1.0, -3e9), (0.7, 1.5e9), (2.0, 3e38), (1e-6, -1e29)):
        x = m + noise(3)
        x[1, V // 3:] = m - abs(m) * 1e-3                       # most of the row clearly lower
        x[2] = m                                                # all the same
        rows.append((T, x))
    for fill in (-1e9, -1e10, -2.5e10, -1e15, -1e20, -9.9e29):
        x = noise(3, 3.0)
        x[0, : V // 2] = fill                                   # long runs: lanes that see nothing else for a while or at all
        x[1, V // 4:] = fill
        x[2, torch.rand(V, generator=g) < 0.97] = fill
        rows.append((1.0, x))
    return [(T, x.to(dtype)) for T, x in rows]


def check(got, want, bound, what):
    got = got.double().cpu()
    bad = ~((got == want) | ((got - want).abs() <= bound))      # (equal infinities)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[0].tolist(), float(got[bad][0]), float(want[bad][0]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [5, 3001, 140001])
def test_logits_many_temperatures_from_0(V, dtype):
    g = torch.Generator().manual_seed(V)
    half = torch.finfo(dtype).eps / 2
    for i, (T, x) in enumerate(far_rows(V, dtype, g)):
        print(f"[case] far logits {i} T={T} V={V} {dtype}", flush=True)
        N = 3
        tokens = torch.tensor([V - 1, 0, V // 2], dtype=torch.int32)
        gpu = padded(x)
        f = R.softmax_rows(x.double(), T, tokens)
        n = espo.espo_logprobs_workspace_bytes(N, V, dtype)
        for ws in ([None, torch.full((n,), 0xCD, dtype=torch.uint8, device="cuda")] if n else [None]):
            lp, H, stats = (torch.full((m,), math.nan, device="cuda") for m in (N, N, 2 * N))
            espo.espo_logprobs(gpu, T, tokens.cuda(), lp, entropy=H, stats=stats, workspace=ws)
            want = f["logprob"]
            want = torch.where(want < -torch.finfo(F32).max, -math.inf, want)
            check(lp, want, R.logprob_bound(f, V), "logprob")
            check(H, f["entropy"], R.entropy_bound(f, V), "entropy")
            espo.espo_logprobs(gpu, T, tokens.cuda(), lp, workspace=ws)
            check(lp, want, R.logprob_bound(f, V), "logprob alone")
        dlp, dH = torch.randn(N, generator=g), torch.randn(N, generator=g)
        for h in (None, dH):
            d = padded(torch.full_like(x, 5.0))
            espo.espo_logprobs_backward(gpu, T, tokens.cuda(), stats, dlp.cuda(), d, entropy=None if h is None else H,
                                        dentropy=None if h is None else h.cuda())
            hh = torch.zeros(N).double() if h is None else h.double()
            ref = R.logits_grad(f, dlp.double(), hh)
            check(d, ref, R.grad_bound(f, dlp.double(), hh, ref, half, V), "gradient")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,V,coef,which", [(9, 3001, 0.01, range(16)), (9, 3001, 0.0, range(16)), (1032, 3001, 0.01, range(0, 16, 3)), (1032, 3001, 0.0, range(0, 16, 3)),
                                            (264, 40001, 0.01, (1, 4, 11))])
def test_policy_loss_of_logits_many_temperatures_from_0(N, V, coef, which, dtype):
    """The rows between others, in batches that are read twice and in ones whose rows are held."""
    g = torch.Generator().manual_seed(N)
    half = torch.finfo(dtype).eps / 2
    for i, (T, far) in enumerate(far_rows(V, dtype, g)):
        if i not in which:
            continue
        print(f"[case] policy loss of far logits {i} T={T} N={N} V={V} {dtype}", flush=True)
        x = (3.0 * T * torch.randn(N, V, generator=g)).to(dtype)
        at = torch.randperm(N, generator=g)[:3]
        x[at] = far
        tokens = x.float().argmax(1).to(torch.int32)
        f = R.softmax_rows(x.double(), T, tokens)
        old, adv = f["logprob"].float() - 0.1, torch.randn(N, generator=g)
        ones = torch.ones(N).double()
        gg, h, sums, c = R.policy_terms(f, old.double(), adv.double(), ones, 1.0 / N, 0.2, 0.2, coef)
        out = torch.zeros(espo.POLICY_RESULT_BYTES, dtype=torch.uint8, device="cuda")
        ws = torch.full((espo.espo_policy_loss_workspace_bytes(N, V, dtype),), 0xCD, dtype=torch.uint8, device="cuda")
        lp, H = torch.full((N,), math.nan, device="cuda"), torch.full((N,), math.nan, device="cuda")
        gpu = padded(x)
        whole = torch.full((N, gpu.stride(0)), 5.0, dtype=dtype, device="cuda")
        d = whole[:, :V]
        espo.espo_policy_loss(gpu, T, tokens.cuda(), old.cuda(), adv.cuda(), out, ws, dlogits=d, logprob=lp, entropy=H, entropy_coef=coef,
                              scale=1.0 / N)
        check(lp, f["logprob"], R.logprob_bound(f, V), "logprob")
        check(H, f["entropy"], R.entropy_bound(f, V), "entropy")
        ref = R.logits_grad(f, gg, h)
        # the ratio carries the log-probability's error and its own four roundings, relative to g
        rel = (R.logprob_bound(f, V) + 8 * R.U)[:, None]
        check(d, ref, R.grad_bound(f, gg, h, ref, half, V) + rel * gg.abs()[:, None] * 2 / T, "gradient")
        assert (whole[:, V:] == 5.0).all()
        res = espo.read_policy_result(out)
        lpb, Hb = R.logprob_bound(f, V) + 8 * R.U, R.entropy_bound(f, V)
        # weights are a product of two roundings, the sum is rounded to fp32 once
        err = (c["w"] * (lpb * c["r"] * c["A"].abs() * 2 + coef * Hb)).sum() + 4 * R.U * (c["w"] * (1 + c["r"] * c["A"].abs() + f["entropy"])).sum()
        assert abs(res["loss"] - float(sums[0])) <= float(err) and res["tokens"] == N


@pytest.mark.parametrize("N", [4, 1024])
def test_weight_0_takes_a_token_out_whose_probability_is_0(N):
    """A token that the new policy's mask rules out has r = 0 and ln r = -inf; with weight 0 it adds nothing to any sum."""
    print(f"[case] policy loss, weight 0 and a masked token, N={N}", flush=True)
    V = 2000
    g = torch.Generator().manual_seed(N)
    x = torch.randn(N, V, generator=g)
    tokens = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    x[1, int(tokens[1])] = -math.inf
    x[3, int(tokens[3])] = -1e30
    weights = torch.ones(N)
    weights[1] = weights[3] = 0.0
    f = R.softmax_rows(x.double(), 1.0, tokens)
    old = torch.where(torch.isinf(f["logprob"]), -3.0, f["logprob"]).float() + 0.05
    adv = torch.randn(N, generator=g)
    rest = torch.tensor([n for n in range(N) if n not in (1, 3)])
    part = {k: v[rest] if isinstance(v, torch.Tensor) else v for k, v in f.items()}
    _, _, sums, c = R.policy_terms(part, old[rest].double(), adv[rest].double(), torch.ones(N - 2).double(), 1.0 / N, 0.2, 0.2, 0.01)
    out = torch.zeros(espo.POLICY_RESULT_BYTES, dtype=torch.uint8, device="cuda")
    ws = torch.zeros(espo.espo_policy_loss_workspace_bytes(N, V, F32), dtype=torch.uint8, device="cuda")
    d = torch.full((N, V), 3.0, device="cuda")
    espo.espo_policy_loss(x.cuda(), 1.0, tokens.cuda(), old.cuda(), adv.cuda(), out, ws, dlogits=d, weights=weights.cuda(), entropy_coef=0.01,
                          scale=1.0 / N)
    res = espo.read_policy_result(out)
    assert (d[1] == 0).all() and (d[3] == 0).all() and res["tokens"] == N
    lpb, Hb = R.logprob_bound(part, V) + 8 * R.U, R.entropy_bound(part, V)
    err = [(c["w"] * (lpb * c["r"] * c["A"].abs() * 2 + 0.01 * Hb)).sum(), (c["w"] * lpb * c["r"] * c["A"].abs() * 2).sum(), (c["w"] * Hb).sum(),
           (c["w"] * lpb * (1 + c["r"] + c["d"].abs())).sum()]
    for name, s, e in zip(("loss", "policy", "entropy", "kl"), sums, err):
        # weights are a product of two roundings; the sums are rounded to fp32 once
        assert abs(res[name] - float(s)) <= float(e) + 4 * R.U * float((c["w"] * (1 + c["r"] * c["A"].abs() + part["entropy"] + c["d"].abs())).sum()), name
