"""espo_logprobs, its backward pass and espo_policy_loss against the definitions in 64 bits (needs an MI355X)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import rows_reference as R  # noqa: E402
import paper_2605_29860_amd as espo  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def make(N, V, dtype, seed, pad=0, unused=0.2, masked=0.0, scale=3.0):
    """Logits with a row pitch of at least V + pad, tokens (some rows unused, their logits NaN), and the logits on the CPU."""
    g = torch.Generator().manual_seed(seed)
    E = 8 if dtype == BF16 else 4
    pitch = -(-(V + pad) // E) * E
    buf = torch.full((N, pitch), 7.0, dtype=dtype)
    buf[:, :V] = torch.randn(N, V, generator=g) * scale
    if masked:
        hide = torch.rand(N, V, generator=g) < masked
        fill = torch.where(torch.rand(N, V, generator=g) < 0.5, -math.inf, torch.finfo(dtype).min).to(dtype)
        buf[:, :V] = torch.where(hide, fill, buf[:, :V])
    tokens = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    off = torch.rand(N, generator=g) < unused
    if N > 1:
        off[0], off[1] = False, unused > 0
    tokens[off] = torch.where(torch.rand(int(off.sum()), generator=g) < 0.5, -1, V).int()
    buf[off, :V] = math.nan
    return buf.cuda()[:, :V], tokens.cuda(), buf[:, :V].double(), tokens, g


def pitched(x, fill=5.0):
    """A tensor of x's type and shape with the same pitch, and its whole buffer."""
    buf = torch.full((x.shape[0], x.stride(0)), fill, dtype=x.dtype, device=x.device)
    return buf[:, :x.shape[1]], buf


def check(got, want, bound, what):
    got = got.double().cpu()
    same_inf = torch.isinf(want) & (got == want)
    err = torch.where(same_inf, 0.0, (got - want).abs())
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(err[bad][0]), bad.nonzero()[0].tolist())


def workspace(size, N, V, dtype):
    n = size(N, V, dtype)
    return torch.full((n,), 0xCD, dtype=torch.uint8, device="cuda") if n else None


def forward(x, tokens, T, entropy=True):
    N, V = x.shape
    out = [torch.full((n,), math.nan, device="cuda") for n in (N, N, 2 * N)]
    espo.espo_logprobs(x, T, tokens, out[0], entropy=out[1] if entropy else None, stats=out[2],
                       workspace=workspace(espo.espo_logprobs_workspace_bytes, N, V, x.dtype))
    return out


def check_all(N, V, dtype, T, seed, **kw):
    x, tokens, x64, tok, g = make(N, V, dtype, seed, **kw)
    f = R.softmax_rows(x64, T, tok)
    lp, H, stats = forward(x, tokens, T)
    check(lp, f["logprob"], R.logprob_bound(f, V), "logprob")
    check(H, f["entropy"], R.entropy_bound(f, V), "entropy")
    lp2, _, _ = forward(x, tokens, T, entropy=False)
    check(lp2, f["logprob"], R.logprob_bound(f, V), "logprob alone")
    dlp, dH = torch.randn(N, generator=g), torch.randn(N, generator=g)
    half = torch.finfo(dtype).eps / 2
    for h in (None, dH):
        d, buf = pitched(x)
        espo.espo_logprobs_backward(x, T, tokens, stats, dlp.cuda(), d, entropy=H if h is not None else None,
                                    dentropy=h.cuda() if h is not None else None)
        hh = torch.zeros(N).double() if h is None else h.double()
        want = R.logits_grad(f, dlp.double(), hh)
        check(d, want, R.grad_bound(f, dlp.double(), hh, want, half, V), "gradient")
        assert (buf[:, V:] == 5.0).all()
    copy, whole = pitched(x)
    whole.copy_(x.as_strided(whole.shape, whole.stride()))
    espo.espo_logprobs_backward(copy, T, tokens, stats, dlp.cuda(), copy, entropy=H, dentropy=dH.cuda())
    assert torch.equal(copy.float(), d.float())             # in place: the same bits
    return f, x, tokens, x64, tok, g


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,V,T", [(1, 1, 1.0), (3, 2, 0.5), (2, 7, 1.0), (5, 8, 2.0), (4, 9, 1.0), (3, 511, 1.0), (2, 4096, 0.6), (5, 4099, 1.0),
                                   (3, 16383, 1.3), (2, 16385, 0.6), (7, 32768, 1.0), (3, 50003, 0.3), (2, 152064, 0.6), (300, 1000, 1.0),
                                   (600, 2049, 1.0)])
def test_shapes(N, V, T, dtype):
    print(f"[case] logprobs N={N} V={V} T={T} {dtype}", flush=True)
    check_all(N, V, dtype, T, seed=N * 7 + V, pad=0 if V % 2 else 24)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1e-6, 1e-3, 0.1, 50.0, 1e6, 1e20])
def test_temperatures(T, dtype):
    print(f"[case] logprobs temperature {T} {dtype}", flush=True)
    check_all(4, 3001, dtype, T, seed=5)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shift", [1000.0, -5000.0, -1e6])
def test_shifted_and_wide_logits(shift, dtype):
    print(f"[case] logprobs shifted {shift} {dtype}", flush=True)
    V, T = 5003, 0.7
    x, tokens, x64, tok, g = make(5, V, dtype, 17, unused=0.0, scale=30.0)
    x += shift
    x[3] = torch.linspace(-90, 90, V).to(dtype).cuda()          # every part of the row has a larger logit than the one before
    x[4] = torch.linspace(90, -90, V).to(dtype).cuda()
    f = R.softmax_rows(x.double().cpu(), T, tok)
    lp, H, stats = forward(x, tokens, T)
    check(lp, f["logprob"], R.logprob_bound(f, V), "logprob")
    check(H, f["entropy"], R.entropy_bound(f, V), "entropy")
    w = torch.randn(5, generator=g)
    d, _ = pitched(x)
    espo.espo_logprobs_backward(x, T, tokens, stats, w.cuda(), d, entropy=H, dentropy=w.cuda())
    want = R.logits_grad(f, w.double(), w.double())
    check(d, want, R.grad_bound(f, w.double(), w.double(), want, torch.finfo(dtype).eps / 2, V), "gradient")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,masked", [(40, 0.5), (5000, 0.9), (20011, 0.999)])
def test_masked_vocabulary(V, masked, dtype):
    print(f"[case] logprobs masked {masked} V={V} {dtype}", flush=True)
    check_all(9, V, dtype, 0.8, seed=11, masked=masked)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_without_any_logit_and_masked_tokens(dtype):
    print(f"[case] logprobs empty rows {dtype}", flush=True)
    N, V = 4, 777
    x, _, _, _, _ = make(N, V, dtype, 3, unused=0.0)
    x[0] = -math.inf
    x[1] = torch.finfo(dtype).min
    x[2, 5] = -math.inf                                      # the token itself is masked
    x[3, 1:] = -math.inf                                     # one logit is all there is
    tokens = torch.tensor([3, 4, 5, 0], dtype=torch.int32, device="cuda")
    lp, H, stats = forward(x, tokens, 1.0)
    assert lp.tolist()[:3] == [-math.inf] * 3 and lp[3] == 0 and H[0] == 0 and H[1] == 0 and H[3] == 0 and H[2] > 0
    d, _ = pitched(x)
    one = torch.ones(N, device="cuda")
    espo.espo_logprobs_backward(x, 1.0, tokens, stats, one, d, entropy=H, dentropy=one)
    assert torch.isfinite(d.float()).all() and (d[:2] == 0).all() and d[2, 5] == 0 and (d[3, 1:] == 0).all() and abs(float(d[3, 0])) < 1e-6
    f = R.softmax_rows(x.double().cpu(), 1.0, tokens.cpu())
    want = R.logits_grad(f, one.double().cpu(), one.double().cpu())
    check(d, want, R.grad_bound(f, one.double().cpu(), one.double().cpu(), want, torch.finfo(dtype).eps / 2, V), "gradient")


def test_gradient_against_differences():
    print("[case] logprobs differences", flush=True)
    N, V, T, step = 6, 37, 0.7, 2.0 ** -6
    x, tokens, _, _, g = make(N, V, F32, 9, unused=0.0, scale=1.0)
    gl, gh = torch.randn(N, generator=g).cuda(), torch.randn(N, generator=g).cuda()
    lp, H, stats = forward(x, tokens, T)
    d, _ = pitched(x)
    espo.espo_logprobs_backward(x, T, tokens, stats, gl, d, entropy=H, dentropy=gh)
    got = torch.zeros(N, V, device="cuda")
    for v in range(V):
        side = []
        for s in (step, -step):
            y, buf = pitched(x)
            buf.zero_()
            y.copy_(x)
            y[:, v] += s
            a, b, _ = forward(y, tokens, T)
            side.append(gl.double() * a.double() + gh.double() * b.double())
        got[:, v] = ((side[0] - side[1]) / (2 * step)).float()
    # central differences: third derivatives of ln pi and H over T^3 stay below 2 |g| and 8 |h| (|ln pi| <= 10 here), so the
    # error is below step^2 / 6 * (2 |g| + 8 |h|) / T^3; both sides carry forward errors of at most 1e-6 (|g| + |h|) / step
    size = gl.abs() + 4 * gh.abs()
    bound = step ** 2 / 3 * size / T ** 3 + 2e-6 * size / step
    assert ((got - d).abs() <= bound[:, None]).all(), float((got - d).abs().max())


def loss_inputs(f, N, g, spread=0.15):
    old = torch.where(torch.isinf(f["logprob"]), -5.0, f["logprob"]).float() + spread * torch.randn(N, generator=g)
    return old, torch.randn(N, generator=g), torch.rand(N, generator=g)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,V,T,coef,weighted", [(1, 5, 1.0, 0.0, False), (7, 4096, 1.0, 0.01, True), (40, 50003, 0.6, 0.0, True), (300, 1003, 1.0, 0.02, False),
                                                 (257, 33000, 1.0, 0.5, False), (260, 70001, 1.0, 0.0, True), (256, 152064, 0.8, 0.01, False),
                                                 (1500, 9, 1.0, 0.1, True), (530, 82001, 0.9, 0.0, False), (600, 8192, 1.0, 0.01, False), (192, 38912, 1.0, 0.0, True), (260, 19457, 1.0, 0.01, False), (450, 38912, 1.0, 0.0, True), (110, 140001, 1.0, 0.01, False),
                                                 (210, 77825, 1.0, 0.0, False), (700, 19457, 1.0, 0.01, True),
                                                 (1100, 5121, 1.0, 0.01, False)])
def test_policy_loss(N, V, T, coef, weighted, dtype):
    print(f"[case] policy loss N={N} V={V} T={T} coef={coef} {dtype}", flush=True)
    x, tokens, x64, tok, g = make(N, V, dtype, N + V, pad=8)
    f = R.softmax_rows(x64, T, tok)
    old, adv, weights = loss_inputs(f, N, g)
    lo, hi = 0.2, 0.28
    # a row whose ratio lies within the log-probability's error of an end of the clip range may fall on either side: move it
    near = sum(((f["logprob"] - old.double()).exp() - b).abs() < 1e-4 for b in (1 - lo, 1 + hi)) > 0
    old[near] += 0.01
    poison = lambda t: torch.where(f["used"], t, math.nan).cuda()
    gg, h, sums, c = R.policy_terms(f, old.double(), adv.double(), weights.double() if weighted else torch.ones(N).double(), 1.0 / N, lo, hi, coef)
    out = torch.full((espo.POLICY_RESULT_BYTES,), 0xAB, dtype=torch.uint8, device="cuda")
    ws = workspace(espo.espo_policy_loss_workspace_bytes, N, V, dtype)
    lp, H = torch.full((N,), math.nan, device="cuda"), torch.full((N,), math.nan, device="cuda")
    d, buf = pitched(x)
    call = lambda x, d, **kw: espo.espo_policy_loss(x, T, tokens, poison(old), poison(adv), out, ws, dlogits=d,
                                                    weights=poison(weights) if weighted else None, clip_low=lo, clip_high=hi, entropy_coef=coef,
                                                    scale=1.0 / N, **kw)
    call(x, d, logprob=lp, entropy=H)
    check(lp, f["logprob"], R.logprob_bound(f, V), "logprob")
    check(H, f["entropy"], R.entropy_bound(f, V), "entropy")
    # the ratio carries the log-probability's error and its own four roundings: relative to g
    want = R.logits_grad(f, gg, h)
    rel = (R.logprob_bound(f, V) + 8 * R.U)[:, None]
    check(d, want, R.grad_bound(f, gg, h, want, torch.finfo(dtype).eps / 2, V) + rel * gg.abs()[:, None] * 2 / T, "gradient")
    assert (buf[:, V:] == 5.0).all()
    res = espo.read_policy_result(out)
    assert res["tokens"] == int(f["used"].sum())
    lpb, Hb = R.logprob_bound(f, V) + 8 * R.U, R.entropy_bound(f, V)
    err = [(c["w"] * (lpb * c["r"] * c["A"].abs() * 2 + coef * Hb)).sum(), (c["w"] * lpb * c["r"] * c["A"].abs() * 2).sum(), (c["w"] * Hb).sum(),
           (c["w"] * lpb * (1 + c["r"] + c["d"].abs())).sum(), 0.0]
    def check_sums(res):
        for name, s, e in zip(("loss", "policy", "entropy", "kl", "clipped"), sums, err):
            # weights are a product of two roundings; the sums are rounded to fp32 once
            assert abs(res[name] - float(s)) <= float(e) + 4 * R.U * float((c["w"] * (1 + c["r"] * c["A"].abs() + f["entropy"] + c["d"].abs())).sum()), (name, res[name], float(s))

    check_sums(res)
    first = (res, d.clone())
    # without the optional outputs, and in place: the same bits
    copy, whole = pitched(x)
    whole.copy_(x.as_strided(whole.shape, whole.stride()))
    call(copy, copy)
    assert torch.equal(copy.float(), first[1].float()) and espo.read_policy_result(out) == res
    call(x, None)                                              # the loss alone: the rows' sums may be formed in another order
    check_sums(espo.read_policy_result(out))


def test_policy_loss_of_no_rows_and_of_unused_rows():
    print("[case] policy loss empty", flush=True)
    zero = dict(loss=0.0, policy=0.0, entropy=0.0, kl=0.0, clipped=0.0, tokens=0)
    out = torch.full((espo.POLICY_RESULT_BYTES,), 0xAB, dtype=torch.uint8, device="cuda")
    ws = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    f = torch.zeros(0, device="cuda")
    espo.espo_policy_loss(torch.zeros(0, 16, device="cuda"), 1.0, f.int(), f, f, out, ws)
    assert espo.read_policy_result(out) == zero
    x = torch.full((5, 64), math.nan, device="cuda")
    d = torch.full_like(x, 3.0)
    nan = torch.full((5,), math.nan, device="cuda")
    out.fill_(0xAB)
    espo.espo_policy_loss(x, 1.0, torch.full((5,), -1, dtype=torch.int32, device="cuda"), nan, nan, out, ws, dlogits=d, weights=nan, entropy_coef=0.1)
    assert espo.read_policy_result(out) == zero and (d == 0).all()


def test_extreme_ratios_stay_finite():
    print("[case] policy loss extreme ratios", flush=True)
    x = torch.zeros(4, 64, device="cuda")
    x[1, 3] = -math.inf                                      # the token has become impossible: ratio 0
    tokens = torch.full((4,), 3, dtype=torch.int32, device="cuda")
    old = torch.tensor([-500.0, -1.0, -500.0, 500.0], device="cuda")
    adv = torch.tensor([1.0, -1.0, 0.0, 1.0], device="cuda")
    out = torch.zeros(espo.POLICY_RESULT_BYTES, dtype=torch.uint8, device="cuda")
    ws = workspace(espo.espo_policy_loss_workspace_bytes, 4, 64, F32)
    d = torch.full_like(x, 3.0)
    espo.espo_policy_loss(x, 1.0, tokens, old, adv, out, ws, dlogits=d)
    assert torch.isfinite(d).all()
    r = espo.read_policy_result(out)
    # -1.2 (clipped above), 0.8 (clipped below: A < 0), 0, and a ratio of e^-504
    assert r["policy"] == pytest.approx(-1.2 + 0.8, rel=1e-6) and r["clipped"] == 3.0 and r["tokens"] == 4
    assert (d[0] == 0).all() and (d[1] == 0).all() and (d[2] == 0).all()


def test_captured_and_replayed():
    print("[case] logprobs graph", flush=True)
    N, V, T = 20, 5001, 0.7
    x, tokens, x64, tok, g = make(N, V, BF16, 21)
    f = R.softmax_rows(x64, T, tok)
    old, adv, _ = (t.cuda() for t in loss_inputs(f, N, g))
    lp, H, stats = torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda"), torch.zeros(2 * N, device="cuda")
    d, _ = pitched(x)
    d2, _ = pitched(x)
    out = torch.zeros(espo.POLICY_RESULT_BYTES, dtype=torch.uint8, device="cuda")
    ws, ws2 = workspace(espo.espo_logprobs_workspace_bytes, N, V, BF16), workspace(espo.espo_policy_loss_workspace_bytes, N, V, BF16)

    def calls():
        espo.espo_logprobs(x, T, tokens, lp, entropy=H, stats=stats, workspace=ws)
        espo.espo_logprobs_backward(x, T, tokens, stats, adv, d, entropy=H, dentropy=old)
        espo.espo_policy_loss(x, T, tokens, old, adv, out, ws2, dlogits=d2, entropy_coef=0.01, scale=0.1)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        calls()
    rows = x.as_strided((N, x.stride(0)), x.stride())
    for turn in range(4):
        rows[:, :V] = (torch.randn(N, V, generator=g) * 3).cuda().to(BF16)
        adv.copy_(torch.randn(N, generator=g))
        calls()
        torch.cuda.synchronize()
        want = [t.clone() for t in (lp, H, d, d2, out)]
        for t in (lp, H, stats, d, d2, out):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (lp, H, d, d2, out)):
            assert torch.equal(a, b), turn


def test_another_stream_and_results_that_repeat():
    print("[case] logprobs stream", flush=True)
    N, V = 300, 33001
    x, tokens, _, _, _ = make(N, V, BF16, 31, unused=0.0)
    a = [t.clone() for t in forward(x, tokens, 1.0)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = [torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda")]
    torch.cuda.synchronize()
    espo.espo_logprobs(x, 1.0, tokens, out[0], entropy=out[1], workspace=workspace(espo.espo_logprobs_workspace_bytes, N, V, BF16), stream=s)
    s.synchronize()
    assert torch.equal(out[0], a[0]) and torch.equal(out[1], a[1])


def test_row_offsets_beyond_32_bits():
    print("[case] logprobs far rows", flush=True)
    N, V, pitch = 6, 1000, 1 << 30                           # bf16: rows 2 GiB apart, the last 10 GiB from the first
    buf = torch.empty(5 * pitch + 1008, dtype=BF16, device="cuda")
    x = buf.as_strided((N, V), (pitch, 1))
    small, tokens, x64, tok, g = make(N, V, BF16, 41, unused=0.0)
    x.copy_(small)
    lp, H, stats = forward(x, tokens, 1.0)
    a, b, _ = forward(small, tokens, 1.0)
    assert torch.equal(lp, a) and torch.equal(H, b)
    w = torch.randn(N, generator=g).cuda()
    d, _ = pitched(small)
    espo.espo_logprobs_backward(small, 1.0, tokens, stats, w, d)
    espo.espo_logprobs_backward(x, 1.0, tokens, stats, w, x)
    assert torch.equal(x.float(), d.float())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_few_long_rows_split_with_a_workspace(dtype):
    for N, V in ((1, 152064), (3, 140001), (32, 152064), (60, 131072), (5, 1 << 20)):
        print(f"[case] logprobs split N={N} V={V} {dtype}", flush=True)
        x, tokens, x64, _, _ = make(N, V, dtype, seed=N + V, masked=0.1, pad=5)
        tokens[0] = V - 1
        if N > 1:
            tokens[N // 2] = -1
        n = espo.espo_logprobs_workspace_bytes(N, V, dtype)
        assert n > 0
        ws = torch.full((n + 16,), 0xFF, dtype=torch.uint8, device="cuda")
        out = lambda: [torch.full((N,), math.nan, device="cuda") for _ in range(2)] + [torch.full((2 * N,), math.nan, device="cuda")]
        whole, split, offset = out(), out(), out()
        espo.espo_logprobs(x, 0.8, tokens, whole[0], entropy=whole[1], stats=whole[2])
        espo.espo_logprobs(x, 0.8, tokens, split[0], entropy=split[1], stats=split[2], workspace=ws[:n])
        espo.espo_logprobs(x, 0.8, tokens, offset[0], entropy=offset[1], stats=offset[2], workspace=ws[4:])   # misaligned: not used
        assert all(torch.equal(a, b) for a, b in zip(whole, offset)) and (ws[n:] == 0xFF).all()
        f = R.softmax_rows(x64, 0.8, tokens.cpu())
        for got in (whole, split):
            check(got[0], f["logprob"], R.logprob_bound(f, V), "logprob")
            check(got[1], f["entropy"], R.entropy_bound(f, V), "entropy")
        assert torch.equal(whole[2][0::2], split[2][0::2])     # the maximum is the same number
        alone = torch.full((N,), math.nan, device="cuda")
        espo.espo_logprobs(x, 0.8, tokens, alone, workspace=ws)
        check(alone, f["logprob"], R.logprob_bound(f, V), "logprob without the entropy")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_policy_loss_of_few_long_rows(dtype):
    test_policy_loss(20, 152064, 0.9, 0.01, True, dtype)


def test_rows_that_do_not_fit_are_refused():
    x, tokens, out = torch.zeros(4, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    espo.espo_logprobs(x, 1.0, tokens, out)
    for bad in (x.t(), x[0], x.cpu(), x[:, ::2]):
        with pytest.raises(TypeError):
            espo.espo_logprobs(bad, 1.0, tokens, out)
    with pytest.raises(espo.EspoError):
        espo.espo_logprobs(x, 1.0, tokens, out, V=65)
    with pytest.raises(espo.EspoError):
        espo.espo_logprobs(x, 1.0, tokens, out, V=-1)
    with pytest.raises(ValueError):
        espo.espo_logprobs(torch.zeros(5, 64, device="cuda"), 1.0, tokens, out)
    espo.espo_logprobs(x[:1, :63], 1.0, tokens, out)            # a single row's stride does not matter
    assert abs(float(out[0]) + math.log(63)) < 1e-6 and (out[1:] + math.log(64)).abs().max() < 1e-6
