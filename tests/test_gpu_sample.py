"""espo_sample against its definition in 64 bits (needs an MI355X).

Tokens have to be equal.  Sums of V doubles in any order differ by less than V * 2^-53 of the total and the weights by a
few 2^-53 * |t|, together below 1e-10 for the sizes here; a case whose u comes closer than that to a running sum would
not decide anything, and `run` says so.  logprob is a double rounded to fp32: half a step, and 1e-9 for the sums."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import rows_reference as R  # noqa: E402
import paper_2605_29860_amd as espo  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def logits(B, V, dtype, seed, pad=0, scale=3.0, masked=0.0, grid=None):
    g = torch.Generator().manual_seed(seed)
    E = 8 if dtype == BF16 else 4
    buf = torch.full((B, -(-(V + pad) // E) * E), 50.0, dtype=dtype)     # beyond V: larger than any logit
    x = torch.randn(B, V, generator=g) * scale
    if grid:
        x = (x / grid).round() * grid
    if masked:
        fill = torch.where(torch.rand(B, V, generator=g) < 0.5, -math.inf, torch.finfo(dtype).min)
        x = torch.where(torch.rand(B, V, generator=g) < masked, fill, x)
    buf[:, :V] = x
    return buf.cuda()[:, :V], g


def run(x, u, T=None, k=None, p=None, min_p=None, alive=None, V=None):
    B = x.shape[0]
    n = espo.espo_sample_workspace_bytes(B, V or x.shape[1], x.dtype)
    ws = torch.full((n,), 0xCD, dtype=torch.uint8, device="cuda") if n else None
    dev = lambda t, dtype: None if t is None else torch.as_tensor(t, dtype=dtype).expand(B).contiguous().cuda()
    tokens, lp = torch.full((B,), -7, dtype=torch.int32, device="cuda"), torch.full((B,), math.nan, device="cuda")
    s = dict(temperature=dev(T, F32), top_k=dev(k, torch.int32), top_p=dev(p, F32), min_p=dev(min_p, F32), alive=dev(alive, torch.uint8))
    espo.espo_sample(x, u.cuda(), tokens, logprob=lp, V=V, workspace=ws, **s)
    again = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    espo.espo_sample(x, u.cuda(), again, V=V, **s)             # without the log-probability and without a workspace
    assert torch.equal(tokens, again)
    row = lambda t, b, off: off if t is None else float(t[b])
    x64 = x.double().cpu()
    for b in range(B):
        tok, want, near = R.sample_row(x64[b, :V], *(row(s[n], b, off) for n, off in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0))),
                                       float(u[b])) if alive is None or int(s["alive"][b]) else (-1, 0.0, 1.0)
        assert near > 1e-10, ("this input decides nothing", b, near)
        assert int(tokens[b]) == tok, (b, int(tokens[b]), tok)
        assert abs(float(lp[b]) - want) <= 2.0 ** -24 * abs(want) + 1e-9, (b, float(lp[b]), want)
    return tokens, lp


MODES = [dict(), dict(T=0.6), dict(k=5), dict(k=1), dict(p=0.7), dict(p=0.999), dict(min_p=0.1), dict(T=1.3, k=40, p=0.9), dict(T=0.7, k=300, p=0.95, min_p=0.02),
         dict(T=2.5, k=20000), dict(T=2.0, p=0.97, min_p=1e-4), dict(T=0.0)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("mode", range(len(MODES)))
def test_modes(mode, dtype):
    for B, V in ((5, 1000), (3, 33333), (2, 152064)):
        print(f"[case] sample {MODES[mode]} B={B} V={V} {dtype}", flush=True)
        x, g = logits(B, V, dtype, seed=mode * 100 + B, pad=9)
        run(x, torch.rand(B, generator=g), **MODES[mode])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 63, 64, 65, 511, 513, 1023, 4097, 8191, 16385, 65537, 131073])
def test_sizes(V, dtype):
    print(f"[case] sample V={V} {dtype}", flush=True)
    x, g = logits(6, V, dtype, seed=V)
    u = torch.rand(6, generator=g)
    run(x, u)
    run(x, u, T=0.8, k=3, p=0.9)
    run(x, u, p=0.5, min_p=0.01)
    run(x, u, k=V)                                             # at V and beyond the filter is off
    run(x, u, k=V - 1)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_row_its_own_settings(dtype):
    for B, V in ((64, 5003), (300, 2001), (33, 140001)):
        print(f"[case] sample mixed B={B} V={V} {dtype}", flush=True)
        x, g = logits(B, V, dtype, seed=B, masked=0.3)
        pick = lambda v: torch.tensor(v)[torch.randint(len(v), (B,), generator=g)]
        run(x, torch.rand(B, generator=g), T=pick([0.0, 0.5, 0.8, 1.0, 1.7, -1.0]), k=pick([0, -3, 1, 30, 200, V + 5]), p=pick([0.0, 1.0, 1.5, 0.3, 0.9, 0.99]),
            min_p=pick([0.0, -1.0, 0.05, 1.0, 7.0]), alive=pick([1, 1, 1, 0, 255]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("mode", [dict(), dict(k=7), dict(p=0.6), dict(T=0.5, k=50, p=0.8, min_p=0.01), dict(T=0.0), dict(k=400), dict(p=0.98)])
def test_ties(mode, dtype):
    print(f"[case] sample ties {mode} {dtype}", flush=True)
    x, g = logits(9, 3001, dtype, seed=77, grid=2.0)           # a dozen values, hundreds of tokens each
    x[1] = torch.where(x[1] == 0, torch.full_like(x[1], -0.0), x[1])   # both zeros are one value
    x[2, ::2] = torch.where(x[2, ::2] == 0, torch.full_like(x[2, ::2], -0.0), x[2, ::2])
    run(x, torch.rand(9, generator=g), **mode)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [8, 64, 1024, 65536])
def test_equal_logits_at_exact_borders(V, dtype):
    print(f"[case] sample equal V={V} {dtype}", flush=True)
    # equal logits: the running sums are whole numbers, u V too, and a sum equal to u V does not exceed it
    n = min(V, 64)
    at = torch.arange(n) * (V // n)
    x = torch.full((n, V), 1.5, dtype=dtype, device="cuda")
    tokens, lp = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    for mode in (dict(), dict(top_k=3), dict(top_p=0.5), dict(min_p=1.0)):
        s = {k: torch.full((n,), v, device="cuda", dtype=torch.int32 if k == "top_k" else F32) for k, v in mode.items()}
        espo.espo_sample(x, (at / V).cuda(), tokens, logprob=lp, **s)
        assert torch.equal(tokens.cpu(), at.int()), mode
        assert ((lp.cpu() + math.log(V)).abs() < 1e-6).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ends_of_the_range(dtype):
    print(f"[case] sample ends {dtype}", flush=True)
    V = 20001
    x, _ = logits(6, V, dtype, seed=5)
    x[:, 0] = -math.inf
    x[:, -1] = torch.finfo(dtype).min
    out = {}
    for name, u in (("first", 0.0), ("below", -0.5), ("last", 1.0 - 2.0 ** -24), ("beyond", 1.5)):
        tokens = torch.zeros(6, dtype=torch.int32, device="cuda")
        espo.espo_sample(x, torch.full((6,), u, device="cuda"), tokens)
        out[name] = tokens.cpu().tolist()
    assert out["first"] == [1] * 6 and out["below"] == [1] * 6 and out["beyond"] == [V - 2] * 6
    assert all(t <= V - 2 for t in out["last"])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_without_any_logit_and_with_one(dtype):
    print(f"[case] sample empty rows {dtype}", flush=True)
    for mode in MODES:
        x, g = logits(6, 4099, dtype, seed=8)
        x[0] = -math.inf
        x[1] = torch.finfo(dtype).min
        x[2, :-1] = -math.inf
        x[3, 1:] = -1e30
        x[4] = -math.inf
        x[4, 17] = -1e29                                       # far down, but not masked
        tokens, lp = run(x, torch.rand(6, generator=g), **mode)
        assert tokens[:5].tolist() == [-1, -1, 4098, 0, 17] and (lp[:5] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1e-6, 1e-2, 30.0, 1e8])
def test_temperatures(T, dtype):
    print(f"[case] sample temperature {T} {dtype}", flush=True)
    x, g = logits(5, 9001, dtype, seed=3)
    u = torch.rand(5, generator=g)
    run(x, u, T=T)
    run(x, u, T=T, k=60, p=0.5)
    run(x, u, T=T, p=0.9)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_wide_and_shifted_logits(dtype):
    print(f"[case] sample wide {dtype}", flush=True)
    x, g = logits(6, 6001, dtype, seed=4, scale=40.0)
    x[1] += 1000.0
    x[2] -= 5000.0
    x[3] = torch.linspace(-80, 80, 6001).to(dtype)             # rising: every part of the row has a larger logit than the one before
    x[4] = torch.linspace(80, -80, 6001).to(dtype)
    x[5, :3000] = -200.0
    u = torch.rand(6, generator=g)
    for mode in (dict(), dict(p=0.9), dict(k=100), dict(T=20.0, p=0.99), dict(T=20.0, k=2000, min_p=1e-3)):
        run(x, u, **mode)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,left", [(4099, 7), (4099, 350), (40001, 900), (40001, 1)])
def test_filters_over_fewer_logits_than_top_k(V, left, dtype):
    """A grammar's mask leaves `left` logits: a top-k beyond that is no filter, and the nucleus is of what is left."""
    print(f"[case] sample mask leaves {left} of {V} {dtype}", flush=True)
    x, g = logits(5, V, dtype, seed=left)
    for b in range(5):
        out = torch.randperm(V, generator=g)[left:].cuda()
        x[b, out] = [-math.inf, torch.finfo(dtype).min, -1e30][b % 3]
    u = torch.rand(5, generator=g)
    for k in (left, left + 1, left + 40, V - 1):
        run(x, u, k=k)
        run(x, u, T=0.8, k=k, p=0.9)
        run(x, u, k=k, min_p=0.05)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1.0, 4.0, 9.0])
def test_filters_around_128(T, dtype):
    print(f"[case] sample around 128, T={T} {dtype}", flush=True)
    x, g = logits(6, 5003, dtype, seed=31)
    x[0, ::2] = -128.0
    x[1, ::3] = -130.0 - torch.rand(1668, generator=g).to(dtype).cuda() * 20
    x[2] -= 300.0                                              # all of it beyond
    x[3, :40] += 135.0                                         # the maximum beyond on the other side
    x[4, ::2] = torch.linspace(-160, 100, 2502).to(dtype).cuda()
    x[5, 10:] = -200.0
    u = torch.rand(6, generator=g)
    for mode in (dict(k=5), dict(k=4000), dict(k=4000, p=0.99), dict(p=0.9), dict(p=0.9999), dict(k=300, p=0.8, min_p=0.01)):
        run(x, u, T=T, **mode)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("members", [400, 600, 1500, 2048, 2049, 6000])
def test_crowded_bins(members, dtype):
    """Many logits next to each other, from a run that is ranked to one that is not, above and below the others."""
    print(f"[case] sample {members} logits within 1 / 32 {dtype}", flush=True)
    V = 20001
    for B, level in ((3, 4.0), (260, -4.03125)):
        x, g = logits(B, V, dtype, seed=members, scale=1.0)
        at = torch.randperm(V, generator=g)[:members].cuda()
        x[:, at] = (level + torch.rand(B, members, generator=g) * 0.031).to(dtype).cuda()
        if B > 3:
            x[:, at[0]] = 9.0
        u = torch.rand(B, generator=g)
        keep = slice(0, 3)
        for mode in (dict(p=0.6), dict(k=300), dict(k=350, p=0.4), dict(k=V - members // 2), dict(k=V - members // 2, p=0.99), dict(p=0.9999)):
            s = {name: torch.full((B,), float(v), device="cuda") if name == "p" else torch.full((B,), v, dtype=torch.int32, device="cuda") for name, v in mode.items()}
            run(x[keep], u[keep], **mode)
            tokens, few = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B, 3))
            espo.espo_sample(x, u.cuda(), tokens, top_k=s.get("k"), top_p=s.get("p"))
            espo.espo_sample(x[keep], u[keep].cuda(), few, top_k=s["k"][keep] if "k" in s else None, top_p=s["p"][keep] if "p" in s else None)
            assert torch.equal(tokens[keep], few)              # 8 waves a row in large batches, 16 in small ones


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_longest_rows(dtype):
    print(f"[case] sample longest rows {dtype}", flush=True)
    for V, modes in ((1 << 19, (dict(), dict(k=60, p=0.9), dict(p=0.8), dict(T=3.0, k=30000, min_p=1e-4))), (1 << 20, (dict(), dict(T=0.4), dict(T=0.0)))):
        x, g = logits(2, V, dtype, seed=V % 1000)
        for mode in modes:
            run(x, torch.rand(2, generator=g), **mode)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_with_nan_leave_the_others_alone(dtype):
    print(f"[case] sample rows with NaN and +inf {dtype}", flush=True)
    for B, V in ((12, 3001), (8, 152064)):
        x, g = logits(B, V, dtype, seed=51)
        x[1] = math.nan
        x[3, ::2] = math.nan
        x[4, 77] = math.inf
        x[6, V - 1] = -math.nan
        bad = torch.tensor([1, 3, 4, 6])
        good = torch.tensor([b for b in range(B) if b not in (1, 3, 4, 6)])
        u = torch.rand(B, generator=g)
        for mode in (dict(), dict(top_k=7), dict(top_p=0.7), dict(min_p=0.1), dict(top_k=50, top_p=0.9), dict(top_k=2900)):
            s = {k: torch.full((B,), v, device="cuda", dtype=torch.int32 if k == "top_k" else F32) for k, v in mode.items()}
            n = espo.espo_sample_workspace_bytes(B, V, dtype)
            ws = torch.zeros(n, dtype=torch.uint8, device="cuda") if n else None
            tokens = torch.full((B,), -7, dtype=torch.int32, device="cuda")
            espo.espo_sample(x, u.cuda(), tokens, workspace=ws, **s)
            alive = torch.ones(B, dtype=torch.uint8)
            alive[bad] = 0
            alone = torch.full((B,), -7, dtype=torch.int32, device="cuda")
            espo.espo_sample(x, u.cuda(), alone, alive=alive.cuda(), **s)
            assert torch.equal(tokens[good.cuda()], alone[good.cuda()]) and (alone[good.cuda()] >= 0).all()
            assert ((tokens[bad.cuda()] >= -1) & (tokens[bad.cuda()] < V)).all()


def test_frequencies_are_the_distribution():
    print("[case] sample frequencies", flush=True)
    n, V = 4096, 300
    x, _ = logits(1, V, F32, seed=12, scale=2.0)
    rows = x.expand(n, V).contiguous()
    tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
    u = (torch.arange(n) + 0.5) / n
    espo.espo_sample(rows, u.cuda(), tokens, top_k=torch.full((n,), 50, dtype=torch.int32, device="cuda"))
    v = x[0].double().cpu()
    w = torch.where(v >= v.sort(descending=True).values[49], (v - v.max()).exp(), 0.0)
    got = torch.bincount(tokens.cpu().long(), minlength=V).double()
    assert (got - n * w / w.sum()).abs().max() <= 1.0          # equally spaced numbers: every interval holds its length's share


def test_captured_and_replayed_on_another_stream():
    print("[case] sample graph", flush=True)
    B, V = 40, 30001
    x, g = logits(B, V, BF16, seed=6)
    dev = lambda t: t.cuda()
    u, T = dev(torch.rand(B, generator=g)), dev(torch.full((B,), 0.8))
    k, p = dev(torch.randint(0, 60, (B,), generator=g, dtype=torch.int32)), dev(torch.rand(B, generator=g))
    tokens, lp = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, device="cuda")
    n = espo.espo_sample_workspace_bytes(B, V, BF16)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda") if n else None
    call = lambda: espo.espo_sample(x, u, tokens, logprob=lp, temperature=T, top_k=k, top_p=p, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call()
    for turn in range(4):
        x.copy_((torch.randn(B, V, generator=g) * 3).to(BF16))
        u.copy_(torch.rand(B, generator=g))
        call()
        torch.cuda.synchronize()
        want = tokens.clone(), lp.clone()
        tokens.zero_(), lp.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, want[0]) and torch.equal(lp, want[1]), turn
    s = torch.cuda.Stream()
    tokens.zero_()
    torch.cuda.synchronize()
    espo.espo_sample(x, u, tokens, temperature=T, top_k=k, top_p=p, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(tokens, want[0])


def test_row_offsets_beyond_32_bits():
    print("[case] sample far rows", flush=True)
    B, V, pitch = 4, 3001, 1 << 30
    buf = torch.empty(3 * pitch + 3008, dtype=BF16, device="cuda")
    x = buf.as_strided((B, V), (pitch, 1))
    small, g = logits(B, V, BF16, seed=2)
    x.copy_(small)
    u = torch.rand(B, generator=g)
    a, b = run(x, u, p=0.9), run(small, u, p=0.9)
    assert torch.equal(a[0], b[0])
    buf_n = x[:, :2000]                                        # fewer columns than the tensor has
    run(buf_n, u, k=9)


def test_rollout_and_update_together():
    """A batch drawn, its advantages, and the loss with its gradient on the logits of the same tokens, as a trainer chains them."""
    print("[case] rollout, advantages, whitening, loss", flush=True)
    B, S, V, T = 6, 9, 2003, 0.9
    g = torch.Generator().manual_seed(99)
    lengths = torch.tensor([9, 1, 5, 9, 3, 7], dtype=torch.int32)
    valid = torch.arange(S)[None, :] < lengths[:, None]
    buf = torch.zeros(B * S, 2008, dtype=BF16, device="cuda")   # the old policy's logits of every position
    buf[:, :V] = torch.randn(B * S, V, generator=g).to(BF16).cuda()
    old = buf[:, :V]
    tokens, old_lp = torch.full((B, S), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, S, device="cuda")
    tau = torch.full((B,), T, device="cuda")
    for s in range(S):                                         # rows that have ended are not drawn from
        rows = old.view(B, S, V)[:, s] if old.is_contiguous() else buf.view(B, S, 2008)[:, s, :V]
        tok, lp = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, device="cuda")
        espo.espo_sample(rows, torch.rand(B, generator=g).cuda(), tok, logprob=lp, temperature=tau, alive=valid[:, s].to(torch.uint8).cuda())
        tokens[:, s], old_lp[:, s] = tok, lp
    assert torch.equal(tokens.cpu() >= 0, valid)
    flat = tokens.view(-1)
    again = torch.zeros(B * S, device="cuda")
    espo.espo_logprobs(old, T, flat, again)                    # the draw's log-probability is the forward pass's
    assert (again - old_lp.view(-1)).abs().max() < 2e-5        # fp32 sums of 2003 weights against double ones: sum_bound below 1e-5
    values = torch.rand(B, S, generator=g).cuda()
    td, adv = torch.zeros(B, S, device="cuda"), torch.zeros(B, S, device="cuda")
    stopped = torch.tensor([0, 1, 0, 0, 1, 0], dtype=torch.uint8, device="cuda")
    espo.espo_advantages_terminal(values, lengths.cuda(), stopped, torch.ones(B, device="cuda"), -1.0, 1.0, 0.95, td, adv)
    wws = torch.empty(espo.espo_whiten_workspace_bytes(B, S), dtype=torch.uint8, device="cuda")
    espo.espo_whiten(adv, lengths.cuda(), adv, wws)
    new = torch.zeros_like(buf)                                # the policy has moved
    new[:, :V] = (old.float() + 0.05 * torch.randn(B * S, V, generator=g).cuda()).to(BF16)
    n = int(lengths.sum())
    out = torch.zeros(espo.POLICY_RESULT_BYTES, dtype=torch.uint8, device="cuda")
    ws = torch.empty(espo.espo_policy_loss_workspace_bytes(B * S, V, BF16), dtype=torch.uint8, device="cuda")
    d = torch.full_like(new, 3.0)
    espo.espo_policy_loss(new[:, :V], T, flat, old_lp.view(-1), adv.view(-1), out, ws, dlogits=d[:, :V], entropy_coef=0.01, scale=1.0 / n)
    f = R.softmax_rows(new[:, :V].double().cpu(), T, flat.cpu())
    gg, h, sums, _ = R.policy_terms(f, old_lp.view(-1).double().cpu(), adv.view(-1).double().cpu(), torch.ones(B * S).double(), 1.0 / n, 0.2, 0.2, 0.01)
    want = R.logits_grad(f, gg, h)
    bound = R.grad_bound(f, gg, h, want, 2.0 ** -8, V) + (R.logprob_bound(f, V) + 8 * R.U)[:, None] * gg.abs()[:, None] * 2 / T
    assert ((d[:, :V].double().cpu() - want).abs() <= bound).all()
    assert (d[~valid.view(-1).cuda(), :V] == 0).all() and (d[:, V:] == 3.0).all()
    res = espo.read_policy_result(out)
    assert res["tokens"] == n and abs(res["loss"] - float(sums[0])) < 1e-4 * (1 + abs(float(sums[0])))
