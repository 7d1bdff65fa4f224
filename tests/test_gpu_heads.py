"""Token log probabilities and distillation from top log probabilities against the 64-bit oracle.

Tolerances.  With t = (x - m) log2(e) / T: the difference, the factor and the product round once each, so t is off by at most
3 * 2^-24 |t|, and the exponential adds 2 ulp: a term that matters to a sum (t > -24) is off by at most 55 * 2^-24 relative.  A thread
adds at most V/256 + 32 terms, one rounding each, and the joining about 16 more.  SUM(V) = (128 + V / 256) * 2^-24 covers them."""
import numpy as np
import pytest
import torch

from oracle import heads
from paper_2111_09389_b200 import api

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24
f32 = lambda v: float(np.float32(v))          # the entry points take fp32 temperatures


def SUM(V):
    return (128 + V / 256) * U


def within(got, want, tol):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - want) <= tol)
    assert ok.all(), (np.argwhere(~ok)[:5].tolist(), got[~ok][:5], want[~ok][:5])


def logits_of(rows, V, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, V, generator=g) * spread).to(dtype)


def report(x, tokens, k=0, temperature=1.0, V=None, row_stride=None):
    """The forward call on rows of x (device); numpy outputs, whole."""
    rows = x.shape[0]
    V = x.shape[1] if V is None else V
    new = lambda *s, dtype=torch.float32: torch.full(s, 77, dtype=dtype, device="cuda")
    o = {n: new(rows) for n in ("logprob", "entropy", "lse")}
    if k:
        o |= {"top_logprob": new(rows, k), "top_index": new(rows, k, dtype=torch.int32)}
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.lpdt_token_logprobs(rows, V, x, torch.from_numpy(tokens.astype(np.int32)).cuda(), o["logprob"], o["entropy"], o["lse"],
                            o.get("top_logprob"), o.get("top_index"), top_k=k, temperature=temperature, row_stride=row_stride, dev_status=status)
    return o, api.lpdt_check_status(status)


def check_report(x, tokens, k, temperature, **kw):
    V = x.shape[1]
    o, status = report(x.cuda() if not x.is_cuda else x, tokens, k, temperature, **kw)
    want = heads.token_logprobs(x.double().cpu().numpy(), tokens, f32(temperature), k)
    assert status == (1 if (tokens >= V).any() else 0)
    within(o["lse"], want["lse"], SUM(V) + 2 * U * np.abs(want["lse"]))
    within(o["logprob"], want["logprob"], SUM(V) + 2 * U * np.abs(want["logprob"]))
    within(o["entropy"], want["entropy"], SUM(V) * (1 + 2 * np.log(V)) + 2 * U * np.abs(want["entropy"]))
    if k:
        assert np.array_equal(o["top_index"].cpu().numpy(), want["top_index"])
        within(o["top_logprob"], want["top_logprob"], SUM(V) + 2 * U * np.abs(want["top_logprob"]))
    return o, want


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V,k,temperature", [
    (1, 1, 1, 1.0), (3, 2, 2, 0.5), (40, 10, 3, 2.0), (5, 64, 64, 1.0), (7, 65, 20, 1.0), (9, 256, 8, 0.7), (6, 257, 128, 1.0),
    (130, 1000, 5, 1.0), (3, 1024, 128, 1.3), (4, 1025, 1, 1.0), (4, 1031, 128, 1.0), (2, 2049, 100, 1.0), (300, 3001, 7, 1.0),
    (1, 5000, 20, 0.7), (2, 32003, 64, 1.0), (1, 131072, 128, 1.0), (700, 9001, 16, 1.0), (3, 300001, 50, 1.0)])
def test_logprobs(rows, V, k, temperature, dtype):
    x = logits_of(rows, V, dtype, rows + V)
    tokens = np.random.default_rng(V).integers(0, V, rows)
    check_report(x, tokens, k, temperature)
    check_report(x, tokens, 0, temperature)


def hard_rows(V, dtype):
    """Rows on which a running top-k or a running softmax goes wrong first."""
    rng = np.random.default_rng(V)
    low = torch.finfo(dtype).min
    r = [np.arange(V) * 0.01, -np.arange(V) * 0.01, np.zeros(V), np.full(V, -np.inf), np.full(V, low), rng.standard_normal(V) * 30,
         np.where(rng.random(V) < 0.5, -np.inf, rng.standard_normal(V)), np.where(rng.random(V) < 0.5, low, rng.standard_normal(V)),
         rng.integers(0, 3, V), rng.integers(-1, 1, V) * 0.0]
    few = np.full(V, -np.inf)
    few[[0, V // 3, V - 1]] = [1.0, 5.0, 1.0]
    late = rng.standard_normal(V)
    late[-(V // 4):] += 50
    spike = np.zeros(V)
    spike[V // 2] = 100
    zeros = np.where(np.arange(V) % 2 == 0, -0.0, 0.0)
    steep = np.repeat(np.arange((V + 63) // 64), 64)[:V] * 0.125
    r += [few, late, spike, zeros, steep]
    with np.errstate(over="ignore"):
        return torch.from_numpy(np.stack(r)).to(dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,k", [(4, 3), (50, 10), (700, 128), (1500, 128), (9000, 1), (40001, 128), (150000, 64)])
def test_logprobs_of_hard_rows(V, k, dtype):
    x = hard_rows(V, dtype)
    tokens = np.random.default_rng(1).integers(0, V, len(x))
    tokens[0], tokens[1], tokens[2] = -1, V, V - 1
    check_report(x, tokens, k, 1.0)
    check_report(x[:3], tokens[:3], k, 1.0)                 # few rows: several CTAs a row


@pytest.mark.parametrize("V", [10, 300, 1024, 5003, 70001])
def test_logprobs_of_rows_with_nan_and_infinity(V):
    """NaN or +inf anywhere: the row answers NaN; NaN is never among the top; the other rows are as they were."""
    x = logits_of(6, V, torch.float32, V)
    x[1, V // 2] = np.nan
    x[2, 0] = np.inf
    x[3] = np.nan
    x[3, V - 1] = 2.0
    x[4] = np.nan
    tokens = np.full(6, 1)
    k = min(V, 6)
    o, _ = report(x.cuda(), tokens, k)
    want = heads.token_logprobs(x.double().numpy(), tokens, 1.0, k)
    for n in ("logprob", "entropy", "lse", "top_logprob"):
        got = o[n].cpu().numpy().reshape(6, -1)
        assert np.isnan(got[1:5]).all() and np.isfinite(got[[0, 5]]).all(), n
        within(got[[0, 5]], want[n].reshape(6, -1)[[0, 5]], SUM(V) * 20 + 1e-6)
    index = o["top_index"].cpu().numpy()
    assert np.array_equal(index[[0, 1, 5]], want["top_index"][[0, 1, 5]]) and index[2, 0] == 0
    assert index[3].tolist() == [V - 1] + [-1] * (k - 1) and (index[4] == -1).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,stride,offset", [(10, 11, 1), (1000, 1001, 3), (5003, 5003, 1), (5000, 5013, 7), (33000, 33001, 2)])
def test_rows_that_start_anywhere(V, stride, offset, dtype):
    """Odd strides and offsets; what lies between the rows is neither read (NaN there) nor written."""
    rows, k = 5, 9
    flat = torch.full((offset + rows * stride + 64,), float("nan"), dtype=dtype, device="cuda")
    x = torch.as_strided(flat, (rows, V), (stride, 1), offset)
    x.copy_(logits_of(rows, V, dtype, 3))
    tokens = np.arange(rows)
    o, _ = check_report(x, tokens, k, 1.0, row_stride=stride)
    gout = torch.full((offset + 1 + rows * (stride + 2) + 64,), 5.0, dtype=dtype, device="cuda")
    for target, off, st in ((gout, offset + 1, stride + 2), (flat.clone(), offset, stride)):
        before = target.clone()
        d = torch.as_strided(target, (rows, V), (st, 1), off)
        g = torch.ones(rows, device="cuda")
        api.lpdt_token_logprobs_bwd(rows, V, x, torch.arange(rows, dtype=torch.int32, device="cuda"), o["lse"], o["entropy"], d,
                                    d_logprob=g, row_stride=stride, dlogits_row_stride=st)
        mask = torch.ones_like(target, dtype=torch.bool)
        torch.as_strided(mask, (rows, V), (st, 1), off).fill_(False)
        assert torch.equal(torch.nan_to_num(target[mask]), torch.nan_to_num(before[mask]))
        want = heads.token_logprobs_bwd(x.double().cpu().numpy(), tokens, np.ones(rows))
        within(d, want, 64 * U + torch.finfo(dtype).eps / 2 * np.abs(want) + 2.0 ** -25)
    loss, row_loss = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda")
    value, index = o["top_logprob"], o["top_index"]
    for target, off, st in ((gout, offset + 1, stride + 2), (flat, offset, stride)):                    # the second: in place
        ref = heads.distill_topk(x.double().cpu().numpy()[None], value.cpu().numpy()[None], index.cpu().numpy()[None], True)
        before = target.clone()
        d = torch.as_strided(target, (rows, V), (st, 1), off)
        api.lpdt_distill_topk(1, rows, V, x, k, value, index, loss, row_loss, dlogits=d, row_stride=stride, dlogits_row_stride=st)
        mask = torch.ones_like(target, dtype=torch.bool)
        torch.as_strided(mask, (rows, V), (st, 1), off).fill_(False)
        assert torch.equal(torch.nan_to_num(target[mask]), torch.nan_to_num(before[mask]))
        within(d, ref[2][0], 4 * SUM(V) / rows + torch.finfo(dtype).eps / 2 * np.abs(ref[2][0]) + 2.0 ** -25)


def test_offsets_beyond_32_bits():
    """Rows 2^31 + 8 elements apart: logits, gradients, the quantizer's input and the product's result."""
    rows, V, k, stride = 3, 5001, 4, 2 ** 31 + 8
    far = torch.empty((rows - 1) * stride + 8192, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(far, (rows, V), (stride, 1), 0)
    near = logits_of(rows, V, torch.bfloat16, 8)
    x.copy_(near)
    tokens = np.arange(rows)
    o, _ = check_report(x, tokens, k, 1.0, row_stride=stride)
    q, s = (torch.empty(rows, api.lpdt_e4m3_pitch(V), dtype=torch.uint8, device="cuda"), torch.empty(rows, api.lpdt_e4m3_scale_pitch(V), dtype=torch.uint8, device="cuda"))
    qt, st = (torch.empty(V, 16, dtype=torch.uint8, device="cuda"), torch.empty(V, 4, dtype=torch.uint8, device="cuda"))
    api.lpdt_quantize_e4m3(x, 1, rows, V, q, s, qt, st, x_row_stride=stride)
    qr, sr = heads.quantize_e4m3(near.double().numpy())
    assert np.array_equal(q.cpu().numpy()[:, :V], qr) and np.array_equal(s.cpu().numpy()[:, :sr.shape[1]], sr)
    assert np.array_equal(qt.cpu().numpy()[:, :rows], heads.quantize_e4m3(near.double().numpy().T)[0])
    loss, row_loss = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda")
    lists = o["top_logprob"], o["top_index"]
    api.lpdt_distill_topk(1, rows, V, x, k, *lists, loss, row_loss, dlogits=x, row_stride=stride, dlogits_row_stride=stride)
    ref = heads.distill_topk(near.double().numpy()[None], lists[0].cpu().numpy()[None], lists[1].cpu().numpy()[None], True)
    within(x, ref[2][0], 4 * SUM(V) / rows + 2.0 ** -8 * np.abs(ref[2][0]) + 2.0 ** -25)
    x.copy_(near)
    api.lpdt_token_logprobs_bwd(rows, V, x, torch.arange(rows, dtype=torch.int32, device="cuda"), o["lse"], o["entropy"], x,
                                d_logprob=torch.ones(rows, device="cuda"), row_stride=stride, dlogits_row_stride=stride)
    want = heads.token_logprobs_bwd(near.double().numpy(), tokens, np.ones(rows))
    within(x, want, 64 * U + 2.0 ** -8 * np.abs(want) + 2.0 ** -25)
    api.lpdt_matmul_e4m3(1, rows, V, 16, qt.view(-1, 16), st, qt, st, x, c_row_stride=stride)         # its first three rows with all
    v = heads.dequantize_e4m3(qt.cpu().numpy(), st.cpu().numpy()[:, :1])
    v[:, rows:] = 0
    within(x, v[:rows] @ v.T, 2.0 ** -8 * np.abs(v[:rows] @ v.T) + 1e-5)


def test_the_same_bits_every_time():
    """Lists with tokens listed twice, ties among the top: ten calls on two streams at once give the same bits."""
    rows, V, k = 6, 70001, 64
    x = logits_of(rows, V, torch.bfloat16, 1).cuda()
    value, index = lists_of(1, rows, V, k, 3, duplicates=True)
    index[..., k // 2:] = index[..., :k // 2]
    value, index = torch.from_numpy(value).cuda(), torch.from_numpy(index).cuda()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for i in range(10):
        with torch.cuda.stream(streams[i % 2]):
            loss, row_loss, d = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
            api.lpdt_distill_topk(1, rows, V, x, k, value, index, loss, row_loss, dlogits=d)
            o, _ = report(x, np.zeros(rows), k)
            got.append([loss, row_loss, d] + [o[n] for n in sorted(o)])
    torch.cuda.synchronize()
    for g in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(g, got[0]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V,temperature", [(1, 1, 1.0), (40, 10, 2.0), (3, 333, 0.7), (2, 1025, 1.0), (5, 32003, 1.0), (1, 140000, 0.5)])
@pytest.mark.parametrize("which", ["logprob", "entropy", "lse", "all"])
def test_logprobs_backward(rows, V, temperature, which, dtype):
    x = logits_of(rows, V, dtype, V + rows)
    if V > 20:
        x[0, 5:V // 2] = -float("inf")
    rng = np.random.default_rng(V)
    tokens = np.where(rng.random(rows) < 0.2, -1, rng.integers(0, V, rows))
    tokens[0] = 0
    gs = {n: rng.standard_normal(rows).astype(np.float32) if which in (n, "all") else None for n in ("logprob", "entropy", "lse")}
    xd = x.cuda()
    o, _ = report(xd, tokens, 0, temperature)
    d = torch.empty_like(xd)
    api.lpdt_token_logprobs_bwd(rows, V, xd, torch.from_numpy(tokens.astype(np.int32)).cuda(), o["lse"], o["entropy"], d, temperature=temperature,
                                **{"d_" + n: None if g is None else torch.from_numpy(g).cuda() for n, g in gs.items()})
    temperature = f32(temperature)
    z = x.double().numpy() / temperature
    want = heads.token_logprobs_bwd(x.double().numpy(), tokens, gs["logprob"], gs["entropy"], gs["lse"], temperature)
    ref = heads.token_logprobs(x.double().numpy(), tokens, temperature)
    lse, H = ref["lse"][:, None], ref["entropy"][:, None]
    with np.errstate(invalid="ignore"):
        lp = np.where(z == -np.inf, 0, z - lse)
        p = np.where(z == -np.inf, 0, np.exp(z - lse))
    a = {n: np.zeros((rows, 1)) if g is None else np.abs(g.astype(np.float64))[:, None] for n, g in gs.items()}
    off = (np.abs(lse) + np.abs(np.where(z == -np.inf, 0, z)) + 3 * np.abs(lp) + 8) * 2 * U + SUM(V)        # of ln p, and of p relative
    size = a["logprob"] + a["lse"] + a["entropy"] * (np.abs(lp) + H + 1)
    tol = (p * (off * size + a["entropy"] * (off + SUM(V) * (1 + 2 * np.log(V))) + 8 * U * size) + 4 * U * a["logprob"]) / temperature
    within(d, want, tol + torch.finfo(dtype).eps / 2 * np.abs(want) + 2.0 ** -25)


@pytest.mark.parametrize("V", [5, 3001])
def test_logprobs_backward_of_logits_beyond_fp32(V):
    """Logits / temperature whose lse no fp32 holds: the forward's log probabilities are right, lse is infinite, and the gradient, which has
    nothing else to go by, is NaN and not that of probabilities 0.  Rows that stay in range beside them are as ever."""
    x = logits_of(4, V, torch.float32, V)
    x[1] = (x[1] * 4).round() * 1024 + 1e10
    x[2] = -1e-29
    x[2, 3] = 2e-30
    tokens, T = np.array([0, 1, 3, 2]), 1e-30
    x[0], x[3] = x[0] * 1e-30, x[3] * 1e-30
    o, _ = report(x.cuda(), tokens, 0, T)
    ref = heads.token_logprobs(x.double().numpy(), tokens, f32(T))
    within(o["logprob"], ref["logprob"], SUM(V) + 2 * U * np.abs(ref["logprob"]))
    d = torch.empty(4, V, device="cuda")
    api.lpdt_token_logprobs_bwd(4, V, x.cuda(), torch.from_numpy(tokens.astype(np.int32)).cuda(), o["lse"], o["entropy"], d,
                                d_logprob=torch.full((4,), 1e-30, device="cuda"), temperature=T)
    assert torch.isinf(o["lse"][1]) and torch.isnan(d[1]).all()
    want = heads.token_logprobs_bwd(x.double().numpy(), tokens, np.full(4, np.float32(1e-30), np.float64), temperature=f32(T))
    keep = [0, 2, 3]
    z = x.double().numpy()[keep] / f32(T)
    within(d[keep], want[keep], (2 * np.abs(z).max() + SUM(V) / U + 16) * 2 * U)


@pytest.mark.parametrize("V", [100, 3001])
@pytest.mark.parametrize("shift", [0.0, 100.0, -1e4, 3e4])
def test_logprobs_backward_of_shifted_rows(V, shift):
    """The forward of shifted logits loses nothing but the rounding of the logits themselves; the gradient loses what the header says of
    the fp32 lse, 2^-23 (|lse| + 2 |ln p|) of p, beside the sums' own rounding."""
    x = (logits_of(3, V, torch.float32, V) * 64).round() / 64 + shift              # exact
    tokens, g = np.arange(3), np.array([1.0, -2.0, 0.5], np.float32)
    o, want = check_report(x, tokens, 0, 1.0)
    base, _ = report((x - shift).cuda(), tokens)
    within(o["logprob"], base["logprob"].double().cpu().numpy(), 2 * SUM(V) + 4 * U * np.abs(want["logprob"]))
    d = torch.empty(3, V, device="cuda")
    api.lpdt_token_logprobs_bwd(3, V, x.cuda(), torch.arange(3, dtype=torch.int32, device="cuda"), o["lse"], o["entropy"], d, d_logprob=torch.from_numpy(g).cuda())
    ref = heads.token_logprobs_bwd(x.double().numpy(), tokens, g)
    lp = x.double().numpy() - want["lse"][:, None]
    off = 2 * U * (np.abs(want["lse"])[:, None] + 2 * np.abs(lp)) + SUM(V) + 8 * U
    within(d, ref, np.abs(g)[:, None] * (np.exp(lp) * off + 2 * U))


def test_logprobs_gradient_against_differences():
    """Central differences of the forward call itself: step 2^-4 of the logits; third derivatives are below 1, so the differences are
    off by at most step^2 / 6, and by the rounding of the forward over the step."""
    rows, V = 4, 12
    x = logits_of(rows, V, torch.float32, 0, spread=1.0)
    x = (x * 64).round() / 64                                  # steps leave the values exact
    tokens = np.arange(rows)
    g, h, l = (np.random.default_rng(i).standard_normal(rows).astype(np.float32) for i in range(3))
    o, _ = report(x.cuda(), tokens)
    d = torch.empty(rows, V, device="cuda")
    api.lpdt_token_logprobs_bwd(rows, V, x.cuda(), torch.from_numpy(tokens.astype(np.int32)).cuda(), o["lse"], o["entropy"], d,
                                *(torch.from_numpy(v).cuda() for v in (g, h, l)))
    step = 2.0 ** -4
    def value(x):
        o, _ = report(x.cuda(), tokens)
        return sum(w * o[n].cpu().double().numpy() for w, n in ((g, "logprob"), (h, "entropy"), (l, "lse")))
    for v in range(V):
        up, down = x.clone(), x.clone()
        up[:, v] += step
        down[:, v] -= step
        diff = (value(up) - value(down)) / (2 * step)
        scale = np.abs(g) + np.abs(h) * 4 + np.abs(l)
        assert (np.abs(diff - d[:, v].double().cpu().numpy()) <= scale * (step ** 2 / 6 + SUM(V) * 8 / step)).all()


# ------------------------------------------------------------------ distillation
def lists_of(nodes, B, V, k, seed, duplicates=False):
    rng = np.random.default_rng(seed)
    index = rng.integers(0, V, (nodes, B, k)) if duplicates or k > V else np.argsort(rng.random((nodes, B, V)), -1)[..., :k]
    raw = np.sort(rng.standard_normal((nodes, B, k)) * 2)[..., ::-1]
    value = raw - np.log(np.exp(raw).sum(-1, keepdims=True)) + np.log(rng.uniform(0.3, 1.0, (nodes, B, 1)))
    return value.astype(np.float32), index.astype(np.int32)


def distill(x, value, index, tail=True, weight=None, temperature=1.0, grad=True, **kw):
    nodes, B, V = x.shape
    k = value.shape[-1]
    loss, row_loss = torch.full((nodes,), 7.0, device="cuda"), torch.full((nodes, B), 7.0, device="cuda")
    d = torch.full(x.shape, 3.0, dtype=x.dtype, device="cuda") if grad else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.lpdt_distill_topk(nodes, B, V, x.cuda(), k, torch.from_numpy(value).cuda(), torch.from_numpy(index).cuda(), loss, row_loss,
                          dlogits=d, row_weight=None if weight is None else torch.from_numpy(weight).cuda(), tail=tail, temperature=temperature,
                          dev_status=status)
    return loss, row_loss, d, api.lpdt_check_status(status)


def check_distill(x, value, index, tail, weight=None, temperature=1.0):
    nodes, B, V = x.shape
    loss, row_loss, d, status = distill(x, value, index, tail, weight, temperature)
    temperature = f32(temperature)
    L, R, G = heads.distill_topk(x.double().numpy(), value, index, tail, temperature, weight)
    w = np.abs(np.ones((nodes, B)) if weight is None else weight)
    assert status == (1 if ((index >= V) & (w[..., None] != 0)).any() else 0)
    total = np.exp(value.astype(np.float64)).sum(-1) + 1 if tail else np.full((nodes, B), 2.0)
    tolR = 3 * SUM(V) * total + 2 * U * np.abs(R)
    within(row_loss, R, tolR)
    within(loss, L, (w * np.where(np.isfinite(tolR), tolR, 0)).mean(1) + 2 * U * np.abs(L))
    # outside the list |p total - left p / p_R| <= p (total + 1 / p_R); inside p total.  exp2 of far values: 3 |t| roundings, |t| <= 149
    z = x.double().numpy() / temperature
    with np.errstate(invalid="ignore", divide="ignore"):
        logp, _ = heads._log_softmax(z)
        p = np.exp(np.nan_to_num(logp, nan=-np.inf))
        inside = np.zeros(x.shape, bool)
        for n in range(nodes):
            for b in range(B):
                have = index[n, b][(index[n, b] >= 0) & (index[n, b] < V)]
                inside[n, b, have] = True
        p_r = np.where(inside, 0, p).sum(-1, keepdims=True)
        size = np.where(inside | (p_r == 0), p * total[..., None], p * (total[..., None] + (1 / np.maximum(p_r, 1e-300) if tail else 0)))
    tol = (SUM(V) * 2 + 450 * U) * size * (w / (B * temperature))[..., None] + torch.finfo(x.dtype).eps / 2 * np.abs(G) + 2.0 ** -25 * (x.dtype == torch.float16) + 1e-37
    within(d, G, tol)
    only = distill(x, value, index, tail, weight, temperature, grad=False)
    assert torch.equal(only[0], loss) and torch.equal(only[1], row_loss)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("nodes,B,V,k,temperature", [(1, 1, 1, 1, 1.0), (3, 5, 10, 3, 2.0), (2, 3, 10, 10, 1.0), (2, 2, 65, 64, 1.0), (1, 7, 300, 128, 0.7),
                                                     (2, 3, 1024, 20, 1.0), (1, 2, 1025, 128, 1.0), (2, 2, 5003, 5, 1.0), (1, 1, 131072, 64, 1.0),
                                                     (2, 150, 2500, 16, 1.0), (1, 1, 60001, 1, 0.5), (1, 3, 5, 128, 1.0)])
def test_distill(nodes, B, V, k, temperature, tail, dtype):
    x = logits_of(nodes * B, V, dtype, V + k).view(nodes, B, V)
    value, index = lists_of(nodes, B, V, k, V)
    weight = np.random.default_rng(k).uniform(0.2, 2, (nodes, B)).astype(np.float32)
    check_distill(x, value, index, tail, weight, temperature)
    check_distill(x, value, index, tail, None, temperature)


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V", [12, 200, 1000, 4099, 90001])
@pytest.mark.parametrize("B", [9, 170])                       # few rows are shared by clusters
def test_distill_of_hard_lists(V, tail, B):
    """Tokens listed twice, short and empty lists, ids out of range, rows of weight 0, a teacher sure of itself, a student that has
    (nearly) all of its mass on the list, masked tokens on and off the list, a student's row of nothing but masks."""
    nodes, k = 2, 8
    x = logits_of(nodes * B, V, torch.float32, V).view(nodes, B, V)
    value, index = lists_of(nodes, B, V, k, V + 1)
    weight = np.ones((nodes, B), np.float32)
    index[0, 0, 3:] = index[0, 0, :5]                          # the same tokens again
    index[0, 1, 2:] = -1
    index[0, 2] = -1
    index[0, 3, 1], index[0, 3, 4] = V, 2 ** 31 - 1
    weight[0, 4] = 0
    x[0, 4, 0] = float("nan")                                  # not read
    index[0, 4, 0] = V + 5
    value[0, 5] = [0.0] + [-200.0] * (k - 1)
    for j in range(k):
        x[0, 6, index[0, 6, j]] += 60                          # e^-60 of the mass is left: beyond 1 - sum p in any float
    x[0, 7, index[0, 7, 3]] = -float("inf")                    # listed but masked: an infinite loss, a finite gradient
    rest = np.setdiff1d(np.arange(V), index[1, 0])
    x[1, 0, rest] = -float("inf")                              # nothing outside the list
    x[1, 1] = -float("inf")
    x[1, 2] = torch.finfo(torch.float32).min
    value[1, 3] = -float("inf")
    value[1, 4, 2] = -float("inf")
    x[1, 5, V // 2] = -float("inf")
    if B > 100:
        for a in (x, value, index, weight):
            a[0, 140:149], a[1, 150:159] = a[0, :9], a[1, :9]
        weight[:, 9::13] = 0
    check_distill(x, value, index, tail, weight)


@pytest.mark.parametrize("dtype,V", [(torch.bfloat16, 16400), (torch.bfloat16, 131072), (torch.float16, 50021), (torch.float32, 9003), (torch.float32, 70001),
                                     (torch.float32, 131200)])
def test_distill_of_many_long_rows(dtype, V):
    """Hundreds of rows at every number of threads, odd strides, in place; weights that are 0 or negative."""
    nodes, B, k, stride = 3, 113, 20, V + 1 + V % 2
    flat = torch.full((2 + nodes * B * stride,), 7.0, dtype=dtype, device="cuda")
    view = torch.as_strided(flat, (nodes, B, V), (B * stride, stride, 1), 2)
    x = logits_of(nodes * B, V, dtype, V).view(nodes, B, V)
    view.copy_(x)
    value, _ = lists_of(nodes, B, 1000, k, V)
    index = np.random.default_rng(V).integers(0, V, (nodes, B, k)).astype(np.int32)
    weight = np.random.default_rng(1).uniform(0.5, 2, (nodes, B)).astype(np.float32)
    weight[:, ::4], weight[:, 1::8] = 0, -1
    loss, row_loss = torch.empty(nodes, device="cuda"), torch.empty(nodes, B, device="cuda")
    api.lpdt_distill_topk(nodes, B, V, view, k, torch.from_numpy(value).cuda(), torch.from_numpy(index).cuda(), loss, row_loss, dlogits=view,
                          row_weight=torch.from_numpy(weight).cuda(), row_stride=stride, dlogits_row_stride=stride)
    result = view.clone()
    view.fill_(7)
    assert (flat == 7).all()
    some = slice(0, None, 16)
    L, R, G = heads.distill_topk(x[:, some].double().numpy(), value[:, some], index[:, some], True, 1.0, weight[:, some])
    G = G * G.shape[1] / B
    within(row_loss[:, some], R, 6 * SUM(V) + 2 * U * np.abs(R))
    within(loss, (row_loss.double().cpu().numpy() * weight).mean(1), 2 * U * np.abs(row_loss.cpu().numpy() * weight).mean(1) + 1e-30)
    within(result[:, some], G, 8 * SUM(V) / B + torch.finfo(dtype).eps / 2 * np.abs(G) + 2.0 ** -25 * (dtype == torch.float16))


@pytest.mark.parametrize("V", [10, 700, 3000, 50000])
def test_distill_of_rows_with_nan(V):
    """NaN or +inf, listed or not, makes its own row NaN and no other."""
    x = logits_of(5, V, torch.float32, V).view(1, 5, V)
    value, index = lists_of(1, 5, V, 4, V)
    index[0, :, 0] = [1, 1, 2, 1, 1]
    index[0, :, 1:] = [3, 4, 5]
    x[0, 1, 7] = float("nan")                                  # not listed
    x[0, 2, 2] = float("nan")                                  # listed
    x[0, 3, 8] = float("inf")
    loss, row_loss, d, _ = distill(x, value, index)
    assert torch.isnan(row_loss[0]).tolist() == [False, True, True, True, False] and torch.isnan(loss).all()
    assert torch.isnan(d[0, 1:4]).all() and torch.isfinite(d[0, [0, 4]]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V,B", [(10, 6), (700, 6), (1024, 40), (3000, 6), (3000, 170), (50000, 6)])
def test_distill_of_rows_with_nan_beside_masks(V, B, tail, dtype):
    """One token allowed and its logit NaN or +inf, listed or not, masks of -inf or of the type's lowest value around it, with a list or
    without any: loss and gradient of the row are NaN, other rows are as they were.  A weight of 0 leaves the row out."""
    x = logits_of(B, V, dtype, V).view(1, B, V)
    value, index = lists_of(1, B, V, 4, V)
    index[0, :, :] = [1, 3, 4, 5]
    weight = np.ones((1, B), np.float32)
    low = torch.finfo(dtype).min
    for row in range(1, B - 1):
        bad = float("nan") if row % 3 else float("inf")
        x[0, row] = low if row % 2 else -float("inf")
        x[0, row, (1, V - 1)[row // 2 % 2]] = bad
        if row % 5 == 4:
            index[0, row] = -1
        if row % 8 == 7:
            weight[0, row] = 0
    loss, row_loss, d, _ = distill(x, value, index, tail, weight)
    bad = np.arange(B) % 8 != 7
    bad[[0, -1]] = False
    assert np.array_equal(torch.isnan(row_loss[0]).cpu().numpy(), bad) and torch.isnan(loss).all()
    assert torch.isnan(d[0, torch.from_numpy(bad).cuda()]).all()
    L, R, G = heads.distill_topk(x.double().numpy(), value, index, tail, 1.0, weight)
    within(row_loss, R, 9 * SUM(V) + 2 * U * np.abs(R))
    within(d, G, 9 * SUM(V) / B + torch.finfo(dtype).eps / 2 * np.abs(G) + 2.0 ** -25)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,B", [(10, 5), (700, 5), (1024, 40), (3000, 5), (3000, 170), (50001, 5)])
def test_distill_with_masks_of_the_lowest_value(V, B, dtype):
    """Every token outside the list masked by the type's lowest value: no class of others, as with -inf; some of them masked: those count
    for nothing.  Listed and masked: a loss near the largest floats or beyond."""
    x = logits_of(B, V, dtype, V).view(1, B, V)
    value, index = lists_of(1, B, V, 4, V)
    low = torch.finfo(dtype).min
    for row in range(B):
        rest = np.setdiff1d(np.arange(V), index[0, row])
        if row % 4 == 0:
            x[0, row, rest] = low
        elif row % 4 == 1:
            x[0, row, rest[::2]] = low
        elif row % 4 == 2:
            x[0, row, index[0, row, 2]] = low
    for tail in (True, False):
        check_distill(x, value, index, tail)


@pytest.mark.parametrize("V", [10, 700, 3000, 50001])
def test_distill_of_students_far_from_the_others(V):
    """The tokens outside the list 300 to 5000 below it: ln p_R counts, however little p_R is."""
    B, k = 5, 4
    x = logits_of(B, V, torch.float32, V).view(1, B, V)
    value, index = lists_of(1, B, V, k, V)
    for row in range(B):
        x[0, row, index[0, row]] += (300, 1000, 2000, 5000, 0)[row]
    _, row_loss, d, _ = distill(x, value, index)
    _, R, G = heads.distill_topk(x.double().numpy(), value, index, True)
    logp, _ = heads._log_softmax(x.double().numpy())
    inside = np.zeros(x.shape, bool)
    np.put_along_axis(inside, index.astype(np.int64), True, -1)
    rest = np.where(inside, -np.inf, logp)
    share = np.exp(rest - np.logaddexp.reduce(rest, -1, keepdims=True))      # p / p_R
    within(row_loss, R, 6 * SUM(V) + 2 * U * np.abs(R))
    within(d, G, (2 * SUM(V) + 450 * U) * (np.exp(logp) * 2 + share) / B + U * np.abs(G) + 1e-37)      # as in check_distill


def test_distill_against_differences():
    """Central differences of the loss itself (step 2^-4, third derivatives below 1)."""
    V, k, step = 9, 3, 2.0 ** -4
    x = (logits_of(4, V, torch.float32, 5, spread=1.0) * 64).round().view(2, 2, V) / 64
    value, index = lists_of(2, 2, V, k, 1)
    for tail in (True, False):
        d = distill(x, value, index, tail)[2]
        for v in range(V):
            up, down = x.clone(), x.clone()
            up[..., v] += step
            down[..., v] -= step
            diff = (distill(up, value, index, tail)[1] - distill(down, value, index, tail)[1]).double() / (2 * step) / 2
            assert (diff - d[..., v].double()).abs().max() <= step ** 2 / 6 + 8 * SUM(V) / step


def test_a_head_from_products_to_gradients():
    """The run as a node makes it: 8-bit products to logits, a teacher's report, distillation from it, 8-bit gradients;
    captured into a graph it gives the same bits."""
    n, B, D, V, k = 2, 64, 384, 2500, 16
    g = torch.Generator().manual_seed(4)
    X, W, WT = (torch.randn(*s, generator=g).cuda() for s in ((n, B, D), (n, V, D), (n, V, D)))
    W, WT = W * 0.1, WT * 0.1
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")
    form = lambda r, c: (e(n, r, api.lpdt_e4m3_pitch(c), dtype=torch.uint8), e(n, r, api.lpdt_e4m3_scale_pitch(c), dtype=torch.uint8))
    fX, fXt, fW, fWT, fd, fdt = form(B, D), form(D, B), form(V, D), form(V, D), form(B, V), form(V, B)
    logits, teacher, dlogits, dW = e(n, B, V, dtype=torch.bfloat16), e(n, B, V, dtype=torch.bfloat16), e(n, B, V, dtype=torch.bfloat16), e(n, V, D)
    lp, index, loss, row_loss = e(n, B, k), e(n, B, k, dtype=torch.int32), e(n), e(n, B)

    def step():
        api.lpdt_quantize_e4m3(X, n, B, D, *fX, *fXt)
        api.lpdt_quantize_e4m3(WT, n, V, D, *fWT)
        api.lpdt_matmul_e4m3(n, B, V, D, *fX, *fWT, teacher)
        api.lpdt_token_logprobs(n * B, V, teacher, top_logprob=lp, top_index=index, top_k=k)
        api.lpdt_quantize_e4m3(W, n, V, D, *fW)
        api.lpdt_matmul_e4m3(n, B, V, D, *fX, *fW, logits)
        api.lpdt_distill_topk(n, B, V, logits, k, lp, index, loss, row_loss, dlogits=dlogits)
        api.lpdt_quantize_e4m3(dlogits, n, B, V, *fd, *fdt)
        api.lpdt_matmul_e4m3(n, V, D, B, *fdt, *fXt, dW)

    step()
    first = [t.clone() for t in (logits, lp, index, loss, row_loss, dlogits, dW)]
    z = logits.double().cpu().numpy()
    ref = heads.distill_topk(z, lp.cpu().numpy(), index.cpu().numpy(), True)
    within(loss, ref[0], 8 * SUM(V))
    want = np.matmul(ref[2].transpose(0, 2, 1), X.double().cpu().numpy())
    got = dW.double().cpu().numpy()
    assert np.linalg.norm(got - want) <= (2.0 ** -4 + 2.0 ** -4 + 2.0 ** -8 + 2.0 ** -7) * np.linalg.norm(want) * 1.1     # two operands of 8 bits, bf16 gradient
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for t in (logits, dlogits, dW, loss):
            t.zero_()
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(first, (logits, lp, index, loss, row_loss, dlogits, dW)):
        assert torch.equal(a, b)
