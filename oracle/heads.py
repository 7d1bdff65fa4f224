"""Oracle of the output head's operators, in 64 bits from their definitions: 8-bit floats with a scale for each block of
128 values and their product, token log probabilities, distillation from a teacher's top log probabilities.

TEST INFRASTRUCTURE ONLY, like the rest of this package; numpy, no code shared with the CUDA library.
"""
import numpy as np

BLOCK = 128


def _e4m3_table():
    """Value of each code: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN, there is no infinity."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        mag = (m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = -mag if c & 128 else mag
    v[0x7f] = v[0xff] = np.nan
    return v


E4M3 = _e4m3_table()
_POSITIVE = E4M3[:0x7f]


def e4m3_encode(v):
    """Codes of values of magnitude at most 448: the nearest one, of two as near the one with an even last bit."""
    a = np.abs(v)
    hi = np.searchsorted(_POSITIVE, a)                       # first code whose value is at least a
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[np.minimum(hi, 0x7e)] - a, a - _POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def quantize_e4m3(x):
    """x [..., cols] -> codes (uint8, shape of x), scale bytes [..., ceil(cols/128)]."""
    x = np.asarray(x, np.float64)
    cols = x.shape[-1]
    q = np.zeros(x.shape, np.uint8)
    s = np.zeros(x.shape[:-1] + (-(-cols // BLOCK),), np.uint8)
    for b in range(s.shape[-1]):
        part = x[..., b * BLOCK:(b + 1) * BLOCK]
        bad = ~np.isfinite(part).all(-1)
        amax = np.abs(np.where(bad[..., None], 0, part)).max(-1)
        e = np.full(amax.shape, -127)
        while (over := amax > 448 * np.exp2(e.astype(np.float64))).any():
            e += over
        e = np.where(amax == 0, 0, e)
        s[..., b] = np.where(bad, 255, e + 127)
        v = np.where(bad[..., None], 0, part) * np.exp2(-e.astype(np.float64))[..., None]
        q[..., b * BLOCK:(b + 1) * BLOCK] = np.where(bad[..., None], 0x7f, e4m3_encode(v))
    return q, s


def dequantize_e4m3(q, s):
    scale = np.where(s == 255, np.nan, np.exp2(s.astype(np.float64) - 127))
    return E4M3[q] * np.repeat(scale, BLOCK, -1)[..., :q.shape[-1]]


def matmul_e4m3(qa, sa, qb, sb, bias=None, addend=None):
    """(A B^T (+ bias) (+ addend), sum |a| |b|) of [nodes][rows][K] operands."""
    a, b = dequantize_e4m3(qa, sa), dequantize_e4m3(qb, sb)
    c = np.matmul(a, b.transpose(0, 2, 1))
    if bias is not None:
        c = c + np.asarray(bias, np.float64)[:, None, :]
    if addend is not None:
        c = c + np.asarray(addend, np.float64)
    return c, np.matmul(np.abs(a), np.abs(b).transpose(0, 2, 1))


def _log_softmax(z):
    """Rows without anything above -inf: every log probability is -inf."""
    m = z.max(-1, keepdims=True)
    m = np.where(m == -np.inf, 0, m)
    with np.errstate(divide="ignore", invalid="ignore"):
        log_sum = np.log(np.exp(z - m).sum(-1, keepdims=True))
        return np.where((z == -np.inf) & ~np.isnan(log_sum), -np.inf, (z - m) - log_sum), m + log_sum


def token_logprobs(logits, tokens, temperature=1.0, top_k=0):
    """logits [rows][V], tokens [rows] (outside [0, V): none) -> dict of logprob, entropy, lse, top_logprob, top_index."""
    z = np.asarray(logits, np.float64) / temperature
    with np.errstate(invalid="ignore"):
        logp, lse = _log_softmax(z)
        p = np.exp(logp)
        entropy = -np.where(p == 0, 0, p * np.where(p == 0, 0, logp)).sum(-1)
    at = np.arange(len(z))
    some = (tokens >= 0) & (tokens < z.shape[1])
    out = {"logprob": np.where(some, logp[at, np.where(some, tokens, 0)], 0.0), "entropy": entropy, "lse": lse[:, 0]}
    if top_k:
        index = np.argsort(-z, -1, kind="stable")[:, :top_k]               # equal values: lower index first; NaN last
        value = np.take_along_axis(logp, index, -1)
        out["top_index"] = np.where(np.isnan(np.take_along_axis(z, index, -1)), -1, index)
        out["top_logprob"] = value
    return out


def token_logprobs_bwd(logits, tokens, d_logprob=None, d_entropy=None, d_lse=None, temperature=1.0):
    """Gradient with respect to the logits of sum(d_logprob*logprob + d_entropy*entropy + d_lse*lse)."""
    z = np.asarray(logits, np.float64) / temperature
    with np.errstate(invalid="ignore"):
        logp, _ = _log_softmax(z)
        p = np.exp(logp)
        plogp = np.where(p == 0, 0, p * np.where(p == 0, 0, logp))
    col = lambda g: np.zeros((len(z), 1)) if g is None else np.asarray(g, np.float64)[:, None]
    g, h, l = col(d_logprob), col(d_entropy), col(d_lse)
    some = ((tokens >= 0) & (tokens < z.shape[1]))[:, None]
    onehot = np.zeros_like(z)
    np.put_along_axis(onehot, np.where(some, tokens[:, None], 0), some.astype(float), -1)
    g = np.where(some, g, 0)
    none = z.max(-1, keepdims=True) < -1e30                   # nothing but mask values: no gradient
    return np.where(none, 0, (onehot - p) * g - h * (plogp - p * plogp.sum(-1, keepdims=True)) + l * p) / temperature


def distill_topk(logits, value, index, tail, temperature=1.0, row_weight=None):
    """logits [nodes][B][V], value/index [nodes][B][k] (an index outside [0, V): no entry) -> loss [nodes], row_loss
    [nodes][B], gradient of sum(loss) with respect to the logits."""
    z = np.asarray(logits, np.float64) / temperature
    nodes, B, V = z.shape
    w = np.ones((nodes, B)) if row_weight is None else np.asarray(row_weight, np.float64)
    row_loss, grad = np.zeros((nodes, B)), np.zeros_like(z)
    for n in range(nodes):
        for b in range(B):
            if w[n, b] == 0 or z[n, b].max() < -1e30:         # left out, or nothing but mask values
                continue
            have = (index[n, b] >= 0) & (index[n, b] < V)
            ids, lt = index[n, b][have], np.asarray(value[n, b], np.float64)[have]
            logp, _ = _log_softmax(z[n, b][None])
            logp = logp[0]
            with np.errstate(divide="ignore", invalid="ignore"):
                p = np.exp(logp)
                if not tail and len(lt) and lt.max() > -np.inf:       # a list without any mass stays without
                    lt = lt - lt.max() - np.log(np.exp(lt - lt.max()).sum())
                t = np.exp(lt)
                live = t > 0
                loss = (t[live] * (lt[live] - logp[ids[live]])).sum()
                target = np.zeros(V)
                np.add.at(target, ids, t)
                g = p * t.sum() - target
                rest = np.ones(V, bool)
                rest[ids] = False
                left = max(0.0, 1 - t.sum()) if tail else 0.0
                # the others' class by its own logarithm, which does not run out where its mass would; mask values have none
                if left > 0 and rest.any() and not z[n, b, rest].max() < -1e30:
                    log_mass = np.logaddexp.reduce(logp[rest])
                    loss += left * (np.log(left) - log_mass)
                    g += left * (p - np.exp(np.where(rest, logp - log_mass, -np.inf)))
            row_loss[n, b] = np.nan if np.isnan(p).any() else loss         # NaN or +inf in the row: also without a list
            grad[n, b] = g * w[n, b] / (B * temperature)
    return (row_loss * w).mean(1), row_loss, grad
